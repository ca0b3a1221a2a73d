"""How exactly the softmax weights of the paged attention enter the product with the values, on inputs where nothing else hides it: values of neighbouring tokens
cancel, so that a result is a small difference of large terms and the rounding of each weight shows.

Tolerance, from the formula: scores are sums of D exact products in binary32 and a few factors, off by (D + 16) 2^-24 of their magnitude; a weight enters as a pair of
binary16 numbers (2^-22 of it) or, where several tokens have bfloat16 results, as one (half a step: at most 2^-11 of it).  Numerator and denominator: twice that, beside n roundings of a
sum in binary32; the result is rounded once, by at most half a step."""
import pytest
import torch

import kv8_reference as ref
import paper_2502_15779_amd as rcp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _int(v):
    return torch.tensor(v, dtype=torch.int32)


def _run(q, lengths, starts, table, caches, scale, out_dtype):
    got = rcp.kv8_attn(q.to(DEV), _int(lengths).to(DEV), table.to(DEV), *[t.to(DEV) for t in caches], scale, starts=None if starts is None else _int(starts).to(DEV),
                       out_dtype=out_dtype)
    return got.cpu().double(), ref.attention(q, lengths, starts, table, *caches, scale)


@pytest.mark.parametrize("one,out,weight", [(True, "f16", 2.0 ** -22), (True, "bf16", 2.0 ** -22), (True, "f32", 2.0 ** -22), (False, "f16", 2.0 ** -22),
                                            (False, "f32", 2.0 ** -22), (False, "bf16", 2.0 ** -11)])
@pytest.mark.parametrize("D", [64, 128])
def test_values_that_cancel(D, one, out, weight):
    page, H, rep = 16, 2, 4
    g = torch.Generator().manual_seed(D)
    kc = (8 + torch.randint(0, 8, (6, H, page, D), generator=g)).float().to(ref.E4M3)
    values = torch.randn((6, H, page, D), generator=g) * 60
    values[:, :, 1::2] = -values[:, :, 0::2]
    vc = values.clamp(-448, 448).to(ref.E4M3)
    scales = torch.full((6, H), 2.0 ** -5)
    lengths = [2, 4, 10, 30, 46, 16] if one else [30, 46]
    starts = None if one else [0, 30, 60]
    table = torch.arange(6).int().view(6, 1).expand(6, 3).contiguous() if one else torch.arange(6).int().view(2, 3)
    q = torch.zeros((6 if one else 60, H * rep, D))
    q[..., :3] = torch.randn((*q.shape[:2], 3), generator=g)   # few elements, so that scores are all but exact
    q = q.to(torch.float32 if out == "f32" else DTYPES[out])
    got, (exact, mag, size, seen) = _run(q, lengths, starts, table, [kc, scales, vc, scales], 0.25, DTYPES[out])
    e = (weight + 2 * ((D + 16) * 2.0 ** -24 + (2.0 ** -21 if out == "f32" else 0.0)) * size + (seen + 16) * 2.0 ** -24) * 2 * mag
    tol = e + torch.finfo(DTYPES[out]).eps / 2 * exact.abs()
    off = (got - exact).abs()
    assert bool((exact.abs() < 0.05 * mag).any())
    assert bool((off <= tol).all()), f"{float((off / tol).max()):.2f} of what is allowed"
