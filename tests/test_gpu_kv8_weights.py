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


@pytest.mark.parametrize("one", [True, False])
@pytest.mark.parametrize("out,low,high", [("f16", -20, 3), ("f16", -22, 6), ("bf16", -20, 6), ("bf16", -30, 6), ("f32", -20, 3), ("f32", -22, 6), ("f32", -40, 10)])
def test_values_of_very_different_size_that_are_attended_to_alike(one, out, low, high):
    """Pages of values 2^23 to 2^50 apart whose tokens have weights of the same size, the large page zero in half of its elements: what stands there comes from
    weights that, with their page's scale, are subnormal binary16 numbers or none.  A weight times its scale is then off by up to 2^-34 of the row's largest one (2^-25 where that is
    2^9 or more), and no element by more than the sum of that over the tokens."""
    D, page, rep = 64, 16, 2
    g = torch.Generator().manual_seed(high - low)
    kc = torch.randn((3, 1, page, D), generator=g).to(ref.E4M3)
    vc = (torch.randn((3, 1, page, D), generator=g) * 60).clamp(-448, 448).to(ref.E4M3)
    vc[1, :, :, ::2] = torch.zeros_like(vc[1, :, :, ::2])
    ks, vs = torch.full((3, 1), 1.0), torch.tensor([[2.0 ** low], [2.0 ** high], [2.0 ** (low + 3)]])
    q = (0.5 * torch.randn((3, rep, D), generator=g)).to(DTYPES[out])
    lengths, starts, table = ([48, 40, 34], None, _int([[0, 1, 2], [2, 1, 0], [1, 0, 2]])) if one else ([48], [0, 3], _int([[0, 1, 2]]))
    got, (exact, mag, size, seen) = _run(q, lengths, starts, table, [kc, ks, vc, vs], 0.2, DTYPES[out])
    floor = torch.zeros_like(exact)
    for i in range(3):
        n, ids = (lengths[i], table[i]) if one else (46 + i, table[0])
        at, slots = ids.long().repeat_interleave(page)[:n], torch.arange(n) % page
        for h in range(rep):
            p = torch.softmax(0.2 * (kc[at, 0, slots].double() @ q[i, h].double()), 0) * vs[at, 0].double()
            floor[i, h] = 2.0 ** -34 * p.max() * vc[at, 0, slots].double().abs().sum(0)
    weight = 2.0 ** -11 if out == "bf16" and not one else 2.0 ** -22
    e = (weight + 2 * ((D + 16) * 2.0 ** -24 + (2.0 ** -21 if out == "f32" else 0.0)) * size + (seen + 16) * 2.0 ** -24) * 2 * mag
    tol = e + floor + torch.finfo(DTYPES[out]).eps / 2 * exact.abs() + (2.0 ** -25 if out == "f16" else 0.0)
    off = (got - exact).abs()
    assert bool((off <= tol).all()), f"{float((off / tol).max()):.2f} of what is allowed"
    if high - low >= 46:
        assert bool((off > e).any()), "the range of the weights does not show here"
