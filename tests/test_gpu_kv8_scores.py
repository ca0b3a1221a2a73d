"""Scores are sums of binary32 in every form of the paged attention: small products count beside a large one.

Two tokens whose keys differ in the small elements only, beside a first product of `large` times theirs: the difference of their scores is softmax_scale times the sum of those, exact in
64 bits.  Tolerance: a score of D exact products summed in binary32 is off by (D + 16) 2^-24 of softmax_scale sum |q_d K_td|, the result 1 / (1 + e^-difference) by half a step."""
import pytest
import torch

import paper_2502_15779_amd as rcp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("one", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("large", [448.0, 64.0, 8.0, 1.0])
def test_small_products_beside_a_large_one(one, D, dtype, large):
    g = torch.Generator().manual_seed(int(large))
    kc = torch.zeros((1, 1, 16, D))
    kc[0, 0, :, 0] = large
    kc[0, 0, 0, 1:] = torch.randint(4, 15, (D - 1,), generator=g) / 8   # exact codes
    vc = torch.zeros((1, 1, 16, D))
    vc[0, 0, 0] = 1.0
    rows = 6
    q = torch.zeros((rows, 4, D))
    q[..., 0] = large
    q[..., 1:] = torch.randint(1, 120, (rows, 4, D - 1), generator=g) / 64
    q = q.to(DTYPES[dtype])
    caches = [kc.to(torch.float8_e4m3fn), torch.ones((1, 1)), vc.to(torch.float8_e4m3fn), torch.ones((1, 1))]
    scale = 1.5 / float(q[0, 0, 1:].double() @ kc[0, 0, 0, 1:].double())
    # (several tokens: each sees one more that is like the second)
    lengths, starts, table = ([2] * rows, None, torch.zeros((rows, 1))) if one else ([rows + 1], _int([0, rows]), torch.zeros((1, 1)))
    out = rcp.kv8_attn(q.to(DEV), _int(lengths), table.int().to(DEV), *[t.to(DEV) for t in caches], scale, starts=starts).cpu().double()
    others = torch.ones(rows) if one else 1.0 + torch.arange(rows)
    k = caches[0].double()[0, 0]
    difference, size = scale * (q.double() @ (k[0] - k[1])), scale * (q.double().abs() @ k[0])
    exact = 1 / (1 + others.double()[:, None] * torch.exp(-difference))
    tol = exact * (2 * ((D + 16) * 2.0 ** -24 + (2.0 ** -21 if dtype == "f32" else 0.0)) * size + 2.0 ** -19)
    off = (out[:, :, 0] - exact).abs()
    assert bool((off <= tol).all()), f"{float((off / tol).max()):.2f} of what is allowed"
    assert bool((out == out[:, :, :1]).all())
