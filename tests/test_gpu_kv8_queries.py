"""How exactly small elements of a query enter beside its largest one: keys that are zero everywhere else make the score that element's alone, and a large softmax
scale makes its last bits show."""
import pytest
import torch

import paper_2502_15779_amd as rcp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _score(q, code, scale, one):
    """The score of a token whose key is `code` in element 0 and zero elsewhere, beside one whose key is zero: values 1 and 0, so that a row's result is 1 / (1 + e^-score)."""
    rows, H_q, D = q.shape
    kc, vc = torch.zeros((1, 1, 16, D)), torch.zeros((1, 1, 16, D))
    kc[0, 0, 0, 0], vc[0, 0, 0] = code, 1.0
    s = torch.ones((1, 1), device=DEV)
    caches = [kc.to(torch.float8_e4m3fn).to(DEV), s, vc.to(torch.float8_e4m3fn).to(DEV), s]
    starts = None if one else _int([0, rows])
    table = torch.zeros((rows if one else 1, 1), dtype=torch.int32, device=DEV)
    lengths = _int([2] * rows) if one else _int([rows + 1])
    out = rcp.kv8_attn(q.to(DEV), lengths, table, *caches, scale, starts=starts).cpu().double()[:, :, 0]
    seen = torch.full((rows, 1), 2.0) if one else 2.0 + torch.arange(rows)[:, None]   # (several tokens: the others' keys are zero, too)
    return torch.log(out * (seen - 1) / (1 - out))


@pytest.mark.parametrize("one", [True, False])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_small_elements_beside_a_large_one(one, dtype):
    """Elements of 2^-14 to 2^-29 of the largest, with all the bits of their type: off by 2^-38 of the largest at most (pairs of binary16 numbers: or by 2^-22 of themselves)."""
    dtype = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    g = torch.Generator().manual_seed(7)
    largest, rows, H_q, D = 2.0 ** 15, 8, 16, 64
    q = torch.zeros((rows, H_q, D), dtype=dtype)
    down = torch.arange(16).repeat(rows, 1)
    q[..., 0] = ((1 + torch.rand((rows, H_q), generator=g)) * largest * 2.0 ** -14 * 2.0 ** -down).to(dtype)
    q[0, :, 0] = (largest * 2.0 ** -15 * (1 + torch.finfo(dtype).eps) * 2.0 ** -torch.arange(16)).to(dtype)
    q[..., 1] = largest
    small = q[..., 0].double()
    worst = 0.0
    for d in range(16):   # a scale for each magnitude: scores of 1 to 4
        scale = 2.0 ** (14 + d) / largest / 16
        got = _score(q[:, d:d + 1].contiguous(), 16.0, scale, one)
        exact = small[:, d:d + 1] * 16 * scale
        # the score's own binary32 steps, and the result's: 1 / (1 + e^-s) is at least 0.1 away from 0 and 1, rounded a few times
        off = (got - exact).abs() - (2.0 ** -19 + 2.0 ** -22 * exact)
        worst = max(worst, float((off / (16 * scale * largest)).max()))
    assert worst <= 2.0 ** -38, f"2^{float(torch.tensor(worst).log2()):.2f} of the largest element"
