"""The adapters' kernels for more than 128 tokens: every number of pieces in a row of B, outputs that end inside a wavefront's part, tiles of many adapters, and the sizes on either side of the
rule that picks them.  References and tolerances are those of the other tests of these calls."""
import pytest
import torch

from test_gpu_lowrank import _check, _inputs, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,r,adapters,dtype,out", [
    (129, 1028, 64, 64, 3, "bf16", "bf16"), (228, 516, 96, 40, 100, "f16", "f32"), (194, 1140, 32, 48, 2, "bf16", "f16"), (205, 36, 160, 96, 9, "f16", "f16"),
    (209, 640, 64, 112, 2, "bf16", "f32"), (198, 4, 64, 56, 5, "f16", "bf16"), (257, 300, 224, 8, 5, "f16", "bf16"), (130, 512, 2048, 16, 130, "bf16", "f16"),
    (191, 2048, 640, 72, 7, "f16", "f16"), (128, 1028, 640, 64, 3, "bf16", "bf16"), (128, 388, 1312, 128, 128, "bf16", "f32")])
def test_many_tokens_and_ranks(M, N, K, r, adapters, dtype, out):
    print("many", M, N, K, r, adapters, dtype, out, flush=True)
    g, x, A, B, scaling, base = _inputs(3 * M + r, M, N, K, r, adapters, dtype, out)
    which = torch.randint(-1, adapters, (M,), generator=g)
    which[:2] = torch.tensor([0, 1])
    got = _run(x, A, B, which, scaling, base)
    _check(x, A, B, which, scaling, base, got)
    B[1, :, 3] = float("inf")
    A[1, 5] = float("nan")
    other = _run(x, A, B, which, scaling, base)
    assert torch.equal(other[which != 1], got[which != 1]) and not bool(other[1].isfinite().any())


def test_an_infinity_stays_with_its_request():
    g, x, A, B, scaling, base = _inputs(3, 200, 128, 128, 16, 4, "f16", "f32")
    which = torch.arange(200) % 3
    want = _run(x, A, B, which, scaling, base).cpu()
    x[5, 7], x[5, 9] = float("inf"), float("nan")
    A[2, 3, 11], B[2, 40, 5], B[3] = float("-inf"), float("nan"), float("nan")
    got = _run(x, A, B, which, scaling, base).cpu()
    keep = which != 2
    keep[5] = False
    assert torch.equal(got[keep], want[keep])


def test_no_adapter_at_all():
    g, x, A, B, scaling, base = _inputs(2, 140, 64, 64, 8, 2, "bf16", "f32")
    which = torch.full((140,), -1)
    assert torch.equal(_run(x, A, B, which, scaling, base).cpu(), base)
