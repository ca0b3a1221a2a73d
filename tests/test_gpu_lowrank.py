"""Low-rank adapters beside a shared projection against 64 bits.

Tolerance, from the formula: t = x A^T is a sum of K exact products in binary32, off by at most (K + 16) 2^-24 sum_k |x_k A_rk|; it enters the second product with a
relative 2^-20 of the token's largest |t| (two binary16 numbers; three bfloat16 numbers are closer); that product sums r terms, and the
result is rounded once: |out - exact| <= |s| sum_r |B_nr| ((K + 16) 2^-24 sum_k |x_k A_rk| + (2^-20 + (r + 16) 2^-24) max_r |t_r|) + (half a step + 2^-23)
of the larger of |out| and |base|."""
import pytest
import torch

import paper_2502_15779_amd as rcp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(seed, M, N, K, r, adapters, dtype, out):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, K), generator=g).to(DTYPES[dtype])
    A = (torch.randn((adapters, r, K), generator=g) / K ** 0.5).to(DTYPES[dtype])
    B = (torch.randn((adapters, N, r), generator=g) * 0.1).to(DTYPES[dtype])
    return g, x, A, B, torch.rand((adapters,), generator=g) + 0.5, torch.randn((M, N), generator=g).to(DTYPES[out])


def _check(x, A, B, which, scaling, base, got):
    exact, tol = base.double(), torch.zeros(base.shape, dtype=torch.float64)
    r, K = A.shape[1:]
    for a in range(A.shape[0]):
        rows = torch.nonzero(which == a).flatten()
        if rows.numel() == 0:
            continue
        s, xa, Aa, Ba = scaling[a].double(), x[rows].double(), A[a].double(), B[a].double()
        t, size = xa @ Aa.t(), xa.abs() @ Aa.abs().t()
        exact[rows] += s * (t @ Ba.t())
        e = (K + 16) * 2.0 ** -24 * size + (2.0 ** -20 + (r + 16) * 2.0 ** -24) * t.abs().amax(1, keepdim=True)
        tol[rows] += s * (e @ Ba.abs().t())
    tol += (torch.finfo(base.dtype).eps / 2 + 2.0 ** -23) * torch.maximum(exact.abs(), base.double().abs())
    off = (got.cpu().double() - exact).abs()
    assert bool((off <= tol).all()), f"off by {float(off.max()):.2e}, {float((off / tol).max()):.2f} of what is allowed"
    alone = (which < 0) | (which >= A.shape[0])
    assert torch.equal(got.cpu()[alone], base[alone])


def _run(x, A, B, which, scaling, base, **more):
    return rcp.lowrank_add(*(t.to(DEV) for t in (x, A, B, which.int(), scaling, base)), **more)


@pytest.mark.parametrize("M,N,K,r,adapters,dtype,out", [
    (1, 64, 32, 8, 1, "f16", "f16"), (1, 4, 4096, 16, 3, "bf16", "f32"), (16, 260, 96, 16, 20, "f16", "f32"), (15, 1028, 544, 24, 4, "bf16", "bf16"),
    (17, 132, 1056, 40, 2, "f16", "f16"), (64, 512, 2048, 64, 64, "bf16", "f16"), (65, 300, 224, 8, 5, "f16", "bf16"), (130, 388, 1312, 128, 3, "bf16", "f32"),
    (333, 2048, 640, 72, 7, "f16", "f16"), (200, 40, 14336, 32, 1, "bf16", "bf16")])
def test_against_64_bits(M, N, K, r, adapters, dtype, out):
    """Adapters in any order, some tokens without one, entries far outside."""
    print("lowrank", M, N, K, r, adapters, dtype, out, flush=True)
    g, x, A, B, scaling, base = _inputs(M + N, M, N, K, r, adapters, dtype, out)
    which = torch.randint(-1, adapters, (M,), generator=g)
    if M > 3:
        which[1], which[2] = adapters, -2 ** 31
        which[3] = 2 ** 31 - 1
    else:
        which[0] = adapters - 1
    _check(x, A, B, which, scaling, base, _run(x, A, B, which, scaling, base))


def test_onto_the_base_itself_and_with_a_workspace():
    g, x, A, B, scaling, base = _inputs(1, 20, 256, 128, 16, 3, "f16", "f16")
    which = torch.arange(20) % 4 - 1
    want = _run(x, A, B, which, scaling, base)
    dev = [t.to(DEV) for t in (x, A, B, which.int(), scaling, base)]
    work = torch.empty(rcp.lowrank_workspace_bytes(20, 256, 128, 16), dtype=torch.uint8, device=DEV)
    got = rcp.lowrank_add(*dev, out=dev[5], workspace=work)
    assert got is dev[5] and torch.equal(got, want)
    with pytest.raises(rcp.RcpError) as e:
        rcp.lowrank_add(*dev, workspace=work[:16])
    assert e.value.code == -5
    empty = rcp.lowrank_add(dev[0][:0], dev[1], dev[2], dev[3][:0], dev[4], dev[5][:0])
    assert empty.shape == (0, 256)
    for i, bad in ((0, dev[0].float()), (1, dev[1][:2]), (3, dev[3].long()), (3, dev[3][:5]), (4, dev[4].double()), (5, dev[5][:, :128]), (3, dev[3].cpu())):
        with pytest.raises(ValueError):
            rcp.lowrank_add(*dev[:i], bad, *dev[i + 1:])


def test_no_adapter_at_all():
    g, x, A, B, scaling, base = _inputs(2, 70, 64, 64, 8, 2, "bf16", "f32")
    which = torch.full((70,), -1)
    assert torch.equal(_run(x, A, B, which, scaling, base).cpu(), base)


@pytest.mark.parametrize("M", [12, 100])
def test_an_infinity_stays_with_its_request(M):
    """Infinities and NaN in one token's input, and in the adapter of another one, change no other token's result."""
    g, x, A, B, scaling, base = _inputs(3, M, 128, 128, 16, 4, "f16", "f32")
    which = torch.arange(M) % 3
    want = _run(x, A, B, which, scaling, base).cpu()
    x[5, 7], x[5, 9] = float("inf"), float("nan")
    A[2, 3, 11], B[2, 40, 5] = float("-inf"), float("nan")
    B[3] = float("nan")
    got = _run(x, A, B, which, scaling, base).cpu()
    keep = which != 2
    keep[5] = False
    assert torch.equal(got[keep], want[keep])


@pytest.mark.parametrize("M,N,K,r,adapters,dtype,out", [
    (129, 1028, 64, 64, 3, "bf16", "bf16"), (100, 516, 96, 40, 100, "f16", "f32"), (66, 1140, 32, 48, 2, "bf16", "f16"), (77, 36, 160, 96, 9, "f16", "f16"),
    (81, 640, 64, 112, 2, "bf16", "f32"), (70, 4, 64, 56, 5, "f16", "bf16")])
def test_many_tokens_and_ranks(M, N, K, r, adapters, dtype, out):
    """Rows of B of every number of pieces, wavefronts whose outputs end early or are none, tiles of many adapters; infinities and NaN stay with their adapter."""
    print("ranks", M, N, K, r, adapters, dtype, out, flush=True)
    g, x, A, B, scaling, base = _inputs(5 * M + r, M, N, K, r, adapters, dtype, out)
    which = torch.randint(-1, adapters, (M,), generator=g)
    which[:2] = torch.tensor([0, 1])
    got = _run(x, A, B, which, scaling, base)
    _check(x, A, B, which, scaling, base, got)
    B[1, :, 3] = float("inf")
    A[1, 5] = float("nan")
    other = _run(x, A, B, which, scaling, base)
    assert torch.equal(other[which != 1], got[which != 1]) and not bool(other[1].isfinite().any())


@pytest.mark.parametrize("size", [1e-4, 1.0, 60000.0])
def test_magnitudes(size):
    """Inner products far from 1: binary16 operands are scaled per token."""
    g, x, A, B, scaling, base = _inputs(4, 9, 64, 256, 16, 2, "f16", "f32")
    x = (x.float() * size / 4).clamp(-65504, 65504).half()
    x[3] = 0
    which = torch.arange(9) % 2
    base = base * size
    _check(x, A, B, which, scaling, base, _run(x, A, B, which, scaling, base))


def test_results_do_not_depend_on_the_neighbours():
    """A token alone and among others, in another order, with the same splits of K: the same bits."""
    g, x, A, B, scaling, base = _inputs(5, 16, 128, 256, 16, 6, "bf16", "f32")
    which = torch.randint(0, 6, (16,), generator=g)
    want = _run(x, A, B, which, scaling, base).cpu()
    order = torch.randperm(16, generator=g)
    got = _run(x[order], A, B, which[order], scaling, base[order]).cpu()
    assert torch.equal(got, want[order])


def test_a_capture_follows_the_adapters():
    g, x, A, B, scaling, base = _inputs(6, 10, 192, 128, 8, 5, "f16", "f16")
    dev = [t.to(DEV) for t in (x, A, B, torch.zeros(10).int(), scaling, base)]
    out = torch.zeros_like(dev[5])
    work = torch.empty(rcp.lowrank_workspace_bytes(10, 192, 128, 8), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        rcp.lowrank_add(*dev, out=out, workspace=work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        rcp.lowrank_add(*dev, out=out, workspace=work)
    for _ in range(4):
        dev[0].copy_(torch.randn((10, 128), generator=g))
        dev[3].copy_(torch.randint(-1, 6, (10,), generator=g))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, rcp.lowrank_add(*dev))
