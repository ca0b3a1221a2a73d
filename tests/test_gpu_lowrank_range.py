"""How exactly small inner products enter the second product of the adapters beside large ones of the same token: B is zero for the ranks of the large ones.

t = x A^T is off by at most (K + 16) 2^-24 sum_k |x_k A_rk|; binary16: as a pair of numbers, off by 2^-22 of it or by 2^-38 of the token's largest; bfloat16: as three numbers, 2^-24.
The second product sums r terms in binary32, and the result is binary32."""
import pytest
import torch

import paper_2502_15779_amd as rcp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,r", [(5, 16), (5, 64), (100, 16), (100, 64), (100, 128)])
@pytest.mark.parametrize("down", [10, 16, 20, 26])
def test_small_inner_products_beside_large_ones(M, r, down, dtype):
    N, K = 64, 64
    T = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(M + r + down)
    # the even columns of x and A make the large inner products, the odd ones the small
    x = (torch.rand((M, K), generator=g) + 0.5) * 16
    x[:, 1::2] *= 2.0 ** -(down // 2)
    A = torch.zeros((1, r, K))
    large = torch.arange(r) % 2 == 0
    A[0, large, ::2] = torch.rand((r // 2, K // 2), generator=g) + 0.5
    A[0, ~large, 1::2] = (torch.rand((r // 2, K // 2), generator=g) + 0.5) * 2.0 ** -(down - down // 2)
    B = torch.randn((1, N, r), generator=g)
    B[:, :, large] = 0.0
    x, A, B = x.to(T), A.to(T), B.to(T)
    base, which, scaling = torch.zeros((M, N)), torch.zeros(M, dtype=torch.int32), torch.tensor([1.5])
    got = rcp.lowrank_add(*(t.to(DEV) for t in (x, A, B, which, scaling, base))).cpu().double()
    t = x.double() @ A[0].double().t()
    exact = 1.5 * t @ B[0].double().t()
    piece = torch.maximum(2.0 ** -22 * t.abs(), 2.0 ** -38 * t.abs().amax(1, keepdim=True)) if dtype == "f16" else 2.0 ** -24 * t.abs()
    e = (K + 16) * 2.0 ** -24 * (x.double().abs() @ A[0].double().abs().t()) + piece + (r + 16) * 2.0 ** -24 * t.abs()
    tol = 1.5 * e @ B[0].double().abs().t() + 2.0 ** -23 * exact.abs()
    off = (got - exact).abs()
    assert bool((off <= tol).all()), f"{float((off / tol).max()):.2f} of what is allowed"
