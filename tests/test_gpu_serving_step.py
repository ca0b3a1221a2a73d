"""A serving step of several requests as a program runs it: one quantised projection for all, each request's adapter beside it, keys and values into
the paged cache with the rotations on the way, attention over it -- prompts first, then captured single-token steps whose lengths advance inside
the graph."""
import pytest
import torch

import kv8_reference as ref
import paper_2502_15779_amd as rcp
from test_gpu_kv8_attn import _tolerance

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
K, HEADS, KV_HEADS, D, PAGE, R, REQUESTS = 512, 8, 2, 64, 16, 8, 3
N = (HEADS + 2 * KV_HEADS) * D


class Program:
    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.g = g
        w = (torch.randn((N, K), generator=g) * 0.02).half().to(DEV)
        self.packed, self.codebook = rcp.pack_weights(w, torch.full((N,), -0.04, device=DEV), torch.full((N,), 0.04, device=DEV),
                                                      torch.full((N, 3), 1 / 3, device=DEV))
        self.A = (torch.randn((2, R, K), generator=g) / K ** 0.5).half().to(DEV)
        self.B = (torch.randn((2, N, R), generator=g) * 0.1).half().to(DEV)
        self.scaling = torch.tensor([2.0, 0.5], device=DEV)
        self.table = torch.randperm(30, generator=g).view(REQUESTS, 10).int().to(DEV)
        self.caches = [t for _ in range(2) for t in rcp.kv8_new_cache(30, KV_HEADS, DEV, PAGE, D)]
        self.rope = ref.rope_table(10 * PAGE, D).to(DEV)
        self.lengths = torch.zeros(REQUESTS, dtype=torch.int32, device=DEV)

    def project(self, x, which):
        """[rows, N]: in calls of sixteen tokens at most, as the product takes them."""
        base = torch.empty((x.shape[0], N), dtype=torch.float16, device=DEV)
        for at in range(0, x.shape[0], rcp.MAX_M):
            part = x[at:at + rcp.MAX_M]
            xq, s = rcp.rotate_quant_act(part, None, 0.9)
            rcp.w2a4_gemv(self.packed, self.codebook, N, K, xq, s, part.shape[0], out=base[at:at + rcp.MAX_M])
        return rcp.lowrank_add(x, self.A, self.B, which, self.scaling, base, out=base)

    def attend(self, qkv, starts, out=None):
        qkv = qkv.view(-1, HEADS + 2 * KV_HEADS, D)
        q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]
        q = rcp.kv8_append(k, v, self.lengths, self.table, *self.caches, starts=starts, rope=self.rope, rotate=True, q=q)
        return q, rcp.kv8_attn(q, self.lengths, self.table, *self.caches, D ** -0.5, starts=starts, out=out, out_dtype=torch.float16)


def _against_64_bits(p, q, out, starts):
    host = [t.cpu() for t in p.caches]
    lengths = p.lengths.tolist()
    exact, mag, size, seen = ref.attention(q.cpu(), lengths, starts, p.table.cpu(), *host, D ** -0.5)
    tol = _tolerance(exact, mag, size, seen, q, out.dtype, starts is None)
    assert bool(((out.cpu().double() - exact).abs() <= tol).all())


def test_prompts_then_captured_steps():
    p = Program(1)
    new = [37, 5, 18]
    starts = [0, 37, 42, 60]
    which = torch.tensor([0] * 37 + [-1] * 5 + [1] * 18, dtype=torch.int32, device=DEV)
    x = torch.randn((60, K), generator=p.g).half().to(DEV)
    p.lengths += torch.tensor(new, dtype=torch.int32, device=DEV)
    q, out = p.attend(p.project(x, which), torch.tensor(starts, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    _against_64_bits(p, q, out, starts)

    # one token of each request: eager on a copy of the state, captured on the other
    which = torch.tensor([0, -1, 1], dtype=torch.int32, device=DEV)
    e = Program(1)
    e.lengths.copy_(p.lengths)
    for a, b in zip(e.caches, p.caches):
        a.copy_(b)
    token = torch.zeros((REQUESTS, K), dtype=torch.float16, device=DEV)
    result = torch.zeros((REQUESTS, HEADS, D), dtype=torch.float16, device=DEV)
    saved = [t.clone() for t in [p.lengths] + p.caches]

    def step():
        p.lengths.add_(1)
        return p.attend(p.project(token, which), None, result)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        q, _ = step()
    for t, s in zip([p.lengths] + p.caches, saved):   # the warm-up took a step
        t.copy_(s)
    for i in range(20):
        x = torch.randn((REQUESTS, K), generator=p.g).half().to(DEV)
        token.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        e.lengths += 1
        eq, want = e.attend(e.project(x, which), None)
        torch.cuda.synchronize()
        assert torch.equal(result, want) and torch.equal(q, eq), i
        assert torch.equal(p.lengths, e.lengths)
        assert all(torch.equal(a.float(), b.float()) for a, b in zip(p.caches, e.caches))
        if i % 7 == 0:
            _against_64_bits(p, q, result, None)
