"""Calls whose launches pass what one dimension of a grid holds: 2^24 workgroups of 256 threads."""
import pytest
import torch

import paper_2502_15779_amd as rcp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("with_queries", [False, True])
def test_append_of_as_many_sequences_and_heads_as_there_may_be(with_queries):
    """1024 sequences of 4096 heads, three of which have new tokens: what a call of those three alone writes."""
    H, D, page, sequences, some = 4096, 64, 16, 1024, {3: 2, 700: 17, 1023: 1}
    g = torch.Generator(device=DEV).manual_seed(1)
    new = [some.get(b, 0) for b in range(sequences)]
    starts = [1]
    for n in new:
        starts.append(starts[-1] + n)
    rows = starts[-1] + 2
    k, v, q = (torch.randn((rows, H, D), generator=g, device=DEV).half() for _ in range(3))
    lengths, table = [5 * (n > 0) + n for n in new], torch.full((sequences, 2), -1, dtype=torch.int32)
    for i, b in enumerate(some):
        table[b] = torch.tensor([2 * i, 2 * i + 1])
    rope = torch.randn((2 * page, D), generator=g, device=DEV)
    codes = (torch.randn((6, H, page, D), generator=g, device=DEV) * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    scales = torch.full((6, H), 2.0 ** -9, device=DEV)
    made = []
    for which in (range(sequences), list(some)):
        caches = [codes.clone(), scales.clone(), codes.clone(), scales.clone()]
        first = [starts[b] for b in which]
        out = rcp.kv8_append(k, v, _int([lengths[b] for b in which]), table[list(which)].to(DEV), *caches, starts=_int(first + [starts[-1]]), rope=rope, rotate=True,
                             q=q if with_queries else None)
        torch.cuda.synchronize()
        made.append([t.view(torch.uint8) if t.dtype == codes.dtype else t for t in caches] + ([out] if with_queries else []))
    assert all(torch.equal(a, b) for a, b in zip(*made))
    assert not torch.equal(made[0][0], codes.view(torch.uint8))
