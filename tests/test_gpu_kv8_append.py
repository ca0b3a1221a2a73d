"""Appending to the paged 8-bit cache, bit for bit against the written order of its operations: codes, scales, rotated queries, and every byte that no
new token has."""
import pytest
import torch

import kv8_reference as ref
import paper_2502_15779_amd as rcp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _int(v):
    return torch.tensor(v, dtype=torch.int32)


def _state(seed, n_pages, H, page, D, low=-9, high=-3):
    """A used cache: random finite codes, powers of two."""
    g = torch.Generator().manual_seed(seed)
    caches = []
    for _ in range(2):
        codes = (torch.randn((n_pages, H, page, D), generator=g) * 60).clamp(-448, 448).to(ref.E4M3)
        caches += [codes, torch.exp2(torch.randint(low, high, (n_pages, H), generator=g).float())]
    return g, caches


def _tables(g, lengths, page, extra=0):
    """Random distinct pages, as many as the lengths take and `extra` columns more."""
    width = max(-(-n // page) for n in lengths) + extra
    ids = torch.randperm(width * len(lengths), generator=g)
    return ids.view(len(lengths), width).int(), width * len(lengths)


def _check(k, v, lengths, starts, table, caches, angles, rotate, q=None, in_place=False):
    """Appends on both sides and compares everything."""
    dev = [t.clone().to(DEV) for t in caches]
    opt = lambda t: None if t is None else t.to(DEV)
    kd, vd = k.to(DEV), v.to(DEV)
    H, D = k.shape[1], k.shape[2]
    qd = opt(q)
    q_out = None if q is None else (qd if in_place else torch.full_like(qd, 7.0))
    got = rcp.kv8_append(kd, vd, _int(lengths).to(DEV), table.to(DEV), *dev, starts=None if starts is None else _int(starts).to(DEV),
                         rope=opt(angles), rotate=rotate, q=qd, q_out=q_out)
    torch.cuda.synchronize()
    want = [t.clone() for t in caches]
    ref.append(k, lengths, starts, table, want[0], want[1], angles, rotate)
    ref.append(v, lengths, starts, table, want[2], want[3])
    for name, a, b in zip(("k codes", "k scales", "v codes", "v scales"), dev, want):
        a = a.cpu()
        same = torch.equal(a.view(torch.uint8), b.view(torch.uint8)) if a.dtype == ref.E4M3 else torch.equal(a, b)
        assert same, f"{name}: {int((a.float() != b.float()).sum())} differ"
    if q is None:
        assert got is None
        return dev
    assert got is q_out
    expect = q.clone() if in_place else torch.full_like(q, 7.0)
    for first, count, pos0 in ref.runs(len(lengths), lengths, starts, q.shape[0]):
        for i in range(count):
            if 0 <= pos0 + i < table.shape[1] * caches[0].shape[2]:
                expect[first + i] = ref.turn(q[first + i].float(), None if angles is None else angles[pos0 + i], rotate).to(q.dtype)
    assert torch.equal(got.cpu(), expect)
    return dev


@pytest.mark.parametrize("D,page,dtype,H,rotate,rope", [
    (128, 64, "f16", 32, True, True), (128, 16, "bf16", 8, False, True), (64, 32, "f32", 3, True, True), (64, 16, "f16", 5, False, False),
    (128, 128, "f32", 1, True, False), (64, 128, "bf16", 8, True, True)])
def test_one_token_each(D, page, dtype, H, rotate, rope):
    print("one token each", D, page, dtype, H, flush=True)
    lengths = [1, 2, page, page + 1, 3 * page, 0, 37, 2 * page + 9]
    g, _ = _state(1, 1, 1, 16, 64)
    table, n = _tables(g, lengths, page, 1)
    _, caches = _state(2, n, H, page, D)
    k, v = (torch.randn((len(lengths), H, D), generator=g).to(DTYPES[dtype]) * s for s in (3.0, 0.7))
    q = torch.randn((len(lengths), 2 * H, D), generator=g).to(DTYPES[dtype])
    angles = ref.rope_table(table.shape[1] * page, D) if rope else None
    _check(k, v, lengths, None, table, caches, angles, rotate, q)


@pytest.mark.parametrize("D,page,dtype,H,rotate", [
    (128, 16, "bf16", 2, False), (128, 32, "f16", 3, True), (128, 64, "f32", 1, False), (128, 128, "bf16", 2, True),
    (64, 16, "f16", 4, True), (64, 32, "f32", 2, False), (64, 64, "bf16", 1, True), (64, 128, "f16", 3, False)])
def test_ragged_runs(D, page, dtype, H, rotate):
    """Runs that start and end inside pages, empty ones, one token, padding rows before and behind; keys, values and queries as views of one
    projection's output."""
    print("ragged", D, page, dtype, H, flush=True)
    new = [3, 0, page, 1, 2 * page + 5, page - 1, 70]
    lengths = [3, 9, 2 * page + 7, page + 1, 2 * page + 5, 3 * page, 200]
    starts = [2]
    for n in new:
        starts.append(starts[-1] + n)
    rows = starts[-1] + 3
    g, _ = _state(3, 1, 1, 16, 64)
    table, n = _tables(g, lengths, page)
    _, caches = _state(4, n, H, page, D)
    x = (torch.randn((rows, 4 * H, D), generator=g) * torch.exp(torch.randn((1, 4 * H, 1), generator=g))).to(DTYPES[dtype])
    _check(x[:, 2 * H:3 * H], x[:, 3 * H:], lengths, starts, table, caches, ref.rope_table(table.shape[1] * page, D), rotate, x[:, :2 * H])


def test_more_sequences_than_lanes():
    D, page, H = 64, 16, 2
    new = [(b * 7) % 4 for b in range(140)]
    lengths, starts = [n + (b * 5) % 40 for b, n in enumerate(new)], [1]
    for x in new:
        starts.append(starts[-1] + x)
    g, _ = _state(16, 1, 1, 16, 64)
    table, n = _tables(g, lengths, page)
    _, caches = _state(17, n, H, page, D)
    k, v = (torch.randn((starts[-1] + 2, H, D), generator=g).half() for _ in range(2))
    _check(k, v, lengths, starts, table, caches, ref.rope_table(table.shape[1] * page, D), True, torch.randn((starts[-1] + 2, 3, D), generator=g).half())


def test_scales_grow_and_pages_start_anew():
    """Token after token with magnitudes that rise and fall: the scale only grows within a page, older codes are rounded to it, and the next page's first token
    ignores what the page held (a scale of 2^30)."""
    D, page, H = 64, 16, 2
    g, caches = _state(5, 4, H, page, D)
    caches[1].fill_(2.0 ** 30)
    table = _int([[2, 0, 3]])
    size = [1.0, 1.0, 30.0, 0.01, 900.0, 1e-6, 5000.0, 1.0] * 5
    for i, s in enumerate(size):
        k, v = (torch.randn((1, H, D), generator=g) * s for _ in range(2))
        if i == 20:
            k.zero_()   # nothing to represent: the page keeps its scale
        starts = [0, 1] if i % 2 else None
        caches = [t.cpu() for t in _check(k, v, [i + 1], starts, table, caches, None, False)]


def test_a_run_at_once_and_token_by_token():
    """The same tokens in one call and one by one leave the same scales, and the same codes but where an older code fell into the subnormals before a growth."""
    D, page, H, n = 128, 32, 3, 75
    g = torch.Generator().manual_seed(6)
    k, v = (torch.randn((n, H, D), generator=g).cuda() for _ in range(2))
    table = _int([[1, 0, 2]]).cuda()
    a, b = (rcp.kv8_new_cache(3, H, DEV, page, D) + rcp.kv8_new_cache(3, H, DEV, page, D) for _ in range(2))
    rcp.kv8_append(k, v, _int([n]).cuda(), table, *a, starts=_int([0, n]).cuda(), rotate=True)
    for i in range(n):
        rcp.kv8_append(k[i:i + 1], v[i:i + 1], _int([i + 1]).cuda(), table, *b, rotate=True)
    for i in (0, 2):
        assert torch.equal(a[i + 1], b[i + 1])
        x, y = (c[i].float() * c[i + 1][..., None, None] for c in (a, b))
        assert bool(((x - y).abs() <= a[i + 1][..., None, None] * 2.0 ** -9).all())


@pytest.mark.parametrize("one", [True, False])
def test_tokens_without_a_page(one):
    """Table entries that are no page, positions beyond the table, more new tokens than the length: nothing of those is written."""
    D, page, H = 128, 16, 2
    g, caches = _state(7, 5, H, page, D)
    table = _int([[0, -1, 1], [5, 2, 2 ** 31 - 1], [-2 ** 31, 3, 4]])
    angles = ref.rope_table(3 * page, D)
    if one:
        cases = [[17, 16, 49], [16, 17, 48], [0, 33, 20], [-5, 2 ** 30, 1]]
        rows, starts = 3, None
    else:
        cases = [[40, 45, 60], [30, 3, 48]]
        rows, starts = 72, [0, 30, 50, 72]
    for lengths in cases:
        k, v, q = (torch.randn((rows, h, D), generator=g).half() for h in (H, H, 2 * H))
        caches = [t.cpu() for t in _check(k, v, lengths, starts, table, caches, angles, True, q)]


def test_numbers_at_the_ends():
    """Infinities, NaN, zeros of both signs, subnormals, the largest numbers, and magnitudes on and next to 448 * 2^E."""
    D, page, H = 64, 16, 1
    g, caches = _state(8, 6, H, page, D)
    inf, nan = float("inf"), float("nan")
    rows = [[inf, 1.0], [-inf, nan], [nan, nan], [0.0, -0.0], [1e-45, -3e-39], [3.4028234663852886e38, -1.0], [inf, 3.4028234663852886e38], [448.0, 1.0],
            [448.00003, 1.0], [224.0, 0.5], [1.75 * 2.0 ** -32, 2.0 ** -49], [2.0 ** -50, 2.0 ** -51], [28.0, 17.0 / 1024]]
    for pair in rows:
        k = torch.zeros((1, H, D))
        k[0, 0, 0::2], k[0, 0, 1::2] = pair[0], pair[1]
        v = k.flip(-1)
        for lengths, starts in (([1], None), ([2], [0, 1])):
            caches = [t.cpu() for t in _check(k, v, lengths, starts, _int([[3, 1]]), caches, None, False)]


def test_queries_in_place_and_alone():
    D, page, H = 128, 64, 4
    g, caches = _state(9, 4, H, page, D)
    k, v, q = (torch.randn((2, h, D), generator=g).bfloat16() for h in (H, H, 12))
    table = _int([[0, 1], [2, 3]])
    angles = ref.rope_table(2 * page, D)
    _check(k, v, [70, 5], None, table, caches, angles, True, q, in_place=True)
    made = rcp.kv8_append(k.to(DEV), v.to(DEV), _int([70, 5]).to(DEV), table.to(DEV), *[t.clone().to(DEV) for t in caches], rope=angles.to(DEV), q=q.to(DEV))
    want = torch.stack([ref.turn(q[i].float(), angles[p], False).to(q.dtype) for i, p in enumerate((69, 4))])
    assert torch.equal(made.cpu(), want)


def test_pages_beyond_32_bits():
    """A pool of 5 GB: the last page's codes start beyond 2^32 bytes."""
    D, page, H, n = 128, 128, 64, 5200
    codes, scales = rcp.kv8_new_cache(n, H, DEV, page, D)
    vc, vs = rcp.kv8_new_cache(n, H, DEV, page, D)
    g = torch.Generator().manual_seed(10)
    k, v = (torch.randn((150, H, D), generator=g).half() for _ in range(2))
    table, last = _int([[n - 1, 4999]]), [n - 1, 4999]
    rcp.kv8_append(k.to(DEV), v.to(DEV), _int([150]).to(DEV), table.to(DEV), codes, scales, vc, vs, starts=_int([0, 150]).to(DEV))
    small = [t[last].cpu() for t in (codes, scales, vc, vs)]
    want = [torch.zeros_like(t) for t in small]
    ref.append(k, [150], [0, 150], _int([[0, 1]]), want[0], want[1])
    ref.append(v, [150], [0, 150], _int([[0, 1]]), want[2], want[3])
    assert all(torch.equal(a.float(), b.float()) for a, b in zip(small, want))
    q = torch.randn((1, H, D), generator=g).half()
    a = rcp.kv8_attn(q.to(DEV), _int([150]).to(DEV), table.to(DEV), codes, scales, vc, vs, 0.09)
    b = rcp.kv8_attn(q.to(DEV), _int([150]).to(DEV), _int([[0, 1]]).to(DEV), *[t.to(DEV) for t in want], 0.09)
    assert torch.equal(a, b)


def test_a_capture_follows_lengths_and_tables():
    """One captured call, replayed on other tokens, lengths and pages, with eager work between the replays."""
    D, page, H = 64, 16, 2
    g, caches = _state(11, 6, H, page, D)
    lengths, table = _int([1, 1]).to(DEV), _int([[0, 1, 2], [3, 4, 5]]).to(DEV)
    k, v, q = (torch.zeros((2, h, D), dtype=torch.float16, device=DEV) for h in (H, H, 4))
    q_out, angles = torch.zeros_like(q), ref.rope_table(3 * page, D).to(DEV)
    dev = [t.to(DEV) for t in caches]
    call = lambda into: rcp.kv8_append(k, v, lengths, table, *into, rope=angles, rotate=True, q=q, q_out=q_out)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call([t.clone() for t in dev])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(dev)
    for n in ([7, 40], [17, 0], [48, 16], [1, 2]):
        other = [t.clone() for t in dev]
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g))
        lengths.copy_(_int(n))
        table.copy_(torch.randperm(6, generator=g).view(2, 3))
        graph.replay()
        torch.cuda.synchronize()
        replayed = q_out.clone()
        q_out.fill_(0)
        call(other)
        torch.cuda.synchronize()
        rows = [b for b in range(2) if n[b] > 0]
        assert torch.equal(replayed[rows], q_out[rows])
        assert all(torch.equal(a.float(), b.float()) for a, b in zip(dev, other))


@pytest.mark.parametrize("change, message", [
    (dict(rope=(47, 64)), "rope must be"), (dict(rope=(48, 32)), "rope must be"), (dict(rope=(48, 64), rope_dtype=torch.float64), "rope must be"),
    (dict(q=(2, 4, 32)), "q"), (dict(q=(3, 4, 64)), "q must be"), (dict(q=(2, 4, 64), q_dtype=torch.bfloat16), "q must be"),
    (dict(q=(2, 4, 64), q_out=(2, 3, 64)), "q_out must be"), (dict(q_out=(2, 4, 64)), "q_out without q"), (dict(k=(2, 2, 32)), "k"), (dict(k=(1, 2, 64)), "as many tokens"),
    (dict(wide=8 + 2), "multiple"), (dict(lengths=(3,)), "lengths"), (dict(table=(1, 3)), "table")])
def test_refusals(change, message):
    caches = [t.to(DEV) for t in _state(15, 6, 2, 16, 64)[1]]
    before = [t.clone() for t in caches]
    made = lambda name, shape, dtype=torch.float16: torch.zeros(change.get(name, shape), dtype=change.get(name + "_dtype", dtype), device=DEV)
    k = made("k", (2, 2, 64))
    if "wide" in change:   # a token stride that is no multiple of 8
        k = torch.zeros((2, 2 * 64 + change["wide"]), dtype=torch.float16, device=DEV)[:, :128].unflatten(1, (2, 64))
    more = {name: made(name, None) for name in ("q", "q_out") if name in change}
    if "rope" in change:
        more["rope"] = made("rope", None, torch.float32)
    with pytest.raises((ValueError, RuntimeError), match=message):
        rcp.kv8_append(k, torch.zeros((2, 2, 64), dtype=torch.float16, device=DEV), made("lengths", (2,), torch.int32), made("table", (2, 3), torch.int32), *caches, **more)
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(caches, before))
