"""What a step of several requests costs in the operators around the quantised products.

Three operators, each through the package's public calls on buffers that a serving program keeps:

  append   new keys and values of one or many requests enter a paged 8-bit cache (E4M3 codes, one power-of-two scale for each
           page and head), with the position rotation of keys and queries, and the Hadamard rotation where it is wanted, on the way
  attn     attention of the new tokens over that cache: one token per request, whole prompts, or a chunk behind a long context
  lowrank  every token's own low-rank adapter beside the shared projection: base + scaling (x A^T) B^T

Head counts, widths and contexts are those of the repository's configurations (LLaMA-3.2-1B-, LLaMA-2-7B- and LLaMA-3-8B-shaped
layers).  Where `own` is false the same results come from elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
E4M3_TOP = 448.0
SCALE_MIN = -40   # the smallest scale of a page is 2^-40
WORKSPACE = 64 << 20   # scratch that a program keeps for its calls on one stream


# ---- the cases ------------------------------------------------------------------------------------
def listed():
    return [
        # one request's new token: latency only (7B heads)
        {"name": "append_one_7b", "kind": "append", "b": 1, "hq": 32, "hkv": 32, "d": 128, "page": 64, "lmin": 1501, "lmax": 1501,
         "nmin": 1, "nmax": 1, "one": True, "rotate": True, "dtype": "f16"},
        # one token each of sixteen requests, keys rotated by the Hadamard matrix as for the 4-bit cache (8B heads)
        {"name": "append_batch16_8b", "kind": "append", "b": 16, "hq": 32, "hkv": 8, "d": 128, "page": 64, "lmin": 300, "lmax": 6000,
         "nmin": 1, "nmax": 1, "one": True, "rotate": True, "dtype": "bf16"},
        # prompts of several requests enter together, some behind a context that is there already
        {"name": "append_prompts_8b", "kind": "append", "b": 7, "hq": 32, "hkv": 8, "d": 128, "page": 32, "lmin": 900, "lmax": 2500,
         "nmin": 77, "nmax": 2001, "one": False, "rotate": False, "dtype": "bf16"},
        # decode of a short context, heads of 64 (1B)
        {"name": "attn_short_1b", "kind": "attn", "b": 1, "hq": 32, "hkv": 8, "d": 64, "page": 16, "lmin": 333, "lmax": 333,
         "nmin": 1, "nmax": 1, "one": True, "dtype": "f16", "out": "f16"},
        # decode of one request, a query head for each cache head, binary32 result as the activation quantiser takes it
        {"name": "attn_step_7b", "kind": "attn", "b": 1, "hq": 32, "hkv": 32, "d": 128, "page": 64, "lmin": 4001, "lmax": 4001,
         "nmin": 1, "nmax": 1, "one": True, "dtype": "f16", "out": "f32"},
        # decode of sixteen requests of very different lengths
        {"name": "attn_batch16_8b", "kind": "attn", "b": 16, "hq": 32, "hkv": 8, "d": 128, "page": 64, "lmin": 300, "lmax": 6000,
         "nmin": 1, "nmax": 1, "one": True, "dtype": "bf16", "out": "bf16"},
        # three requests, a chunk of new tokens each behind a long context, heads of 64
        {"name": "attn_chunk_1b", "kind": "attn", "b": 3, "hq": 32, "hkv": 8, "d": 64, "page": 128, "lmin": 5000, "lmax": 17003,
         "nmin": 5, "nmax": 130, "one": False, "dtype": "f16", "out": "f16"},
        # prompts of several requests, nothing before them
        {"name": "attn_prompts_8b", "kind": "attn", "b": 4, "hq": 32, "hkv": 8, "d": 128, "page": 64, "lmin": 301, "lmax": 2000,
         "nmin": 301, "nmax": 2000, "one": False, "dtype": "bf16", "out": "bf16"},
        # one long prompt: the largest
        {"name": "attn_prompt_long_8b", "kind": "attn", "b": 1, "hq": 32, "hkv": 8, "d": 128, "page": 64, "lmin": 8192, "lmax": 8192,
         "nmin": 8192, "nmax": 8192, "one": False, "dtype": "bf16", "out": "bf16"},
        # one token with one adapter: latency only
        {"name": "lowrank_one_1b", "kind": "lowrank", "m": 1, "n": 2048, "k": 2048, "r": 8, "adapters": 3, "runs": 1, "bare": 0,
         "dtype": "f16", "out": "f16"},
        # sixteen requests with adapters of their own beside the 7B query / key / value projection, two without one
        {"name": "lowrank_batch16_7b", "kind": "lowrank", "m": 16, "n": 12288, "k": 4096, "r": 16, "adapters": 20, "runs": 16,
         "bare": 2, "dtype": "f16", "out": "f16"},
        # prompts of five requests beside the 8B down projection
        {"name": "lowrank_prompts_8b", "kind": "lowrank", "m": 2001, "n": 4096, "k": 14336, "r": 64, "adapters": 8, "runs": 5,
         "bare": 1, "dtype": "bf16", "out": "bf16"},
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "lowrank"])
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    if kind == "lowrank":
        dtype = rng.choice(["f16", "bf16"])
        m = _log(rng, 1, 3000)
        k, n = _log(rng, 1024, 14336, 32), _log(rng, 1024, 22016, 4)
        while m * (n + k) > 2001 * (14336 + 4096):
            m = _log(rng, 1, 3000)
        runs = rng.randint(1, min(m, 16))
        return {"kind": kind, "m": m, "n": n, "k": k, "r": rng.choice([8, 16, 24, 32, 64]), "adapters": rng.randint(1, 20), "runs": runs,
                "bare": rng.randint(0, runs // 2), "dtype": dtype, "out": rng.choice([dtype, "f32"])}
    hkv = rng.choice([2, 4, 8, 16, 32])
    hq = hkv * rng.choice([r for r in (1, 2, 3, 4, 8) if 8 <= hkv * r <= 64])
    d, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
    b = _log(rng, 1, 48)
    case = {"kind": kind, "b": b, "hq": hq, "hkv": hkv, "d": d, "page": page}
    if kind == "append":
        one = rng.random() < 0.5
        nmax = 1 if one else _log(rng, 2, 9000 // b)
        lmin = nmax + _log(rng, 1, 3000)
        return {**case, "lmin": lmin, "lmax": lmin + _log(rng, 1, 2000), "nmin": 1 if one else rng.randint(1, nmax), "nmax": nmax,
                "one": one, "rotate": rng.random() < 0.5, "dtype": dtype}
    if rng.random() < 0.5:   # one token each
        lmax = _log(rng, 100, min(70000, 2_500_000 // (b * hkv)))
        return {**case, "lmin": _log(rng, 1, lmax), "lmax": lmax, "nmin": 1, "nmax": 1, "one": True, "dtype": dtype,
                "out": rng.choice([dtype, "f32"])}
    b = case["b"] = min(b, 8)
    nmax = _log(rng, 2, 4000 // b)
    lmax = nmax + rng.choice([0, _log(rng, 1, 12000 // b)])
    out = dtype if dtype != "f32" else "f32"
    return {**case, "lmin": nmax + rng.randint(0, lmax - nmax), "lmax": lmax, "nmin": rng.randint(1, nmax), "nmax": nmax, "one": False,
            "dtype": dtype, "out": out}


# ---- inputs ---------------------------------------------------------------------------------------
def _spread(lo, hi, b):
    """b whole numbers from lo to hi."""
    return [lo + (hi - lo) * i // (b - 1) if b > 1 else hi for i in range(b)]


def _requests(case, seed):
    """(tokens that each request holds with its new ones, new tokens of each): the same numbers for every seed, in another order."""
    b = case["b"]
    order = torch.randperm(b, generator=torch.Generator().manual_seed(int(seed))).tolist()
    lengths, new = _spread(case["lmin"], case["lmax"], b), _spread(case["nmin"], case["nmax"], b)
    return [lengths[i] for i in order], [min(new[i], lengths[i]) for i in order]


def _cache(g, n_pages, h, page, d):
    """Pages as earlier appends left them: finite codes up to 448 of both signs, a power of two for each page and head."""
    codes = (torch.randn((n_pages, h, page, d), generator=g, device="cuda") * 60).clamp_(-E4M3_TOP, E4M3_TOP).to(torch.float8_e4m3fn)
    octave = torch.randint(-7, -4, (n_pages, h), generator=g, device="cuda")
    return codes, torch.ldexp(torch.ones((), device="cuda"), octave)


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    dtype = DTYPES[case["dtype"]]
    s = {"kind": case["kind"], "work": torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")}
    if case["kind"] == "lowrank":
        m, n, k, r, adapters, runs = (case[x] for x in ("m", "n", "k", "r", "adapters", "runs"))
        x = randn(m, k)
        s["x"] = torch.where(torch.rand((m, k), generator=g, device="cuda") < 0.01, 20 * x, x).to(dtype)
        s["A"] = (randn(adapters, r, k) / math.sqrt(k)).to(dtype)
        s["B"] = (randn(adapters, n, r) * 0.05).to(dtype)
        s["scaling"] = 0.5 + 1.5 * torch.rand((adapters,), generator=g, device="cuda")
        s["base"] = randn(m, n).to(DTYPES[case["out"]])
        s["out"] = torch.empty_like(s["base"])
        # tokens of one request stand together; the first `bare` requests have no adapter
        ids = torch.randperm(max(adapters, runs), generator=g, device="cuda")[:runs].remainder(adapters)
        ids[:case["bare"]] = -1
        order = torch.randperm(runs, generator=g, device="cuda")
        s["which"] = ids[order][torch.arange(m, device="cuda") * runs // m].to(torch.int32)
        return s
    b, hq, hkv, d, page = (case[x] for x in ("b", "hq", "hkv", "d", "page"))
    lengths, new = _requests(case, seed)
    per = -(-max(lengths) // page)
    used = [-(-n // page) for n in lengths]
    n_pages = sum(used) + 3
    ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(int(seed) + 1)).tolist()
    table, at = [], 0
    for u in used:
        table.append(ids[at:at + u] + [-1] * (per - u))
        at += u
    t = sum(new)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s |= {"lengths": _int32(lengths), "table": _int32(table), "starts": None if case["one"] else _int32(starts), "nmax": max(new),
          "seq": torch.repeat_interleave(torch.arange(b, device="cuda"), _int32(new)), "first": _int32(starts[:-1]),
          "new": _int32(new)}
    s["kc"], s["ks"] = _cache(g, n_pages, hkv, page, d)
    s["vc"], s["vs"] = _cache(g, n_pages, hkv, page, d)
    if case["kind"] == "attn":
        s["q"] = (1.5 * randn(t, hq, d)).to(dtype)
        s["scale"] = d ** -0.5
        s["out"] = torch.empty((t, hq, d), dtype=DTYPES[case["out"]], device="cuda")
        return s
    # one projection's output, of which queries, keys and values are views; keys carry a spread and an offset per head
    qkv = randn(t, hq + 2 * hkv, d) * torch.exp(0.4 * randn(hq + 2 * hkv, 1)) + 0.3 * randn(hq + 2 * hkv, 1)
    qkv = qkv.to(dtype)
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    angle = torch.arange(per * page, dtype=torch.float64, device="cuda")[:, None] * \
        torch.pow(500000.0, -torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    s["rope"] = torch.cat([torch.cos(angle), torch.sin(angle)], dim=1).float()
    s["rotate"] = case["rotate"]
    s["q_out"] = torch.empty((t, hq, d), dtype=dtype, device="cuda")
    return s


# ---- one pass -------------------------------------------------------------------------------------
def run(s):
    if own:
        import paper_2502_15779_amd as rcp
        if s["kind"] == "append":
            rcp.kv8_append(s["k"], s["v"], s["lengths"], s["table"], s["kc"], s["ks"], s["vc"], s["vs"], starts=s["starts"],
                           rope=s["rope"], rotate=s["rotate"], q=s["q"], q_out=s["q_out"])
            return [s["kc"], s["ks"], s["vc"], s["vs"], s["q_out"]]
        if s["kind"] == "attn":
            work = s["work"]
            if s["starts"] is not None:   # rows that are split can take more than the scratch: such a call makes its own
                n, hq, d = s["q"].shape
                need = rcp.kv8_workspace_bytes(n, s["lengths"].numel(), hq, s["kc"].shape[1], d, False)
                work = work if need <= work.numel() else None
            return rcp.kv8_attn(s["q"], s["lengths"], s["table"], s["kc"], s["ks"], s["vc"], s["vs"], s["scale"], starts=s["starts"],
                                out=s["out"], workspace=work)
        return rcp.lowrank_add(s["x"], s["A"], s["B"], s["which"], s["scaling"], s["base"], out=s["out"], workspace=s["work"])
    return {"append": _plain_append, "attn": _plain_attn, "lowrank": _plain_lowrank}[s["kind"]](s)


def _butterfly(x, stride):
    v = x.unflatten(-1, (-1, 2, stride))
    return torch.stack([v[..., 0, :] + v[..., 1, :], v[..., 0, :] - v[..., 1, :]], dim=-2).flatten(-3)


def _hadamard(x):
    """The normalised Hadamard transform of the last axis (64 or 128 elements), strides in ascending order."""
    y = _butterfly(_butterfly(_butterfly(_butterfly(_butterfly(_butterfly(x, 1), 2), 4), 8), 16), 32)
    y = _butterfly(y, 64) if x.shape[-1] == 128 else y
    return y * torch.tensor(1.0 / math.sqrt(x.shape[-1]), dtype=x.dtype, device=x.device)


def _position_rotation(x, rows):
    """x [t, h, d] by the angles of rows [t, d] = (cosines, sines): element j with element j + d / 2."""
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    c, s = rows[:, None, :half], rows[:, None, half:]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _plain_write(x, codes, scales, pages, slots):
    """x [t, h, d] into slots of pages; a page that gets its slot 0 starts anew, another one keeps its older codes at the larger scale."""
    n, h, page, d = codes.shape
    at = pages[:, None].expand(-1, h)
    top = torch.zeros((n, h), device=x.device).scatter_reduce_(0, at, x.abs().amax(-1), "amax")
    first = torch.full((n,), page, device=x.device).scatter_reduce_(0, pages, slots, "amin")
    mantissa, exponent = torch.frexp(top)
    octave = torch.where(mantissa <= 0.875, exponent - 9, exponent - 8)
    scale = torch.ldexp(torch.ones((), device=x.device), torch.where(top > 0, octave, SCALE_MIN).clamp(SCALE_MIN, 120))
    grown = torch.where((first > 0)[:, None], torch.maximum(scales, scale), scale)
    touched = torch.unique(pages)
    old = codes[touched].float() * (scales[touched] / grown[touched])[:, :, None, None]
    kept = torch.arange(page, device=x.device) < first[touched][:, None]
    raw = codes.view(torch.uint8)
    raw[touched] = torch.where(kept[:, None, :, None], old.to(torch.float8_e4m3fn).view(torch.uint8), raw[touched])
    scales[touched] = grown[touched]
    raw[pages, :, slots] = (x / scales[pages][:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)


def _places(s, page):
    """Position, page and slot of every new token."""
    i = torch.arange(s["seq"].numel(), device="cuda") - s["first"][s["seq"]]
    pos = (s["lengths"] - s["new"])[s["seq"]] + i
    return pos, s["table"][s["seq"], pos // page].long(), pos % page


def _plain_append(s):
    pos, pages, slots = _places(s, s["kc"].shape[2])
    rows = s["rope"][pos]
    turn = _hadamard if s["rotate"] else (lambda x: x)
    _plain_write(turn(_position_rotation(s["k"].float(), rows)), s["kc"], s["ks"], pages, slots)
    _plain_write(s["v"].float(), s["vc"], s["vs"], pages, slots)
    s["q_out"].copy_(turn(_position_rotation(s["q"].float(), rows)))
    return [s["kc"], s["ks"], s["vc"], s["vs"], s["q_out"]]


def _gathered(codes, scales, table):
    """[b, h, tokens, d] in 32 bits from the pages of each request."""
    at = table.clamp(min=0).long()
    return (codes[at].float() * scales[at][..., None, None]).permute(0, 2, 1, 3, 4).flatten(2, 3)


def _plain_attn(s):
    b, hkv, d = s["lengths"].numel(), s["kc"].shape[1], s["kc"].shape[3]
    t, hq, _ = s["q"].shape
    n = s["nmax"]
    k, v = _gathered(s["kc"], s["ks"], s["table"]), _gathered(s["vc"], s["vs"], s["table"])
    i = torch.arange(t, device="cuda") - s["first"][s["seq"]]
    q = torch.zeros((b, n, hq, d), device="cuda")
    q[s["seq"], i] = s["q"].float()
    q = q.view(b, n, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, n * (hq // hkv), d)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"]).view(b, hkv, n, hq // hkv, -1)
    last = (s["lengths"] - s["new"])[:, None] + torch.arange(n, device="cuda")
    masked = torch.arange(k.shape[2], device="cuda") > last[:, :, None]
    scores.masked_fill_(masked[:, None, :, None, :], -math.inf)
    scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    total = scores.sum(-1, keepdim=True)
    o = torch.matmul(scores.view(b, hkv, n * (hq // hkv), -1), v).view(b, hkv, n, hq // hkv, d) / total
    return o.permute(0, 2, 1, 3, 4).reshape(b, n, hq, d)[s["seq"], i].to(s["out"].dtype)


def _plain_lowrank(s):
    adapters, r, _ = s["A"].shape
    x = s["x"].float()
    chosen = s["which"].long()[:, None] == torch.arange(adapters, device="cuda")
    t = torch.matmul(x, s["A"].float().flatten(0, 1).t()).view(-1, adapters, r)   # every adapter for every token, the others dropped
    t = torch.where(chosen[:, :, None], t * s["scaling"][:, None], 0.0).flatten(1)
    return (s["base"].float() + torch.matmul(t, s["B"].float().transpose(1, 2).reshape(adapters * r, -1))).to(s["base"].dtype)


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    size = {"f16": 2, "bf16": 2, "f32": 4}
    e = size[case["dtype"]]
    if case["kind"] == "lowrank":
        m, n, k, r = case["m"], case["n"], case["k"], case["r"]
        with_one = min(case["runs"] - case["bare"], case["adapters"])
        tokens = sum(1 for i in range(m) if i * case["runs"] // m >= case["bare"])
        return {"bytes": e * (tokens * k + with_one * r * (n + k)) + 2 * size[case["out"]] * m * n, "flops": 2 * tokens * r * (n + k)}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    lengths, new = _requests(case, 0)
    t = sum(new)
    if case["kind"] == "append":
        return {"bytes": t * d * (e * (2 * hq + 2 * hkv) + 2 * hkv + 4), "flops": t * (hq + hkv) * d * (3 + (math.log2(d) if case["rotate"] else 0))}
    seen = sum(sum(range(n - m + 1, n + 1)) for n, m in zip(lengths, new))
    return {"bytes": 2 * hkv * d * sum(lengths) + t * hq * d * (e + size[case["out"]]), "flops": 4 * seen * hq * d}


# ---- the definitions in 64 bits -----------------------------------------------------------------------
def _sylvester(d):
    h = torch.ones((1, 1), dtype=torch.float64, device="cuda")
    while h.shape[0] < d:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h / math.sqrt(d)


def _exact_write(x, codes, scales, b, lengths, new, table, page):
    """The pages after the append, one request and page at a time."""
    values, scales = codes.double(), scales.double()
    at = 0
    for i in range(b):
        pos = lengths[i] - new[i]
        while pos < lengths[i]:
            slot = pos % page
            m = min(page - slot, lengths[i] - pos)
            p = table[i][pos // page]
            y = x[at:at + m].transpose(0, 1)   # [h, m, d]
            top = y.abs().amax((1, 2))
            octave = torch.ceil(torch.log2(torch.where(top > 0, top, 2.0 ** (SCALE_MIN + 8)) / E4M3_TOP)).clamp(SCALE_MIN, 120)
            scale = torch.exp2(octave)
            if slot > 0:
                scale = torch.maximum(scale, scales[p])
                values[p, :, :slot] = (values[p, :, :slot] * (scales[p] / scale)[:, None, None]).to(torch.float8_e4m3fn).double()
            values[p, :, slot:slot + m] = (y / scale[:, None, None]).to(torch.float8_e4m3fn).double()
            scales[p] = scale
            pos += m
            at += m
    return values, scales


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "lowrank":
        out = s["base"].double()
        for a in range(case["adapters"]):
            rows = torch.nonzero(s["which"] == a).flatten()
            if rows.numel():
                out[rows] += s["scaling"][a].double() * (s["x"][rows].double() @ s["A"][a].double().t() @ s["B"][a].double().t())
        return out
    lengths, new = _requests(case, seed)
    table, page, hkv, rep, d = s["table"].tolist(), case["page"], case["hkv"], case["hq"] // case["hkv"], case["d"]
    if case["kind"] == "append":
        pos = torch.cat([torch.arange(n - m, n, device="cuda") for n, m in zip(lengths, new)])
        c, sn = s["rope"].double()[pos].chunk(2, dim=1)
        turn = _sylvester(d) if case["rotate"] else torch.eye(d, dtype=torch.float64, device="cuda")

        def rotated(x):
            a, b = x.double().chunk(2, dim=2)
            return torch.cat([a * c[:, None] - b * sn[:, None], b * c[:, None] + a * sn[:, None]], 2) @ turn

        kc, ks = _exact_write(rotated(s["k"]), s["kc"], s["ks"], case["b"], lengths, new, table, page)
        vc, vs = _exact_write(s["v"].double(), s["vc"], s["vs"], case["b"], lengths, new, table, page)
        return [kc, ks, vc, vs, rotated(s["q"])]
    out, at = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda"), 0
    for i in range(case["b"]):
        p = s["table"][i, :-(-lengths[i] // page)].long()
        hidden = torch.arange(lengths[i], device="cuda") > torch.arange(lengths[i] - new[i], lengths[i], device="cuda")[:, None]
        for h in range(hkv):
            k, v = ((c[p, h].double() * sc[p, h].double()[:, None, None]).flatten(0, 1)[:lengths[i]]
                    for c, sc in ((s["kc"], s["ks"]), (s["vc"], s["vs"])))
            for j in range(h * rep, h * rep + rep):
                w = (s["q"][at:at + new[i], j].double() @ k.t()) * s["scale"]
                w = torch.softmax(w.masked_fill_(hidden, -math.inf), dim=1)
                out[at:at + new[i], j] = w @ v
        at += new[i]
    return out
