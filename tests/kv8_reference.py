"""Plain references of the paged 8-bit cache: the append in the written order of its binary32 operations (bit for bit, on the CPU), the attention
in 64 bits."""
import math

import torch

E4M3, TOP = torch.float8_e4m3fn, 448.0


def rope_table(positions, D, base=10000.0):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def turn(x, angles, rotate):
    """One token's heads [H, D] (binary32 on the CPU, every operation rounded on its own); angles [D] or None."""
    D = x.shape[-1]
    if angles is not None:
        a, b, c, s = x[:, :D // 2], x[:, D // 2:], angles[:D // 2], angles[D // 2:]
        x = torch.cat([a * c - b * s, b * c + a * s], 1)
    if rotate:
        stride = 1
        while stride < D:
            v = x.unflatten(1, (-1, 2, stride))
            x = torch.stack([v[:, :, 0] + v[:, :, 1], v[:, :, 0] - v[:, :, 1]], 2).flatten(1)
            stride *= 2
        x = x * torch.tensor(1.0 / math.sqrt(D), dtype=torch.float32)
    return x


def encode(x, scale):
    """Codes of x / scale (a power of two), infinities saturated, NaN as 0."""
    t = (x.double() / scale.double()).clamp(-TOP, TOP)
    return torch.where(t.isnan(), torch.zeros_like(t), t).float().to(E4M3)


def scale_of(top):
    """2^E: the smallest power with top <= 448 * 2^E, E in -40 .. 120."""
    E = -40
    while E < 120 and float(top) > TOP * 2.0 ** E:
        E += 1
    return 2.0 ** E


def runs(B, lengths, starts, rows):
    """(first row, count, position of the first) of each sequence"""
    if starts is None:
        return [(b, 1, lengths[b] - 1) for b in range(B)]
    return [(starts[b], starts[b + 1] - starts[b], lengths[b] - (starts[b + 1] - starts[b])) for b in range(B)]


def append(x, lengths, starts, table, codes, scales, angles=None, rotate=False):
    """x [rows, H, D] (any dtype, CPU) into codes [n, H, page, D] (E4M3) and scales [n, H], in place."""
    n_pages, H, page, D = codes.shape
    raw = codes.view(torch.uint8)
    for b, (first, count, pos0) in enumerate(runs(len(lengths), lengths, starts, x.shape[0])):
        pages = {}
        for i in range(count):
            pos = pos0 + i
            if 0 <= pos < table.shape[1] * page and 0 <= int(table[b, pos // page]) < n_pages:
                y = turn(x[first + i].float(), None if angles is None else angles[pos], rotate)
                pages.setdefault(int(table[b, pos // page]), []).append((pos % page, y))
        for p, new in pages.items():
            for h in range(H):
                block = torch.stack([y[h] for _, y in new])
                mags = block.abs()[block.isfinite()]
                scale = scale_of(mags.max() if mags.numel() else 0.0)
                slot = new[0][0]
                if slot > 0:
                    old = float(scales[p, h])
                    if scale > old:
                        raw[p, h, :slot] = encode(codes[p, h, :slot].float() * old, torch.tensor(scale)).view(torch.uint8)
                    scale = max(scale, old)
                raw[p, h, slot:slot + len(new)] = encode(block, torch.tensor(scale)).view(torch.uint8)
                scales[p, h] = scale


def attention(q, lengths, starts, table, kc, ks, vc, vs, softmax_scale):
    """-> (out in 64 bits, sum_t w_t |V_t|, largest softmax_scale sum_d |q_d K_td|, tokens seen), each per row and head; rows of no sequence: NaN."""
    n_pages, H, page, D = kc.shape
    rows, H_q, _ = q.shape
    rep = H_q // H
    out = torch.full((rows, H_q, D), math.nan, dtype=torch.float64)
    mag, size, seen = torch.zeros_like(out), torch.zeros((rows, H_q, 1), dtype=torch.float64), torch.zeros((rows, H_q, 1), dtype=torch.float64)
    for b, (first, count, pos0) in enumerate(runs(len(lengths), lengths, starts, rows)):
        n = max(0, min(lengths[b], table.shape[1] * page))
        ids = table[b].long().repeat_interleave(page)[:n]
        slots = torch.arange(n) % page
        there = (ids >= 0) & (ids < n_pages)
        at, slots, where = ids[there], slots[there], torch.arange(n)[there]
        for h in range(H):
            K = kc[at, h, slots].double() * ks[at, h].double()[:, None]
            V = vc[at, h, slots].double() * vs[at, h].double()[:, None]
            for i in range(count):
                visible = int((where <= pos0 + i).sum())
                for j in range(h * rep, h * rep + rep):
                    x, k, v = q[first + i, j].double(), K[:visible], V[:visible]
                    w = torch.softmax(softmax_scale * (k @ x), 0)
                    out[first + i, j] = w @ v
                    mag[first + i, j] = w @ v.abs()
                    size[first + i, j] = softmax_scale * (k.abs() @ x.abs()).max() if visible else 0.0
                    seen[first + i, j] = visible
    return out, mag, size, seen
