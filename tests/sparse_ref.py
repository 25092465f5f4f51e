"""Plain implementations, in 64 bits, of rotary positions and block-sparse attention (numpy, host).

TEST INFRASTRUCTURE ONLY: written from the definitions in include/vpp_rope.h and
include/vpp_block_attn.h, without blocking and without the library's code. Each returns, where
the library rounds, what is needed for an elementwise bound on its error.
"""
import math

import numpy as np
import torch

HALF_BF16 = 2.0 ** -8   # a rounding to bf16, relative to the value
HALF_FP32 = 2.0 ** -24


def f64(t):
    return t.detach().double().cpu().numpy()


def rotated(x, positions, freq, offset, interleaved, scale=1.0, inverse=False):
    """Rotated rows [T, H, d] and, for each value, the magnitudes that its rounding errors go by.

    The angle is reduced with 64-bit integers of the position and the frequency's fixed point
    (Python's own, not the library's) so that positions of any size are exact."""
    x = np.asarray(x, dtype=np.float64)
    y, mag = x.copy(), np.zeros_like(x)
    n = len(freq)
    for i, f in enumerate(freq):
        turn = round((f / (2 * math.pi)) * 2 ** 64)
        t = np.array([((int(p) * turn) % 2 ** 64) / 2 ** 64 * 2 * math.pi for p in positions])[:, None]
        c, s = np.cos(t) * scale, np.sin(t) * scale * (-1 if inverse else 1)
        a, b = (offset + 2 * i, offset + 2 * i + 1) if interleaved else (offset + i, offset + n + i)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        mag[..., a] = mag[..., b] = abs(scale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, mag


def rotation_bound(y, mag):
    """One rounding to bf16; cos and sin within 2e-7 (and the angle's last bits); three fp32 roundings."""
    return HALF_BF16 * np.abs(y) + mag * (2.5e-7 + 4 * HALF_FP32)


def grid(x):
    """x [.., d] on the grid of its values (see vpp_block_summarize_paged)."""
    x = np.where(np.isnan(x), 0.0, np.clip(x, -2.0 ** 60, 2.0 ** 60))
    top = np.maximum(np.abs(x).max(-1, keepdims=True), 2.0 ** -55)
    step = np.exp2(np.frexp(top)[1] - 8.0)
    return np.rint(x / step) * step


def summary(keys):
    """Summary of a block of keys [n, d]."""
    with np.errstate(invalid="ignore"):
        return grid(keys.sum(0) / len(keys))


def rows_of(pages, table_row, kv_start, n, page):
    """Cache rows kv_start .. kv_start + n - 1 of a request: [n, ...]."""
    j = kv_start + np.arange(n)
    return pages[table_row[j // page], j % page]


def query_blocks(cu, prefix, size):
    """(first row, rows, segment, position) of each."""
    return [(a, min(size, cu[s + 1] - a), s, prefix[s] + a - cu[s])
            for s in range(len(prefix)) for a in range(cu[s], cu[s + 1], size)]


def selected(q, sums, table, cu, kv_start, prefix, *, hkv, block, size, most, sink, local):
    """Lists [query blocks, hkv, most] from q [T, Hq, d] and summaries [pages, blocks, hkv, d] (fp64)."""
    group = q.shape[1] // hkv
    per = sums.shape[1]
    qb = query_blocks(cu, prefix, size)
    out = np.full((len(qb), hkv, most), -1, dtype=np.int64)
    gq = grid(q)
    for n, (r0, rows, s, pos) in enumerate(qb):
        f, c = pos // block, (pos + rows - 1) // block
        sure = [b for b in range(c + 1) if b < sink or b > f - local]
        rest = [b for b in range(c + 1) if not (b < sink or b > f - local)]
        for h in range(hkv):
            mine = gq[r0:r0 + rows, h * group:(h + 1) * group].reshape(-1, q.shape[2])
            best = rest
            if rest:
                at = kv_start[s] // block + np.array(rest)
                k = sums[table[s][at // per], at % per, h]
                score = (mine @ k.T).max(0)
                order = sorted(range(len(rest)), key=lambda i: (-score[i], rest[i]))
                best = [rest[i] for i in order[:most - len(sure)]]
            got = sorted(sure + best)
            out[n, h, :len(got)] = got
    return out


def attended(q, k_pages, v_pages, table, lists, cu, kv_start, prefix, *, block, size, scale=None):
    """out [T, Hq, dv], lse [Hq, T] and bounds on their errors, for rows of the chunk (fp64 inputs).

    Bounds: a score is a fp32 sum of d products (and one product with the scale): off by at most
    (d + 4) half steps of the sum of their magnitudes; a probability by that much relatively, by
    two steps of exp2 and its rounding to bf16; the sums of n terms by n half steps; out is
    rounded to bf16 once."""
    hq, d = q.shape[1:]
    hkv, dv, page = k_pages.shape[2], v_pages.shape[3], k_pages.shape[1]
    group = hq // hkv
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, bound = np.zeros((q.shape[0], hq, dv)), np.zeros((q.shape[0], hq, dv))
    lse, lse_bound = np.full((hq, q.shape[0]), -np.inf), np.zeros((hq, q.shape[0]))
    for n, (r0, rows, s, pos) in enumerate(query_blocks(cu, prefix, size)):
        for h in range(hq):
            hk = h // group
            at = np.concatenate([np.arange(b * block, (b + 1) * block) for b in lists[n, hk]
                                 if 0 <= b <= (pos + rows - 1) // block] or [np.zeros(0, dtype=np.int64)])
            for t in range(rows):
                j = at[at <= pos + t]
                if not len(j):
                    continue
                c = kv_start[s] + j
                k, v = k_pages[table[s][c // page], c % page, hk], v_pages[table[s][c // page], c % page, hk]
                x = k @ q[r0 + t, h] * scale
                m = x.max()
                w = np.exp(x - m)
                l = w.sum()
                with np.errstate(invalid="ignore"):
                    out[r0 + t, h] = (w[:, None] * v).sum(0) / l
                lse[h, r0 + t] = m + math.log(l)
                off = (d + 4) * HALF_FP32 * (np.abs(k) @ np.abs(q[r0 + t, h])).max() * scale + HALF_FP32 * abs(m) * 4
                off += (len(j) + 8) * HALF_FP32
                lse_bound[h, r0 + t] = 2 * off + 4 * HALF_FP32 * abs(lse[h, r0 + t])
                with np.errstate(invalid="ignore"):
                    away = (w[:, None] * np.abs(v)).sum(0) / l
                bound[r0 + t, h] = HALF_BF16 * np.abs(out[r0 + t, h]) * 1.01 + away * (HALF_BF16 + 4 * off)
    return out, lse, bound, lse_bound


def paged(rng, seg_rows, page, *shapes, extra=3):
    """A block table (pages in random order; entries past a segment's rows: any page) and page pools of
    random bf16 values, one for each shape behind [pages, page]."""
    per = [-(-r // page) for r in seg_rows]
    total = sum(per) + extra
    order = rng.permutation(total).astype(np.int32)
    table = rng.integers(0, total, size=(len(seg_rows), max(per + [1]) + 1)).astype(np.int32)
    at = 0
    for s, n in enumerate(per):
        table[s, :n] = order[at:at + n]
        at += n
    return table, [torch.from_numpy(rng.standard_normal((total, page) + shape).astype(np.float32)).to(torch.bfloat16)
                   for shape in shapes]
