"""Plain forms of the rotary positions, the 4-bit cache and its attention, in 64 bits.

Written from the formulas of include/conduit.h; the tests compare the kernels with these.
"""

import numpy as np
import torch

CLIP = 61440.0


def rotate(x, pos, table, axis, layout="halves", inverse=False):
    """x [..., T, H, d] float64; pos int [A, T]; table [n, pairs, 2]."""
    x = x.double().clone()
    half = len(axis)
    p = torch.arange(half)
    ax = torch.as_tensor(list(axis))
    cs = table.double().cpu()[pos.cpu().long()[ax].T, p].to(x.device)  # [T, pairs, 2]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1] * (-1.0 if inverse else 1.0)
    i1, i2 = (p, p + half) if layout == "halves" else (2 * p, 2 * p + 1)
    i1, i2 = i1.to(x.device), i2.to(x.device)
    a, b = x[..., i1].clone(), x[..., i2].clone()
    x[..., i1] = a * c - b * s
    x[..., i2] = b * c + a * s
    return x


def pack_groups(x):
    """float32 rows [..., d] -> (codes -8..7, s, m as fp16 [..., d/32, 1]): the formula in fp32, one rounding an operation."""
    f = np.float32
    x = np.asarray(x, dtype=f)
    x = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = np.isnan(x).any(-1, keepdims=True)
    x = np.clip(np.where(np.isnan(x), f(0), x), f(-CLIP), f(CLIP))
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    s = ((hi - lo) * f(1 / 15)).astype(np.float16)
    m = (lo + f(8) * s.astype(f)).astype(np.float16)
    sf = s.astype(f)
    inv = np.where(sf > 0, f(1) / np.where(sf > 0, sf, f(1)), f(0)).astype(f)
    c = np.clip(np.rint((x - m.astype(f)) * inv), -8, 7)
    c = np.where(bad, 0, c)
    return c, np.where(bad, np.float16(0), s), np.where(bad, np.float16(np.nan), m)


def values(c, s, m):
    """What packed groups stand for, float64 [..., d]."""
    y = m.astype(np.float64) + s.astype(np.float64) * c
    return y.reshape(*y.shape[:-2], y.shape[-2] * 32)


def page_record(kc, ks, km, vc, vs, vm):
    """The bytes of a page from the groups of its K and V rows [ps, d/32, 32] (codes) and [ps, d/32, 1]."""
    out = []
    for c, lanes, width in ((kc, 4, 8), (vc, 8, 4)):
        ps, groups = c.shape[:2]
        u = (c + 8).astype(np.uint32).reshape(ps, groups, lanes, width)
        word = (u << (4 * np.arange(width, dtype=np.uint32))).sum(-1).astype("<u4" if width == 8 else "<u2")
        out.append(np.ascontiguousarray(word.transpose(0, 2, 1)).tobytes())
    for s, m in ((ks, km), (vs, vm)):
        out.append(np.ascontiguousarray(np.concatenate([s, m], -1)).astype("<f2").tobytes())
    return np.frombuffer(b"".join(out), dtype=np.uint8)


def attend(q, k, v, seen, scale):
    """q [n, H, d], k / v [N, Hkv, d], seen [n] keys a row sees, all float64. Returns out [n, H, d], lse [H, n] and, for
    tolerances, the largest scale sum |q||k| and |v| of what each (row, head) sees."""
    n, H, d = q.shape
    G = H // k.shape[1]
    out, lse = np.zeros((n, H, d)), np.full((H, n), -np.inf)
    reach, big = np.zeros((n, H)), np.zeros((n, H))
    for i in range(n):
        for h in range(H):
            N = int(seen[i])
            if N == 0:
                continue
            kk, vv = k[:N, h // G], v[:N, h // G]
            x = scale * (kk @ q[i, h])
            top = x.max()
            p = np.exp(x - top)
            out[i, h] = p @ vv / p.sum()
            lse[h, i] = top + np.log(p.sum())
            reach[i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max()
            big[i, h] = np.abs(vv).max()
    return out, lse, reach, big
