"""Plain 64-bit implementations of the operators around the pages, for tests: from the definitions
in include/prefixplace.h."""

import math

import numpy as np
import torch

from tests.serve_ref import UNIT

E4 = torch.float8_e4m3fn


def frequencies(dim, base=10000.0, factor=1.0, original=0.0, slow=1.0, fast=32.0):
    w = np.array([base ** (-2.0 * i / dim) for i in range(dim // 2)])
    if factor != 1:
        turns = original * w / (2 * math.pi)
        g = np.clip((turns - slow) / (fast - slow), 0, 1) if original else 0 * w
        w = g * w + (1 - g) * w / factor
    return w


def rotary(x, weight, radians, position, first, interleaved, amplitude, eps):
    """(rows, bound of the error before the last rounding) in 64 bits on the CPU.

    The bound, before any run, in units of 2^-24, of what an element is made of:
      - a norm: squares summed in 32 bits, 16 a lane and 6 steps over lanes, (16 + 6) / 2 by the root,
        and a root, a division and two products, 3 more: 15
      - sine and cosine are 4 off (2^-22), times the amplitude, rounded, 1 more; a product and the sum
        of two 2 more: 7, and as much again for frequencies that the host rounds (2^-53 of the angle, which is
        at most 2^31 radians: 2^-22, 4) and for what 64 bits here make of the same: 16
    So 32 of |a| + |b|."""
    x = x.cpu().double()
    if weight is not None:
        n = weight.shape[0]
        y = x[..., :n]
        x = torch.cat([y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.cpu().double(), x[..., n:]], -1)
    size = x.abs()
    if radians is not None and len(radians):
        n = len(radians)
        # whole turns off the angle in long doubles
        angle = position.cpu().numpy().astype(np.longdouble)[:, None] * np.asarray(radians, np.longdouble)
        angle = np.remainder(angle, 2 * np.longdouble("3.14159265358979323846264338327950288"))
        c = torch.from_numpy(np.cos(angle).astype(np.float64) * amplitude)[:, None]
        s = torch.from_numpy(np.sin(angle).astype(np.float64) * amplitude)[:, None]
        at = torch.arange(n)
        ia, ib = (first + 2 * at, first + 2 * at + 1) if interleaved else (first + at, first + n + at)
        a, b = x[..., ia], x[..., ib]
        x, size = x.clone(), size.clone()
        x[..., ia], x[..., ib] = a * c - b * s, a * s + b * c
        size[..., ia] = size[..., ib] = (a.abs() + b.abs()) * abs(amplitude)
    return x, 32 * 2.0 ** -24 * size


def rounded(want, bound, dtype):
    """Bound with the rounding into the type on top."""
    t = bound + UNIT[dtype] * (want.abs() + bound)
    return t + 2.0 ** -25 if dtype == torch.float16 else t


def in_e4m3(want, bound, scale):
    """(value / scale held to the type's range, its bound): half a step is 2^-4 of the value, 2^-10 below the
    normal numbers; the quotient is rounded before, 2^-23 of itself."""
    y = (want / scale).clamp(-448, 448)
    b = bound / scale + 2.0 ** -23 * y.abs()
    return y, b + 2.0 ** -4 * (y.abs() + b) + 2.0 ** -10


def latent(q, cache, block_table, query_start, length, value_dim, *, scale, window=0, k_scale=None):
    """(out, lse, tolerance of out, tolerance of lse) in 64 bits on the CPU.  The tolerances are those of
    tests/serve_ref.py's attend: weights and the output are rounded once to the type, scores are sums of D
    products in 32 bits."""
    T, H, D = q.shape
    page, u = cache.shape[2], UNIT[q.dtype]
    begin, length = query_start.tolist(), length.tolist()
    qd, table = q.cpu().double(), block_table.cpu()
    out = torch.zeros((T, H, value_dim), dtype=torch.float64)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    pages = cache[:, 0].cpu()
    for r, n in enumerate(length):
        new = begin[r + 1] - begin[r]
        if new == 0 or n <= 0:
            continue
        room = min(n, table.shape[1] * page)
        rows = pages[table[r, :-(-room // page)].long().clamp(0, pages.shape[0] - 1)].double().flatten(0, 1)[:room]
        if k_scale is not None:
            rows = rows * k_scale.item()
        for i in range(new):
            pos = n - new + i
            if pos < 0:
                continue
            c = rows[max(0, pos - window + 1) if window else 0:pos + 1]
            if not len(c):
                continue
            x, v = qd[begin[r] + i], c[:, :value_dim]
            s = (x @ c.T) * scale
            m = s.max(1, keepdim=True).values
            dead = m.squeeze(1) == -math.inf
            w = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
            l = w.sum(1, keepdim=True)
            w = w / torch.where(l == 0, torch.ones_like(l), l)
            o = w @ v
            o[dead] = 0
            a = w @ v.abs()
            sure = torch.where(torch.isfinite(c).all(1, keepdim=True), c.abs(), torch.zeros_like(c))
            e = (D + 8) * 2.0 ** -24 * (x.abs() @ sure.T).max(1, keepdim=True).values * abs(scale)
            count = (c.shape[0] + 64) * 2.0 ** -23
            at = begin[r] + i
            out[at] = o
            lse[at] = torch.where(dead, torch.full_like(l, -math.inf).squeeze(1), (m + l.log()).squeeze(1))
            tol[at] = u * (a + o.abs()) + (2 * e + count) * a + 1e-30
            if q.dtype == torch.float16:
                tol[at] += 2.0 ** -24 * v.abs().sum(0)[None, :] + 2.0 ** -25
            tol_lse[at] = e.squeeze(1) + count + 2.0 ** -22 * lse[at].abs().nan_to_num(posinf=0)
    return out, lse, tol, tol_lse


def fork(parent, length, table, free, out_table, page):
    """pp_fork_tables' outputs; out_table is not changed."""
    P, blocks = table.shape
    R = len(parent)
    out = out_table.copy()
    got = dict(out_length=np.zeros(R, np.int32), source=np.full(R, -1, np.int32), target=np.full(R, -1, np.int32),
               tokens=np.zeros(R, np.int32))
    kept, taken = set(), 0
    for r in range(R):
        p = int(parent[r])
        if not 0 <= p < P:
            continue
        n = max(int(length[p]), 0)
        got["out_length"][r] = n
        held = min(-(-n // page), blocks)
        out[r, :held] = table[p, :held]
        last = n // page
        if n % page and last < blocks:
            if p in kept:
                got["source"][r], got["tokens"][r] = table[p, last], n % page
                got["target"][r] = out[r, last] = free[taken] if taken < len(free) else -1
                taken += 1
            kept.add(p)
    return dict(out_table=out, taken=np.array([taken], np.int32), **got)


def free_pages(table, length, n_pages, first, page):
    named = set()
    for r, n in enumerate(length):
        named.update(int(x) for x in table[r, :min(max(-(-int(n) // page), 0), table.shape[1])])
    return np.array([p for p in range(first, n_pages) if p not in named], np.int32)
