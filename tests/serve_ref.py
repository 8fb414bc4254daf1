"""Plain 64-bit implementations of the prefix cache's operators, for tests: request by
request, from the definitions in include/prefixplace.h."""

import math

import numpy as np
import torch

# largest relative error of rounding to nearest: half a unit in the last place
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def tables(leaf, length, cached, parent, slot, free, table, *, page, chunk, n_slots, max_new,
           max_tokens):
    """Returns a dict of pp_block_tables' outputs; `table` is not changed."""
    n, per = len(parent), chunk // page
    table = np.array(table)
    blocks = table.shape[1]
    starts, ends, query_start, taken = [], [], [0], 0
    slot_map = np.full(max_tokens, -1, np.int64)
    position = np.zeros(max_tokens, np.int32)
    for r in range(len(leaf)):
        len_r = max(int(length[r]), 0)
        if cached[r] < 0:
            path, v = [], int(leaf[r]) if 0 <= leaf[r] < n else -1
            while v >= 0:
                path.append(v)
                v = int(parent[v])
            start = 0
            for v in reversed(path):
                if not 0 <= slot[v] < n_slots or start + chunk >= len_r:
                    break
                for j in range(per):
                    if start // page + j < blocks:
                        table[r, start // page + j] = slot[v] * per + j
                start += chunk
        else:
            start = min(int(cached[r]), len_r)
        end = len_r if max_new == 0 else min(len_r, start + max_new)
        for b in range(-(-start // page), -(-end // page)):
            if b < blocks:
                table[r, b] = free[taken] if taken < len(free) else -1
            taken += 1
        for i, pos in enumerate(range(start, end)):
            t = query_start[-1] + i
            if t < max_tokens:
                b = pos // page
                p = int(table[r, b]) if b < blocks else -1
                slot_map[t] = -1 if p < 0 else p * page + pos % page
                position[t] = pos
        starts.append(start)
        ends.append(end)
        query_start.append(query_start[-1] + end - start)
    return dict(block_table=table, query_start=np.array(query_start, np.int32),
                start=np.array(starts, np.int32), end=np.array(ends, np.int32),
                slot_map=slot_map, position=position, taken=np.array([taken], np.int32))


def cache_rows(cache, pages, head, count):
    """Rows 0..count-1 of one request and head, in 64 bits on the CPU."""
    page = cache.shape[2]
    out = [cache[p, head].cpu().to(torch.float64) for p in pages[:-(-count // page)]]
    return torch.cat(out)[:count] if out else torch.zeros((0, cache.shape[3]), dtype=torch.float64)


def attend(q, k_cache, v_cache, block_table, query_start, length, *, scale, window=0,
           k_scale=None, v_scale=None):
    """(out, lse, tolerance of out, tolerance of lse) in 64 bits on the CPU.

    Tolerances, before any run: u is the type's unit roundoff, A = sum_j w_j |v_j| with the exact
    weights, n the keys seen, D the dim.
      - each weight is rounded once to the type: u A (and, in f16, up to 2^-25 where a weight is
        below the normal range: 2^-24 sum_j |v_j| covers it, the largest weight being near 1)
      - the output is rounded once: u |o|
      - a score's 32-bit sum of D products and its scaling are off by up to
        (D + 8) 2^-24 sum_d |q_d k_d| scale =: e, which moves every weight by a factor of e^(+-e),
        the weights and their sum by 2 e A together; the exponential and the 32-bit sums over the
        keys by (n + 64) 2^-23 A more.
    lse moves by e, by the sum's (n + 64) 2^-23 and by its own rounding."""
    T, Hq, D = q.shape
    Hkv, page = k_cache.shape[1], k_cache.shape[2]
    G, u = Hq // Hkv, UNIT[q.dtype]
    begin, length = query_start.tolist(), length.tolist()
    qd = q.cpu().to(torch.float64)
    table = block_table.cpu()
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for r, n in enumerate(length):
        u_r = begin[r + 1] - begin[r]
        if u_r == 0 or n <= 0:
            continue
        for h in range(Hkv):
            k = cache_rows(k_cache, table[r].tolist(), h, n)
            v = cache_rows(v_cache, table[r].tolist(), h, n)
            if k_scale is not None:
                k = k * k_scale[h].item()
                v = v * v_scale[h].item()
            for i in range(u_r):
                pos = n - u_r + i
                if pos < 0:
                    continue
                lo = max(0, pos - window + 1) if window else 0
                kk, vv, x = k[lo:pos + 1], v[lo:pos + 1], qd[begin[r] + i, h * G:(h + 1) * G]
                s = (x @ kk.T) * scale
                m = s.max(1, keepdim=True).values
                dead = m.squeeze(1) == -math.inf
                w = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
                l = w.sum(1, keepdim=True)
                w = w / torch.where(l == 0, torch.ones_like(l), l)
                o = w @ vv
                o[dead] = 0
                a = w @ vv.abs()
                # a key of an infinite element scores -infinity or makes the row NaN: no rounding in it
                sure = torch.where(torch.isfinite(kk).all(1, keepdim=True), kk.abs(), torch.zeros_like(kk))
                e = (D + 8) * 2.0 ** -24 * (x.abs() @ sure.T).max(1, keepdim=True).values * abs(scale)
                count = (kk.shape[0] + 64) * 2.0 ** -23
                t = slice(h * G, (h + 1) * G)
                at = begin[r] + i
                out[at, t] = o
                lse[at, t] = torch.where(dead, torch.full_like(l, -math.inf).squeeze(1), (m + l.log()).squeeze(1))
                tol[at, t] = u * (a + o.abs()) + (2 * e + count) * a + 1e-30
                if q.dtype == torch.float16:
                    tol[at, t] += 2.0 ** -24 * vv.abs().sum(0)[None, :] + 2.0 ** -25
                tol_lse[at, t] = e.squeeze(1) + count + 2.0 ** -22 * lse[at, t].abs().nan_to_num(posinf=0)
    return out, lse, tol, tol_lse
