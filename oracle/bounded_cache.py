"""Plain definitions, in numpy float64, of the calls of a bounded K/V cache with shared heads: grouped attention, the
accepted nodes' attention sums, eviction, rotary positions.  Loops over everything; no code of the library."""
import numpy as np


def root_path(parent, i):
    path = []
    while i >= 0:
        path.append(int(i))
        i = int(parent[i])
    return path[::-1]


def score(q, k, rule, head, back):
    """rule: dict(scale, cap, window, slopes); back = p_i - p_j, an array over the keys of k"""
    s = rule["scale"] * (k @ q)
    if rule["cap"]:
        s = rule["cap"] * np.tanh(s / rule["cap"])
    if rule["slopes"] is not None:
        s = s - float(rule["slopes"][head]) * back
    return s


def in_window(back, rule):
    return back < rule["window"] if rule["window"] else np.ones(back.shape, bool)


def cached_positions(b, hk, L, position, dropped):
    if position is not None:
        return position[b, hk, :L].astype(np.int64)
    return int(dropped[b]) + np.arange(L, dtype=np.int64)


def grouped_attention(n_nodes, parent, q, k_cache, v_cache, k_tree, v_tree, seq_lens, dropped, position, rule):
    """-> out, lse, weighted |V| (what an error of the weights counts against), largest |score| parts; NaN where nothing is written"""
    B, H, T, d = q.shape
    group = H // k_tree.shape[1]
    out, lse, mag = np.full(q.shape, np.nan), np.full((B, H, T), np.nan), np.full(q.shape, np.nan)
    for b in range(B):
        L, now = int(seq_lens[b]), int(seq_lens[b]) + int(dropped[b])
        for h in range(H):
            hk = h // group
            at = cached_positions(b, hk, L, position, dropped)
            for i in range(int(n_nodes[b])):
                path = root_path(parent[b], i)
                p_i = now + len(path) - 1
                back = np.concatenate((p_i - at, len(path) - 1 - np.arange(len(path))))
                seen = in_window(back, rule)
                seen[:L] &= (at >= 0) & (at < now)
                # (only what the node sees is looked at: hidden rows may hold anything)
                k = np.concatenate((k_cache[b, hk, :L], k_tree[b, hk, path]))[seen]
                v = np.concatenate((v_cache[b, hk, :L], v_tree[b, hk, path]))[seen]
                s = score(q[b, h, i], k, rule, h, back[seen])
                m = s.max()
                e = np.exp(s - m)
                out[b, h, i] = e @ v / e.sum()
                with np.errstate(invalid="ignore"):
                    mag[b, h, i] = e @ np.abs(v) / e.sum()
                lse[b, h, i] = m + np.log(e.sum())
    return out, lse, mag


def cache_observe(n_nodes, accept_len, accept_path, q, lse, k_cache, k_tree, seq_lens, dropped, position, weight, rule, decay,
                  weight_out, position_out):
    """-> weight_out, position_out (copies, untouched entries as given), paid"""
    B, H, T, d = q.shape
    Hk, L_max = k_cache.shape[1], k_cache.shape[2]
    group, weight_out, paid_out = H // Hk, weight_out.astype(np.float64), np.zeros(weight_out.shape)
    position_out = None if position is None else position_out.copy()
    for b in range(B):
        L, now, a = int(seq_lens[b]), int(seq_lens[b]) + int(dropped[b]), min(max(int(accept_len[b]), 0), accept_path.shape[1])
        path = [int(x) if 0 <= x < n_nodes[b] else None for x in accept_path[b, :a]]
        for hk in range(Hk):
            at = cached_positions(b, hk, L, position, dropped)
            paid = np.zeros(L + a)
            for r, node in enumerate(path):
                if node is None:
                    continue
                places = [x for x in range(r + 1) if path[x] is not None]
                back = np.concatenate((now + r - at, r - np.array(places)))
                seen = in_window(back, rule)
                seen[:L] &= (at >= 0) & (at < now)
                to = np.concatenate((np.arange(L), L + np.array(places)))[seen]
                k = np.concatenate((k_cache[b, hk, :L], k_tree[b, hk, [path[x] for x in places]]))[seen]
                for h in range(hk * group, (hk + 1) * group):
                    if lse[b, h, node] == -np.inf:  # saw nothing
                        continue
                    paid[to] += np.exp(score(q[b, h, node], k, rule, h, back[seen]) - float(lse[b, h, node]))
            room = min(L + a, L_max)
            weight_out[b, hk, :L] = decay * weight[b, hk, :L].astype(np.float64) + paid[:L]
            weight_out[b, hk, L:room] = paid[L:room]
            paid_out[b, hk, :room] = paid[:room]
            if position is not None:
                position_out[b, hk, :L] = position[b, hk, :L]
                position_out[b, hk, L:room] = [-1 if path[r] is None else now + r for r in range(room - L)]
    return weight_out, position_out, paid_out


def cache_evict(k_cache, v_cache, seq_lens, dropped, position, weight, budget, recent, sinks, out):
    """In place on k_cache and v_cache; out: the four per-row arrays, written where the call writes."""
    B, Hk = k_cache.shape[:2]
    for b in range(B):
        L, now = int(seq_lens[b]), int(seq_lens[b]) + int(dropped[b])
        left = min(L, budget)
        for hk in range(Hk):
            def rank(j):
                p, w = int(position[b, hk, j]), float(weight[b, hk, j])
                if p < 0:
                    return (2, 0.0, j)
                if p >= now - recent or p < sinks:
                    return (0, 0.0, j)
                return (2, 0.0, j) if np.isnan(w) or w == -np.inf else (1, -w, j)
            kept = set(sorted(range(L), key=rank)[:left])
            source = list(range(left))
            moving = iter(sorted(j for j in kept if j >= left))
            for j in range(left):
                if j not in kept:
                    source[j] = next(moving)
            for a in (k_cache, v_cache):
                a[b, hk, :left] = a[b, hk, source].copy()
            out["position"][b, hk, :left] = position[b, hk, source].copy()
            out["weight"][b, hk, :left] = weight[b, hk, source].copy()
        out["seq_lens"][b], out["dropped"][b] = left, int(dropped[b]) + L - left


def rotary(x, inv_freq, offset, start, axis_of, n_rows, adjacent, out):
    """x [B,H,S,d] float64 -> a copy of `out` with the turned rows"""
    out = out.astype(np.float64)
    pairs = len(inv_freq)
    for b in range(x.shape[0]):
        for s in range(int(n_rows[b]) if n_rows is not None else x.shape[2]):
            out[b, :, s] = x[b, :, s]
            for c in range(pairs):
                axis = int(axis_of[c]) if axis_of is not None else 0
                p = int(offset[b, axis, s] if offset.ndim == 3 else offset[b, s]) + (int(start[b, axis]) if start is not None else 0)
                angle = np.longdouble(p) * np.longdouble(inv_freq[c])
                cos, sin = float(np.cos(angle)), float(np.sin(angle))
                i, j = (2 * c, 2 * c + 1) if adjacent else (c, c + pairs)
                out[b, :, s, i] = x[b, :, s, i] * cos - x[b, :, s, j] * sin
                out[b, :, s, j] = x[b, :, s, j] * cos + x[b, :, s, i] * sin
    return out
