"""Plain definitions, in numpy float64, of the calls of a paged K/V cache and of acceptance by sampling: rows in 8 bits, rows in
and out of pages, attention over pages, the accepted path.  Loops over everything; no code of the library."""
import numpy as np

from oracle import bounded_cache

LEAST_POWER, MOST_POWER = -117, 119


def e4m3_values():
    """The value of every code 0..127 (the other half are their negatives); NaN for 127."""
    values = []
    for code in range(128):
        exponent, fraction = code >> 3, code & 7
        values.append(fraction * 2.0 ** -9 if exponent == 0 else (8 + fraction) * 2.0 ** (exponent - 10))
    values[127] = np.nan
    return np.array(values)


VALUES = e4m3_values()


def code_of(x):
    """The code of a float64 value of at most 448: the nearest, ties to the even code."""
    sign = 128 if np.signbit(x) else 0
    distance = np.abs(VALUES[:127] - abs(x))
    nearest = np.flatnonzero(distance == distance.min())
    return sign | int(nearest[0] if len(nearest) == 1 or nearest[0] % 2 == 0 else nearest[1])


def quantise(row):
    """-> codes uint8, scale byte"""
    row = np.asarray(row, np.float64)
    fine = np.isfinite(row)
    most = np.abs(row[fine]).max() if fine.any() else 0.0
    power = LEAST_POWER
    while power < MOST_POWER and most > 448 * 2.0 ** power:
        power += 1
    codes = np.array([code_of(np.clip(x / 2.0 ** power, -448, 448)) if np.isfinite(x) else 127 for x in row], np.uint8)
    return codes, power + 127


def decode(codes, scale_byte):
    """Codes [...,d] and scale bytes [...] as float64 values"""
    codes = np.asarray(codes)
    return np.where(codes >> 7, -1.0, 1.0) * VALUES[codes & 127] * 2.0 ** (np.asarray(scale_byte, np.float64)[..., None] - 127)


def place(table, n_pages, page_rows, b, row):
    """-> page, row in page; page None if there is none"""
    page = int(table[b, row // page_rows])
    return (page if 0 <= page < n_pages else None), row % page_rows


def append(rows, taken, pages, scales, table, seq_lens):
    """Writes, into pages [n_pages,Hk,R,d] (float64 values or, with scales, codes) in place: rows[b,:,i] for the i in taken[b] (None: no row).
    -> new lengths"""
    n_pages, Hk, R, _ = pages.shape
    room, out = table.shape[1] * R, []
    for b, which in enumerate(taken):
        L = min(max(int(seq_lens[b]), 0), room)
        for j, i in enumerate(which[:room - L]):
            page, at = place(table, n_pages, R, b, L + j)
            if page is None or i is None:
                continue
            for h in range(Hk):
                if scales is None:
                    pages[page, h, at] = rows[b, h, i]
                else:
                    pages[page, h, at], scales[page, h, at] = quantise(rows[b, h, i])
        out.append(min(L + len(which), room))
    return np.array(out, np.int32)


def dense(pages, table, seq_lens, L_max):
    """Rows [B,Hk,L_max,d] (zeros where there is no page, NaN behind the sequence), and which have a page [B,L_max]"""
    n_pages, Hk, R, d = pages.shape
    B = len(seq_lens)
    out, there = np.full((B, Hk, L_max, d), np.nan), np.zeros((B, L_max), bool)
    for b in range(B):
        for j in range(min(int(seq_lens[b]), L_max)):
            page, at = place(table, n_pages, R, b, j)
            there[b, j] = page is not None
            out[b, :, j] = 0.0 if page is None else pages[page, :, at]
    return out, there


def attention(n_nodes, parent, q, k_pages, v_pages, table, k_tree, v_tree, seq_lens, rule):
    """-> as bounded_cache.grouped_attention; pages in float64"""
    L_max = max(int(np.max(seq_lens)), 1)
    k, there = dense(k_pages, table, seq_lens, L_max)
    v, _ = dense(v_pages, table, seq_lens, L_max)
    position = np.where(there, np.arange(L_max), -1)[:, None].repeat(k.shape[1], 1)
    return bounded_cache.grouped_attention(n_nodes, parent, q, k, v, k_tree, v_tree, seq_lens, np.zeros(len(seq_lens), np.int64), position, rule)


def softmax(logits, inv_temperature):
    """NaN is -inf; several +inf share; -inf alone: zeros"""
    x = np.where(np.isnan(logits), -np.inf, logits)
    most = x.max()
    if most == -np.inf:
        return np.zeros(x.shape)
    with np.errstate(invalid="ignore"):
        e = np.where(x == most, 1.0, np.exp((x - most) * inv_temperature))
    return e / e.sum()


def accept_sampled(n_nodes, parent, token, logits, inv, draft, draft_inv, u, u_next, path_stride):
    """-> accept_len, accept_path, next_token, and the least distance of a decision or a draw from its border"""
    B, _, V = logits.shape
    lengths, paths, tokens, margin = [], np.full((B, path_stride), -1, np.int32), [], np.inf
    for b in range(B):
        node, path = 0, [0]
        while True:
            target = softmax(logits[b, node].astype(np.float64), inv)
            drawn_from = None if draft is None else softmax(draft[b, node].astype(np.float64), draft_inv)
            left, taken = target.copy(), None  # what is left of the target, as probabilities
            for c in range(node + 1, int(n_nodes[b])):
                if parent[b, c] != node or not 0 <= token[b, c] < V:
                    continue
                t = int(token[b, c])
                have, need = left[t], float(u[b, c]) * (1.0 if drawn_from is None else drawn_from[t])
                if have > 0 or (drawn_from is not None and need > 0):  # (a given candidate without probability is refused without rounding)
                    margin = min(margin, abs(have - need))
                if need < have:
                    taken = c
                    break
                if drawn_from is None:
                    left[t] = 0.0
                else:
                    left = np.maximum(left - drawn_from, 0.0)
                left = left / left.sum() if left.sum() > 0 else left
            if taken is None:
                break
            path.append(taken)
            node = taken
        n = min(len(path), path_stride)
        lengths.append(n)
        paths[b, :n] = path[:n]
        if len(path) > n:
            tokens.append(int(token[b, path[n]]))
        elif left.sum() > 0:
            upto = np.cumsum(left)
            goal = float(u_next[b]) * upto[-1]
            margin = min(margin, np.abs(upto[:-1][left[1:] > 0] - goal).min(initial=np.inf))
            tokens.append(int(np.flatnonzero(upto > goal)[0]))
        else:
            x = np.where(np.isnan(logits[b, node]), -np.inf, logits[b, node])
            tokens.append(int(np.argmax(x)))
    return np.array(lengths, np.int32), paths, np.array(tokens, np.int32), margin
