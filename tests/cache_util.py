"""Inputs of the calls of a bounded cache: host arrays, with NaN wherever nothing may be read."""
import numpy as np

from paper_2402_13485_amd import synth


def rule_of(d, cap=0.0, window=0, slopes=None):
    return dict(scale=float(np.float32(1 / np.sqrt(d))), cap=cap, window=window, slopes=slopes)


def slopes_of(H):
    return (2.0 ** (-1 - 7 * np.arange(H) / H)).astype(np.float32)


def make_inputs(rng, dtype, H, Hk, d, shapes, lens, T_max=None, L_max=None, placed=False, holes=0.0, sigma=1.0):
    """shapes: a tree per sequence.  placed: rows out of order at positions of their own; holes: share of rows without one."""
    B = len(shapes)
    T_max = T_max or max(len(s.parent) for s in shapes)
    L_max = max(lens) if L_max is None else L_max
    n_nodes, parent, _ = synth.pad_trees(shapes, T_max)

    def tensor(*shape, scale=1.0):
        return synth.from_float((rng.normal(size=shape) * scale).astype(np.float32), dtype)
    x = dict(dtype=dtype, n_nodes=n_nodes, parent=parent, q=tensor(B, H, T_max, d, scale=sigma), k_tree=tensor(B, Hk, T_max, d),
             v_tree=tensor(B, Hk, T_max, d), k_cache=tensor(B, Hk, L_max, d), v_cache=tensor(B, Hk, L_max, d),
             seq_lens=np.array(lens, np.int32), dropped=np.zeros(B, np.int32), position=None)
    if placed:
        x["dropped"] = rng.integers(0, 2 * L_max + 2, B).astype(np.int32)
        x["position"] = np.full((B, Hk, L_max), -7, np.int32)
    for b in range(B):
        for name in ("q", "k_tree", "v_tree"):
            poison(x[name], (b, slice(None), slice(int(n_nodes[b]), None)))
        for name in ("k_cache", "v_cache"):
            poison(x[name], (b, slice(None), slice(lens[b], None)))
        for hk in range(Hk if placed else 0):
            at = rng.permutation(lens[b] + int(x["dropped"][b]))[:lens[b]].astype(np.int32)
            hole = rng.random(lens[b]) < holes
            at[hole] = -1 - rng.integers(0, 3, hole.sum())
            x["position"][b, hk, :lens[b]] = at
            poison(x["k_cache"], (b, hk, np.flatnonzero(hole)))
            poison(x["v_cache"], (b, hk, np.flatnonzero(hole)))
    return x


def poison(a, where):
    a[where] = 0x7fc0 if a.dtype == np.uint16 else np.nan


def f64(a):
    return synth.as_float(a).astype(np.float64)


def score_error(x, rule, n_keys_d):
    """A bound of the fp32 error of any score: d products and sums, the scale, the cap, the bias."""
    size = lambda name: np.where(np.isfinite(f64(x[name])), np.abs(f64(x[name])), 0.0)  # rows that count are finite
    q, k = size("q"), max(size(n).max() if x[n].size else 0.0 for n in ("k_cache", "k_tree"))
    u = 2.0 ** -24
    most = rule["scale"] * q.sum(-1).max() * k
    reach = int(x["seq_lens"].max()) + int(x["dropped"].max()) + 128
    if rule["window"]:
        reach = min(reach, rule["window"])
    bias = float(rule["slopes"].max()) * reach if rule["slopes"] is not None else 0.0
    return u * ((n_keys_d + 4) * most + 8 * rule["cap"] + 3 * bias)
