"""The plain definitions of oracle/bounded_cache.py against library routines, closed forms and invariants (CPU only)."""
import numpy as np
import pytest
import torch

from cache_util import f64, make_inputs, rule_of, slopes_of
from oracle import bounded_cache as ref
from paper_2402_13485_amd import synth


def case(rng, H, Hk, **kw):
    return make_inputs(rng, "f32", H, Hk, 64, [synth.random_tree(rng, 11), synth.chain_tree(5)], [23, 0], **kw)


def attention(x, rule):
    return ref.grouped_attention(x["n_nodes"], x["parent"], f64(x["q"]), f64(x["k_cache"]), f64(x["v_cache"]), f64(x["k_tree"]), f64(x["v_tree"]),
                                 x["seq_lens"], x["dropped"], x["position"], rule)


def test_attention_without_rule_is_the_tree_attention(oracle):
    x = case(np.random.default_rng(1), 6, 6)
    out = attention(x, rule_of(64))[0]
    want = oracle.tree_attention(x["n_nodes"], x["parent"], x["seq_lens"], x["q"], x["k_cache"], x["v_cache"], x["k_tree"], x["v_tree"], rule_of(64)["scale"])
    for b, T in enumerate(x["n_nodes"]):
        assert np.abs(out[b, :, :T] - want[b, :, :T]).max() < 1e-12


def test_attention_with_rule_is_the_library_attention_with_a_bias():
    """SDPA in float64 on repeated heads, the bias and the mask given as one additive tensor."""
    rng = np.random.default_rng(2)
    H, Hk, L, T = 6, 2, 31, 9
    x = make_inputs(rng, "f32", H, Hk, 64, [synth.chain_tree(T)], [L], placed=True)
    slopes, window = slopes_of(H), 25
    out, lse, _ = attention(x, rule_of(64, window=window, slopes=slopes))
    rep = lambda a: torch.from_numpy(f64(a)).repeat_interleave(H // Hk, 1)
    now = L + int(x["dropped"][0])
    rows = np.concatenate((np.repeat(x["position"], H // Hk, 1)[0], np.broadcast_to(now + np.arange(T), (H, T))), 1).astype(np.int64)
    back = (now + np.arange(T))[None, :, None] - rows[:, None]
    bias = np.where((back >= 0) & (back < window), -slopes[:, None, None] * back, -np.inf)
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(f64(x["q"])), torch.cat((rep(x["k_cache"]), rep(x["k_tree"])), 2),
                                                            torch.cat((rep(x["v_cache"]), rep(x["v_tree"])), 2),
                                                            attn_mask=torch.from_numpy(bias)[None], scale=rule_of(64)["scale"])
    assert np.abs(out - want.numpy()).max() < 1e-6  # the scale is an fp32 number there
    s = torch.from_numpy(f64(x["q"])) @ torch.cat((rep(x["k_cache"]), rep(x["k_tree"])), 2).transpose(-1, -2) * rule_of(64)["scale"]
    assert np.abs(lse - torch.logsumexp(s + torch.from_numpy(bias), -1).numpy()).max() < 1e-12


def test_cap_bounds_scores_and_vanishes_for_large_caps():
    x = case(np.random.default_rng(3), 4, 2, sigma=3.0)
    plain, capped, wide = (attention(x, rule_of(64, cap=c)) for c in (0.0, 2.0, 1e6))
    assert np.nanmax(np.abs(plain[0] - wide[0])) < 1e-9 and np.nanmax(np.abs(plain[0] - capped[0])) > 0.1
    # every score lies within the cap: so does lse less the logarithm of the number of keys
    for b, n in enumerate(x["n_nodes"]):
        keys = np.array([int(x["seq_lens"][b]) + len(ref.root_path(x["parent"][b], i)) for i in range(n)], float)
        assert (np.abs(capped[1][b, :, :n] - np.log(keys)) <= 2.0).all()


@pytest.mark.parametrize("placed", [False, True])
def test_observed_weights_of_a_query_sum_to_one(placed):
    rng = np.random.default_rng(4)
    x = make_inputs(rng, "f32", 6, 2, 64, [synth.chain_tree(6), synth.chain_tree(6)], [17, 9], L_max=20, placed=placed, holes=0.2 if placed else 0.0)
    rule = rule_of(64, cap=20.0, window=12, slopes=slopes_of(6))
    lse = attention(x, rule)[1]
    a, path = np.array([4, 1], np.int32), np.tile(np.arange(6, dtype=np.int32), (2, 1))
    zero = np.zeros((2, 2, 20))
    weight, position, _ = ref.cache_observe(x["n_nodes"], a, path, f64(x["q"]), lse, f64(x["k_cache"]), f64(x["k_tree"]), x["seq_lens"], x["dropped"],
                                            x["position"], zero, rule, 1.0, np.full(zero.shape, np.nan), x["position"])
    # three query heads share a K/V head: each accepted node pays three in all; 17 + 4 rows do not fit 20
    assert abs(np.nansum(weight[1], -1) - 3).max() < 1e-12
    assert (np.nansum(weight[0], -1) < 12).all() and (np.nansum(weight[0], -1) > 9).all()
    assert np.isnan(weight[1, :, 10:]).all()
    if placed:
        assert (position[1, :, 9] == 9 + x["dropped"][1]).all() and (position[0, :, 17:20] == 17 + x["dropped"][0] + np.arange(3)).all()


def test_evict_keeps_the_best_and_moves_the_least():
    rng = np.random.default_rng(5)
    B, Hk, L_max, d, budget = 3, 2, 40, 4, 16
    k, v = (rng.normal(size=(B, Hk, L_max, d)) for _ in range(2))
    lens, dropped = np.array([40, 16, 29], np.int32), np.array([5, 0, 60], np.int32)
    position = np.stack([[rng.permutation(int(n + m))[:L_max] if n + m >= L_max else np.arange(L_max) for _ in range(Hk)]
                         for n, m in zip(lens, dropped)]).astype(np.int32)
    weight = rng.integers(0, 6, (B, Hk, L_max)).astype(np.float32)
    out = dict(position=position.copy(), weight=weight.copy(), seq_lens=lens.copy(), dropped=dropped.copy())
    k2, v2 = k.copy(), v.copy()
    ref.cache_evict(k2, v2, lens, dropped, position, weight, budget, 3, 2, out)
    assert out["seq_lens"].tolist() == [16, 16, 16] and out["dropped"].tolist() == [29, 0, 73]
    assert (k2[1] == k[1]).all() and (out["weight"][1] == weight[1]).all()
    for b in (0, 2):
        now = lens[b] + dropped[b]
        for h in range(Hk):
            p, w = position[b, h, :lens[b]], weight[b, h, :lens[b]]
            safe = (p >= now - 3) | (p < 2)
            order = np.lexsort((np.arange(lens[b]), np.where(safe, 0, -w), ~safe))
            assert sorted(out["position"][b, h, :16]) == sorted(p[order[:16]])
            stay = [j for j in order[:16] if j < 16]
            assert (k2[b, h, stay] == k[b, h, stay]).all() and (out["position"][b, h, stay] == p[stay]).all()
            at = {int(x): j for j, x in enumerate(p)}  # rows, positions and weights moved together
            for j in range(16):
                j0 = at[int(out["position"][b, h, j])]
                assert (k2[b, h, j] == k[b, h, j0]).all() and (v2[b, h, j] == v[b, h, j0]).all() and out["weight"][b, h, j] == w[j0]


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotary_products_depend_on_distances_alone(adjacent):
    rng = np.random.default_rng(6)
    d, pairs = 24, 8
    freq = (100.0 ** (-np.arange(pairs) / pairs)).astype(np.float32)
    x, y = rng.normal(size=(1, 1, 1, d)), rng.normal(size=(1, 1, 1, d))
    turn = lambda a, p, axis_of=None: ref.rotary(a, freq, np.array(p, np.int32).reshape(1, -1, 1), None, axis_of, None, adjacent, np.zeros(a.shape))
    assert abs((turn(x, 7) * turn(y, 3)).sum() - (turn(x, 1004) * turn(y, 1000)).sum()) < 1e-9
    assert (turn(x, 0) == x).all() and abs((turn(x, 55) ** 2).sum() - (x ** 2).sum()) < 1e-9 and (turn(x, 9)[..., 16:] == x[..., 16:]).all()
    axis_of = np.array([0, 0, 1, 1, 1, 2, 2, 2])
    mixed = turn(x, [5, 900, 31], axis_of)
    for c in range(pairs):
        i = [2 * c, 2 * c + 1] if adjacent else [c, c + pairs]
        assert (mixed[..., i] == turn(x, [5, 900, 31][axis_of[c]])[..., i]).all()
