"""The calls of a bounded cache where values, not shapes, are the hard part, against the float64 definitions: weights that must
not lose bits, results near the end of the type's range, values that are not finite, rows that see nothing, lengths outside their range."""
import numpy as np
import pytest
import torch

from cache_util import f64, make_inputs, rule_of, score_error
from gpu_util import sentinel_like, to_dev, to_host
from oracle import bounded_cache as ref
from paper_2402_13485_amd import synth
from test_gpu_bounded_cache import (RULES, U, check_observe, dev_tree, evict_case, make_rule, observe_case, run_attention,
                                    run_observe)
from test_gpu_marshal import both
from test_gpu_parity import pb  # noqa: F401
from test_gpu_values import timed

pytestmark = pytest.mark.gpu


def weight_step(dtype, d):
    """How far a softmax weight w, 2^e <= w < 2^(e+1), is from the fp32 one where it meets V.  d = 64 multiplies all 24 bits.  d = 128: two bf16
    values.  The first has steps of 2^(e-7) and leaves at most half of one, 2^(e-8).  That value is exact or lies in a binade whose
    steps are 2^(e-16) at most, and is rounded by half of one: 2^(e-17) <= 2^-17 w."""
    return 2.0 ** -17 if dtype == "bf16" and d == 128 else 0.0


def check_exactly(x, rule, out, lse):
    """As check_attention of test_gpu_bounded_cache, with the weights' own step; NaN and the signs of infinities are compared too."""
    d = x["q"].shape[3]
    with np.errstate(invalid="ignore"):
        want, want_lse, mag = ref.grouped_attention(x["n_nodes"], x["parent"], *(f64(x[n]) for n in ("q", "k_cache", "v_cache", "k_tree", "v_tree")),
                                                    x["seq_lens"], x["dropped"], x["position"], rule)
    keys = int(x["seq_lens"].max()) + x["q"].shape[2]
    e = score_error(x, rule, d)
    share = 2 * e + (keys + 16) * U + weight_step(x["dtype"], d)
    for b, T in enumerate(x["n_nodes"]):
        got, r = synth.as_float(out[b, :, :T]).astype(np.float64), want[b, :, :T]
        fine = np.isfinite(r)
        assert (np.isnan(got) == np.isnan(r)).all(), (b, np.argwhere(np.isnan(got) != np.isnan(r))[:5])
        assert (got[~fine & ~np.isnan(r)] == r[~fine & ~np.isnan(r)]).all(), b
        with np.errstate(invalid="ignore"):
            bound = share * mag[b, :, :T] + (2.0 ** -8 if x["dtype"] == "bf16" else U) * np.abs(r) + 1e-37
            assert (np.abs(got - r)[fine] <= bound[fine]).all(), (b, float((np.abs(got - r) / bound)[fine].max()))
        bound = e + (keys + 16) * U + 4 * U * np.abs(want_lse[b, :, :T])
        assert (np.abs(lse[b, :, :T] - want_lse[b, :, :T]) <= bound).all(), (b, float((np.abs(lse[b, :, :T] - want_lse[b, :, :T]) / bound).max()))
        assert (out[b, :, T:] == sentinel_like(x["q"])[b, :, T:]).all() and (lse[b, :, T:] == 12345.5).all()


def by_hand(rng, dtype, H, Hk, d, T, L, score, second, values):
    """Queries (1, 1, 0, ...), so that a cached key's score is the sum of its first two entries (scale 1); T children of the root whose own
    keys weigh next to nothing.  score, second [Hk,L], values [Hk,L,d]."""
    x = make_inputs(rng, dtype, H, Hk, d, [synth.star_tree(T)], [L])
    k, q, kt = np.zeros((1, Hk, L, d), np.float32), np.zeros((1, H, T, d), np.float32), np.zeros((1, Hk, T, d), np.float32)
    k[0, :, :, 0], k[0, :, :, 1] = score, second
    q[..., :2], kt[..., 0] = 1.0, -80.0
    x.update(q=synth.from_float(q, dtype), k_cache=synth.from_float(k, dtype), k_tree=synth.from_float(kt, dtype),
             v_cache=synth.from_float(values[None].astype(np.float32), dtype), v_tree=synth.from_float(np.zeros((1, Hk, T, d), np.float32), dtype))
    return x


def rounded(a):
    return synth.as_float(synth.f32_to_bf16_bits(np.asarray(a, np.float32)))


ONE = dict(scale=1.0, cap=0.0, window=0, slopes=None)


# ---- weights

@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_weights_that_nearly_cancel(pb, d, cut):
    """Two keys per column of V with values +1 and -1 and weights w and w (1 + 2^-11): 2^-11 w is left.  The weights' own roundings count 2^11
    times: exponent (2^-22 of 4 and below), exponential and sums 3e-3 of the result together, and at d = 128 twice the weights' step.
    Then the result is rounded.  cut: one K/V head, whose few stages are cut and merged; otherwise 1200 units."""
    rng = np.random.default_rng(6)
    Hk, L = 1 if cut else 1200, 2 * d + 1
    score, second, v = np.zeros((Hk, L)), np.zeros((Hk, L)), np.zeros((Hk, L, d))
    s = rounded(rng.uniform(-2.0, -0.05, (Hk, d)))
    score[:, 1::2], score[:, 2::2] = s, s
    second[:, 2::2] = 2.0 ** -11
    for i in range(d):
        v[:, 1 + 2 * i, i], v[:, 2 + 2 * i, i] = -1.0, 1.0
    x = by_hand(rng, "bf16", 2 * Hk, Hk, d, 2, L, score, second, v)
    out, _ = run_attention(pb, x, ONE)
    want, _, _ = ref.grouped_attention(x["n_nodes"], x["parent"], *(f64(x[n]) for n in ("q", "k_cache", "v_cache", "k_tree", "v_tree")), x["seq_lens"], x["dropped"],
                                       None, ONE)
    off = np.abs(synth.as_float(out) - want) / np.abs(want)
    assert (off <= 2.0 ** -8 + 3e-3 + 2 * weight_step("bf16", d) * 2.0 ** 11).all(), off.max()


@pytest.mark.parametrize("placed", [False, True])
@pytest.mark.parametrize("name", list(RULES))
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_attention_rounds_once(pb, dtype, d, name, placed):
    """Results are the definition's, rounded once: the weights add next to nothing to that."""
    rng = np.random.default_rng(7)
    x = make_inputs(rng, dtype, 8, 2, d, [synth.random_tree(rng, 40), synth.random_tree(rng, 9)], [300, 77], placed=placed, holes=0.1)
    rule = make_rule(name, 8, d)
    check_exactly(x, rule, *run_attention(pb, x, rule))


@pytest.mark.parametrize("scale", [2.0 ** -130, 2.0 ** -149])
@pytest.mark.parametrize("name", ["plain", "cap", "bias"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_attention_and_sums_with_next_to_no_scale(pb, dtype, d, name, scale):
    """A subnormal scale makes all scores zero, up to the bias."""
    rng = np.random.default_rng(21)
    x = observe_case(rng, dtype, 4, 2, d, [100, 9], [4, 5], T=20, L_max=110, placed=True)
    rule = dict(make_rule(name, 4, d), scale=scale)
    out, lse = run_attention(pb, x, rule)
    check_exactly(x, rule, out, lse)
    x["lse"] = lse
    check_observe(x, rule, 0.5, *run_observe(pb, x, rule, 0.5))


# ---- V

@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("name", ["plain", "cap", "bias"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_attention_values_near_the_largest(pb, dtype, d, name, cut):
    """A maximum that rises after the first rows, and V values within a factor of four of the largest float: weights above 1
    would overflow where the result does not.  cut: two K/V heads whose stages are cut and merged; otherwise 520 units."""
    rng = np.random.default_rng(9)
    Hk, L = 2 if cut else 520, 200
    score = rounded(rng.uniform(-3.0, -1.0, (Hk, L)))
    score[:, 40], score[:, 130] = 3.0, 4.5
    v = rounded(rng.uniform(-1.0, 1.0, (Hk, L, d)))
    v[:, 40], v[:, 130] = 1e38, -5e37
    x = by_hand(rng, dtype, Hk, Hk, d, 2, L, score, np.zeros((Hk, L)), v)
    rule = dict(ONE, cap=30.0 if name == "cap" else 0.0, slopes=np.full(Hk, 2.0 ** -9, np.float32) if name == "bias" else None)
    out, lse = run_attention(pb, x, rule)
    assert np.isfinite(synth.as_float(out[0, :, :2])).all()
    check_exactly(x, rule, out, lse)


# ---- one long sequence among short ones

@pytest.mark.parametrize("B,Hk,T,L,short", [(32, 8, 2, 2100, 40), (32, 16, 2, 2100, 40), (40, 8, 3, 1500, 5), (64, 16, 1, 1900, 33), (70, 16, 2, 1700, 20),
                                            (300, 1, 2, 900, 0), (257, 1, 1, 3000, 31)])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_plans_of_one_long_sequence(pb, d, B, Hk, T, L, short):
    """256 to 1120 units, the last sequence's much longer than the others': cut where ranges leave room for it, or in shares of all
    stages, fewer of them than workgroups where there are few stages."""
    rng = np.random.default_rng(B + L)
    x = make_inputs(rng, "bf16", Hk, Hk, d, [synth.chain_tree(T)] * B, [short] * (B // 2) + [max(0, short - 3)] * (B - B // 2 - 1) + [L])
    rule = rule_of(d)
    check_exactly(x, rule, *run_attention(pb, x, rule))


@pytest.mark.parametrize("B,Hk,group", [(32, 8, 2), (32, 8, 4), (64, 8, 4)])
def test_attention_of_one_long_sequence_takes_no_longer_than_its_rows(pb, B, Hk, group):
    """256, 512 and 1024 units whose stages are nearly all one sequence's, against as many stages in equal sequences: 1.3 to 1.5 times as long
    (3.1 to 7.2 where the long units are not cut)."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    L, T, d = [8192] + [256] * (B - 1), 64, 128
    n_nodes, parent, _ = synth.pad_trees([synth.rank_product_tree(T, 4)] * B, T)
    tree = dev_tree(pb, dict(n_nodes=n_nodes, parent=parent))
    normal = lambda *s: torch.empty(s, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    q, kt, vt, kc, vc = normal(B, Hk * group, T, d), normal(B, Hk, T, d), normal(B, Hk, T, d), normal(B, Hk, max(L), d), normal(B, Hk, max(L), d)
    ws = torch.empty(pb.workspace_bytes(pb.WS_GROUPED_ATTENTION, B, T, Hk * group, d, max(L)), dtype=torch.uint8, device="cuda")
    out, took = torch.empty_like(q), []
    for lens in ([sum(L) // B] * B, L):
        seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):  # the kernels without the host's time
            for _ in range(10):
                pb.propd_grouped_attention(tree, q, kc, vc, kt, vt, seq, 0.09, out=out, workspace=ws)
        graph.replay()
        took.append(timed(graph.replay))
    assert took[1] < 2.3 * took[0], took


def test_attention_of_very_many_sequences(pb):
    """64000 sequences of different lengths: every node sees itself and its rows of ones; it takes about as long as with equal lengths (twenty times
    as long where each search for a unit's sequence starts in front)."""
    B, d, L = 64000, 64, 40
    gen = torch.Generator(device="cuda").manual_seed(20)
    normal = lambda *s: torch.empty(s, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    n_nodes, parent = torch.ones(B, dtype=torch.int32, device="cuda"), torch.full((B, 1), -1, dtype=torch.int32, device="cuda")
    tree = pb.Tree(n_nodes, parent, anc=pb.propd_tree_mask(n_nodes, parent)[1])
    q, kt, vt = normal(B, 1, 1, d), torch.zeros((B, 1, 1, d), device="cuda", dtype=torch.bfloat16), normal(B, 1, 1, d)
    kc, vc = torch.zeros((B, 1, L, d), device="cuda", dtype=torch.bfloat16), torch.ones((B, 1, L, d), device="cuda", dtype=torch.bfloat16)
    took = []
    for seq in (torch.full((B,), 33, device="cuda").int(), torch.randint(0, L + 1, (B,), device="cuda", generator=gen).int()):
        out, lse = torch.zeros_like(q), torch.zeros((B, 1, 1), device="cuda")
        took.append(timed(lambda: pb.propd_grouped_attention(tree, q, kc, vc, kt, vt, seq, 0.125, out=out, lse=lse)))
        n = seq.double()[:, None, None, None]
        want = (vt.double() + n) / (n + 1)  # scores of zero: the mean
        assert bool(((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + 64 * U).all())
        assert bool(((lse.double() - torch.log(n[..., 0] + 1)).abs() <= 16 * U).all())
    assert took[1] < 4 * took[0], took


# ---- sums of attention

@pytest.mark.parametrize("placed", [False, True])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_observe_long_paths_with_steep_slopes(pb, dtype, d, placed):
    """A path of 120 nodes, products of zero: a key pays exp(-slope * distance - lse).  Roundings: slope, its factor log2(e) and the product 3 of the
    distance's part, lse with its own and its factor 3, their difference one of both, the exponential 2, the sum one for every term that is not
    zero (adding zero is exact), the decayed weight 2; none of the root's distance, which is up to 1.4 * 120 in the exponent."""
    rng = np.random.default_rng(12)
    H, Hk, T, L = 4, 2, 120, 60
    x = observe_case(rng, dtype, H, Hk, d, [L, 17], [1, 1], T=T, L_max=L + T, placed=placed, stride=T, holes=0.0)
    x["parent"][:] = np.arange(T) - 1
    x["accept_path"][:], x["accept_len"][:] = np.arange(T), [T, T - 5]
    for name in ("q", "k_cache", "k_tree"):
        x[name] = np.zeros_like(x[name])
    slopes = np.array([0.97, 0.71, 0.33, 0.13], np.float32)
    rule = dict(scale=0.125, cap=0.0, window=0, slopes=slopes)
    _, lse, _ = ref.grouped_attention(x["n_nodes"], x["parent"], *(f64(x[n]) for n in ("q", "k_cache", "k_cache", "k_tree", "k_tree")), x["seq_lens"], x["dropped"],
                                      x["position"], rule)
    x["lse"] = lse.astype(np.float32)
    weight, position = run_observe(pb, x, rule, 1.0)
    want, want_position, _ = ref.cache_observe(x["n_nodes"], x["accept_len"], x["accept_path"], f64(x["q"]), x["lse"], f64(x["k_cache"]), f64(x["k_tree"]),
                                               x["seq_lens"], x["dropped"], x["position"], x["weight"], rule, 1.0, sentinel_like(x["weight"]),
                                               None if x["position"] is None else sentinel_like(x["position"]))
    assert position is None or (position == want_position).all()
    for b, n in enumerate(x["seq_lens"]):
        a, root = int(x["accept_len"][b]), int(x["seq_lens"][b]) + int(x["dropped"][b])
        for hk in range(Hk):
            at = np.concatenate((ref.cached_positions(b, hk, n, x["position"], x["dropped"]), root + np.arange(a))).astype(np.float64)
            bound, total, terms = np.zeros(n + a), np.zeros(n + a), np.zeros(n + a)
            for h in (2 * hk, 2 * hk + 1):
                for r in range(a):
                    bias, y = float(slopes[h]) * (root + r - at), float(x["lse"][b, h, r])
                    paid = np.where(bias >= 0, np.exp(np.minimum(-bias - y, 50.0)), 0.0)
                    bound += paid * U * (4 * bias + 4 * abs(y) + 4)
                    total += paid
                    terms += paid > 0
            bound += terms * U * total
            bound[:n] += 2 * U * np.abs(x["weight"][b, hk, :n])
            off = np.abs(weight[b, hk, :n + a] - want[b, hk, :n + a])
            assert (off <= bound + 1e-30).all(), (b, hk, float((off / (bound + 1e-30)).max()))


# ---- refusals

def test_outputs_and_workspaces_that_overlap_are_refused(pb, monkeypatch):
    """Every output and workspace against every argument that the call reads, by both marshallings; nothing is enqueued, so that the
    inputs stay as they were."""
    rng = np.random.default_rng(13)
    H, Hk, d, T, L = 4, 2, 64, 32, 64  # lse of 2 * 4 * 32 floats
    x = observe_case(rng, "f32", H, Hk, d, [40, 20], [3, 3], T=T, L_max=L)
    names = ("q", "k_cache", "v_cache", "k_tree", "v_tree", "seq_lens", "dropped", "position", "weight", "lse", "accept_len", "accept_path")
    tree, t = dev_tree(pb, x), {n: to_dev(x[n]) for n in names}
    big = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")
    as_f32 = lambda a, shape: a.view(-1).view(torch.float32)[:int(np.prod(shape))].view(shape)
    slopes_at, lse_shape, state = big[4096:].view(torch.float32)[:H], (2, H, T), (2, Hk, L)
    inside = big[:int(np.prod(lse_shape)) * 4 + 4096]  # a piece of `big` that holds slopes_at
    att = lambda **k: lambda: pb.propd_grouped_attention(tree, t["q"], t["k_cache"], t["v_cache"], t["k_tree"], t["v_tree"], t["seq_lens"], 0.125,
                                                         position=t["position"], dropped=t["dropped"], **k)
    rows = pb.CacheRows(*(t[n] for n in ("seq_lens", "dropped", "position", "weight")))
    obs = lambda **k: lambda: pb.propd_cache_observe(tree, t["accept_len"], t["accept_path"], t["q"], t["lse"], t["k_cache"], t["k_tree"], rows, 0.125, **k)
    swap = lambda **k: pb.CacheRows(**{**dict(seq_lens=t["seq_lens"].clone(), dropped=t["dropped"].clone(), position=t["position"].clone(),
                                              weight=t["weight"].clone()), **k})
    evict = lambda k_cache=None, v_cache=None, **k: lambda: pb.propd_cache_evict(t["k_cache"] if k_cache is None else k_cache,
                                                                                 t["v_cache"] if v_cache is None else v_cache, rows, 8, 2, 1, **k)
    inv, offset = torch.ones(32, device="cuda"), torch.zeros((2, T), dtype=torch.int32, device="cuda")
    rot = lambda **k: lambda: pb.propd_rotary(**{**dict(q=t["q"], k=t["k_tree"], inv_freq=inv, offset=offset), **k})
    bad = [att(lse=as_f32(t[n], lse_shape)) for n in ("q", "k_cache", "v_cache", "k_tree", "v_tree", "position")]
    bad += [att(lse=as_f32(inside, lse_shape), slopes=as_f32(inside, lse_shape).view(-1)[8:8 + H]), att(out=as_f32(big, t["q"].shape), slopes=slopes_at),
            att(out=as_f32(big, t["q"].shape), lse=as_f32(big, lse_shape)), att(out=as_f32(big, t["q"].shape), workspace=big),
            att(lse=as_f32(big, lse_shape), workspace=big), att(slopes=slopes_at, workspace=big)]
    bad += [obs(weight_out=as_f32(t[n], state)) for n in ("q", "k_cache", "k_tree", "lse", "position")]
    bad += [obs(position_out=as_f32(t[n], state).view(torch.int32)) for n in ("q", "k_cache", "k_tree", "lse", "weight")]
    both_out = torch.zeros(state, device="cuda")
    bad += [obs(weight_out=both_out, position_out=both_out.view(torch.int32))]
    bad += [evict(rows_out=swap(weight=as_f32(t[n], state))) for n in ("k_cache", "v_cache", "position")]
    bad += [evict(rows_out=swap(position=as_f32(t[n], state).view(torch.int32))) for n in ("k_cache", "v_cache", "weight")]
    bad += [evict(rows_out=swap(seq_lens=t["dropped"])), evict(rows_out=swap(dropped=t["seq_lens"])), evict(k_cache=t["v_cache"]),
            evict(workspace=t["k_cache"]), evict(k_cache=as_f32(big, t["k_cache"].shape), workspace=big)]
    bad += [rot(q_out=as_f32(big, t["q"].shape), inv_freq=big[4096:].view(torch.float32)[:32]),
            rot(q_out=as_f32(big, t["q"].shape), offset=big[4096:].view(torch.int32)[:2 * T].view(2, T)),
            rot(k_out=as_f32(big, t["k_tree"].shape), n_rows=big[4096:].view(torch.int32)[:2])]
    torch.cuda.synchronize()
    before = {n: v.clone() for n, v in t.items()}
    for n, call in enumerate(bad):
        for got in both(pb, monkeypatch, call):
            assert isinstance(got, ValueError) and "overlaps" in str(got), (n, got)
    no_tensor = torch.zeros(1 << 26, dtype=torch.uint8)
    for call in (att(workspace=no_tensor), evict(workspace=no_tensor), att(workspace=torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1 << 26)),
                 lambda: pb.propd_tree_attention(tree, t["q"], *(torch.zeros(2, H, L, d, device="cuda") for _ in "kv"), t["q"], t["q"], t["seq_lens"], 0.125,
                                                 workspace=no_tensor)):
        for got in both(pb, monkeypatch, call):
            assert isinstance(got, TypeError) and "workspace" in str(got), got
    torch.cuda.synchronize()
    assert all(torch.equal(before[n].view(torch.uint8), v.view(torch.uint8)) for n, v in t.items())


def test_attention_f32_takes_the_workspace_it_asked_for(pb):
    """1040 pieces of 32 columns and 1084 tiles, which more ranges would suit than there is room for: a larger workspace makes no
    difference to the results, in no bit."""
    B, H, T, d, L = 16, 26, 80, 128, 17264
    gen = torch.Generator(device="cuda").manual_seed(14)
    n_nodes, parent, _ = synth.pad_trees([synth.chain_tree(T)] * B, T)
    tree = dev_tree(pb, dict(n_nodes=n_nodes, parent=parent))
    normal = lambda *s: torch.empty(s, device="cuda").normal_(generator=gen)
    q, kt, vt, kc, vc = normal(B, H, T, d), normal(B, 1, T, d), normal(B, 1, T, d), normal(B, 1, L, d), normal(B, 1, L, d)
    seq = torch.full((B,), L, dtype=torch.int32, device="cuda")
    nbytes = pb.workspace_bytes(pb.WS_GROUPED_ATTENTION, B, T, H, d, L)
    outs = [pb.propd_grouped_attention(tree, q, kc, vc, kt, vt, seq, 0.09, want_lse=True, workspace=torch.empty(n, dtype=torch.uint8, device="cuda"))
            for n in (nbytes, 2 * nbytes, 4 * nbytes)]
    for out, lse in outs[1:]:
        assert torch.equal(out, outs[0][0]) and torch.equal(lse, outs[0][1])


# ---- values of V that are not finite, rows that see nothing

@pytest.mark.parametrize("Hk,L", [(2, 5), (2, 700), (600, 70)])
@pytest.mark.parametrize("name", ["plain", "all"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_attention_infinities_of_both_signs(pb, dtype, d, name, Hk, L):
    """NaN, +inf and -inf in V, alone in a column and together, in cached rows (the last one too) and in tree rows that some nodes see
    and others do not: every result is the sum of what the node sees.  One range to a unit, several of them, 600 units."""
    rng = np.random.default_rng(15)
    x = make_inputs(rng, dtype, 2 * Hk, Hk, d, [synth.rank_product_tree(40, 4)], [L])
    put = lambda v: synth.from_float(np.array([v], np.float32), dtype)[0]
    for row, column, v in ((L - 1, 2, np.inf), (1, 3, -np.inf), (0, 4, np.inf), (L - 1, 4, -np.inf), (L - 2, 7, np.nan), (L // 2, 8, np.inf), (L // 3, 8, np.inf)):
        x["v_cache"][0, ::2, row, column] = put(v)
    for row, column, v in ((7, 5, np.inf), (39, 5, -np.inf), (12, 6, -np.inf), (1, 9, np.nan), (39, 4, np.inf)):
        x["v_tree"][0, ::2, row, column] = put(v)
    rule = make_rule(name, 2 * Hk, d)
    out, lse = run_attention(pb, x, rule)
    assert np.isposinf(synth.as_float(out)).any() and np.isneginf(synth.as_float(out)).any()
    check_exactly(x, rule, out, lse)


@pytest.mark.parametrize("name", ["plain", "all"])
@pytest.mark.parametrize("Hk,L,placed", [(2, 0, False), (2, 0, True), (2, 700, True), (600, 40, True), (1100, 0, False)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_attention_of_nodes_that_see_nothing(pb, dtype, d, Hk, L, placed, name):
    """Nodes whose set is empty, over an empty cache and over one whose rows have no position (NaN in them): zeros, lse -inf.  The
    other nodes' results are bit for bit those without such nodes.  Whole units, pieces that are merged, fp32 with one range and several."""
    rng = np.random.default_rng(16)
    x = make_inputs(rng, dtype, Hk, Hk, d, [synth.star_tree(37), synth.star_tree(5)], [L, L], L_max=max(L, 1), placed=placed, holes=1.0)
    rule, tree = make_rule(name, Hk, d), dev_tree(pb, x)
    whole = run_attention(pb, x, rule, tree)
    for b, nodes in ((0, [1, 30, 36]), (1, [4])):
        tree.anc[b, nodes] = 0
    out, lse = run_attention(pb, x, rule, tree)
    for b, nodes in ((0, [1, 30, 36]), (1, [4])):
        assert (synth.as_float(out[b][:, nodes]) == 0).all() and (lse[b][:, nodes] == -np.inf).all()
        rest = [i for i in range(37) if i not in nodes]
        assert (out[b][:, rest].view(np.uint8) == whole[0][b][:, rest].view(np.uint8)).all() and (lse[b][:, rest] == whole[1][b][:, rest]).all()


# ---- lengths from device memory, outside their range

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_outside_their_range_are_clamped(pb, dtype):
    """Lengths, numbers of nodes, of dropped positions and of accepted nodes below and above what there is: the results are those of the
    nearest that there is, bit for bit."""
    rng = np.random.default_rng(17)
    H, Hk, d, T, L = 4, 2, 64, 24, 90
    x = observe_case(rng, dtype, H, Hk, d, [L, L, 60, 30], [8] * 4, T=T, L_max=L, placed=True, holes=0.0)
    x["weight"] = np.exp(rng.normal(size=x["weight"].shape)).astype(np.float32)
    wild = dict(seq_lens=[-5, 2 ** 31 - 1, 60, 30], n_nodes=[0, 2 ** 31 - 1, -2 ** 31, 7], dropped=[-1, 40, -2 ** 31, 0], accept_len=[3, -7, 2 ** 31 - 1, 8])
    tame = dict(seq_lens=[0, L, 60, 30], n_nodes=[1, T, 1, 7], dropped=[0, 40, 0, 0], accept_len=[3, 0, 8, 8])
    rule, results = make_rule("all", H, d), []
    for given in (wild, tame):
        y = dict(x, **{n: np.array(v, np.int32) for n, v in given.items()})
        tree = dev_tree(pb, dict(n_nodes=np.array(tame["n_nodes"], np.int32), parent=x["parent"]))
        tree.n_nodes = to_dev(y["n_nodes"])
        got = list(run_attention(pb, y, rule, tree))
        got += run_observe(pb, y, rule, 0.5)
        rows = pb.CacheRows(*(to_dev(y[n]) for n in ("seq_lens", "dropped", "position", "weight")))
        k, v = to_dev(y["k_cache"]), to_dev(x["v_cache"])
        pb.propd_cache_evict(k, v, rows, 40, 5, 1)
        results.append(got + [to_host(t) for t in (k, v, rows.seq_lens, rows.dropped, rows.position, rows.weight)])
    for i, (a, b) in enumerate(zip(*results)):
        # (a sequence of at most `budget` rows keeps its numbers as they are clamped too)
        assert (a.view(np.uint8) == b.view(np.uint8)).all(), i
    assert results[1][6].tolist() == [0, 40, 40, 30] and results[1][7].tolist() == [0, 90, 20, 0]


# ---- eviction with some of the rows' arrays in place

@pytest.mark.parametrize("mine", range(16))
def test_evict_with_some_arrays_in_place(pb, mine):
    """Every choice of the four arrays that are written in place; the others get their entries and nothing else."""
    rng = np.random.default_rng(mine)
    x = evict_case(rng, "bf16", 2, 64, [200, 50, 0, 51], 200, True)
    names = ("seq_lens", "dropped", "position", "weight")
    rows = pb.CacheRows(*(to_dev(x[n]) for n in names))
    out = pb.CacheRows(*(getattr(rows, n) if mine >> i & 1 else to_dev(sentinel_like(x[n])) for i, n in enumerate(names)))
    k, v = to_dev(x["k"]), to_dev(x["v"])
    pb.propd_cache_evict(k, v, rows, 50, 9, 3, rows_out=out)
    want = {n: (x[n] if mine >> i & 1 else sentinel_like(x[n])).copy() for i, n in enumerate(names)}
    k_ref, v_ref = x["k"].copy(), x["v"].copy()
    ref.cache_evict(k_ref, v_ref, x["seq_lens"], x["dropped"], x["position"], x["weight"], 50, 9, 3, want)
    for i, n in enumerate(names):
        assert (to_host(getattr(out, n)).view(np.uint8) == want[n].view(np.uint8)).all(), n
        if not mine >> i & 1:
            assert (to_host(getattr(rows, n)).view(np.uint8) == x[n].view(np.uint8)).all(), n
    assert (to_host(k) == k_ref).all() and (to_host(v) == v_ref).all()


# ---- calls as they are made most: one token for each sequence, a prompt as chains of nodes

@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("name", ["plain", "all"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_one_token_for_each_of_many_sequences(pb, dtype, d, name, ragged):
    rng = np.random.default_rng(18)
    x = make_inputs(rng, dtype, 8, 2, d, [synth.chain_tree(1)] * 32, [900 - (25 * b if ragged else 0) for b in range(32)])
    rule = make_rule(name, 8, d)
    check_exactly(x, rule, *run_attention(pb, x, rule))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_as_chains_of_nodes(pb, dtype):
    """A prompt of 300 rows as three chains: attention, sums and commit of each, whose state then is that of the definitions; its last rows'
    results are those of one causal attention over the whole prompt."""
    rng = np.random.default_rng(19)
    H, Hk, d, n, T = 4, 2, 64, 300, 128
    rule = dict(scale=0.125, cap=0.0, window=0, slopes=None)
    q, k, v = (synth.from_float(rng.normal(size=(1, h, n, d)).astype(np.float32), dtype) for h in (H, Hk, Hk))
    k_dev, v_dev = to_dev(np.zeros_like(k)), to_dev(np.zeros_like(v))
    weight = np.zeros((1, Hk, n), np.float32)
    rows = pb.CacheRows(torch.zeros(1, dtype=torch.int32, device="cuda"), weight=to_dev(weight))
    results = []
    for start in range(0, n, T):
        a = min(T, n - start)
        pad = lambda t: np.ascontiguousarray(np.concatenate((t[:, :, start:start + a], np.zeros((1, t.shape[1], T - a, d), t.dtype)), 2))
        x = dict(dtype=dtype, n_nodes=np.array([a], np.int32), parent=np.concatenate((np.arange(a) - 1, np.full(T - a, -1)))[None].astype(np.int32), q=pad(q),
                 k_tree=pad(k), v_tree=pad(v), k_cache=to_host(k_dev), v_cache=to_host(v_dev), seq_lens=np.array([start], np.int32),
                 dropped=np.zeros(1, np.int32), position=None, accept_len=np.array([a], np.int32), accept_path=np.arange(T, dtype=np.int32)[None], weight=weight)
        out, lse = run_attention(pb, x, rule)
        check_exactly(x, rule, out, lse)
        results.append(out[:, :, :a])
        x["lse"] = lse
        tree, path = dev_tree(pb, x), to_dev(x["accept_path"])
        tree.token = torch.zeros((1, T), dtype=torch.int32, device="cuda")
        pb.propd_cache_observe(tree, to_dev(x["accept_len"]), path, to_dev(x["q"]), to_dev(lse), k_dev, to_dev(x["k_tree"]), rows, rule["scale"])
        check_observe(x, rule, 1.0, to_host(rows.weight), None, weight)
        weight = to_host(rows.weight)
        pb.propd_commit_path(tree, to_dev(x["accept_len"]), path, torch.zeros(1, dtype=torch.int32, device="cuda"), to_dev(x["k_tree"]), to_dev(x["v_tree"]),
                             k_dev, v_dev, rows.seq_lens)
    assert rows.seq_lens.tolist() == [n] and (to_host(k_dev) == k).all() and (to_host(v_dev) == v).all()
    assert abs(weight.sum() - H * n) < 1e-3 * H * n  # every query's weights sum to one
    s = np.einsum("hid,hjd->hij", f64(q)[0], np.repeat(f64(k)[0], 2, axis=0)) * rule["scale"]
    s[:, np.triu(np.ones((n, n), bool), 1)] = -np.inf
    p = np.exp(s - s.max(-1, keepdims=True))
    want = p @ np.repeat(f64(v)[0], 2, axis=0) / p.sum(-1, keepdims=True)
    off = np.abs(synth.as_float(np.concatenate(results, 2))[0] - want)
    assert (off <= (2.0 ** -8 if dtype == "bf16" else U) * np.abs(want) + 1e-4).all(), off.max()
