"""The calls of a bounded cache where values, not shapes, are the hard part, against the float64 definitions: weights that must
not lose bits, results near the end of the type's range, values that are not finite, rows that see nothing, lengths outside their range."""
import numpy as np
import pytest
import torch

from cache_util import f64, make_inputs, rule_of, score_error
from gpu_util import sentinel_like, to_dev
from oracle import bounded_cache as ref
from paper_2402_13485_amd import synth
from test_gpu_bounded_cache import RULES, U, dev_tree, make_rule, observe_case, run_attention, run_observe
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
