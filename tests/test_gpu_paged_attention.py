"""Attention over a paged cache on the GPU against the float64 definition of oracle/paged_cache.py.

Tolerances.  A score is off by at most `score_error` (products, sums, cap and bias in fp32), a softmax weight by that and a few units
of 2^-24 relative, a weight of two bf16 values by 2^-17 more, a sum of n by n * 2^-24; what an error of the weights counts against is
sum_j p_j |v_j|.  A bf16 result is rounded by half a step (2^-8) at the end.  Rows in 8 bits are exact as values."""
import numpy as np
import pytest
import torch

from cache_util import f64, poison, rule_of, score_error, slopes_of
from gpu_util import sentinel_like, to_dev, to_host
from oracle import paged_cache as ref
from paged_util import dev_cache, make_case
from paper_2402_13485_amd import synth
from test_gpu_bounded_cache import RULES, dev_rule, dev_tree, make_rule
from test_gpu_parity import pb  # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)]


def run_attention(pb, x, rule, cache=None, tree=None, **kw):
    out, lse = to_dev(sentinel_like(x["q"])), to_dev(sentinel_like(np.zeros(x["q"].shape[:3], np.float32)))
    pb.propd_paged_attention(tree or dev_tree(pb, x), to_dev(x["q"]), cache or dev_cache(pb, x), *(to_dev(x[n]) for n in ("k_tree", "v_tree", "seq_lens")),
                             out=out, lse=lse, **dev_rule(rule), **kw)
    torch.cuda.synchronize()
    return to_host(out), to_host(lse)


def check_attention(x, rule, out, lse):
    with np.errstate(invalid="ignore"):
        want, want_lse, mag = ref.attention(x["n_nodes"], x["parent"], f64(x["q"]), x["k64"], x["v64"], x["page_table"], f64(x["k_tree"]), f64(x["v_tree"]),
                                            x["seq_lens"], rule)
    bf16, d = x["dtype"] == "bf16", x["q"].shape[3]
    keys = int(x["seq_lens"].max()) + x["q"].shape[2]
    largest = max(np.abs(a[np.isfinite(a)]).max(initial=0.0) for a in (x["k64"], f64(x["k_tree"])))
    e = score_error({**x, "k_cache": np.full(1, largest, np.float32), "dropped": np.zeros(1)}, rule, d)
    share = 2 * e + (keys + 16) * U + (2.0 ** -17 if bf16 else 0.0)
    for b, T in enumerate(x["n_nodes"]):
        got, r = synth.as_float(out[b, :, :T]).astype(np.float64), want[b, :, :T]
        fine = np.isfinite(r)
        assert (np.isfinite(got) == fine).all(), (b, np.argwhere(np.isfinite(got) != fine)[:5])
        assert ((got == r) | (np.isnan(got) & np.isnan(r)))[~fine].all(), b
        with np.errstate(invalid="ignore"):
            bound = share * mag[b, :, :T] + (2.0 ** -8 if bf16 else U) * np.abs(r) + 1e-37
            assert (np.abs(got - r)[fine] <= bound[fine]).all(), float((np.abs(got - r) / bound)[fine].max())
        bound = e + (keys + 16) * U + 4 * U * np.abs(want_lse[b, :, :T])
        assert (np.abs(lse[b, :, :T] - want_lse[b, :, :T]) <= bound).all(), float((np.abs(lse[b, :, :T] - want_lse[b, :, :T]) / bound).max())
        assert (out[b, :, T:] == sentinel_like(x["q"])[b, :, T:]).all() and (lse[b, :, T:] == 12345.5).all()


@pytest.mark.parametrize("name", list(RULES))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,codes", TYPES)
def test_rules(pb, dtype, codes, d, name):
    """Every rule: ragged lengths, an empty cache, a tree of one node, NaN in padding, behind sequences and in pages of nobody."""
    rng = np.random.default_rng(len(name) + d + codes)
    shapes = [synth.random_tree(rng, 45), synth.chain_tree(1), synth.rank_product_tree(20, 4), synth.random_tree(rng, 13)]
    x = make_case(rng, dtype, codes, 6, 2, d, shapes, [131, 64, 0, 33], 16, T_max=47)
    rule = make_rule(name, 6, d)
    check_attention(x, rule, *run_attention(pb, x, rule))


@pytest.mark.parametrize("H,Hk,T,L,R", [(1, 1, 1, 0, 16), (1, 1, 1, 1, 16), (8, 8, 3, 31, 32), (8, 1, 1, 700, 64), (40, 8, 1, 97, 16), (5, 1, 128, 64, 64), (16, 2, 128, 95, 16),
                                        (64, 2, 16, 40, 32), (3, 3, 128, 32, 1024), (8, 4, 64, 1100, 256), (16, 1, 1, 300, 16), (17, 1, 1, 300, 16), (8, 2, 16, 513, 128),
                                        (65, 1, 1, 40, 16), (13, 13, 5, 129, 16)])
@pytest.mark.parametrize("dtype,codes", TYPES)
def test_heads_lengths_and_pages(pb, dtype, codes, H, Hk, T, L, R):
    """One column to several blocks of 128 (every shape of the waves), one key to many ranges, pages that end inside a stage and that hold many."""
    rng = np.random.default_rng(H + T + L)
    x = make_case(rng, dtype, codes, H, Hk, 128, [synth.random_tree(rng, T)], [L], R)
    check_attention(x, rule_of(128), *run_attention(pb, x, rule_of(128)))


@pytest.mark.parametrize("L", [15, 16, 17, 31, 32, 33, 127, 128, 129])
@pytest.mark.parametrize("dtype,codes,T", [("bf16", False, 1), ("bf16", True, 1), ("bf16", True, 9), ("f32", False, 40)])
def test_edges_of_stages(pb, dtype, codes, T, L):
    rng = np.random.default_rng(L)
    x = make_case(rng, dtype, codes, 4, 2, 64, [synth.chain_tree(T), synth.chain_tree(T)], [L, max(L - 16, 0)], 16)
    check_attention(x, rule_of(64), *run_attention(pb, x, rule_of(64)))


@pytest.mark.parametrize("B", [65, 130])
@pytest.mark.parametrize("dtype,codes", TYPES)
def test_many_sequences(pb, dtype, codes, B):
    rng = np.random.default_rng(B)
    shapes = [synth.random_tree(rng, int(rng.integers(1, 9))) for _ in range(B)]
    x = make_case(rng, dtype, codes, 4, 2, 64, shapes, rng.integers(0, 90, B).tolist(), 16)
    rule = make_rule("all", 4, 64)
    check_attention(x, rule, *run_attention(pb, x, rule))


@pytest.mark.parametrize("B,Hk,L,ragged", [(43, 16, 230, True), (38, 16, 200, False), (66, 16, 70, True), (130, 16, 40, True), (9, 2, 1300, True), (3, 1, 2600, True),
                                           (1, 1, 4000, False)])
@pytest.mark.parametrize("T,codes,d", [(2, True, 64), (2, False, 128), (33, True, 128)])
def test_plans(pb, T, codes, d, B, Hk, L, ragged):
    """Units cut to run all at once, more units than that, units that are not cut (1056 and 2080), one long sequence; few columns and many."""
    if T > 2 and B * Hk > 600:
        B, Hk = B // 4, Hk // 4
    rng = np.random.default_rng(B + L)
    H = 4 * Hk if T > 2 else Hk
    if T > 2 and B * H * T > 3000:
        B, Hk, H = 3, 2, 8
    x = make_case(rng, "bf16", codes, H, Hk, d, [synth.chain_tree(T)] * B, [L - (L * (b % 7)) // 9 if ragged else L for b in range(B)], 32)
    check_attention(x, rule_of(d), *run_attention(pb, x, rule_of(d)))


def test_one_long_sequence_among_short_ones(pb):
    rng = np.random.default_rng(11)
    x = make_case(rng, "bf16", True, 8, 8, 64, [synth.chain_tree(1)] * 31, [9000] + [20 + b for b in range(30)], 64)
    check_attention(x, rule_of(64), *run_attention(pb, x, rule_of(64)))


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 200])
@pytest.mark.parametrize("dtype,codes", TYPES)
def test_window_edges(pb, dtype, codes, window):
    """Windows that end on, before and behind a stage's edge, shorter than the tree is deep, longer than everything."""
    rng = np.random.default_rng(window)
    x = make_case(rng, dtype, codes, 4, 2, 128, [synth.chain_tree(40), synth.random_tree(rng, 40), synth.chain_tree(1)], [130, 17, 99], 16)
    rule = rule_of(128, window=window)
    check_attention(x, rule, *run_attention(pb, x, rule))


@pytest.mark.parametrize("dtype,codes", TYPES)
@pytest.mark.parametrize("T", [1, 30])
def test_entries_that_are_no_pages(pb, dtype, codes, T):
    """Rows there are seen by nobody: negative, one behind the last, far away; a whole sequence without pages."""
    rng = np.random.default_rng(T)
    x = make_case(rng, dtype, codes, 4, 2, 64, [synth.random_tree(rng, T)] * 3, [150, 64, 40], 16)
    n = x["k_pages"].shape[0]
    x["page_table"][0, [1, 4, 9]] = [-1, n, 2 ** 31 - 1]
    x["page_table"][1] = -2 ** 31
    check_attention(x, rule_of(64), *run_attention(pb, x, rule_of(64)))


@pytest.mark.parametrize("dtype,codes", TYPES)
def test_pages_shared_by_sequences(pb, dtype, codes):
    """A common prefix of three pages."""
    rng = np.random.default_rng(5)
    x = make_case(rng, dtype, codes, 4, 2, 128, [synth.random_tree(rng, 7)] * 3, [100, 61, 48], 16)
    x["page_table"][1:, :3] = x["page_table"][0, :3]
    check_attention(x, rule_of(128), *run_attention(pb, x, rule_of(128)))


@pytest.mark.parametrize("where", ["page", "window", "stranger"])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("dtype,codes,T", [("bf16", False, 40), ("bf16", True, 5), ("f32", False, 40), ("f32", True, 5), ("bf16", True, 40)])
def test_values_that_are_not_finite(pb, dtype, codes, T, value, where):
    """In V of a cached row all see, of one that a window hides from some, of a node that is an ancestor of some only."""
    if codes and where != "stranger" and not np.isnan(value):
        pytest.skip("8-bit rows have no infinities")
    rng = np.random.default_rng(T)
    x = make_case(rng, dtype, codes, 4, 2, 128, [synth.random_tree(rng, T)] * 2, [90, 70], 16)
    rule = rule_of(128, window=60 if where == "window" else 0)
    if where == "stranger":
        x["v_tree"] = np.array(x["v_tree"])
        x["v_tree"][0, 1, T // 2, 5] = synth.from_float(np.array([value], np.float32), dtype)[0]
    else:
        row = 90 - 60 + 2 if where == "window" else 37
        page, at = x["page_table"][0, row // 16], row % 16
        if codes:
            x["v_pages"][page, 1, at, 5] = 0x7f
        else:
            x["v_pages"][page, 1, at, 5] = synth.from_float(np.array([value], np.float32), dtype)[0]
        x["v64"][page, 1, at, 5] = value
    check_attention(x, rule, *run_attention(pb, x, rule))


def test_nan_of_a_hidden_row_of_k(pb):
    rng = np.random.default_rng(8)
    x = make_case(rng, "bf16", False, 4, 2, 64, [synth.star_tree(9)] * 2, [50, 70], 16)
    poison(x["k_tree"], (0, 0, 3))
    rule = rule_of(64)
    out, lse = run_attention(pb, x, rule)
    assert np.isnan(synth.as_float(out[0, :2, 3])).all() and np.isnan(lse[0, :2, 3]).all()
    # every other row as if the node's row held zeros (two heads' results of the node itself are not there to compare)
    clean = dict(x, k_tree=np.array(x["k_tree"]))
    clean["k_tree"][0, 0, 3] = 0
    want, want_lse = run_attention(pb, clean, rule)
    out[0, :2, 3], lse[0, :2, 3] = want[0, :2, 3], want_lse[0, :2, 3]
    check_attention(clean, rule, out, lse)


@pytest.mark.parametrize("dtype,codes", TYPES)
def test_rows_that_see_nothing(pb, dtype, codes):
    """Sets without the node itself over an empty cache: zeros, lse -inf."""
    rng = np.random.default_rng(9)
    x = make_case(rng, dtype, codes, 4, 2, 64, [synth.chain_tree(3)] * 2, [0, 20], 16)
    tree = dev_tree(pb, x)
    tree.anc[:, 1] = 0
    out, lse = run_attention(pb, x, rule_of(64), tree=tree)
    assert (synth.as_float(out[0, :, 1]) == 0).all() and (lse[0, :, 1] == -np.inf).all()
    assert np.isfinite(synth.as_float(out[1, :, 1])).all() and np.isfinite(lse[1]).all() and np.isfinite(lse[0, :, [0, 2]]).all()


@pytest.mark.parametrize("dtype,codes", TYPES)
def test_moving_maximum(pb, dtype, codes):
    """Scores that grow by hundreds over the rows, and that fall: the reference moves at every stage, or never."""
    rng = np.random.default_rng(10)
    for rising in (True, False):
        x = make_case(rng, dtype, codes, 2, 1, 64, [synth.chain_tree(2)], [200], 16)
        for j in range(200):
            page, at = x["page_table"][0, j // 16], j % 16
            s = 4.0 * ((j if rising else 200 - j) // 8) / 8
            if codes:
                x["k_pages"][page, 0, at], x["k_scale"][page, 0, at] = ref.quantise(np.full(64, s))
                x["k64"][page, 0, at] = ref.decode(x["k_pages"][page, 0, at][None], x["k_scale"][page, 0, at][None])[0]
            else:
                x["k_pages"][page, 0, at] = synth.from_float(np.full(64, s, np.float32), dtype)
                x["k64"][page, 0, at] = s
        x["q"][...] = synth.from_float(np.full(x["q"].shape, 3.0, np.float32), dtype)
        check_attention(x, rule_of(64), *run_attention(pb, x, rule_of(64)))


def test_large_values_stay_finite(pb):
    """Values of V near the largest number, with weights that exceed 1 before the reference moves."""
    rng = np.random.default_rng(12)
    for dtype in ("bf16", "f32"):
        x = make_case(rng, dtype, False, 2, 1, 64, [synth.chain_tree(2)], [150], 16)
        big = synth.as_float(x["v_pages"]) * np.float32(5e37)
        x["v_pages"] = synth.from_float(big, dtype)
        x["v64"] = f64(x["v_pages"])
        x["v_tree"][...] = synth.from_float(np.full(x["v_tree"].shape, 1e38, np.float32), dtype)
        check_attention(x, rule_of(64), *run_attention(pb, x, rule_of(64)))


@pytest.mark.parametrize("T,codes", [(1, True), (1, False), (20, True), (64, False)])
def test_lengths_out_of_range_and_a_dirty_workspace(pb, T, codes):
    """Lengths beyond the table and below zero are clamped; what a workspace holds does not matter, and padding columns are not there."""
    rng = np.random.default_rng(13)
    x = make_case(rng, "bf16", codes, 4, 2, 64, [synth.random_tree(rng, T)] * 3, [96, 96, 50], 32)
    good = run_attention(pb, dict(x, seq_lens=np.array([96, 0, 50], np.int32)), rule_of(64))
    ws = torch.full((pb.workspace_bytes(pb.WS_PAGED_ATTENTION, 3, T, 4, 64, 96),), 0xff, dtype=torch.uint8, device="cuda")
    got = run_attention(pb, dict(x, seq_lens=np.array([2 ** 31 - 1, -5, 50], np.int32)), rule_of(64), workspace=ws)
    for a, b in zip(good, got):
        assert np.array_equal(a, b)


def test_pool_beyond_32_bits(pb):
    """The last pages of a pool of 9 GB of K and of V, fp32 and 8 bits, against the same rows in a small pool."""
    for dtype in (torch.float32, torch.float8_e4m3fn):
        R, Hk, d = 1024, 8, 128
        n_pages = (9 << 30) // (R * Hk * d * (4 if dtype == torch.float32 else 1)) + 2
        pages = [torch.empty((n_pages, Hk, R, d), dtype=dtype, device="cuda") for _ in range(2)]
        gen = torch.Generator(device="cuda").manual_seed(3)
        table = torch.tensor([[n_pages - 1, n_pages - 3]], dtype=torch.int32, device="cuda")
        scale = None if dtype == torch.float32 else torch.full((n_pages, Hk, R), 121, dtype=torch.uint8, device="cuda")
        for x in pages:
            x[table[0].long()] = torch.randn((2, Hk, R, d), generator=gen, device="cuda").mul(1 if scale is None else 64).to(dtype)
        few = [x[table[0].long()].clone() for x in pages]
        small = pb.PagedCache(*few, torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), *(() if scale is None else (scale[:2].clone(), scale[:2].clone())))
        large = pb.PagedCache(*pages, table, *(() if scale is None else (scale, scale.clone())))
        one = torch.ones(1, dtype=torch.int32, device="cuda")
        parent = torch.full((1, 1), -1, dtype=torch.int32, device="cuda")
        tree = pb.Tree(one, parent, anc=pb.propd_tree_mask(one, parent)[1])
        q, kt, vt = (torch.randn((1, h, 1, d), generator=gen, device="cuda") for h in (16, 8, 8))
        lens = torch.tensor([1900], dtype=torch.int32, device="cuda")
        got, want = (pb.propd_paged_attention(tree, q, c, kt, vt, lens, 0.09) for c in (large, small))
        assert torch.equal(got, want) and bool(got.isfinite().all())
        del pages, few, small, large, scale
        torch.cuda.empty_cache()


def test_other_streams_and_a_captured_graph(pb):
    """On a stream of its own, and replayed from a graph with eager work between the replays: the same bits every time."""
    rng = np.random.default_rng(15)
    for T, dtype, codes in ((1, "bf16", True), (24, "bf16", False), (40, "f32", True)):
        x = make_case(rng, dtype, codes, 4, 2, 64, [synth.random_tree(rng, T)] * 2, [900, 333], 16)
        tree, cache = dev_tree(pb, x), dev_cache(pb, x)
        q, kt, vt, lens = (to_dev(x[n]) for n in ("q", "k_tree", "v_tree", "seq_lens"))
        ws = torch.empty(pb.workspace_bytes(pb.WS_PAGED_ATTENTION, 2, T, 4, 64, cache.capacity), dtype=torch.uint8, device="cuda")
        out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
        call = lambda: pb.propd_paged_attention(tree, q, cache, kt, vt, lens, 0.125, out=out, lse=lse, workspace=ws)
        call()
        torch.cuda.synchronize()
        want = out.clone(), lse.clone()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            out.zero_()
            call()
        side.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for n in range(4):
            out.zero_(), lse.zero_()
            lens.copy_(to_dev(np.array([900 - 100 * n, 333], np.int32)))
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone(), lse.clone()
            call()
            torch.cuda.synchronize()
            assert torch.equal(got[0], out) and torch.equal(got[1], lse)
            if n == 0:
                assert torch.equal(got[0], want[0])


def test_dense_and_paged_caches_agree(pb):
    """The same rows in a dense cache: the results of propd_grouped_attention within both calls' rounding."""
    rng = np.random.default_rng(16)
    for T in (1, 30, 128):
        x = make_case(rng, "bf16", False, 8, 2, 128, [synth.random_tree(rng, T)] * 2, [700, 301], 64)
        tree, cache = dev_tree(pb, x), dev_cache(pb, x)
        q, kt, vt, lens = (to_dev(x[n]) for n in ("q", "k_tree", "v_tree", "seq_lens"))
        k, v = (torch.zeros((2, 2, 700, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        pb.propd_paged_read(cache, lens, k, v)
        a, al = pb.propd_paged_attention(tree, q, cache, kt, vt, lens, 0.088, want_lse=True)
        b, bl = pb.propd_grouped_attention(tree, q, k, v, kt, vt, lens, 0.088, want_lse=True)
        n = int(x["n_nodes"][0])
        # half a step of each, and 2^-15 for weights and sums
        assert ((a - b).float().abs()[:, :, :n] <= 2.0 ** -7 * b.float().abs()[:, :, :n] + 2.0 ** -12).all()
        assert ((al - bl).abs()[:, :, :n] <= 2.0 ** -18 * (1 + bl.abs()[:, :, :n])).all()


@pytest.mark.parametrize("B,H,Hk,T,dtype,codes", [(84, 16, 4, 40, "bf16", True), (84, 16, 4, 40, "bf16", False), (70, 16, 4, 40, "f32", False), (150, 16, 4, 16, "bf16", True),
                                                  (150, 16, 4, 4, "bf16", True), (90, 8, 4, 2, "f32", True)])
def test_more_units_than_run_at_once(pb, B, H, Hk, T, dtype, codes):
    """Whole units first and the others cut, in every shape of the waves, with one sequence so long that its units among the first are cut too."""
    rng = np.random.default_rng(B + T)
    lens = [int(x) for x in rng.integers(0, 60, B)]
    lens[1], lens[B - 2] = 2500, 700
    x = make_case(rng, dtype, codes, H, Hk, 64, [synth.chain_tree(min(T, 3 + b % T)) for b in range(B)], lens, 64, T_max=T)
    check_attention(x, rule_of(64), *run_attention(pb, x, rule_of(64)))


def test_two_streams_at_once(pb):
    """Calls on two streams with workspaces of their own give the bits that they give alone."""
    rng = np.random.default_rng(21)
    calls = []
    for T, L in ((1, 1500), (30, 900)):
        x = make_case(rng, "bf16", True, 8, 2, 128, [synth.random_tree(rng, T)] * 3, [L, L // 2, 7], 32)
        tree, cache = dev_tree(pb, x), dev_cache(pb, x)
        q, kt, vt, lens = (to_dev(x[n]) for n in ("q", "k_tree", "v_tree", "seq_lens"))
        out = torch.zeros_like(q)
        ws = torch.empty(pb.workspace_bytes(pb.WS_PAGED_ATTENTION, 3, T, 8, 128, cache.capacity), dtype=torch.uint8, device="cuda")
        calls.append((out, lambda a=(tree, q, cache, kt, vt, lens), o=out, w=ws: pb.propd_paged_attention(*a, 0.088, out=o, workspace=w)))
    want = []
    for out, call in calls:
        call()
        torch.cuda.synchronize()
        want.append(out.clone())
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(10):
        for (out, call), stream in zip(calls, streams):
            with torch.cuda.stream(stream):
                out.zero_()
                call()
        torch.cuda.synchronize()
        assert all(torch.equal(out, w) for (out, _), w in zip(calls, want))
