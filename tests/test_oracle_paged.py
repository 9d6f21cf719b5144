"""The plain definitions of oracle/paged_cache.py against library routines, closed forms and distributions (CPU only)."""
import numpy as np
import pytest
import torch

from cache_util import f64, make_inputs, rule_of
from oracle import bounded_cache, paged_cache as ref
from paper_2402_13485_amd import synth


def test_codes_are_the_library_types_values():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = ref.decode(codes.numpy()[:, None], np.full(256, 127))[:, 0]
    assert ((got == want) | (np.isnan(got) & np.isnan(want))).all()


def test_quantised_rows_against_the_library_cast():
    """The cast of values of at most 448, ties among them; the scale is the least power of two that gets them there."""
    rng = np.random.default_rng(1)
    for size in (1e-30, 1e-3, 1.0, 448.0, 449.0, 1e30):
        row = (rng.normal(size=64) * size).astype(np.float32)
        row[:8] = row[8] * np.array([1, 2, -3, 0.5, 17 / 16, 19 / 16, 0, 0.03125], np.float32)
        codes, byte = ref.quantise(row)
        scaled = row.astype(np.float64) / 2.0 ** (byte - 127)
        assert np.abs(scaled).max() <= 448 and np.abs(scaled).max() > 224
        assert (codes == torch.from_numpy(scaled).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()).all()
        # half a step: 2^-4 of the value, or of the least normal one
        assert (np.abs(ref.decode(codes[None], [byte])[0] - row) <= 2.0 ** -4 * np.maximum(np.abs(row), 2.0 ** (byte - 127 - 6))).all()


def test_quantised_rows_that_are_special():
    assert ref.quantise(np.zeros(4))[1] == 10 and (ref.quantise(np.zeros(4))[0] == 0).all()
    codes, byte = ref.quantise([np.inf, -np.inf, np.nan, 448.0])
    assert byte == 127 and codes.tolist() == [127, 127, 127, 126]
    codes, byte = ref.quantise([3.39e38, -3.39e38, 1.0, 0.0])
    assert byte == 127 + 119 and codes.tolist()[:2] == [126, 254]


def test_pages_in_any_order_are_the_dense_cache():
    rng = np.random.default_rng(2)
    x = make_inputs(rng, "f32", 4, 2, 64, [synth.random_tree(rng, 9), synth.chain_tree(3)], [37, 16])
    R, table = 16, np.array([[4, 0, 2], [1, 5, 3]], np.int32)
    pages = {}
    for name in ("k", "v"):
        pages[name] = np.full((6, 2, R, 64), np.nan)
        got = ref.append(np.where(np.isnan(f64(x[name + "_cache"])), 0, f64(x[name + "_cache"])), [list(range(37)), list(range(16))], pages[name], None,
                         table, np.zeros(2, np.int32))
        assert got.tolist() == [37, 16]
    args = f64(x["k_tree"]), f64(x["v_tree"]), x["seq_lens"]
    got = ref.attention(x["n_nodes"], x["parent"], f64(x["q"]), pages["k"], pages["v"], table, *args, rule_of(64, window=20))
    want = bounded_cache.grouped_attention(x["n_nodes"], x["parent"], f64(x["q"]), f64(x["k_cache"]), f64(x["v_cache"]), *args, np.zeros(2, int), None,
                                           rule_of(64, window=20))
    for a, b in zip(got, want):
        assert np.array_equal(a, b, equal_nan=True)


def run(rng, parent, token, p, q, n, tries):
    """First token behind the root of a step, and the token after that if the first was accepted, over many random numbers."""
    T, V = len(parent), len(p[0])
    counts = np.zeros((V, V + 1))
    with np.errstate(divide="ignore"):
        logits = np.log(p)[None]
        draft = None if q is None else np.log(q)[None]
    for _ in range(tries):
        if q is not None:
            for i in range(1, T):
                token[0, i] = rng.choice(V, p=q[parent[i]])
        u, u_next = rng.random((1, T)), rng.random(1)
        a, path, last, _ = ref.accept_sampled([T], np.array([parent]), token, logits, 1.0, draft, 1.0, u, u_next, n)
        out = [int(token[0, i]) for i in path[0, 1:a[0]]] + [int(last[0])]
        counts[out[0], out[1] if len(out) > 1 else V] += 1
    return counts


@pytest.mark.parametrize("drawn", [False, True])
def test_accepted_tokens_are_distributed_as_the_target(drawn):
    """A root with three candidates, one of them with two more: the first token is distributed as p at the root, and the second, where
    there is one, as p at the node that was accepted."""
    rng = np.random.default_rng(3)
    V, parent, tries = 5, [-1, 0, 0, 0, 1, 1], 20000
    p = rng.dirichlet(np.ones(V), size=len(parent))
    q = rng.dirichlet(np.ones(V), size=len(parent)) if drawn else None
    token = np.array([[0, 2, 4, 1, 3, 0]])
    counts = run(rng, parent, token, p, q, 6, tries)
    first = counts.sum(1)
    assert (np.abs(first - tries * p[0]) < 5 * np.sqrt(tries * p[0] * (1 - p[0]))).all()
    if not drawn:  # token 2 is node 1: what follows it is p there
        second = counts[2, :V]
        n = second.sum()
        assert counts[2, V] == 0 and (np.abs(second - n * p[1]) < 5 * np.sqrt(n * p[1] * (1 - p[1]))).all()


def test_chain_is_the_usual_rejection_sampling():
    """One drawn candidate: accepted with probability min(1, p / q), else the rest is max(p - q, 0)."""
    p, q = np.array([0.5, 0.3, 0.2]), np.array([0.2, 0.7, 0.1])
    with np.errstate(divide="ignore"):
        logits, draft = np.log(np.stack((p, p)))[None], np.log(np.stack((q, q)))[None]
    for token, u, want in ((0, 0.999, 2), (1, 0.42, 2), (1, 0.43, 1), (2, 0.999, 2)):
        a, _, last, _ = ref.accept_sampled([2], np.array([[-1, 0]]), np.array([[0, token]]), logits, 1.0, draft, 1.0, np.array([[0, u]]), np.array([0.7]), 2)
        assert a[0] == want
        if want == 1:  # left of p: 0.3 of token 0, 0.1 of token 2
            assert last[0] == 0
    a, _, last, _ = ref.accept_sampled([2], np.array([[-1, 0]]), np.array([[0, 1]]), logits, 1.0, draft, 1.0, np.array([[0, .99]]), np.array([0.76]), 2)
    assert a[0] == 1 and last[0] == 2


def test_rows_without_probability_and_without_numbers():
    x = np.array([np.nan, -np.inf, -np.inf])
    assert (ref.softmax(x, 1.0) == 0).all() and ref.softmax(np.array([np.inf, 0, np.inf, np.nan]), 2.0).tolist() == [0.5, 0, 0.5, 0]
    a, _, last, _ = ref.accept_sampled([2], np.array([[-1, 0]]), np.array([[0, 2]]), np.stack((x, x))[None], 1.0, None, 1.0, np.zeros((1, 2)), np.zeros(1), 2)
    assert a[0] == 1 and last[0] == 0
