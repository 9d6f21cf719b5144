"""The calls of a paged cache and of sampled acceptance together, as a decoding loop makes them."""
import numpy as np
import pytest
import torch

from cache_util import f64
from decode_loop_util import root_path
from gpu_util import to_dev, to_host
from oracle import bounded_cache, paged_cache as ref
from paged_util import numbers
from paper_2402_13485_amd import synth
from test_gpu_parity import pb  # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("dtype,codes", [("bf16", True), ("bf16", False), ("f32", True)])
def test_steps_of_a_paged_cache(pb, dtype, codes, drawn, captured):
    """Prompts, then steps of rotary positions, attention over pages, sampled acceptance and commit: every step against the float64
    definitions on what the pages hold, eagerly or replayed from a graph of one step."""
    rng = np.random.default_rng(17)
    B, H, Hk, d, T, V, R, S, steps, stride = 3, 8, 2, 64, 12, 61, 16, 20, 5, 6
    B_pages = 6
    n_pages = B * B_pages
    kind = torch.float8_e4m3fn if codes else torch.bfloat16 if dtype == "bf16" else torch.float32
    pages = [torch.zeros((n_pages, Hk, R, d), dtype=torch.uint8 if codes else kind, device="cuda").view(kind) for _ in range(2)]
    scales = [torch.full((n_pages, Hk, R), 127, dtype=torch.uint8, device="cuda") for _ in range(2)] if codes else []
    table = rng.permutation(n_pages).reshape(B, B_pages).astype(np.int32)
    cache, seq = pb.PagedCache(*pages, to_dev(table), *scales), torch.zeros(B, dtype=torch.int32, device="cuda")
    inv_freq = to_dev((100.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32))
    prompt_rows = np.array([20, 11, 16], np.int32)
    pb.propd_paged_prompt(to_dev(numbers(rng, dtype, B, Hk, S, d)), to_dev(numbers(rng, dtype, B, Hk, S, d)), cache, seq, n_rows=to_dev(prompt_rows))
    assert to_host(seq).tolist() == prompt_rows.tolist()
    scale = float(np.float32(0.125))

    def draw_step():
        x = {}
        shapes = [synth.random_tree(rng, int(rng.integers(2, T + 1))) for _ in range(B)]
        x["n_nodes"], x["parent"], _ = synth.pad_trees(shapes, T)
        x["logits"] = numbers(rng, dtype, B, T, V, scale=2.0)
        x["draft"] = numbers(rng, dtype, B, T, V, scale=2.0)
        x["token"] = rng.integers(0, V, (B, T)).astype(np.int32)
        for b in range(B):  # the first child of most nodes carries the target's likeliest token
            for i in range(1, x["n_nodes"][b]):
                if rng.random() < 0.7:
                    x["token"][b, i] = np.argmax(f64(x["logits"][b, x["parent"][b, i]]))
        x["q"], x["k"], x["v"] = (numbers(rng, dtype, B, h, T, d) for h in (H, Hk, Hk))
        x["u"], x["u_next"] = rng.random((B, T)).astype(np.float32) * 0.7, rng.random(B).astype(np.float32)
        return {n: x[n].astype(x[n].dtype) for n in x}

    first = draw_step()
    t = {n: to_dev(a) for n, a in first.items()}
    tree = pb.Tree(t["n_nodes"], t["parent"], t["token"], *pb.propd_tree_mask(t["n_nodes"], t["parent"]))
    ws = torch.empty(max(pb.workspace_bytes(pb.WS_PAGED_ATTENTION, B, T, H, d, cache.capacity), pb.workspace_bytes(pb.WS_ACCEPT_SAMPLED, B, T, vocab=V)),
                     dtype=torch.uint8, device="cuda")
    qr, kr, out = torch.zeros_like(t["q"]), torch.zeros_like(t["k"]), torch.zeros_like(t["q"])
    tokens_out, result = torch.zeros((B, stride), dtype=torch.int32, device="cuda"), [None]

    def step():
        depth, anc = pb.propd_tree_mask(t["n_nodes"], t["parent"])
        now = pb.Tree(t["n_nodes"], t["parent"], t["token"], depth, anc)
        pb.propd_rotary(t["q"], t["k"], inv_freq, depth, start=seq.view(B, 1), n_rows=t["n_nodes"], q_out=qr, k_out=kr)
        pb.propd_paged_attention(now, qr, cache, kr, t["v"], seq, scale, out=out, workspace=ws)
        a, path, nxt = pb.propd_accept_sampled(now, t["logits"], t["u"], t["u_next"], draft_logits=t["draft"] if drawn else None, path_stride=stride, workspace=ws)
        tokens_out.copy_(pb.propd_paged_commit(now, a, path, nxt, kr, t["v"], cache, seq))
        result[0] = a, path, nxt

    graph = None
    if captured:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step()
    for n in range(steps):
        x = first if n == 0 else draw_step()
        for name in t:
            t[name].copy_(to_dev(x[name]))
        lens = to_host(seq)
        values = {}
        for name in "kv":
            p = getattr(cache, name + "_pages")
            values[name] = ref.decode(p.view(torch.uint8).cpu().numpy(), to_host(getattr(cache, name + "_scale"))) if codes else f64(to_host(p))
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        # the attention of this step, on what the pages held
        q, k, v = f64(to_host(qr)), f64(to_host(kr)), f64(x["v"])
        want, _, mag = ref.attention(x["n_nodes"], x["parent"], q, values["k"], values["v"], table, k, v, lens, dict(scale=scale, cap=0.0, window=0, slopes=None))
        e = U * (d + 4) * scale * np.nanmax(np.abs(q).sum(-1)) * max(np.abs(values["k"]).max(), np.nanmax(np.abs(k)))
        for b, m in enumerate(x["n_nodes"]):
            bound = (2 * e + 200 * U + 2.0 ** -17) * mag[b, :, :m] + 2.0 ** -8 * np.abs(want[b, :, :m]) + 1e-37
            assert (np.abs(f64(to_host(out))[b, :, :m] - want[b, :, :m]) <= bound).all(), (n, b)
        # what was accepted, and where it went
        a, path, nxt, margin = ref.accept_sampled(x["n_nodes"], x["parent"], x["token"], f64(x["logits"]), 1.0, f64(x["draft"]) if drawn else None, 1.0, x["u"],
                                                  x["u_next"], stride)
        assert margin > 1e-9
        assert [to_host(y).tolist() for y in result[0]] == [a.tolist(), path.tolist(), nxt.tolist()]
        line = np.full((B, stride), -1)
        for b in range(B):
            line[b, :a[b]] = [x["token"][b, i] for i in path[b, 1:a[b]]] + [nxt[b]]
        assert to_host(tokens_out).tolist() == line.tolist()
        assert to_host(seq).tolist() == (lens + a).tolist()
        dense = [torch.zeros((B, Hk, stride, d), dtype=t["k"].dtype, device="cuda") for _ in range(2)]
        pb.propd_paged_read(cache, seq, *dense, first=to_dev(lens))
        for got, source in zip(dense, (k, v)):
            for b in range(B):
                for j in range(a[b]):
                    for h in range(Hk):
                        row = source[b, h, path[b, j]]
                        if codes:
                            c, s = ref.quantise(row)
                            row = ref.decode(c[None], [s])[0]
                        assert np.array_equal(f64(to_host(got[b, h, j])), row), (n, b, j)
    assert to_host(seq).sum() > prompt_rows.sum() + steps * B  # some steps accepted more than the root


def test_a_sequence_moves_to_a_dense_cache(pb):
    """Paged rows read into a dense cache go on with the calls for those: the same result."""
    rng = np.random.default_rng(18)
    B, H, d, T, L = 2, 4, 128, 9, 77
    cache = pb.PagedCache(*(torch.zeros((B * 6, H, 16, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)),
                          to_dev(rng.permutation(B * 6).reshape(B, 6).astype(np.int32)),
                          *(torch.full((B * 6, H, 16), 127, dtype=torch.uint8, device="cuda") for _ in range(2)))
    seq = torch.zeros(B, dtype=torch.int32, device="cuda")
    pb.propd_paged_prompt(to_dev(numbers(rng, "bf16", B, H, L, d)), to_dev(numbers(rng, "bf16", B, H, L, d)), cache, seq)
    n_nodes, parent, _ = synth.pad_trees([synth.random_tree(rng, T)] * B, T)
    tree = pb.Tree(to_dev(n_nodes), to_dev(parent))
    tree.depth, tree.anc = pb.propd_tree_mask(tree.n_nodes, tree.parent)
    q, kt, vt = (to_dev(numbers(rng, "bf16", B, H, T, d)) for _ in range(3))
    k, v = pb.propd_paged_read(cache, seq, *(torch.zeros((B, H, 90, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    a = pb.propd_paged_attention(tree, q, cache, kt, vt, seq, 0.088).float()
    b = pb.propd_tree_attention(tree, q, k, v, kt, vt, seq, 0.088).float()
    # half a step of each result; the dense call's weights are single bf16 values, 2^-8 off at most, against sum p |v| <= max |v|
    assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + 2.0 ** -8 * max(float(v.float().abs().max()), float(vt.float().abs().max()))).all()
