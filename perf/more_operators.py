"""The operators of a paged K/V cache and of sampled acceptance, as cases that can be timed and compared.

A server keeps the K/V rows of all its sequences in pages of one pool, as they are or in 8 bits with a power of two as the
scale of each row; a sequence's table names its pages.  Every step the nodes of a sequence's tree attend to its paged
rows, the target's probabilities at the nodes decide by given random numbers which drafted tokens stay, and the rows of the
accepted nodes are written to the pages.  Prompts are written the same way, and a sequence that goes on in a dense cache is read back.

The kinds:
  attention   propd_paged_attention: a tree's nodes, or a single token, over paged rows and their own root paths
  sampled     propd_accept_sampled: the path that the target's probabilities accept, and the token after it
  commit      propd_paged_commit: the accepted nodes' rows to the end of their sequences' pages
  prompt      propd_paged_prompt: whole prompts to the pages
  read        propd_paged_read: paged rows as dense tensors
Head counts, tree sizes, lengths and the vocabulary are those of ``synth.WORKLOADS`` and ``perf/operators.py`` (32 or 40 query heads on
8 K/V heads, heads of 64 or 128, batch 1..32, trees of 1..128 nodes, up to 8192 cached tokens, 32000 tokens); pages are of 16 to 256 rows, in any
order.  Inputs are N(0,1); logits are 4 N(0,1), whose most likely token has a tenth to a half of the probability.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
PATH_STRIDE = 8         # the longest path of an accepting step here, as in perf/operators.py
E4M3_MOST = 448.0       # the largest value of the 8-bit type
LEAST_SCALE, MOST_SCALE = -117, 119  # exponents of a row's scale


def listed():
    return [
        # a single user's next token: one query of 32 heads, latency
        _attention(name="attn_token_b1", B=1, H=32, Hk=8, T=1, L=1024, rows=16),
        # a full server without drafting: long sequences in 8 bits, one token each; every row is read once
        _attention(name="attn_token_b32", pages="e4m3", B=32, H=32, Hk=8, T=1, L=8192, rows=64),
        # a small server with capped scores and a window, mixed lengths, 8 bits
        _attention(name="attn_tree_b4", pages="e4m3", B=4, H=32, Hk=8, T=64, L=2048, rows=32, ragged=True, cap=30.0, window=1500, lse=True),
        # the largest batch of the benchmark, pages as they are, five query heads to a K/V head
        _attention(name="attn_tree_b16", B=16, H=40, Hk=8, T=128, L=4096, rows=256, lse=True),
        # fp32 with a bias per distance, small heads
        _attention(name="attn_f32", dtype="f32", B=2, H=16, Hk=4, d=64, T=48, L=1024, rows=16, ragged=True, slopes=True, lse=True),
        # a single user's step: a small tree of given candidates
        _sampled(name="sampled_b1", B=1, T=16, V=32000, width=3),
        # the benchmark's batch of 64 nodes
        _sampled(name="sampled_b16", B=16, T=64, V=32000, width=4, ragged=True, inv_temperature=1.25),
        # candidates drawn from a draft model's distributions, several per node, fp32
        _sampled(name="sampled_draft_b4", dtype="f32", B=4, T=16, V=32000, width=3, draft=True),
        # the accepted rows of a batch: two dozen rows of 8 heads, latency
        dict(name="commit_b16", kind="commit", dtype="bf16", pages="e4m3", B=16, Hk=8, d=128, T=64, L=500, rows=16, ragged=True),
        # prompts of a small batch into 8 bits
        dict(name="prompt_b4", kind="prompt", dtype="bf16", pages="e4m3", B=4, Hk=8, d=128, S=4096, L=37, rows=64, ragged=False),
        # the smallest: fp32 rows as they are, of a short sequence
        dict(name="read_f32_tiny", kind="read", dtype="f32", pages="same", B=1, Hk=2, d=64, L=100, rows=16, ragged=False),
        # a batch that moves to dense caches
        dict(name="read_b8", kind="read", dtype="bf16", pages="e4m3", B=8, Hk=8, d=128, L=4096, rows=64, ragged=True),
    ]


def _attention(**k):
    return {**dict(kind="attention", dtype="bf16", pages="same", d=128, ragged=False, cap=0.0, slopes=False, window=0, lse=False), **k}


def _sampled(**k):
    return {**dict(kind="sampled", dtype="bf16", ragged=False, draft=False, inv_temperature=1.0), **k}


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = tuple(max(a, b) for a, b in zip(most.get(c["kind"], (0, 0)), (w["bytes"], w["flops"])))
    most["commit"] = most["prompt"]
    while True:
        c = dict(kind=rng.choice(("attention", "attention", "sampled", "commit", "prompt", "read")), dtype=rng.choice(("bf16", "bf16", "f32")),
                 B=log(1, 32), ragged=rng.random() < 0.5)
        if c["kind"] == "sampled":
            c.update(T=log(1, 128), V=log(500, 64000), width=rng.randint(1, 5), draft=rng.random() < 0.4, inv_temperature=rng.choice((1.0, 1.25, 2.0)))
            if c["B"] * c["T"] * c["V"] <= 16 * 64 * 32000 and (not c["draft"] or c["B"] * c["T"] * c["V"] <= 8 * 64 * 32000):
                return c
            continue
        c.update(Hk=rng.choice((1, 2, 4, 5, 8, 16)), d=rng.choice((64, 128, 128)), pages=rng.choice(("same", "e4m3")), rows=rng.choice((16, 32, 64, 256)),
                 L=log(1, 8192))
        if c["kind"] == "attention":
            c.update(H=c["Hk"] * rng.choice((1, 2, 4, 5, 8)), T=rng.choice((1, log(1, 128))), cap=rng.choice((0.0, 0.0, 30.0)), slopes=rng.random() < 0.3,
                     window=rng.choice((0, 0, log(1, 4096))), lse=rng.random() < 0.5)
        elif c["kind"] == "commit":
            c.update(T=log(1, 128), L=log(1, 1000))
        elif c["kind"] == "prompt":
            c.update(S=log(1, 4096), L=log(1, 300))
        w = work(c)
        if w["bytes"] <= most[c["kind"]][0] and w["flops"] <= most[c["kind"]][1] and c["B"] * c["Hk"] * c["L"] <= 32 * 8 * 8192:
            return c


def _lengths(case, n):
    """The sequences' lengths, from a third of `n` to all of it where they differ."""
    return [max(1, n - (n * ((7 * b) % 16)) // 24) if case["ragged"] else n for b in range(case["B"])]


def _row_bytes(case):
    """of a paged row, its scale included"""
    return case["d"] + 1 if case["pages"] == "e4m3" else case["d"] * _size(case)


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def work(case):
    """Every row that is needed once, queries and results once; two products.  Sampled: the rows of nodes on a path of usual length."""
    size, B = _size(case), case["B"]
    if case["kind"] == "sampled":
        rows = sum(min(n, 3) for n in _lengths(case, case["T"])) * (2 if case["draft"] else 1)
        return {"bytes": rows * case["V"] * size, "flops": 4.0 * rows * case["V"]}
    Hk, d = case["Hk"], case["d"]
    if case["kind"] == "read":
        rows = sum(_lengths(case, case["L"])) * Hk
        return {"bytes": 2 * rows * (_row_bytes(case) + d * size), "flops": 2.0 * rows * d}
    if case["kind"] in ("commit", "prompt"):
        rows = Hk * (sum(_lengths(case, case["S"])) if case["kind"] == "prompt" else sum(min(n, 3) for n in _lengths(case, case["T"])))
        return {"bytes": 2 * rows * (_row_bytes(case) + d * size), "flops": 4.0 * rows * d}
    rows, nodes = _lengths(case, case["L"]), _lengths(case, case["T"])
    if case["window"]:
        rows = [min(n, case["window"]) for n in rows]
    return {"bytes": 2 * Hk * sum(rows) * _row_bytes(case) + sum(nodes) * (2 * (case["H"] + Hk) * d * size + 4 * case["H"] * case["lse"]),
            "flops": 4.0 * case["H"] * d * sum((r + n) * n for r, n in zip(rows, nodes))}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev, dt = dict(device="cuda"), DTYPES[case["dtype"]]
    kind, B = case["kind"], case["B"]

    def normal(*shape):
        return torch.randn(shape, generator=g, dtype=dt, **dev)

    def uniform(*shape):
        return torch.rand(shape, generator=g, **dev)

    def whole(values):
        return torch.tensor(values, dtype=torch.int32, **dev)

    s = dict(case)
    if kind in ("attention", "sampled", "commit"):  # the trees
        T = case["T"]
        node = torch.arange(T, **dev)
        if kind == "sampled":  # every node has up to `width` children
            parent = ((node - 1).clamp(min=0) // case["width"]).expand(B, T).contiguous()
        else:
            parent = torch.where(node > 0, (uniform(B, T) ** 0.7 * node).long().clamp(max=T - 1), 0)
        step = torch.nn.functional.one_hot(parent, T).double()
        step[:, 0] = 0
        seen = torch.linalg.matrix_power(torch.eye(T, dtype=torch.float64, **dev) + step, T) > 0  # [B,T,T]: root paths
        parent[:, 0] = -1
        bits = torch.nn.functional.pad(seen, (0, 128 - T)).view(B, T, 2, 64).long() << torch.arange(64, **dev)
        s.update(n_nodes=whole(_lengths(case, T)), parent=parent.int(), anc=bits.sum(-1), seen=seen, depth=(seen.sum(-1) - 1).int(),
                 token=torch.zeros(B, T, dtype=torch.int32, **dev))
    if kind == "sampled":
        V, width, inv = case["V"], case["width"], case["inv_temperature"]
        s.update(logits=4 * normal(B, T, V), u=uniform(B, T), u_next=uniform(B), draft_logits=None)
        rank, above = (node - 1) % width, parent.clamp(min=0)
        if case["draft"]:  # drawn from what the draft says at the parent
            s["draft_logits"] = 0.9 * s["logits"] + normal(B, T, V)
            drawn = torch.multinomial(torch.softmax(s["draft_logits"].float() * inv, -1).view(B * T, V), width, replacement=True, generator=g)
        else:  # the likeliest by an estimate of the target
            drawn = (s["logits"].float() + torch.randn((B, T, V), generator=g, **dev)).topk(width, -1).indices
        s["token"] = drawn.view(B, T, width).gather(1, above[..., None].expand(B, T, width)).gather(2, rank.expand(B, T)[..., None])[..., 0].int()
        return s
    Hk, d, rows, L = case["Hk"], case["d"], case["rows"], _lengths(case, case["L"])
    room = PATH_STRIDE if kind == "commit" else case["S"] if kind == "prompt" else 0
    table_pages = (case["L"] + room + rows - 1) // rows
    n_pages = B * table_pages + 3
    s.update(seq_lens=whole(L), page_table=torch.randperm(n_pages, generator=g, **dev)[:B * table_pages].view(B, table_pages).int(), k_scale=None, v_scale=None)
    if case["pages"] == "e4m3":  # as rows of N(0,1) are held
        for name in ("k", "v"):
            codes = torch.randn((n_pages, Hk, rows, d), generator=g, dtype=torch.bfloat16, **dev)
            s[name + "_pages"] = codes.mul_(128).clamp_(-E4M3_MOST, E4M3_MOST).to(torch.float8_e4m3fn)
            s[name + "_scale"] = torch.randint(119, 122, (n_pages, Hk, rows), generator=g, dtype=torch.uint8, **dev)
    else:
        s.update(k_pages=normal(n_pages, Hk, rows, d), v_pages=normal(n_pages, Hk, rows, d))
    if kind == "read":
        s.update(k_out=torch.zeros(B, Hk, case["L"], d, dtype=dt, **dev), v_out=torch.zeros(B, Hk, case["L"], d, dtype=dt, **dev))
        return s
    if kind == "prompt":
        s.update(k=normal(B, Hk, case["S"], d), v=normal(B, Hk, case["S"], d), n_rows=whole(_lengths(case, case["S"])),
                 seq_lens_out=torch.zeros(B, dtype=torch.int32, **dev))
        return s
    s.update(k_tree=normal(B, Hk, T, d), v_tree=normal(B, Hk, T, d))
    if kind == "commit":
        s["token"] = torch.randint(0, 32000, (B, T), generator=g, dtype=torch.int32, **dev)
        last = (uniform(B) * s["n_nodes"]).long()  # the accepted path ends in some node
        path = torch.where(s["seen"][torch.arange(B, **dev), last], torch.arange(T, **dev), T).sort(-1).values
        path = torch.nn.functional.pad(path, (0, PATH_STRIDE), value=T)[:, :PATH_STRIDE]
        s.update(accept_len=(path < T).sum(-1).int(), accept_path=torch.where(path < T, path, -1).int().contiguous(),
                 next_token=torch.randint(0, 32000, (B,), generator=g, dtype=torch.int32, **dev), seq_lens_out=torch.zeros(B, dtype=torch.int32, **dev))
        return s
    H = case["H"]
    s.update(q=normal(B, H, T, d), scale=1 / math.sqrt(d), out=torch.zeros(B, H, T, d, dtype=dt, **dev),
             lse_out=torch.zeros(B, H, T, **dev) if case["lse"] else None,
             slope=2.0 ** (-4 - 8 * torch.arange(H, **dev) / H) if case["slopes"] else None)  # distances matter over tens to thousands of tokens
    return s


def run(s):
    if own:
        from paper_2402_13485_amd import binding as pb
        kind = s["kind"]
        tree = pb.Tree(s["n_nodes"], s["parent"], s["token"], s["depth"], s["anc"]) if "n_nodes" in s else None
        if kind == "sampled":
            return pb.propd_accept_sampled(tree, s["logits"], s["u"], s["u_next"], inv_temperature=s["inv_temperature"], draft_logits=s["draft_logits"],
                                           draft_inv_temperature=s["inv_temperature"], path_stride=PATH_STRIDE)
        cache = pb.PagedCache(s["k_pages"], s["v_pages"], s["page_table"], s["k_scale"], s["v_scale"])
        if kind == "read":
            return pb.propd_paged_read(cache, s["seq_lens"], k_out=s["k_out"], v_out=s["v_out"])
        if kind == "prompt":
            pb.propd_paged_prompt(s["k"], s["v"], cache, s["seq_lens"], n_rows=s["n_rows"], seq_lens_out=s["seq_lens_out"])
            return s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["seq_lens_out"]
        if kind == "commit":
            tokens = pb.propd_paged_commit(tree, s["accept_len"], s["accept_path"], s["next_token"], s["k_tree"], s["v_tree"], cache, s["seq_lens"],
                                           seq_lens_out=s["seq_lens_out"])
            return s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["seq_lens_out"], tokens
        pb.propd_paged_attention(tree, s["q"], cache, s["k_tree"], s["v_tree"], s["seq_lens"], s["scale"], cap=s["cap"], window=s["window"],
                                 slopes=s["slope"], out=s["out"], lse=s["lse_out"])
        return s["out"], s["lse_out"]
    return {"attention": _plain_attention, "sampled": _plain_sampled, "commit": _plain_commit, "prompt": _plain_prompt, "read": _plain_read}[s["kind"]](s)


def _power_of_two(exponent):
    """fp32, by its bits: a power function need not give it exactly."""
    return ((exponent.int() + 127) << 23).view(torch.float32)


def _plain_rows(s, name):
    """The paged rows of every sequence in order, [B,Hk,pages * rows,d] fp32."""
    table = s["page_table"].long()
    x = s[name + "_pages"][table].float()  # [B,pages,Hk,rows,d]
    if s[name + "_scale"] is not None:
        x = x * _power_of_two(s[name + "_scale"][table].int() - 127)[..., None]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attention(s):
    B, H, T, d = s["q"].shape
    Hk = s["k_tree"].shape[1]
    k, v = (torch.cat((_plain_rows(s, n), s[n + "_tree"].float()), 2) for n in ("k", "v"))
    M, L, depth = k.shape[2] - T, s["seq_lens"][:, None, None], s["depth"].long()
    row = torch.arange(M, device="cuda")
    back = torch.cat(((L + depth[:, :, None] - row), depth[:, :, None] - depth[:, None]), 2)  # [B,T,M + T]
    x = (s["q"].float().view(B, Hk, -1, d) @ k.transpose(-1, -2)).view(B, Hk, -1, T, M + T) * s["scale"]
    if s["cap"]:
        x = s["cap"] * torch.tanh(x / s["cap"])
    if s["slope"] is not None:
        x = x - s["slope"].view(1, Hk, -1, 1, 1) * back[:, None, None].float()
    seen = torch.cat(((row < L).expand(B, T, M), s["seen"]), 2)
    seen = seen & (back < s["window"]) if s["window"] else seen
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    most = x.amax(-1, keepdim=True)
    x = torch.exp(x - most)
    total = x.sum(-1, keepdim=True)
    out = (x.view(B, Hk, H // Hk * T, -1) @ v).view(B, H, T, d) / total.view(B, H, T, 1)
    there = torch.arange(T, device="cuda") < s["n_nodes"][:, None, None]
    out = torch.where(there[..., None], out, 0.0).to(s["q"].dtype)
    return out, torch.where(there, (most + torch.log(total)).view(B, H, T), 0.0) if s["lse_out"] is not None else None


def _plain_quantised(x):
    """Codes and scale bytes of rows [...,d]: the smallest power of two that brings the largest value to 448 or less."""
    most = x.float().abs().amax(-1)
    fraction, exponent = torch.frexp(most)
    power = torch.where(most > 0, exponent - 9 + (fraction > 0.875).int(), LEAST_SCALE).clamp(LEAST_SCALE, MOST_SCALE)
    codes = (x.float() * _power_of_two(-power)[..., None]).clamp(-E4M3_MOST, E4M3_MOST)
    return codes.to(torch.float8_e4m3fn), (power + 127).to(torch.uint8)


def _plain_write(s, rows, there):
    """rows: k and v [B,Hk,N,d]; row n of sequence b goes to place seq_lens[b] + n where there[b,n]."""
    table, N = s["page_table"].long(), there.shape[1]
    at = s["seq_lens"][:, None] + torch.arange(N, device="cuda")
    there = there & (at < table.shape[1] * s["rows"])
    b, n = there.nonzero(as_tuple=True)
    at = at[b, n]
    page, place = table[b, at // s["rows"]], at % s["rows"]
    for name, x in zip("kv", rows):
        x = x.transpose(1, 2)[b, n]  # [rows,Hk,d]
        if s[name + "_scale"] is not None:
            x, scale = _plain_quantised(x)
            s[name + "_scale"][page, :, place] = scale
            s[name + "_pages"].view(torch.uint8)[page, :, place] = x.view(torch.uint8)
        else:
            s[name + "_pages"][page, :, place] = x


def _plain_commit(s):
    path, a = s["accept_path"].long(), s["accept_len"][:, None]
    B, P = path.shape
    step = torch.arange(P, device="cuda")
    node = path.clamp(min=0)
    rows = [x.gather(2, node[:, None, :, None].expand(B, x.shape[1], P, x.shape[3])) for x in (s["k_tree"], s["v_tree"])]
    _plain_write(s, rows, step < a)
    tokens = torch.nn.functional.pad(s["token"].gather(1, node), (0, 1))[:, 1:]  # those behind the root
    tokens = torch.where(step + 1 < a, tokens, torch.where(step + 1 == a, s["next_token"][:, None], -1))
    return s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["seq_lens"] + s["accept_len"], tokens


def _plain_prompt(s):
    _plain_write(s, (s["k"], s["v"]), torch.arange(s["S"], device="cuda") < s["n_rows"][:, None])
    return s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["seq_lens"] + s["n_rows"]


def _plain_read(s):
    there = (torch.arange(s["L"], device="cuda") < s["seq_lens"][:, None])[:, None, :, None]
    return tuple(torch.where(there, _plain_rows(s, n)[:, :, :s["L"]].to(s[n + "_out"].dtype), s[n + "_out"]) for n in "kv")


def _plain_sampled(s):
    B, T, V = s["logits"].shape
    node, inv = torch.arange(T, device="cuda"), s["inv_temperature"]
    parent, token, n = s["parent"].long(), s["token"].long(), s["n_nodes"][:, None]
    above = parent.clamp(min=0)
    is_child = (node > 0) & (node < n)
    earlier = (parent[:, :, None] == parent[:, None]) & (node < node[:, None]) & (is_child[:, :, None] & is_child[:, None])  # [B,T,T]: siblings before
    batch = torch.arange(B, device="cuda")
    if s["draft_logits"] is None:
        x = s["logits"].float()
        most = x.amax(-1, keepdim=True)
        total = torch.exp((x - most) * inv).sum(-1)
        p = torch.exp((x[batch[:, None], above, token] - most[..., 0].gather(1, above)) * inv) / total.gather(1, above)
        again = (earlier & (token[:, :, None] == token[:, None])).any(-1)  # a token that a sibling before has
        p = torch.where(again, 0.0, p)
        left = 1 - torch.where(earlier, p[:, None], 0.0).sum(-1)
        passes = is_child & (s["u"] * left < p)
    else:
        pq = torch.softmax(s["logits"].double() * inv, -1), torch.softmax(s["draft_logits"].double() * inv, -1)
        p, q = (x[batch[:, None], above, token] for x in pq)
        rank = earlier.sum(-1)
        much, mass = torch.zeros(B, T, dtype=torch.float64, device="cuda"), torch.ones(B, T, dtype=torch.float64, device="cuda")  # by parent
        passes = torch.zeros_like(is_child)
        children = (is_child[:, :, None] & (above[:, :, None] == node)).sum(1)
        for k in range(s["width"]):  # (each sibling's test needs what the one before left)
            much_i, mass_i = much.gather(1, above), mass.gather(1, above)
            passes |= is_child & (rank == k) & (s["u"].double() * mass_i * q < (p - much_i * q).clamp(min=0))
            more = children > k
            much = torch.where(more, much + mass, much)
            mass = torch.where(more, (pq[0] - much[..., None] * pq[1]).clamp(min=0).sum(-1), mass)
    chosen = passes & ~(earlier & passes[:, None]).any(-1)
    chosen[:, 0] = True
    on_path = ((~s["seen"] | chosen[:, None]).all(-1)) & (node < n)
    full = on_path.sum(-1)
    path = torch.where(on_path, node, T).sort(-1).values
    path = torch.nn.functional.pad(path, (0, PATH_STRIDE + 1), value=T)
    last = path.gather(1, full[:, None] - 1)[:, 0]
    row = s["logits"][batch, last].double()
    weight = torch.exp((row - row.amax(-1, keepdim=True)) * inv)
    tried = is_child & (parent == last[:, None])  # all of them failed
    if s["draft_logits"] is None:
        hit = torch.zeros(B, V + 1, dtype=torch.bool, device="cuda").scatter(1, torch.where(tried, token, V), True)[:, :V]
        weight = torch.where(hit, 0.0, weight)
    else:
        weight = (pq[0][batch, last] - much[batch, last][:, None] * pq[1][batch, last]).clamp(min=0)
    upto = weight.cumsum(-1)
    next_token = (upto > s["u_next"].double()[:, None] * upto[:, -1:]).int().argmax(-1)
    length = full.clamp(max=PATH_STRIDE)
    cut = path[:, PATH_STRIDE].clamp(max=T - 1)
    next_token = torch.where(full > PATH_STRIDE, token.gather(1, cut[:, None])[:, 0], next_token)
    path = path[:, :PATH_STRIDE]
    return length.int(), torch.where(path < T, path, -1).int(), next_token.int()


def _double_power(exponent):
    return ((exponent.long() + 1023) << 52).view(torch.float64)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sampled":
        return _exact_sampled(s)
    if case["kind"] == "attention":
        return _exact_attention(s)
    Hk, rows, B = case["Hk"], case["rows"], case["B"]
    table, lens = s["page_table"].tolist(), s["seq_lens"].tolist()
    if case["kind"] == "read":
        outs = []
        for name in "kv":
            out = s[name + "_out"].double()
            for b, n in enumerate(lens):
                for first in range(0, n, rows):
                    page, m = table[b][first // rows], min(rows, n - first)
                    x = s[name + "_pages"][page, :, :m].double()
                    if s[name + "_scale"] is not None:
                        x = x * _double_power(s[name + "_scale"][page, :, :m, None].long() - 127)
                    out[b, :, first:first + m] = x
            outs.append(out)
        return tuple(outs)
    after, to, of = [], [], []
    for b, n in enumerate(lens):
        taken = range(int(s["n_rows"][b])) if case["kind"] == "prompt" else s["accept_path"][b, :int(s["accept_len"][b])].tolist()
        to += [(table[b][(n + i) // rows], (n + i) % rows) for i in range(len(taken))]
        of += [(b, i) for i in taken]
        after.append(n + len(taken))
    page, place = (torch.tensor(x, device="cuda") for x in zip(*to))
    b_of, i_of = (torch.tensor(x, device="cuda") for x in zip(*of))
    pages, scales = {}, {}
    for name in "kv":
        source = s[name if case["kind"] == "prompt" else name + "_tree"]
        x = source[b_of, :, i_of].double()
        pages[name], scales[name] = s[name + "_pages"].double(), s[name + "_scale"]
        if scales[name] is not None:
            most = x.abs().amax(-1)
            power = torch.ceil(torch.log2(most / E4M3_MOST)).clamp(LEAST_SCALE, MOST_SCALE)
            y = x / _double_power(power)[..., None]
            step = _double_power(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -9))).clamp(min=-6) - 3)
            x = torch.round(y / step) * step
            scales[name] = scales[name].clone()
            scales[name][page, :, place] = (power + 127).to(torch.uint8)
        pages[name][page, :, place] = x
    outs = pages["k"], pages["v"], scales["k"], scales["v"], torch.tensor(after)
    if case["kind"] == "prompt":
        return outs
    tokens = torch.full((B, PATH_STRIDE), -1)
    for b in range(B):
        path = s["accept_path"][b, :int(s["accept_len"][b])].long()
        tokens[b, :len(path)] = torch.cat((s["token"][b][path[1:]], s["next_token"][b:b + 1])).cpu()
    return (*outs, tokens)


def _exact_attention(s):
    B, H, T, d = s["q"].shape
    Hk, rows = s["k_tree"].shape[1], s["rows"]
    out, lse = torch.zeros(B, H, T, d, dtype=torch.float64, device="cuda"), torch.zeros(B, H, T, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, t = int(s["seq_lens"][b]), int(s["n_nodes"][b])
        pages = s["page_table"][b, :(n + rows - 1) // rows].long()
        depth = s["depth"][b, :t].double()
        hidden = torch.cat((torch.zeros(t, n, dtype=torch.bool, device="cuda"), ~s["seen"][b, :t, :t]), 1)
        back = torch.cat((n + depth[:, None] - torch.arange(n, device="cuda"), depth[:, None] - depth), 1)
        if s["window"]:
            hidden = hidden | (back >= s["window"])
        for hk in range(Hk):
            kv = []
            for name in "kv":
                x = s[name + "_pages"][pages, hk].double()
                if s[name + "_scale"] is not None:
                    x = x * _double_power(s[name + "_scale"][pages, hk].long() - 127)[..., None]
                kv.append(torch.cat((x.reshape(-1, d)[:n], s[name + "_tree"][b, hk, :t].double())))
            for h in range(hk * (H // Hk), (hk + 1) * (H // Hk)):
                x = s["q"][b, h, :t].double() @ kv[0].T.contiguous() * s["scale"]
                if s["cap"]:
                    x = s["cap"] * torch.tanh(x / s["cap"])
                if s["slope"] is not None:
                    x = x - float(s["slope"][h]) * back
                x[hidden] = -math.inf
                lse[b, h, :t] = torch.logsumexp(x, 1)
                out[b, h, :t] = torch.softmax(x, 1) @ kv[1]
    return out, lse if s["lse_out"] is not None else None


def _exact_sampled(s):
    lengths, paths, tokens = [], [], []
    for b in range(s["B"]):
        n, node, path = int(s["n_nodes"][b]), 0, [0]
        parent, token, u = s["parent"][b, :n].tolist(), s["token"][b, :n].tolist(), s["u"][b].tolist()
        while True:
            left = torch.softmax(s["logits"][b, node].double() * s["inv_temperature"], -1)  # what is left of the target
            drawn_from = None if s["draft_logits"] is None else torch.softmax(s["draft_logits"][b, node].double() * s["inv_temperature"], -1)
            taken = None
            for child in [i for i in range(1, n) if parent[i] == node]:
                c = token[child]
                if u[child] * (1.0 if drawn_from is None else float(drawn_from[c])) < float(left[c]):
                    taken = child
                    break
                if drawn_from is None:
                    left[c] = 0
                else:
                    left = (left - drawn_from).clamp(min=0)
                left = left / left.sum()
            if taken is None:
                break
            path.append(taken)
            node = taken
        upto = left.cumsum(-1)
        tokens.append(token[path[PATH_STRIDE]] if len(path) > PATH_STRIDE else int((upto > float(s["u_next"][b]) * upto[-1]).int().argmax()))
        lengths.append(min(len(path), PATH_STRIDE))
        paths.append((path + [-1] * PATH_STRIDE)[:PATH_STRIDE])
    return torch.tensor(lengths), torch.tensor(paths), torch.tensor(tokens)
