"""The operators of a bounded K/V cache, as cases that can be timed and compared.

A long generation with shared K/V heads keeps a cache of a fixed size: every step turns the positions
of the tree's nodes into rotations of q and k, lets the nodes attend to the cached rows that are left,
adds the attention that the accepted nodes paid to every row, and gives up the rows that were looked at least.

The kinds:
  rotary      propd_rotary: rotary positions of one or several axes, for the nodes of a tree or the rows of a prompt
  attention   propd_grouped_attention: a tree's nodes over cached rows whose K/V heads are shared by several
              query heads, with capped scores, a distance bias, a window and rows out of order as the case says
  observe     propd_cache_observe: the accepted nodes' attention weights, added up per cached row
  evict       propd_cache_evict: down to `budget` rows per K/V head, by those sums
Head counts, tree sizes and lengths are those of ``synth.WORKLOADS`` and ``perf/cases.py`` (32 or 40 heads of 64 or
128, batch 1..32, trees of 16..128 nodes, up to 8192 cached tokens) with 1 to 8 query heads to a K/V head, which is
what decoders of these sizes share; inputs are N(0,1), trees random, weights log-normal as sums of attention are.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
PATH_STRIDE = 8   # the longest path of an accepting step here, as in perf/cases.py
SECTIONS = (1, 3, 3)  # parts of the rotated pairs that belong to time, height and width


def listed():
    return [
        # a single user's next token without drafting: one query of 32 heads, latency
        _attention(name="attn_token_b1", B=1, H=32, Hk=8, T=1, L=1024),
        # a small server with capped scores, mixed lengths; lse for the sums of attention
        _attention(name="attn_capped_b4", B=4, H=32, Hk=8, T=64, L=2048, ragged=True, cap=30.0, lse=True),
        # the largest batch of the benchmark, all lengths equal, five query heads to a K/V head
        _attention(name="attn_b16", B=16, H=40, Hk=8, T=128, L=4096, lse=True),
        # evicted caches: rows out of order with positions of their own, a distance bias and a window; small heads
        _attention(name="attn_evicted_b32", B=32, H=32, Hk=8, d=64, T=64, L=2048, ragged=True, evicted=True, slopes=True,
                   window=3000, lse=True),
        # fp32, capped and biased
        _attention(name="attn_f32", dtype="f32", B=2, H=16, Hk=4, T=48, L=1024, ragged=True, cap=30.0, slopes=True, lse=True),
        # the smallest: fp32, two K/V heads
        _observe(name="observe_f32_tiny", dtype="f32", B=1, H=4, Hk=2, d=64, T=16, L=128),
        # one layer of a full batch
        _observe(name="observe_b16", B=16, H=40, Hk=8, T=128, L=4096, evicted=True),
        # every step of a cache that is full: a few rows too many
        dict(name="evict_step_b4", kind="evict", dtype="bf16", B=4, Hk=8, d=128, L=1032, ragged=False, budget=1024, recent=128, sinks=4),
        # after long prompts: down to a quarter
        dict(name="evict_b32", kind="evict", dtype="bf16", B=32, Hk=8, d=128, L=8192, ragged=True, budget=2048, recent=256, sinks=4),
        # the nodes of one tree, text: positions of one axis
        dict(name="rotary_tree_b1", kind="rotary", dtype="bf16", B=1, H=32, Hk=8, d=128, S=64, rot=128, axes=1, adjacent=False, ragged=False),
        # fp32, neighbouring channels in pairs, half of the head rotated, ragged trees
        dict(name="rotary_f32_b16", kind="rotary", dtype="f32", B=16, H=40, Hk=8, d=128, S=128, rot=64, axes=1, adjacent=True, ragged=True),
        # prompts of image patches: time, height and width
        dict(name="rotary_image_b4", kind="rotary", dtype="bf16", B=4, H=32, Hk=8, d=128, S=4096, rot=128, axes=3, adjacent=False, ragged=False),
    ]


def _attention(**k):
    return {**dict(kind="attention", dtype="bf16", d=128, ragged=False, evicted=False, cap=0.0, slopes=False, window=0, lse=False), **k}


def _observe(**k):
    return {**dict(kind="observe", dtype="bf16", d=128, ragged=False, evicted=False, cap=0.0, slopes=False, window=0, decay=0.98), **k}


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {k: (max(work(c)["bytes"] for c in listed() if c["kind"] == k), max(work(c)["flops"] for c in listed() if c["kind"] == k))
            for k in ("attention", "observe", "evict", "rotary")}
    while True:
        kind = rng.choice(("attention", "attention", "observe", "evict", "rotary"))
        Hk = rng.choice((1, 2, 4, 5, 8, 16))
        c = dict(kind=kind, dtype=rng.choice(("bf16", "bf16", "f32")), B=log(1, 32), Hk=Hk, d=rng.choice((64, 128, 128)), ragged=rng.random() < 0.5)
        if kind in ("attention", "observe"):
            c.update(H=Hk * rng.choice((1, 2, 4, 5, 8)), T=log(1, 128), L=log(1, 8192), evicted=rng.random() < 0.4,
                     cap=rng.choice((0.0, 0.0, 30.0)), slopes=rng.random() < 0.3, window=rng.choice((0, 0, log(1, 4096))))
            c.update(dict(lse=rng.random() < 0.5) if kind == "attention" else dict(decay=rng.choice((1.0, 0.98))))
        elif kind == "evict":
            budget = log(8, 4096)
            c.update(L=min(8192, budget + log(1, 2 * budget)), budget=budget, recent=rng.randint(0, budget // 4), sinks=rng.choice((0, 4)))
        else:
            c.update(H=Hk * rng.choice((1, 2, 4, 5, 8)), S=log(1, 4096), rot=rng.choice((c["d"], c["d"], c["d"] // 2)), axes=rng.choice((1, 1, 3)),
                     adjacent=rng.random() < 0.3)
        w = work(c)
        if w["bytes"] <= most[kind][0] and w["flops"] <= most[kind][1] and c["B"] * c["Hk"] * c.get("L", 1) <= 16 * 8 * 4096:
            return c


def _lengths(case, n):
    """The sequences' lengths, from a third of `n` to all of it where they differ."""
    return [max(1, n - (n * ((7 * b) % 16)) // 24) if case["ragged"] else n for b in range(case["B"])]


def work(case):
    """K and V rows once (those that a window leaves), queries, results and per-row numbers once; two products."""
    size = 2 if case["dtype"] == "bf16" else 4
    B, Hk, d = case["B"], case["Hk"], case["d"]
    if case["kind"] == "rotary":
        rows = sum(_lengths(case, case["S"]))
        values = rows * (case["H"] + Hk) * d
        return {"bytes": 2 * values * size + 4 * rows * case["axes"], "flops": 3.0 * values * case["rot"] / d}
    rows = _lengths(case, case["L"])
    if case["kind"] == "evict":
        moved = sum(case["budget"] * (n - case["budget"]) / n for n in rows if n > case["budget"])
        return {"bytes": Hk * (sum(8 * n + 8 * min(n, case["budget"]) for n in rows) + moved * 4 * d * size), "flops": 0}
    if case["window"] and not case["evicted"]:
        rows = [min(n, case["window"]) for n in rows]
    nodes = _lengths(case, case["T"])
    if case["kind"] == "observe":
        nodes = [min(n, 3) for n in nodes]
        return {"bytes": Hk * sum(rows) * (d * size + (16 if case["evicted"] else 8)) + case["H"] * sum(nodes) * (d * size + 4),
                "flops": 2.0 * case["H"] * d * sum(r * n for r, n in zip(rows, nodes))}
    return {"bytes": Hk * sum(rows) * (2 * d * size + 4 * case["evicted"]) + sum(nodes) * (2 * (case["H"] + Hk) * d * size + 4 * case["H"] * case["lse"]),
            "flops": 4.0 * case["H"] * d * sum((r + n) * n for r, n in zip(rows, nodes))}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev, dt = dict(device="cuda"), DTYPES[case["dtype"]]
    kind, B, Hk, d = case["kind"], case["B"], case["Hk"], case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=g, dtype=dt, **dev)

    def uniform(*shape):
        return torch.rand(shape, generator=g, **dev)

    def whole(values):
        return torch.tensor(values, dtype=torch.int32, **dev)

    s = dict(case)
    if kind == "rotary":
        S, rot = case["S"], case["rot"]
        pairs = rot // 2
        per = [pairs * x // sum(SECTIONS) for x in SECTIONS]
        s.update(q=normal(B, case["H"], S, d), k=normal(B, Hk, S, d), q_out=torch.zeros(B, case["H"], S, d, dtype=dt, **dev),
                 k_out=torch.zeros(B, Hk, S, d, dtype=dt, **dev), n_rows=whole(_lengths(case, S)),
                 inv_freq=(1e6 ** (-torch.arange(pairs, dtype=torch.float64, **dev) / pairs)).float(),
                 start=(100000 * uniform(B, case["axes"])).int(), axis_of=None)
        if case["axes"] == 3:  # patches of pictures 64 wide, row by row
            at = torch.arange(S, **dev)
            s["offset"] = torch.stack((at // 4096, at // 64 % 64, at % 64)).int().expand(B, 3, S).contiguous()
            s["axis_of"] = torch.repeat_interleave(torch.arange(3, **dev), torch.tensor([pairs - per[1] - per[2], per[1], per[2]], **dev)).int()
        else:  # a node's depth
            s["offset"] = (8 * uniform(B, S)).int()
        return s
    L, Lm = torch.tensor(_lengths(case, case["L"]), **dev), case["L"] + PATH_STRIDE
    evicted = kind == "evict" or case["evicted"]
    dropped = L // 2 + 3 if evicted else 0 * L
    s.update(seq_lens=L.int(), dropped=dropped.int(), k_cache=normal(B, Hk, Lm, d), position=None)
    if kind != "observe":
        s["v_cache"] = normal(B, Hk, Lm, d)
    if evicted:  # of the positions up to now: the newest quarter, and others at random, in any order
        last = (L + dropped)[:, None, None]
        at = torch.arange(int(last.max()), **dev)
        chosen = torch.where(at < last, torch.where(at >= last - (L // 4)[:, None, None], -1.0, uniform(B, Hk, len(at))), 2.0).argsort(-1)
        chosen = torch.nn.functional.pad(chosen, (0, max(0, Lm - len(at))))[..., :Lm]
        mixed = torch.where(torch.arange(Lm, **dev) < L[:, None, None], uniform(B, Hk, Lm), 2.0).argsort(-1)
        s["position"] = chosen.gather(-1, mixed).int()
    if kind != "attention":
        s.update(weight=torch.exp(2 * torch.randn((B, Hk, Lm), generator=g, **dev)), weight_out=torch.zeros(B, Hk, Lm, **dev),
                 position_out=torch.zeros(B, Hk, Lm, dtype=torch.int32, **dev) if evicted else None)
    if kind == "evict":
        s.update(seq_lens_out=torch.zeros_like(s["seq_lens"]), dropped_out=torch.zeros_like(s["dropped"]))
        return s
    H, T = case["H"], case["T"]
    n_nodes = torch.tensor(_lengths(case, T), **dev)
    node = torch.arange(T, **dev)
    parent = torch.where(node > 0, (uniform(B, T) ** 0.7 * node).long().clamp(max=T - 1), 0)
    step = torch.nn.functional.one_hot(parent, T).double()
    step[:, 0] = 0
    seen = torch.linalg.matrix_power(torch.eye(T, dtype=torch.float64, **dev) + step, T) > 0  # [B,T,T]: root paths
    parent[:, 0] = -1
    bits = torch.nn.functional.pad(seen, (0, 128 - T)).view(B, T, 2, 64).long() << torch.arange(64, **dev)
    s.update(q=normal(B, H, T, d), k_tree=normal(B, Hk, T, d), n_nodes=n_nodes.int(), parent=parent.int(), anc=bits.sum(-1), seen=seen,
             token=torch.zeros(B, T, dtype=torch.int32, **dev), scale=1 / math.sqrt(d), slope=None)
    s["depth"] = (seen.sum(-1) - 1).int()
    if case["slopes"]:  # distances matter over tens to thousands of tokens
        s["slope"] = 2.0 ** (-4 - 8 * torch.arange(H, **dev) / H)
    if kind == "attention":
        s.update(v_tree=normal(B, Hk, T, d), out=torch.zeros(B, H, T, d, dtype=dt, **dev),
                 lse_out=torch.zeros(B, H, T, **dev) if case["lse"] else None)
        return s
    last = (uniform(B) * n_nodes).long()  # the accepted path ends in some node
    path = torch.where(seen[torch.arange(B, **dev), last], node, T).sort(-1).values
    path = torch.nn.functional.pad(path, (0, PATH_STRIDE), value=T)[:, :PATH_STRIDE]
    s["accept_len"] = (path < T).sum(-1).int()
    s["accept_path"] = torch.where(path < T, path, -1).int().contiguous()
    x, seen_by = _path_scores(s)  # what the attention of this step said
    x = torch.where(seen_by, x, -math.inf).logsumexp(-1).view(B, H, PATH_STRIDE)
    s["lse"] = torch.zeros(B, H, T + 1, **dev).scatter(2, path[:, None].expand(B, H, PATH_STRIDE), x)[..., :T].contiguous()
    return s


def run(s):
    if own:
        from paper_2402_13485_amd import binding as pb
        if s["kind"] == "rotary":
            return pb.propd_rotary(s["q"], s["k"], s["inv_freq"], s["offset"], start=s["start"], axis_of=s["axis_of"], n_rows=s["n_rows"],
                                   adjacent=s["adjacent"], q_out=s["q_out"], k_out=s["k_out"])
        rows = pb.CacheRows(s["seq_lens"], s["dropped"], s["position"], s.get("weight"))
        if s["kind"] == "evict":
            out = pb.CacheRows(s["seq_lens_out"], s["dropped_out"], s["position_out"], s["weight_out"])
            pb.propd_cache_evict(s["k_cache"], s["v_cache"], rows, s["budget"], s["recent"], sinks=s["sinks"], rows_out=out)
            return s["k_cache"], s["v_cache"], out.seq_lens, out.dropped, out.position, out.weight
        tree = pb.Tree(s["n_nodes"], s["parent"], s["token"], s["depth"], s["anc"])
        rule = dict(cap=s["cap"], window=s["window"], slopes=s["slope"])
        if s["kind"] == "observe":
            pb.propd_cache_observe(tree, s["accept_len"], s["accept_path"], s["q"], s["lse"], s["k_cache"], s["k_tree"], rows, s["scale"],
                                   decay=s["decay"], weight_out=s["weight_out"], position_out=s["position_out"], **rule)
            return s["weight_out"], s["position_out"]
        pb.propd_grouped_attention(tree, s["q"], s["k_cache"], s["v_cache"], s["k_tree"], s["v_tree"], s["seq_lens"], s["scale"],
                                   dropped=s["dropped"], position=s["position"], out=s["out"], lse=s["lse_out"], **rule)
        return s["out"], s["lse_out"]
    if s["kind"] == "rotary":
        return _plain_rotary(s)
    if s["kind"] == "evict":
        return _plain_evict(s)
    return _plain_observe(s) if s["kind"] == "observe" else _plain_attention(s)


def _plain_rotary(s):
    start, offset = s["start"], s["offset"]
    position = start[:, :, None] + (offset if offset.dim() == 3 else offset[:, None])  # [B,axes,S]
    position = position[:, s["axis_of"].long()] if s["axis_of"] is not None else position  # [B,pairs or 1,S]
    angle = position.transpose(1, 2).double() * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]  # [B,1,S,pairs]
    there = (torch.arange(s["S"], device=angle.device) < s["n_rows"][:, None])[:, None, :, None]
    return _rotated(s, s["q"], cos, sin, there, s["q_out"]), _rotated(s, s["k"], cos, sin, there, s["k_out"])


def _rotated(s, x, cos, sin, there, out):
    y, rot = x.float(), s["rot"]
    if s["adjacent"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.where(there, torch.cat((turned, y[..., rot:]), -1).to(x.dtype), out)


def _scores(s, q, k, distance):
    """q [B,Hk,group*N,d], k [B,Hk,M,d], distance [B,Hk or 1,N,M] -> [B,Hk,group,N,M]"""
    B, Hk, M, N = k.shape[0], k.shape[1], k.shape[2], distance.shape[2]
    x = (q @ k.transpose(-1, -2)).view(B, Hk, -1, N, M) * s["scale"]
    if s["cap"]:
        x = s["cap"] * torch.tanh(x / s["cap"])
    if s["slope"] is not None:
        x = x - s["slope"].view(1, Hk, -1, 1, 1) * distance[:, :, None].float()
    return x


def _row_positions(s, own_positions):
    """positions of the cached rows and of the new ones, [B,Hk or 1,L_max + N]"""
    Lm, B = s["k_cache"].shape[2], len(s["seq_lens"])
    rows = s["position"] if s["position"] is not None else (s["dropped"][:, None] + torch.arange(Lm, device="cuda"))[:, None]
    return torch.cat((rows.long(), own_positions[:, None].expand(B, rows.shape[1], -1)), 2)


def _seen(s, distance, rows, among):
    """which rows a query sees, [B,Hk or 1,N,M]; among: its own kind, [B,N,N]"""
    Lm = s["k_cache"].shape[2]
    cached = (torch.arange(Lm, device="cuda") < s["seq_lens"][:, None])[:, None, None] & (rows[..., :Lm] >= 0)[:, :, None] & (distance[..., :Lm] >= 0)
    seen = torch.cat((cached, among[:, None].expand(-1, cached.shape[1], -1, -1)), 3)
    return seen & (distance < s["window"]) if s["window"] else seen


def _plain_attention(s):
    B, H, T, d = s["q"].shape
    Hk = s["k_tree"].shape[1]
    at = (s["seq_lens"] + s["dropped"])[:, None] + s["depth"].long()  # positions of the nodes
    rows = _row_positions(s, at)
    distance = at[:, None, :, None] - rows[:, :, None]
    x = _scores(s, s["q"].float().view(B, Hk, -1, d), torch.cat((s["k_cache"], s["k_tree"]), 2).float(), distance)
    x = x.masked_fill(~_seen(s, distance, rows, s["seen"])[:, :, None], -math.inf)
    most = x.amax(-1, keepdim=True)
    x = torch.exp(x - most)
    total = x.sum(-1, keepdim=True)
    out = (x.view(B, Hk, H // Hk * T, -1) @ torch.cat((s["v_cache"], s["v_tree"]), 2).float()).view(B, H, T, d) / total.view(B, H, T, 1)
    there = torch.arange(T, device="cuda") < s["n_nodes"][:, None, None]
    out = torch.where(there[..., None], out, 0.0).to(s["q"].dtype)
    return out, torch.where(there, (most + torch.log(total)).view(B, H, T), 0.0) if s["lse_out"] is not None else None


def _path_scores(s):
    """the scores of the accepted nodes, [B,Hk,group,P,L_max + P], and which rows each sees"""
    B, H, T, d = s["q"].shape
    Hk, P = s["k_tree"].shape[1], s["accept_path"].shape[1]
    node, step = s["accept_path"].long().clamp(0, T - 1), torch.arange(P, device="cuda")
    there = (step < s["accept_len"][:, None]) & (s["accept_path"] >= 0) & (s["accept_path"] < s["n_nodes"][:, None])
    q = s["q"].gather(2, node[:, None, :, None].expand(B, H, P, d)).float()
    k = torch.cat((s["k_cache"], s["k_tree"].gather(2, node[:, None, :, None].expand(B, Hk, P, d))), 2).float()
    at = (s["seq_lens"] + s["dropped"])[:, None] + step
    rows = _row_positions(s, at)
    distance = at[:, None, :, None] - rows[:, :, None]
    among = (step <= step[:, None]) & there[:, :, None] & there[:, None]
    return _scores(s, q.view(B, Hk, -1, d), k, distance), (_seen(s, distance, rows, among) & there[:, None, :, None])[:, :, None]


def _plain_observe(s):
    B, H, T, d = s["q"].shape
    Hk, Lm, P = s["k_tree"].shape[1], s["k_cache"].shape[2], s["accept_path"].shape[1]
    x, seen = _path_scores(s)
    lse = s["lse"].gather(2, s["accept_path"].long().clamp(0, T - 1)[:, None].expand(B, H, P)).view(B, Hk, H // Hk, P, 1)
    paid = torch.where(seen, torch.exp(x - lse), 0.0).sum((2, 3))  # [B,Hk,L_max + P]
    new = (torch.arange(Lm, device="cuda") - s["seq_lens"][:, None])[:, None]  # which of the path's rows goes here
    is_new = (new >= 0) & (new < s["accept_len"][:, None, None])
    fresh = paid[..., Lm:].gather(2, new.clamp(0, P - 1).expand(B, Hk, Lm))
    weight = torch.where(new < 0, s["decay"] * s["weight"] + paid[..., :Lm], torch.where(is_new, fresh, s["weight_out"]))
    if s["position"] is None:
        return weight, None
    at = (s["seq_lens"] + s["dropped"])[:, None, None] + new
    return weight, torch.where(new < 0, s["position"], torch.where(is_new, at, s["position_out"])).int()


def _plain_evict(s):
    Lm, budget = s["k_cache"].shape[2], s["budget"]
    row, L = torch.arange(Lm, device="cuda"), s["seq_lens"][:, None, None]
    now = L + s["dropped"][:, None, None]
    p, w = s["position"], s["weight"]
    rank = torch.where((p >= now - s["recent"]) | (p < s["sinks"]), math.inf, torch.where(w.isnan(), -math.inf, w))
    rank = torch.where((row < L) & (p >= 0), rank, -math.inf)
    best = rank.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    kept = torch.where(L > budget, torch.zeros_like(p, dtype=torch.bool).scatter(-1, best, True), row < L)
    hole, late = ~kept & (row < budget) & (L > budget), kept & (row >= budget) & (L > budget)
    late = torch.where(late, row, Lm - 1).sort(-1).values  # the rows that move, in order
    source = torch.where(hole, late.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), row)
    few = source[..., :min(Lm, budget), None].expand(-1, -1, -1, s["k_cache"].shape[3])
    s["k_cache"][:, :, :budget] = s["k_cache"].gather(2, few)
    s["v_cache"][:, :, :budget] = s["v_cache"].gather(2, few)
    left = torch.minimum(L, torch.full_like(L, budget))
    return (s["k_cache"], s["v_cache"], left[:, 0, 0], (now - left)[:, 0, 0], torch.where(row < left, p.gather(-1, source), s["position_out"]),
            torch.where(row < left, w.gather(-1, source), s["weight_out"]))


def exact(case, seed):
    s = prepare(case, seed)
    B, Hk, d = case["B"], case["Hk"], case["d"]
    if case["kind"] == "rotary":
        outs = []
        for x, out in ((s["q"], s["q_out"].double()), (s["k"], s["k_out"].double())):
            for b in range(B):
                n = int(s["n_rows"][b])
                y = x[b, :, :n].double()
                r = y.clone()
                for c in range(case["rot"] // 2):
                    axis = int(s["axis_of"][c]) if s["axis_of"] is not None else 0
                    turn = s["offset"][b, axis, :n] if s["offset"].dim() == 3 else s["offset"][b, :n]
                    z = torch.polar(torch.ones(n, dtype=torch.float64, device="cuda"), (turn.double() + float(s["start"][b, axis])) * float(s["inv_freq"][c]))
                    i, j = (2 * c, 2 * c + 1) if case["adjacent"] else (c, c + case["rot"] // 2)
                    t = torch.complex(y[..., i], y[..., j]) * z
                    r[..., i], r[..., j] = t.real, t.imag
                out[b, :, :n] = r
            outs.append(out)
        return tuple(outs)
    if case["kind"] == "evict":
        k, v = s["k_cache"].double(), s["v_cache"].double()
        position, weight = s["position_out"].cpu(), s["weight_out"].double().cpu()
        p_all, w_all, dropped, left = s["position"].cpu(), s["weight"].cpu(), s["dropped"].tolist(), []
        for b, n in enumerate(s["seq_lens"].tolist()):
            left.append(min(n, case["budget"]))
            for h in range(Hk):
                p, w = p_all[b, h, :n].tolist(), w_all[b, h, :n].tolist()
                rank = [(not (x >= n + dropped[b] - case["recent"] or x < case["sinks"]), -y, j) for j, (x, y) in enumerate(zip(p, w))]
                keep = sorted(x[2] for x in sorted(rank, key=lambda x: (x[0], 0.0 if not x[0] else x[1], x[2]))[:left[b]])
                free = iter(sorted(set(range(left[b])) - set(keep)))
                place = {j: j if j < left[b] else next(free) for j in keep}
                to, of = list(place.values()), list(place)
                position[b, h, to], weight[b, h, to] = p_all[b, h, of], w_all[b, h, of].double()
                k[b, h, to], v[b, h, to] = k[b, h, of], v[b, h, of]
        went = [n - m + x for n, m, x in zip(s["seq_lens"].tolist(), left, dropped)]
        return k, v, torch.tensor(left), torch.tensor(went), position, weight
    H, T = case["H"], case["T"]
    group = H // Hk
    if case["kind"] == "observe":
        weight = s["weight_out"].double()
        position = s["position_out"].clone() if s["position"] is not None else None
    else:
        out, lse = torch.zeros(B, H, T, d, dtype=torch.float64, device="cuda"), torch.zeros(B, H, T, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, now = int(s["seq_lens"][b]), int(s["seq_lens"][b] + s["dropped"][b])
        if case["kind"] == "observe":
            nodes = s["accept_path"][b, :int(s["accept_len"][b])].long()
        else:
            nodes = torch.arange(int(s["n_nodes"][b]), device="cuda")
        at = now + s["depth"][b, nodes].double()
        sees = s["seen"][b][nodes][:, nodes]
        for h in range(H):
            hk = h // group
            x = s["q"][b, h, nodes].double() @ torch.cat((s["k_cache"][b, hk, :n], s["k_tree"][b, hk, nodes])).double().T / math.sqrt(d)
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if case["slopes"] or case["window"] or case["evicted"]:
                rows = s["position"][b, hk, :n].double() if case["evicted"] else torch.arange(n, device="cuda").double() + float(s["dropped"][b])
                back = at[:, None] - torch.cat((rows, at))
                x = x - float(s["slope"][h]) * back if case["slopes"] else x
                hidden = torch.cat((back[:, :n] < 0, ~sees), 1)
                hidden = hidden | (back >= case["window"]) if case["window"] else hidden
            else:
                hidden = torch.cat((torch.zeros(len(nodes), n, dtype=torch.bool, device="cuda"), ~sees), 1)
            x[hidden] = -math.inf
            if case["kind"] == "observe":
                paid = torch.exp(x - s["lse"][b, h, nodes].double()[:, None]).sum(0)
                if h % group == 0:
                    total = torch.zeros_like(paid)
                total += paid
                if h % group == group - 1:
                    total[:n] += case["decay"] * s["weight"][b, hk, :n].double()
                    weight[b, hk, :n + len(nodes)] = total
                    if position is not None:
                        position[b, hk, :n], position[b, hk, n:n + len(nodes)] = s["position"][b, hk, :n], at.int()
            else:
                lse[b, h, :len(nodes)] = torch.logsumexp(x, 1)
                out[b, h, :len(nodes)] = torch.softmax(x, 1) @ torch.cat((s["v_cache"][b, hk, :n], s["v_tree"][b, hk, nodes])).double()
    if case["kind"] == "observe":
        return weight, position
    return out, lse if case["lse"] else None
