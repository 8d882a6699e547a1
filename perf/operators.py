"""Serving operators around the tree-verification pass, as cases to time.

Five operators for batches of sequences that share one page pool: the page
map (block tables, row offsets and slot maps made on the GPU from tree indices
and prefix lengths, with the attention's work list), tree attention over the
pool, compaction of the accepted paths in the pool, penalties / biases /
grammar masks on the verification logits with their statistics, and the token
history those penalties read.  ``listed()`` names fixed sizes, ``draw()`` gives
further ones of the same ranges; ``prepare()`` makes what a serving loop has in
hand, ``run()`` makes one pass (in plain torch, or through the binding where
``own`` is true), ``exact()`` gives the same outputs in 64 bits.
"""
import math
import random

import torch

own = False

D = 128
THETA = 10000.0
BF = torch.bfloat16
I32 = torch.int32
INT_MIN = -(1 << 31)
D_MAX = 31
TREES = [(1, 0), (8, 3), (16, 4), (26, 4), (32, 4), (64, 5), (128, 6)]   # nodes, depth cap


# ------------------------------------------------------------------- cases --

def listed():
    return [
        # one sequence early in a reply, one token at a time: the smallest
        # attention call, where latency and launches count
        {"name": "attn_b1_t1_l63", "kind": "attn", "B": 1, "T": 1, "lo": 63, "hi": 63, "page": 16,
         "Hq": 32, "Hkv": 8, "window": 0, "softcap": 0.0, "slopes": False, "mix": 1},
        # eight sequences with grouped queries, trees and prefixes of their own
        {"name": "attn_b8_mixed_gqa", "kind": "attn", "B": 8, "T": 0, "lo": 512, "hi": 16384,
         "page": 64, "Hq": 32, "Hkv": 8, "window": 0, "softcap": 0.0, "slopes": False, "mix": 5},
        # one long document, a 26-node tree at a 128K context
        {"name": "attn_b1_t26_l128k", "kind": "attn", "B": 1, "T": 26, "lo": 131000, "hi": 131000,
         "page": 16, "Hq": 32, "Hkv": 8, "window": 0, "softcap": 0.0, "slopes": False, "mix": 2},
        # a sliding-window layer with capped scores, 32 sequences, small trees
        {"name": "attn_b32_window_cap", "kind": "attn", "B": 32, "T": 8, "lo": 100, "hi": 16384,
         "page": 32, "Hq": 40, "Hkv": 8, "window": 4096, "softcap": 50.0, "slopes": False, "mix": 3},
        # penalties, a grammar and the statistics for one 26-node tree
        {"name": "adjust_b1_t26_v32000", "kind": "adjust", "B": 1, "T": 26, "V": 32000, "bias": False,
         "masks": 4, "mix": 1},
        # eight 128-node trees at a 128256-entry vocabulary, biases too
        {"name": "adjust_b8_t128_v128k", "kind": "adjust", "B": 8, "T": 128, "V": 128256, "bias": True,
         "masks": 32, "mix": 2},
        # the page map of one sequence, and of a full batch of small trees
        {"name": "map_b1", "kind": "map", "B": 1, "T": 26, "lo": 2000, "hi": 2000, "page": 16, "mix": 1},
        {"name": "map_b256", "kind": "map", "B": 256, "T": 0, "lo": 1, "hi": 32768, "page": 16, "mix": 2},
        # one layer's cache after a 26-node tree, and all 32 layers of a batch
        {"name": "compact_b1_1layer", "kind": "compact", "B": 1, "T": 26, "lo": 2000, "hi": 2000,
         "page": 16, "Hkv": 8, "layers": 1, "mix": 1},
        {"name": "compact_b32_32layer", "kind": "compact", "B": 32, "T": 64, "lo": 100, "hi": 1000,
         "page": 32, "Hkv": 8, "layers": 32, "mix": 2},
        # what a step accepted enters the history of a small batch; prompts of a large one
        {"name": "history_accept_b16", "kind": "accept", "B": 16, "T": 26, "V": 128256, "mix": 1},
        {"name": "history_prompt_b64", "kind": "prompt", "B": 64, "V": 128256, "lo": 100, "hi": 32768,
         "mix": 2},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "adjust", "adjust", "map", "compact", "accept", "prompt"])
    T = rng.choice([0, 1, 8, 16, 26, 32, 64, 128])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    mix = rng.randint(10, 10 ** 6)
    V = rng.choice([32000, 50257, 128256, rng.randint(16000, 128256)])
    if kind == "attn":
        Hq, Hkv = rng.choice([(32, 8), (32, 8), (32, 32), (40, 8), (28, 4), (16, 1)])
        B = _log_int(rng, 1, 64)
        # tokens x KV heads of the whole call, and rows x keys, stay within the largest listed case's
        hi = int(min(131072, 131072 * 8 / (B * Hkv), 131072 * 26 * 32 / (B * (T or 128) * Hq)))
        hi = _log_int(rng, 32, max(32, hi))
        opt = rng.random()
        return {"kind": kind, "B": B, "T": T, "lo": rng.choice([1, max(1, hi // 8), hi]), "hi": hi,
                "page": page, "Hq": Hq, "Hkv": Hkv,
                "window": _log_int(rng, 16, 8192) if opt < 0.3 else 0,
                "softcap": rng.choice([0.0, 30.0, 50.0]) if opt < 0.4 else 0.0,
                "slopes": 0.4 <= opt < 0.6, "mix": mix}
    if kind == "adjust":
        most = 1024 * 128256 // V
        B = _log_int(rng, 1, 64)
        return {"kind": kind, "B": min(B, max(1, most // (T or 128))), "T": T, "V": V,
                "bias": rng.random() < 0.5, "masks": rng.choice([0, 1, 16]), "mix": mix}
    if kind == "map":
        return {"kind": kind, "B": _log_int(rng, 1, 256), "T": T, "lo": 1, "hi": _log_int(rng, 64, 32768),
                "page": page, "mix": mix}
    if kind == "compact":
        return {"kind": kind, "B": _log_int(rng, 1, 32), "T": max(T, 8), "lo": 1,
                "hi": _log_int(rng, 64, 1000), "page": page, "Hkv": rng.choice([1, 4, 8]),
                "layers": _log_int(rng, 1, 32), "mix": mix}
    if kind == "accept":
        return {"kind": kind, "B": _log_int(rng, 1, 64), "T": max(T, 1), "V": V, "mix": mix}
    return {"kind": kind, "B": _log_int(rng, 1, 64), "V": V, "lo": 1, "hi": _log_int(rng, 16, 32768),
            "mix": mix}


# ------------------------------------------------------------------ shapes --

def _tree(n, cap):
    """Parent array of a tree grown node by node under a depth cap."""
    r = random.Random(1000 * n + cap)
    parent, depth = [-1], [0]
    while len(parent) < n:
        p = r.choice([j for j in range(len(parent)) if depth[j] < cap])
        parent.append(p)
        depth.append(depth[p] + 1)
    return parent


_forest_cache = []


def _forest():
    """The bank's trees: parents, node counts, depths, ancestor masks and paths (on the CPU)."""
    if not _forest_cache:
        n, m = len(TREES), max(t for t, _ in TREES)
        trees = [_tree(*t) for t in TREES]
        depth = torch.zeros((n, m), dtype=torch.long)
        anc = torch.zeros((n, m, m), dtype=torch.bool)
        path = torch.full((n, m, D_MAX + 1), -1, dtype=torch.long)
        for k, parent in enumerate(trees):
            for i in range(len(parent)):
                chain = [i]
                while parent[chain[-1]] >= 0:
                    chain.append(parent[chain[-1]])
                chain.reverse()
                depth[k, i] = len(chain) - 1
                anc[k, i, chain] = True
                path[k, i, :len(chain)] = torch.tensor(chain)
        _forest_cache.append({"trees": trees, "T": torch.tensor([t for t, _ in TREES]), "depth": depth,
                              "anc": anc, "path": path})
    return _forest_cache[0]


def _batch(case):
    """Tree index and prefix length of every sequence: the case's own, whatever the seed."""
    r = random.Random(case["mix"])
    index = {t: k for k, (t, _) in enumerate(TREES)}
    topo = [index[case["T"]] if case["T"] else r.randrange(len(TREES)) for _ in range(case["B"])]
    lens = [r.randint(case["lo"], case["hi"]) for _ in range(case["B"])] if "lo" in case else None
    return topo, lens


def _sizes(topo):
    return [TREES[t][0] for t in topo]


def _prompt_lens(case):
    r = random.Random(case["mix"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["B"])]


# ------------------------------------------------------------------ inputs --

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=BF)


def _i32(v):
    return torch.tensor(v, dtype=I32, device="cuda")


def _row_off(topo):
    off = [0]
    for t in _sizes(topo):
        off.append(off[-1] + t)
    return off


def _pages(case, g, topo, lens, spare=3):
    """Block table [B, max_pages] of randomly placed pages that hold every
    prefix and tree, and the number of pages in the pool."""
    page, B = case["page"], case["B"]
    need = [-(-(n + t) // page) for n, t in zip(lens, _sizes(topo))]
    most, total = max(need) + 2, sum(need)
    order = torch.randperm(total + spare, generator=g, device="cuda")[:total].to(I32)
    n = torch.tensor(need, device="cuda")
    held = torch.arange(most, device="cuda")[None] < n[:, None]
    table = torch.full((B, most), -1, dtype=I32, device="cuda")
    table[held] = order
    return table, total + spare


def _slots(case, table, topo, lens):
    """Pool slot of every tree row, in row order."""
    sizes = _sizes(topo)
    seq = torch.repeat_interleave(torch.arange(case["B"]), torch.tensor(sizes)).cuda()
    pos = torch.cat([torch.arange(n, n + t) for n, t in zip(lens, sizes)]).cuda()
    p = case["page"]
    return (table[seq, pos // p].long() * p + pos % p).to(I32)


def _accepted(g, case, topo):
    """Accept lengths and paths [B, D_MAX + 1] of random nodes of the trees."""
    f = _forest()
    node = (torch.rand(case["B"], generator=g, device="cuda").cpu() * f["T"][topo]).long()
    path = f["path"][topo, node]
    return (path >= 0).sum(1).sub(1).to(I32).cuda(), path.to(I32).cuda()


def _inputs(case, seed):
    """The tensors the seed decides."""
    g, kind = _gen(seed), case["kind"]
    if kind == "prompt":
        lens = _prompt_lens(case)
        off = [0]
        for n in lens:
            off.append(off[-1] + n)
        # a text's tokens: some far more often than others
        u = torch.rand(off[-1], generator=g, device="cuda")
        return {"tok": (u.pow(3) * case["V"]).to(I32), "off": _i32(off),
                "history": torch.zeros((case["B"], case["V"]), dtype=I32, device="cuda")}
    topo, lens = _batch(case)
    rows = sum(_sizes(topo))
    s = {"topo": _i32(topo), "row_off": _i32(_row_off(topo))}
    if kind == "attn":
        table, n_pages = _pages(case, g, topo, lens)
        shape = (n_pages, case["Hkv"], case["page"], D)
        s.update(lens=_i32(lens), table=table, slots=_slots(case, table, topo, lens),
                 q=_normal(g, rows, case["Hq"], D).mul_(1.5), k=_normal(g, rows, case["Hkv"], D),
                 v=_normal(g, rows, case["Hkv"], D), kp=_normal(g, *shape), vp=_normal(g, *shape),
                 slopes=None)
        if case["slopes"]:   # a geometric row of slopes over the heads
            s["slopes"] = torch.exp2(-8.0 * torch.arange(1, case["Hq"] + 1, device="cuda") / case["Hq"])
    elif kind == "map":
        table, n_pages = _pages(case, g, topo, lens, spare=40)
        # the prefixes' pages are held, the trees' are still to be taken
        p = case["page"]
        held = _i32([-(-n // p) for n in lens])
        cols = torch.arange(table.shape[1], device="cuda")[None]
        tree = (cols >= held[:, None]) & (table >= 0)
        used = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
        used[table[(table >= 0) & ~tree].long()] = True
        table[tree] = -1
        free = torch.arange(n_pages, device="cuda", dtype=I32)[~used]
        free = free[torch.randperm(free.numel(), generator=g, device="cuda")]
        s.update(lens=_i32(lens), table=table, free=free.contiguous(), n_free=_i32([free.numel()]),
                 n_pages=n_pages)
    elif kind == "compact":
        table, n_pages = _pages(case, g, topo, lens)
        a, path = _accepted(g, case, topo)
        shape = (case["layers"], n_pages, case["Hkv"], case["page"], D)
        s.update(a=a, path=path, slots=_slots(case, table, topo, lens), kp=_normal(g, *shape),
                 vp=_normal(g, *shape))
    elif kind == "accept":
        a, path = _accepted(g, case, topo)
        V = case["V"]
        s.update(a=a, path=path, tok=torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=I32),
                 bonus=torch.randint(0, V, (case["B"],), generator=g, device="cuda", dtype=I32),
                 history=torch.randint(0, 3, (case["B"], V), generator=g, device="cuda", dtype=I32))
    else:
        V, B = case["V"], case["B"]
        z = torch.randn((rows, V), generator=g, device="cuda").mul_(2.5)
        # every row's likely tokens, drafted and repeated ones among them, stand out
        top = torch.randint(0, V, (rows, 6), generator=g, device="cuda")
        z.scatter_add_(1, top, 8 + 4 * torch.rand((rows, 6), generator=g, device="cuda"))
        tok = top[:, 0].to(I32)
        hist = torch.zeros((B, V), dtype=I32, device="cuda")
        said = (torch.rand((B, 600), generator=g, device="cuda").pow(3) * V).long()
        hist.scatter_add_(1, said, torch.ones_like(said, dtype=I32))
        seen = (torch.rand((B, 900), generator=g, device="cuda").pow(3) * V).long()
        hist.scatter_(1, seen, hist.gather(1, seen) | INT_MIN)
        u = torch.rand((B, 4), generator=g, device="cuda")
        params = torch.stack([1 + 0.3 * u[:, 0], 0.5 * u[:, 1], 0.5 * u[:, 2], 1 / (0.5 + u[:, 3])], 1)
        s.update(z=z, tok=tok, history=hist, params=params.contiguous(), bias=None, bias_idx=None,
                 mask=None, mask_idx=None)
        if case["bias"]:
            n = max(1, B // 2)
            bias = torch.zeros((n, V), device="cuda")
            at = torch.randint(0, V, (n, 300), generator=g, device="cuda")
            s["bias"] = bias.scatter_(1, at, 4 * torch.randn((n, 300), generator=g, device="cuda"))
            s["bias_idx"] = torch.randint(-1, n, (B,), generator=g, device="cuda", dtype=I32)
        if case["masks"]:
            words = -(-V // 32)
            s["mask"] = torch.randint(INT_MIN, 1 << 31, (case["masks"], words), generator=g,
                                      device="cuda", dtype=torch.int64).to(I32)
            s["mask_idx"] = torch.randint(-1, case["masks"], (rows,), generator=g, device="cuda", dtype=I32)
    return s


def prepare(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    s["case"] = case
    if kind == "prompt":
        return s
    f = _forest()
    rows, B = int(sum(_sizes(_batch(case)[0]))), case["B"]
    s["rows"] = rows
    s["forest"] = {k: f[k].cuda() for k in ("T", "depth", "anc", "path")}
    new = lambda n, dtype=I32: torch.zeros(n, dtype=dtype, device="cuda")  # noqa: E731
    if kind == "attn":
        s["out"] = torch.zeros_like(s["q"])
        s["status"] = new(B)
    elif kind == "map":
        s["new_off"], s["new_slots"], s["status"] = new(B + 1), new(rows), new(B)
    elif kind == "adjust":
        s["out"] = torch.zeros_like(s["z"])
        s["entropy"], s["top1p"] = new(rows, torch.float32), new(rows, torch.float32)
        s["top"] = new(rows)
    if own:   # the handles, workspaces and work list that a serving loop keeps
        from paper_2606_27550_amd import api
        byte = lambda n: torch.empty(max(int(n), 256), dtype=torch.uint8, device="cuda")  # noqa: E731
        s["bank"] = api.Bank(f["trees"])
        if kind == "attn":
            shape = (rows, case["Hq"], case["Hkv"])
            s["plan"] = byte(api.tree_attn_paged_plan_bytes(s["bank"], B, *shape, s["table"].shape[1],
                                                            case["page"]))
            api.tree_attn_paged_plan(s["bank"], s["topo"], s["lens"], s["row_off"], s["status"],
                                     s["table"], case["page"], s["kp"].shape[0], *shape, s["plan"],
                                     window=case["window"])
            s["ws"] = byte(api.tree_attn_paged_workspace(s["bank"], B, *shape, D, s["table"].shape[1],
                                                         case["page"]))
        elif kind == "map":
            s["plan"] = byte(api.tree_attn_paged_plan_bytes(s["bank"], B, rows, 32, 8, s["table"].shape[1],
                                                            case["page"]))
        elif kind == "adjust":
            s["ws"] = byte(api.logit_adjust_workspace(rows, case["V"]))
    return s


# -------------------------------------------------------------------- pass --

def run(s):
    kind = s["case"]["kind"]
    if own:
        return _run_own(s, kind)
    return {"attn": _plain_attn, "map": _plain_map, "compact": _plain_compact, "adjust": _plain_adjust,
            "accept": _plain_accept, "prompt": _plain_prompt}[kind](s)


def _run_own(s, kind):
    from paper_2606_27550_amd import api
    case = s["case"]
    if kind == "attn":
        api.tree_attn_paged(s["bank"], s["plan"], s["q"], s["k"], s["v"], s["kp"], s["vp"], s["table"],
                            s["slots"], 1 / math.sqrt(D), THETA, s["out"], s["ws"],
                            softcap=case["softcap"], window=case["window"], slopes=s["slopes"])
        return {"out": s["out"], "kp": s["kp"], "vp": s["vp"]}
    if kind == "map":
        api.page_map(s["bank"], s["topo"], s["lens"], s["table"], case["page"], s["n_pages"],
                     s["new_off"], s["new_slots"], s["status"], free_pages=s["free"], n_free=s["n_free"])
        api.tree_attn_paged_plan(s["bank"], s["topo"], s["lens"], s["new_off"], s["status"], s["table"],
                                 case["page"], s["n_pages"], s["rows"], 32, 8, s["plan"])
        return _map_outputs(s)
    if kind == "compact":
        api.kv_compact_paged(s["path"], s["a"], s["row_off"], s["slots"], s["kp"], s["vp"])
        return {"kp": s["kp"], "vp": s["vp"]}
    if kind == "adjust":
        api.logit_adjust(s["bank"], s["topo"], s["row_off"], s["tok"], s["z"], s["params"], s["out"],
                         s["entropy"], s["top1p"], s["top"], s["ws"], history=s["history"],
                         bias=s["bias"], bias_idx=s["bias_idx"], mask=s["mask"], mask_idx=s["mask_idx"])
        return {"out": s["out"], "entropy": s["entropy"], "top1p": s["top1p"], "top": s["top"]}
    if kind == "accept":
        api.token_history_accept(s["row_off"], s["tok"], s["path"], s["a"], s["bonus"], s["history"])
        return {"history": s["history"]}
    api.token_history_prompt(s["tok"], s["off"], s["history"])
    return {"history": s["history"]}


def _map_outputs(s):
    return {"table": s["table"], "row_off": s["new_off"], "slots": s["new_slots"], "status": s["status"],
            "n_free": s["n_free"]}


# ------------------------------------------------------------- plain forms --

def _rope(x, pos):
    """x [rows, H, D] turned to positions pos [rows], in 64 bits (pairs c, c + D / 2)."""
    h = D // 2
    f = THETA ** (-2.0 * torch.arange(h, device="cuda", dtype=torch.float64) / D)
    a = pos.double()[:, None, None] * f
    lo, hi = x[..., :h].double(), x[..., h:].double()
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)


def _rows_of(s):
    """Sequence and node of every tree row."""
    T = s["forest"]["T"][s["topo"].long()]
    seq = torch.repeat_interleave(torch.arange(T.numel(), device="cuda"), T, output_size=s["rows"])
    return seq, torch.arange(s["rows"], device="cuda") - s["row_off"].long()[seq]


def _plain_attn(s):
    case, f = s["case"], s["forest"]
    B, Hq, Hkv, page = case["B"], case["Hq"], case["Hkv"], case["page"]
    G, n = Hq // Hkv, max(_sizes(_batch(case)[0]))
    topo, L = s["topo"].long(), s["lens"].long()
    seq, node = _rows_of(s)
    pos = L[seq] + f["depth"][topo[seq], node]
    slot = s["slots"].long()
    s["kp"][slot // page, :, slot % page] = _rope(s["k"], pos).to(BF)
    s["vp"][slot // page, :, slot % page] = s["v"]
    # every sequence's keys and values side by side, padded to the longest
    longest = max(x + t for x, t in zip(_batch(case)[1], _sizes(_batch(case)[0])))
    cols = -(-longest // page)
    table = s["table"][:, :cols].clamp(min=0).long()

    def dense(pool):
        x = pool[table].permute(0, 2, 1, 3, 4)
        return x.reshape(B, Hkv, cols * page, D).float()

    q = torch.zeros((B, n, Hq, D), device="cuda")
    q[seq, node] = _rope(s["q"], pos).float()
    q = q.reshape(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    z = torch.matmul(q, dense(s["kp"]).transpose(2, 3)).mul_(1 / math.sqrt(D)).view(B, Hkv, G, n, -1)
    if case["softcap"]:
        z = torch.tanh(z / case["softcap"]) * case["softcap"]
    # slot j of a sequence: prefix position j, or tree node j - L
    j = torch.arange(cols * page, device="cuda")
    jn = (j[None] - L[:, None])
    tree = (jn >= 0) & (jn < f["T"][topo][:, None])
    jn = jn.clamp(0, n - 1)
    at = torch.where(tree, L[:, None] + f["depth"][topo].gather(1, jn), j[None])   # [B, keys]
    far = (L[:, None] + f["depth"][topo][:, :n])[:, :, None] - at[:, None]         # [B, n, keys]
    sees = f["anc"][topo][:, :n].gather(2, jn[:, None].expand(B, n, -1)) & tree[:, None]
    sees = sees | (j[None] < L[:, None])[:, None]
    if case["window"]:
        sees = sees & (far < case["window"])
    if s["slopes"] is not None:
        z = z - s["slopes"].view(1, Hkv, G, 1, 1) * far[:, None, None].float()
    z = z.masked_fill(~sees[:, None, None], -math.inf)
    z = (z - z.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    z = z / z.sum(-1, keepdim=True)
    o = torch.matmul(z.view(B, Hkv, G * n, -1), dense(s["vp"]))
    o = o.view(B, Hkv, G, n, D).permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)
    s["out"].copy_(o[seq, node])
    return {"out": s["out"], "kp": s["kp"], "vp": s["vp"]}


def _plain_map(s):
    case, f = s["case"], s["forest"]
    page, table = case["page"], s["table"]
    T, L = f["T"][s["topo"].long()], s["lens"].long()
    s["new_off"][1:] = torch.cumsum(T, 0)
    cols = torch.arange(table.shape[1], device="cuda")[None]
    lack = (cols >= (L // page)[:, None]) & (cols <= ((L + T - 1) // page)[:, None]) & (table < 0)
    k = torch.cumsum(lack.reshape(-1).long(), 0).view_as(lack)   # the k-th page taken, from one
    served = lack & (k[:, -1:] <= s["n_free"])
    at = torch.minimum(s["n_free"] - k, s["n_free"] - 1).clamp(0, s["free"].numel() - 1).long()
    table.copy_(torch.where(served, s["free"][at], table))
    s["n_free"].sub_(served.sum())
    seq = torch.repeat_interleave(torch.arange(T.numel(), device="cuda"), T, output_size=s["rows"])
    pos = L[seq] + torch.arange(s["rows"], device="cuda") - s["new_off"].long()[seq]
    s["new_slots"].copy_(table[seq, pos // page] * page + pos % page)
    s["status"].copy_((lack & ~served).any(1) * 3)
    return _map_outputs(s)


def _plain_compact(s):
    page = s["case"]["page"]
    j = torch.arange(s["path"].shape[1], device="cuda")[None]
    keep = j <= s["a"][:, None]
    seq, j = torch.nonzero(keep & (s["path"] != j), as_tuple=True)   # rows that move
    off = s["row_off"].long()[seq]
    src, dst = s["slots"][off + s["path"][seq, j].long()].long(), s["slots"][off + j].long()
    for pool in (s["kp"], s["vp"]):
        pool[:, dst // page, :, dst % page] = pool[:, src // page, :, src % page]
    return {"kp": s["kp"], "vp": s["vp"]}


def _plain_adjust(s):
    f, topo = s["forest"], s["topo"].long()
    seq, node = _rows_of(s)
    z, p = s["z"], s["params"][seq]
    hist = s["history"][seq]
    # drafted tokens on the way from the root to the node count as said
    path = f["path"][topo[seq], node][:, 1:]
    tok = s["tok"][(s["row_off"].long()[seq][:, None] + path).clamp(0, s["rows"] - 1)].long()
    said = (hist & 0x7FFFFFFF).scatter_add_(1, tok, (path >= 0).to(I32))
    rep, freq, pres, it = p[:, 0:1], p[:, 1:2], p[:, 2:3], p[:, 3:4]
    z = torch.where((said > 0) | (hist < 0), torch.where(z > 0, z / rep, z * rep), z)
    z = z - freq * said.float()
    z = z - pres * (said > 0).float()
    if s["bias"] is not None:
        i = s["bias_idx"][seq]
        z = torch.where((i >= 0)[:, None], z + s["bias"][i.clamp(min=0).long()], z)
    if s["mask"] is not None:
        i = s["mask_idx"]
        v = torch.arange(z.shape[1], device="cuda")
        bit = (s["mask"][i.clamp(min=0).long()][:, v // 32] >> (v % 32)) & 1
        z = z.masked_fill((bit == 0) & (i >= 0)[:, None], -math.inf)
    m, top = z.amax(1, keepdim=True), z.argmax(1)
    some = m > -math.inf
    t = (z - torch.where(some, m, 0.0)) * it
    e = t.exp()
    Z, S = e.sum(1), torch.where(e > 0, t * e, 0.0).sum(1)
    s["out"].copy_(z)
    s["top"].copy_(torch.where(some[:, 0], top, -1))
    s["top1p"].copy_(torch.where(some[:, 0], 1 / Z, 0.0))
    s["entropy"].copy_(torch.where(some[:, 0], Z.log() - S / Z, 0.0))
    return {"out": s["out"], "entropy": s["entropy"], "top1p": s["top1p"], "top": s["top"]}


def _plain_accept(s):
    B, V = s["history"].shape
    j = torch.arange(s["path"].shape[1], device="cuda")[None]
    node = (s["row_off"].long()[:-1, None] + s["path"]).clamp(0, s["rows"] - 1)
    tok = torch.cat([s["tok"][node].long(), s["bonus"].long()[:, None]], 1)
    new = torch.cat([(j >= 1) & (j <= s["a"][:, None]), (s["a"] >= 0)[:, None]], 1)
    s["history"].scatter_add_(1, tok, new.to(I32))
    return {"history": s["history"]}


def _plain_prompt(s):
    h = s["history"]
    n = s["off"].long().diff()
    seq = torch.repeat_interleave(torch.arange(n.numel(), device="cuda"), n, output_size=s["tok"].numel())
    at = seq * h.shape[1] + s["tok"].long()
    h.view(-1)[at] = h.view(-1)[at] | INT_MIN
    return {"history": h}


# ------------------------------------------------------------------- floor --

def work(case):
    kind = case["kind"]
    if kind == "prompt":
        n = sum(_prompt_lens(case))
        return {"bytes": 12 * n, "flops": 0}   # a token read, its counter read and written
    topo, lens = _batch(case)
    sizes = _sizes(topo)
    rows = sum(sizes)
    if kind == "attn":
        w = case["window"] or 1 << 30
        keys = [min(n, w + TREES[t][1]) for n, t in zip(lens, topo)]
        b = sum(keys) * 2 * case["Hkv"] * D * 2 + rows * (2 * case["Hq"] + 4 * case["Hkv"]) * D * 2
        return {"bytes": b, "flops": sum(4 * case["Hq"] * D * t * (min(n, w) + (t + 1) / 2)
                                         for n, t in zip(keys, sizes))}
    if kind == "map":
        pages = sum(-(-(n + t) // case["page"]) for n, t in zip(lens, sizes))
        return {"bytes": 4 * (pages + rows + 5 * case["B"]), "flops": 0}
    if kind == "compact":
        # about half of a tree's depth is accepted, all but the root's row moves
        moved = sum(TREES[t][1] / 2 for t in topo)
        return {"bytes": 2 * moved * 2 * case["Hkv"] * D * 2 * case["layers"] + 12 * moved, "flops": 0}
    if kind == "accept":
        return {"bytes": sum(12 * (TREES[t][1] / 2 + 1) for t in topo), "flops": 0}
    V = case["V"]
    shared = 4 * V * case["B"] * (2 if case["bias"] else 1) + case["masks"] * V / 8
    return {"bytes": 8 * rows * V + shared, "flops": 12 * rows * V}


# --------------------------------------------------------------- in 64 bits --

def _turn(x, pos):
    c = torch.arange(D // 2, device="cuda", dtype=torch.float64)
    w = torch.polar(torch.ones_like(c), float(pos) * THETA ** (-2 * c / D))
    y = torch.complex(x[..., :D // 2].double(), x[..., D // 2:].double()) * w
    return torch.cat([y.real, y.imag], -1)


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind in ("map", "accept", "prompt"):
        return None   # whole numbers
    f = _forest()
    topo, lens = _batch(case)
    off = _row_off(topo)
    if kind == "compact":
        page, slots = case["page"], s["slots"].tolist()
        outs = {"kp": s["kp"].double(), "vp": s["vp"].double()}
        for b, a in enumerate(s["a"].tolist()):
            for j, node in enumerate(s["path"][b, :a + 1].tolist()):
                src, dst = slots[off[b] + node], slots[off[b] + j]
                for pool in ("kp", "vp"):   # the sources as they were at first
                    outs[pool][:, dst // page, :, dst % page] = s[pool][:, src // page, :, src % page].double()
        return outs
    if kind == "attn":
        # pass over (sequence, KV head): its keys by slot, the tree's rotated anew
        page, G = case["page"], case["Hq"] // case["Hkv"]
        if case["B"] * case["Hkv"] > 1024:
            return None
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for b, (t, L) in enumerate(zip(topo, lens)):
            T, r0 = TREES[t][0], off[b]
            depth = f["depth"][t, :T].tolist()
            pages = s["table"][b, :-(-(L + T) // page)].long()
            kt = torch.stack([_turn(s["k"][r0 + i], L + depth[i]) for i in range(T)]).to(BF).double()
            qt = torch.stack([_turn(s["q"][r0 + i], L + depth[i]) for i in range(T)])
            first = max(0, L + 1 - case["window"]) if case["window"] else 0
            where = torch.cat([torch.arange(first, L), L + torch.tensor(depth)]).cuda().double()
            dist = (L + torch.tensor(depth).cuda().double())[:, None] - where[None]
            ok = torch.cat([torch.ones((T, L - first), dtype=torch.bool), f["anc"][t, :T, :T]], 1).cuda()
            if case["window"]:
                ok &= dist < case["window"]
            for g in range(case["Hkv"]):
                k = torch.cat([s["kp"][pages, g].reshape(-1, D)[first:L].double(), kt[:, g]])
                v = torch.cat([s["vp"][pages, g].reshape(-1, D)[first:L].double(),
                               s["v"][r0:r0 + T, g].double()])
                for h in range(g * G, g * G + G):
                    z = qt[:, h] @ k.t() / math.sqrt(D)
                    if case["softcap"]:
                        z = case["softcap"] * torch.tanh(z / case["softcap"])
                    if s["slopes"] is not None:
                        z = z - s["slopes"][h].double() * dist
                    z[~ok] = -math.inf
                    out[r0:r0 + T, h] = torch.softmax(z, 1) @ v
        return {"out": out, "kp": None, "vp": None}
    outs = {"out": torch.zeros(s["z"].shape, dtype=torch.float64, device="cuda"), "top": None,
            "entropy": torch.zeros(off[-1], dtype=torch.float64, device="cuda"),
            "top1p": torch.zeros(off[-1], dtype=torch.float64, device="cuda")}
    for b, t in enumerate(topo):
        rep, freq, pres, it = s["params"][b].double().tolist()
        base = (s["history"][b] & 0x7FFFFFFF).double()
        for i in range(TREES[t][0]):
            r = off[b] + i
            count = base.clone()
            for node in f["path"][t, i, 1:].tolist():
                if node >= 0:
                    count[s["tok"][off[b] + node]] += 1
            z = s["z"][r].double()
            seen = (count > 0) | (s["history"][b] < 0)
            z = torch.where(seen, torch.where(z > 0, z / rep, z * rep), z) - freq * count - pres * (count > 0)
            if s["bias"] is not None and s["bias_idx"][b] >= 0:
                z += s["bias"][s["bias_idx"][b]].double()
            if s["mask"] is not None and s["mask_idx"][r] >= 0:
                word = s["mask"][s["mask_idx"][r]]
                v = torch.arange(z.numel(), device="cuda")
                z[((word[v >> 5] >> (v & 31)) & 1) == 0] = -math.inf
            outs["out"][r] = z
            logp = torch.log_softmax(z * it, 0)
            p = logp.exp()
            outs["top1p"][r] = p.max()
            outs["entropy"][r] = -(p * logp)[p > 0].sum()
    return outs
