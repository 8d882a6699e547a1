"""Operators of a 4-bit page pool and a 4-bit LM head, as cases to time.

Four operators that belong together in a verification step whose cache and
LM-head weights are held in 4 bits: queries and keys of new rows are normed per
head, rotated to their positions and appended to the pages (``append``; also to
bf16 pages), the tree's rows attend over the pages (``attn``), the accepted
path's rows are moved up (``compact``) and the logits are taken from 4-bit
weights with group scales (``logits``).  ``listed()`` names fixed sizes,
``draw()`` gives further ones of the same ranges; ``prepare()`` makes what a
serving loop has in hand, ``run()`` makes one pass (in plain torch, or through
the binding where ``own`` is true), ``exact()`` gives the same outputs in 64 bits.

Four bits: a row's values in groups of 32 along the row; a group has one scale
byte b, 2^(b - 127) (255: not a number), and a code per value, sign and one of
0, 1/2, 1, 3/2, 2, 3, 4, 6, two codes a byte, the lower half first.  Rows of a
page's head lie as page_size x 64 bytes of codes, then page_size x 4 of scales.
"""
import math
import random

import torch

own = False

D = 128
THETA = 10000.0
EPS = 1e-6
BF = torch.bfloat16
I32 = torch.int32
U8 = torch.uint8
D_MAX = 31
TREES = [(1, 0), (8, 3), (16, 4), (26, 4), (32, 4), (64, 5), (128, 6)]   # nodes, depth cap
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------- cases --

def listed():
    return [
        # one sequence early in a reply, one token at a time: the smallest
        # attention call, where latency and launches count
        {"name": "attn4_b1_t1_l63", "kind": "attn", "B": 1, "T": 1, "lo": 63, "hi": 63, "page": 16,
         "Hq": 32, "Hkv": 8, "window": 0, "softcap": 0.0, "slopes": False, "mix": 1},
        # plain decoding of a full batch, a token a sequence: the cache's bytes
        {"name": "attn4_b32_t1_l8k", "kind": "attn", "B": 32, "T": 1, "lo": 8192, "hi": 8192,
         "page": 64, "Hq": 32, "Hkv": 8, "window": 0, "softcap": 0.0, "slopes": False, "mix": 2},
        # one long document, a 26-node tree at a 128K context
        {"name": "attn4_b1_t26_l128k", "kind": "attn", "B": 1, "T": 26, "lo": 131000, "hi": 131000,
         "page": 16, "Hq": 32, "Hkv": 8, "window": 0, "softcap": 0.0, "slopes": False, "mix": 3},
        # eight sequences with trees and prefixes of their own, the large trees
        # bound by the products
        {"name": "attn4_b8_mixed", "kind": "attn", "B": 8, "T": 0, "lo": 512, "hi": 16384,
         "page": 64, "Hq": 32, "Hkv": 8, "window": 0, "softcap": 0.0, "slopes": False, "mix": 5},
        # the rows of one step's trees, normed, rotated and stored in 4 bits: a few rows
        {"name": "append4_b8_t26", "kind": "append", "B": 8, "T": 26, "lo": 300, "hi": 4000, "page": 64,
         "Hq": 32, "Hkv": 8, "norm": True, "bits": 4, "mix": 1},
        # three prompts on their way into 4-bit pages
        {"name": "append4_prompt_8k", "kind": "append", "B": 3, "T": -1, "lo": 2000, "hi": 3400, "page": 16,
         "Hq": 32, "Hkv": 8, "norm": True, "bits": 4, "mix": 2},
        # two prompts of ragged lengths into bf16 pages, every head its own keys, no norm
        {"name": "append16_prompt_4k", "kind": "append", "B": 2, "T": -1, "lo": 1500, "hi": 2500, "page": 32,
         "Hq": 40, "Hkv": 40, "norm": False, "bits": 16, "mix": 3},
        # one sequence's accepted path in one layer, and a batch's in 32 layers
        {"name": "compact4_b1_1layer", "kind": "compact", "B": 1, "T": 26, "lo": 300, "hi": 300, "page": 16,
         "Hkv": 8, "layers": 1, "mix": 4},
        {"name": "compact4_b32_32layer", "kind": "compact", "B": 32, "T": 64, "lo": 100, "hi": 1000, "page": 32,
         "Hkv": 8, "layers": 32, "mix": 5},
        # the LM head of a single token, of a 27-node tree with a large
        # vocabulary, and of a 128-node tree
        {"name": "logits4_t1_v32000", "kind": "logits", "T": 1, "V": 32000, "hid": 4096, "mix": 1},
        {"name": "logits4_t27_v128256", "kind": "logits", "T": 27, "V": 128256, "hid": 4096, "mix": 2},
        {"name": "logits4_t128_v32000", "kind": "logits", "T": 128, "V": 32000, "hid": 5120, "mix": 3},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "append", "compact", "logits", "logits"])
    T = rng.choice([0, 1, 1, 8, 16, 26, 32, 64, 128])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    mix = rng.randint(10, 10 ** 6)
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (32, 32), (40, 8), (28, 4), (16, 1)])
    if kind == "attn":
        B = _log_int(rng, 1, 64)
        # tokens x KV heads of the whole call, and rows x keys, stay within the largest listed cases'
        hi = int(min(131072, 8192 * 32 * 8 / (B * Hkv), 131072 * 26 * 32 / (B * (T or 128) * Hq)))
        hi = _log_int(rng, 32, max(32, hi))
        opt = rng.random()
        return {"kind": kind, "B": B, "T": T, "lo": rng.choice([1, max(1, hi // 8), hi]), "hi": hi,
                "page": page, "Hq": Hq, "Hkv": Hkv,
                "window": _log_int(rng, 16, 8192) if opt < 0.3 else 0,
                "softcap": rng.choice([0.0, 30.0, 50.0]) if opt < 0.4 else 0.0,
                "slopes": 0.4 <= opt < 0.6, "mix": mix}
    if kind == "append":
        B = _log_int(rng, 1, 32)
        T = rng.choice([T, -1])
        hi = _log_int(rng, 1, max(1, 8192 * 48 // (B * (Hq + 2 * Hkv)))) if T < 0 else _log_int(rng, 1, 30000)
        return {"kind": kind, "B": B, "T": T, "lo": max(1, hi // 2), "hi": hi, "page": page, "Hq": Hq, "Hkv": Hkv,
                "norm": rng.random() < 0.6, "bits": rng.choice([4, 4, 16]), "mix": mix}
    if kind == "compact":
        return {"kind": kind, "B": _log_int(rng, 1, 32), "T": max(T, 8), "lo": 1,
                "hi": _log_int(rng, 64, 1000), "page": page, "Hkv": rng.choice([1, 4, 8]),
                "layers": _log_int(rng, 1, 32), "mix": mix}
    V = rng.choice([32000, 50257, 128256, rng.randint(16000, 128256)])
    hid = rng.choice([1024, 2048, 4096, 5120, 32 * rng.randint(20, 200)])
    return {"kind": kind, "T": _log_int(rng, 1, max(1, min(256, 128 * 32000 * 5120 // (V * hid)))), "V": V,
            "hid": hid, "mix": mix}


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
    """Tree index and prefix length of every sequence (of a prompt: -1 and its
    length): the case's own, whatever the seed."""
    r = random.Random(case["mix"])
    index = {t: k for k, (t, _) in enumerate(TREES)}
    if case["T"] < 0:
        return [-1] * case["B"], [r.randint(case["lo"], case["hi"]) for _ in range(case["B"])]
    topo = [index[case["T"]] if case["T"] else r.randrange(len(TREES)) for _ in range(case["B"])]
    return topo, [r.randint(case["lo"], case["hi"]) for _ in range(case["B"])]


def _sizes(case):
    """New rows of every sequence and where they start."""
    topo, lens = _batch(case)
    return [TREES[t][0] if t >= 0 else n for t, n in zip(topo, lens)], [n if t >= 0 else 0 for t, n in zip(topo, lens)]


def _offsets(case):
    off = [0]
    for t in _sizes(case)[0]:
        off.append(off[-1] + t)
    return off


# --------------------------------------------------------------- four bits --

def _quant(x):
    """bf16 x [..., n] in groups of 32 -> codes uint8 [..., n / 2] and scale bytes uint8 [..., n / 32]."""
    g = x.float().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    m, e = torch.frexp(top)   # top = m 2^e, m in [1/2, 1)
    b = torch.where(top > 0, e + (m >= 0.875).to(e.dtype) + 124, 0).clamp(2, 252)
    y = torch.ldexp(g, 127 - b[..., None])
    a = y.abs()
    c = ((a > 0.25).to(U8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    c = (c + 8 * torch.signbit(y).to(U8)).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), b.to(U8)


def _values(codes, scales):
    """What codes and scale bytes stand for, in fp32."""
    lut = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)
    y = torch.stack([lut[(codes & 15).long()], lut[(codes >> 4).long()]], -1).flatten(-2)
    return torch.ldexp(y.unflatten(-1, (-1, 32)), scales.int()[..., None] - 127).flatten(-2)


def _planes(pool):
    """Codes [..., page, 64] and scale bytes [..., page, 4] of a pool's pages (views)."""
    page = pool.shape[-1] // 68
    return (pool[..., :64 * page].unflatten(-1, (page, 64)), pool[..., 64 * page:].unflatten(-1, (page, 4)))


# ------------------------------------------------------------------ inputs --

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=BF)


def _i32(v):
    return torch.tensor(v, dtype=I32, device="cuda")


def _pages(case, g, spare=3):
    """Block table [B, max_pages] of randomly placed pages that hold every
    sequence, and the number of pages in the pool."""
    page, B = case["page"], case["B"]
    need = [-(-(n + t) // page) for t, n in zip(*_sizes(case))]
    most, total = max(need) + 2, sum(need)
    order = torch.randperm(total + spare, generator=g, device="cuda")[:total].to(I32)
    n = torch.tensor(need, device="cuda")
    held = torch.arange(most, device="cuda")[None] < n[:, None]
    table = torch.full((B, most), -1, dtype=I32, device="cuda")
    table[held] = order
    return table, total + spare


def _rows(case):
    """Sequence and place (prefix + row) of every new row, on the CPU."""
    sizes, first = _sizes(case)
    return (torch.repeat_interleave(torch.arange(case["B"]), torch.tensor(sizes)),
            torch.cat([torch.arange(n, n + t) for t, n in zip(sizes, first)]))


def _slots(case, table):
    """Pool slot of every new row, in row order."""
    seq, at = (x.cuda() for x in _rows(case))
    p = case["page"]
    return (table[seq, at // p].long() * p + at % p).to(I32)


def _pool4(g, n_pages, Hkv, page):
    """A pool of 4-bit rows of ordinary keys or values."""
    pool = torch.empty((n_pages, Hkv, page * 68), dtype=U8, device="cuda")
    step = max(1, (1 << 26) // (Hkv * page * D))
    for i in range(0, n_pages, step):
        c, s = _planes(pool[i:i + step])
        x = _normal(g, *c.shape[:-1], D)
        codes, scales = _quant(x)
        c.copy_(codes)
        s.copy_(scales)
    return pool


def _inputs(case, seed):
    """The tensors the seed decides."""
    g, kind = _gen(seed), case["kind"]
    if kind == "logits":
        V, hid = case["V"], case["hid"]
        codes = torch.empty((V, hid // 2), dtype=U8, device="cuda")
        scales = torch.empty((V, hid // 32), dtype=U8, device="cuda")
        step = max(1, (1 << 26) // hid)
        for i in range(0, V, step):
            codes[i:i + step], scales[i:i + step] = _quant(_normal(g, min(step, V - i), hid) * 0.02)
        return {"x": _normal(g, case["T"], hid), "codes": codes, "scales": scales}
    topo, lens = _batch(case)
    off = _offsets(case)
    rows, Hkv, page = off[-1], case["Hkv"], case["page"]
    table, n_pages = _pages(case, g)
    s = {"topo": _i32(topo), "row_off": _i32(off), "lens": _i32(lens), "table": table}
    if kind == "attn":
        s.update(q=_normal(g, rows, case["Hq"], D).mul_(1.5), kp=_pool4(g, n_pages, Hkv, page),
                 vp=_pool4(g, n_pages, Hkv, page), slopes=None)
        if case["slopes"]:   # a geometric row of slopes over the heads
            s["slopes"] = torch.exp2(-8.0 * torch.arange(1, case["Hq"] + 1, device="cuda") / case["Hq"])
        return s
    s["slots"] = _slots(case, table)
    if kind == "append":
        # a projection's output: queries, keys and values of a row side by side
        s["qkv"] = _normal(g, rows, case["Hq"] + 2 * Hkv, D)
        s["pos"] = _rows(case)[1].to(I32).cuda()   # (of a prompt; a tree's come from its depths)
        w = (1 + 0.2 * torch.randn((2, D), generator=g, device="cuda")).to(BF)
        s["q_norm"], s["k_norm"] = (w[0].contiguous(), w[1].contiguous()) if case["norm"] else (None, None)
        if case["bits"] == 4:
            s["kp"], s["vp"] = (torch.zeros((n_pages, Hkv, page * 68), dtype=U8, device="cuda") for _ in "kv")
        else:
            s["kp"], s["vp"] = (torch.zeros((n_pages, Hkv, page, D), dtype=BF, device="cuda") for _ in "kv")
        return s
    f = _forest()
    node = (torch.rand(case["B"], generator=g, device="cuda").cpu() * f["T"][topo]).long()
    path = f["path"][topo, node]
    s.update(a=(path >= 0).sum(1).sub(1).to(I32).cuda(), path=path.to(I32).cuda())
    for name in ("kp", "vp"):
        s[name] = torch.randint(0, 240, (case["layers"], n_pages, Hkv, page * 68), generator=g, device="cuda",
                                dtype=U8)
    return s


def prepare(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    s["case"] = case
    if kind == "logits":
        s["out"] = torch.zeros((case["T"], case["V"]), device="cuda")
        return s
    f = _forest()
    rows, B = _offsets(case)[-1], case["B"]
    s["rows"] = rows
    s["forest"] = {k: f[k].cuda() for k in ("T", "depth", "anc", "path")}
    if kind == "attn":
        s["out"] = torch.zeros_like(s["q"])
        s["status"] = torch.zeros(B, dtype=I32, device="cuda")
    elif kind == "append":
        Hq, Hkv = case["Hq"], case["Hkv"]
        s["q"], s["k"], s["v"] = s["qkv"][:, :Hq], s["qkv"][:, Hq:Hq + Hkv], s["qkv"][:, Hq + Hkv:]
        s["q_out"] = torch.zeros((rows, Hq, D), dtype=BF, device="cuda")
        s["k_out"], s["v_out"] = (torch.zeros((rows, Hkv, D), dtype=BF, device="cuda") for _ in "kv")
    if own and kind != "compact":   # the handles, workspaces and work list that a serving loop keeps
        from paper_2606_27550_amd import api
        byte = lambda n: torch.empty(max(int(n), 256), dtype=U8, device="cuda")  # noqa: E731
        s["bank"] = api.Bank(f["trees"])
        if kind == "attn":
            shape = (rows, case["Hq"], case["Hkv"])
            most = s["table"].shape[1]
            s["plan"] = byte(api.tree_attn_paged_fp4_plan_bytes(s["bank"], B, *shape, most, case["page"]))
            api.tree_attn_paged_fp4_plan(s["bank"], s["topo"], s["lens"], s["row_off"], s["status"], s["table"],
                                         case["page"], s["kp"].shape[0], *shape, s["plan"], window=case["window"])
            s["ws"] = byte(api.tree_attn_paged_fp4_workspace(s["bank"], B, *shape, D, most, case["page"]))
    return s


# -------------------------------------------------------------------- pass --

def run(s):
    kind = s["case"]["kind"]
    if own:
        return _run_own(s, kind)
    return {"attn": _plain_attn, "append": _plain_append, "compact": _plain_compact, "logits": _plain_logits}[kind](s)


def _run_own(s, kind):
    from paper_2606_27550_amd import api
    case = s["case"]
    if kind == "attn":
        api.tree_attn_paged_fp4(s["bank"], s["plan"], s["q"], s["kp"], s["vp"], s["table"], 1 / math.sqrt(D),
                                s["out"], s["ws"], softcap=case["softcap"], window=case["window"],
                                slopes=s["slopes"])
        return {"out": s["out"]}
    if kind == "append":
        if case["T"] >= 0:
            api.tree_positions(s["bank"], s["topo"], s["lens"], s["row_off"], s["pos"])
        append = api.kv_append_paged_fp4 if case["bits"] == 4 else api.kv_append_paged
        append(s["q"], s["k"], s["v"], s["pos"], s["slots"], THETA, s["q_out"], s["kp"], s["vp"],
               q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS, k_out=s["k_out"], v_out=s["v_out"])
        return _append_outputs(s)
    if kind == "compact":
        api.kv_compact_paged_fp4(s["path"], s["a"], s["row_off"], s["slots"], s["kp"], s["vp"])
        return {"kp": s["kp"], "vp": s["vp"]}
    api.verify_logits_fp4(s["x"], s["codes"], s["scales"], s["out"])
    return {"out": s["out"]}


def _append_outputs(s):
    """The rows as the pool holds them, beside the pool itself (in 4 bits its bytes)."""
    return {"pos": s["pos"], "q": s["q_out"], "k": s["k_out"], "v": s["v_out"], "kp": s["kp"], "vp": s["vp"]}


# ------------------------------------------------------------- plain forms --

def _plain_attn(s):
    case, f = s["case"], s["forest"]
    B, Hq, Hkv, page = case["B"], case["Hq"], case["Hkv"], case["page"]
    G, n = Hq // Hkv, max(_sizes(case)[0])
    topo, L = s["topo"].long(), s["lens"].long()
    T = f["T"][topo]
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), T, output_size=s["rows"])
    node = torch.arange(s["rows"], device="cuda") - s["row_off"].long()[seq]
    # every sequence's keys and values side by side, padded to the longest
    cols = -(-max(x + t for t, x in zip(*_sizes(case))) // page)
    table = s["table"][:, :cols].clamp(min=0).long()

    def dense(pool):
        x = _values(*_planes(pool[table]))
        return x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, cols * page, D)

    q = torch.zeros((B, n, Hq, D), device="cuda")
    q[seq, node] = s["q"].float()
    q = q.reshape(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    z = torch.matmul(q, dense(s["kp"]).transpose(2, 3)).mul_(1 / math.sqrt(D)).view(B, Hkv, G, n, -1)
    if case["softcap"]:
        z = torch.tanh(z / case["softcap"]) * case["softcap"]
    # place j of a sequence: prefix position j, or tree node j - L
    j = torch.arange(cols * page, device="cuda")
    jn = (j[None] - L[:, None])
    tree = (jn >= 0) & (jn < T[:, None])
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
    return {"out": s["out"]}


def _plain_append(s):
    case, f = s["case"], s["forest"]
    page = case["page"]
    if case["T"] >= 0:
        topo = s["topo"].long()
        seq = torch.repeat_interleave(torch.arange(case["B"], device="cuda"), f["T"][topo], output_size=s["rows"])
        node = torch.arange(s["rows"], device="cuda") - s["row_off"].long()[seq]
        s["pos"].copy_(s["lens"].long()[seq] + f["depth"][topo[seq], node])
    h = D // 2
    freq = THETA ** (-2.0 * torch.arange(h, device="cuda", dtype=torch.float64) / D)
    a = s["pos"].double()[:, None, None] * freq
    cos, sin = a.cos(), a.sin()

    def turned(x, w):   # (in 64 bits: the keys' values next to a border of two codes)
        x = x.double()
        if w is not None:
            x = x * (x.pow(2).mean(-1, keepdim=True) + EPS).rsqrt() * w.double()
        lo, hi = x[..., :h], x[..., h:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(BF)

    s["q_out"].copy_(turned(s["q"], s["q_norm"]))
    slot = s["slots"].long()
    for x, out, pool in ((turned(s["k"], s["k_norm"]), s["k_out"], s["kp"]), (s["v"], s["v_out"], s["vp"])):
        if case["bits"] == 16:
            out.copy_(x)
            pool[slot // page, :, slot % page] = x
            continue
        codes, scales = _quant(x)
        out.copy_(_values(codes, scales))
        c, b = _planes(pool)
        c[slot // page, :, slot % page] = codes
        b[slot // page, :, slot % page] = scales
    return _append_outputs(s)


def _plain_compact(s):
    page = s["case"]["page"]
    j = torch.arange(s["path"].shape[1], device="cuda")[None]
    keep = j <= s["a"][:, None]
    seq, j = torch.nonzero(keep & (s["path"] != j), as_tuple=True)   # rows that move
    off = s["row_off"].long()[seq]
    src, dst = s["slots"][off + s["path"][seq, j].long()].long(), s["slots"][off + j].long()
    for pool in (s["kp"], s["vp"]):
        for x in _planes(pool):
            x[:, dst // page, :, dst % page] = x[:, src // page, :, src % page]
    return {"kp": s["kp"], "vp": s["vp"]}


def _plain_logits(s):
    s["out"].copy_(torch.matmul(s["x"].float(), _values(s["codes"], s["scales"]).t()))
    return {"out": s["out"]}


# ------------------------------------------------------------------- floor --

def work(case):
    kind = case["kind"]
    if kind == "logits":
        T, V, hid = case["T"], case["V"], case["hid"]
        return {"bytes": V * hid * 17 // 32 + 4 * T * V + 2 * T * hid, "flops": 2 * T * V * hid}
    topo, lens = _batch(case)
    sizes, _ = _sizes(case)
    rows, Hkv = sum(sizes), case["Hkv"]
    if kind == "attn":
        w = case["window"] or 1 << 30
        keys = [min(n, w + TREES[t][1]) for n, t in zip(lens, topo)]
        b = sum(k + t for k, t in zip(keys, sizes)) * 2 * Hkv * 68 + rows * 2 * case["Hq"] * D * 2
        return {"bytes": b, "flops": sum(4 * case["Hq"] * D * t * (min(n, w) + (t + 1) / 2)
                                         for n, t in zip(keys, sizes))}
    if kind == "append":
        # the rows in, queries out, keys and values out twice: to the pool and as they are held there
        held = 68 if case["bits"] == 4 else 256
        return {"bytes": rows * (case["Hq"] * 512 + Hkv * 2 * (512 + held) + 8), "flops": 0}
    # about half of a tree's depth is accepted, all but the root's row moves
    moved = sum(TREES[t][1] / 2 for t in topo)
    return {"bytes": 2 * moved * 2 * Hkv * 68 * case["layers"] + 12 * moved, "flops": 0}


# --------------------------------------------------------------- in 64 bits --

def _held(x):
    """The 4-bit value of every number of a group: the nearest of the scale's levels, of two equally
    near ones that with the even code."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140)))
    e = e + (top >= 1.75 * torch.exp2(e)).double()
    scale = torch.exp2((e - 2).clamp(-125, 125))
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    a = x.abs() / scale
    best = torch.zeros_like(a)
    far = a.clone()   # from level 0
    for i in range(1, 8):
        d = (a - level[i]).abs()
        closer = d <= far if i % 2 == 0 else d < far
        best, far = torch.where(closer, level[i], best), torch.where(closer, d, far)
    return (torch.sign(x) * best * scale).flatten(-2)


def _read(pool, pages, g, lo, hi):
    """Rows lo .. hi - 1 of head g of the sequence with these pages, as they stand, in 64 bits."""
    page = pool.shape[-1] // 68
    raw = pool[pages, g].long()
    codes, b = raw[:, :64 * page].reshape(-1, 64)[lo:hi], raw[:, 64 * page:].reshape(-1, 4)[lo:hi]
    nib = torch.stack([codes % 16, codes // 16], -1).reshape(-1, D)
    mag = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")[nib % 8]
    return mag * (1 - 2 * (nib // 8)) * torch.exp2(b.double() - 127).repeat_interleave(32, 1)


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "compact":
        return None   # bytes
    if kind == "logits":
        V, x = case["V"], s["x"].double()
        out = torch.zeros((case["T"], V), dtype=torch.float64, device="cuda")
        mag = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
        for i in range(0, V, 4096):
            c, b = s["codes"][i:i + 4096].long(), s["scales"][i:i + 4096].double()
            step = torch.exp2(b - 127).repeat_interleave(32, 1)
            for half, nib in ((0, c % 16), (1, c // 16)):
                w = mag[nib % 8] * (1 - 2 * (nib // 8)) * step[:, half::2]
                out[:, i:i + 4096] += x[:, half::2] @ w.t()
        return {"out": out}
    f = _forest()
    topo, lens = _batch(case)
    off = _offsets(case)
    if kind == "append":
        pos = torch.cat([n + f["depth"][t, :TREES[t][0]] if t >= 0 else torch.arange(n)
                         for t, n in zip(topo, lens)]).cuda().double()
        c = torch.arange(D // 2, device="cuda", dtype=torch.float64)
        angle = pos[:, None] * THETA ** (-2 * c / D)
        w = torch.polar(torch.ones_like(angle), angle)[:, None]
        Hq, Hkv = case["Hq"], case["Hkv"]

        def new(x, weight):
            x = x.double()
            if weight is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS) * weight.double()
            y = torch.complex(x[..., :D // 2], x[..., D // 2:]) * w
            return torch.cat([y.real, y.imag], -1)

        # (a key is held as the bf16 number nearest to it, in 4 bits the code of that)
        k, v = new(s["qkv"][:, Hq:Hq + Hkv], s["k_norm"]).to(BF), s["qkv"][:, Hq + Hkv:]
        k, v = (_held(k), _held(v)) if case["bits"] == 4 else (k.double(), v.double())
        return {"pos": None, "q": new(s["qkv"][:, :Hq], s["q_norm"]), "k": k, "v": v, "kp": None, "vp": None}
    # pass over (sequence, KV head): its keys by slot
    page, G = case["page"], case["Hq"] // case["Hkv"]
    if case["B"] * case["Hkv"] > 1024:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, (t, L) in enumerate(zip(topo, lens)):
        T, r0 = TREES[t][0], off[b]
        depth = f["depth"][t, :T]
        pages = s["table"][b, :-(-(L + T) // page)].long()
        first = max(0, L + 1 - case["window"]) if case["window"] else 0
        where = torch.cat([torch.arange(first, L), L + depth]).cuda().double()
        dist = (L + depth.cuda().double())[:, None] - where[None]
        ok = torch.cat([torch.ones((T, L - first), dtype=torch.bool), f["anc"][t, :T, :T]], 1).cuda()
        if case["window"]:
            ok &= dist < case["window"]
        for g in range(case["Hkv"]):
            k, v = (_read(s[n], pages, g, first, L + T) for n in ("kp", "vp"))
            for h in range(g * G, g * G + G):
                z = s["q"][r0:r0 + T, h].double() @ k.t() / math.sqrt(D)
                if case["softcap"]:
                    z = case["softcap"] * torch.tanh(z / case["softcap"])
                if s["slopes"] is not None:
                    z = z - s["slopes"][h].double() * dist
                z[~ok] = -math.inf
                out[r0:r0 + T, h] = torch.softmax(z, 1) @ v
    return {"out": out}
