"""The operators of answers' caches in pages, as cases that can be timed and compared: projected rows rotated into the
pages of a cache, attention over such a cache with a sliding window and first rows that stay visible, attention of a
tree of drafted tokens, and the move of an accepted path's rows.

A case with `own` false is computed from the formulas with elementary torch operations in 32 bits; with `own` true it
is the calls that a user makes of omnimem.Attention.  Shapes are those of perf/cases.py: Qwen-7B-shaped layers (28
query and 4 KV heads of width 128) and the tests' narrower ones.

Formulas, for one sequence (H_q query heads, H_kv KV heads, width d), row r of its cache on page table[r / page_rows]:
  append  x' = x / sqrt(mean(x^2) + eps) * w for each head's row of q and k (or x' = x), then each pair (x'_a, x'_b) of
          frequency j turns by pos[axis_j] * f_j; v is copied; keys and values go to the cache's rows behind `back`.
  window  out_i = sum_j p_ij v_j / sum_j p_ij and lse_i = log sum_j exp(s_ij), s_ij = scale <q_i, k_j>, over every memory
          row and the cache's rows j <= p that are the first `sinks` or past p - window, p = tail - queries + i.
  tree    the same where the cache's last rows are drafts: query i sees those that its mask says, and stands at
          p = cached + (drafts that it sees) - 1.
  keep    the accepted drafts' rows, path[0] < path[1] < .. of those behind `back`, become the rows behind `back`.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
ELT = {"bf16": 2, "f32": 4}
GROUP = 32                          # values that share a scale; rows of a memory block
EPS = 1e-6


def listed():
    qwen = dict(h_q=28, h_kv=4, d=128, dtype="bf16")
    turned = dict(axes=3, rot=128, pairs="half")
    attend = dict(memory=0, window=0, sinks=0, ragged=False, lse=False)
    return [
        # Thirty-two users' next tokens in a 7B layer, each behind a cache of its own length: the launch is all there is.
        dict(name="append-users", kind="append", seqs=32, rows=1, back=500, page=64, norm=False, **turned, **qwen),
        # Three streams' odd prompts in a small fp32 model, part of each head rotated, neighbours paired.
        dict(name="append-ragged-f32", kind="append", seqs=3, rows=777, back=101, page=32, axes=2, rot=48, pairs="neighbours",
             norm=True, h_q=12, h_kv=4, d=64, dtype="f32"),
        # The prompts of eight users in a 7B layer with normalised queries and keys.
        dict(name="append-prompts", kind="append", seqs=8, rows=2048, back=300, page=64, norm=True, **turned, **qwen),
        # One answer token far along a stream, whose older pages are given back: only the window's latency counts.
        dict(name="window-token", kind="window", seqs=1, queries=1, tail=20000, page=16, **{**attend, "window": 1024, "sinks": 4}, **qwen),
        # Thirty-two users' answer tokens at once over whole caches of all lengths: one pass over the pages.
        dict(name="pages-users", kind="window", seqs=32, queries=1, tail=16384, page=64, **{**attend, "ragged": True}, **qwen),
        # A prompt of a streaming layer with a window, behind a long cache.
        dict(name="window-prompt", kind="window", seqs=1, queries=4096, tail=20480, page=64, **{**attend, "window": 4096, "sinks": 4}, **qwen),
        # The same in fp32 at the narrower width, odd sizes (validation runs), with its log-sum-exp.
        dict(name="window-f32", kind="window", seqs=2, queries=333, tail=1501, page=16, **{**attend, "window": 250, "sinks": 3, "lse": True},
             h_q=16, h_kv=4, d=64, dtype="f32"),
        # A few drafts of a small model behind a short memory, where latency counts.
        dict(name="tree-short", kind="tree", seqs=1, queries=7, tail=12, page=16, **{**attend, "memory": 219}, h_q=8, h_kv=2, d=128, dtype="bf16"),
        # Twenty-six drafts of seven streams at the narrower width: memories, a window over the answers so far.
        dict(name="tree-memories", kind="tree", seqs=7, queries=26, tail=200, page=32,
             **{**attend, "memory": 4096, "window": 128, "sinks": 4, "ragged": True}, h_q=16, h_kv=4, d=64, dtype="bf16"),
        # Eight users' full trees over caches of all lengths.
        dict(name="tree-users", kind="tree", seqs=8, queries=64, tail=8192, page=64, **{**attend, "ragged": True}, **qwen),
        # A drafted step of a small model without its attention: a tree's rows appended, the accepted path moved up.
        dict(name="keep-short", kind="keep", layers=4, seqs=1, drafts=16, kept=5, back=77, page=16, h_q=8, h_kv=2, d=128, dtype="bf16"),
        # The same for eight users in 28 layers.
        dict(name="keep-users", kind="keep", layers=28, seqs=8, drafts=32, kept=8, back=90, page=64, **qwen),
    ]


def draw(rng):
    """One more case: sizes over the whole range, odd ones among them, below the largest listed case's cost."""
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["append", "window", "window", "tree", "tree", "keep"])
    h_q, h_kv, d = rng.choice([(28, 4, 128), (8, 2, 128), (16, 4, 64), (12, 4, 64), (32, 8, 128), (5, 1, 128)])
    c = dict(kind=kind, h_q=h_q, h_kv=h_kv, d=d, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), page=rng.choice([16, 32, 64, 128, 256]))
    if kind == "append":
        c.update(seqs=log_uniform(1, 40), rows=log_uniform(1, 4096), back=log_uniform(1, 500), axes=rng.choice([1, 2, 3, 4]),
                 rot=rng.choice([d, d, d // 2, 3 * d // 4]), pairs=rng.choice(["half", "half", "neighbours"]), norm=rng.random() < 0.5)
    elif kind == "keep":
        c.update(layers=log_uniform(1, 28), seqs=log_uniform(1, 12), drafts=log_uniform(2, 64), back=log_uniform(1, 200))
        c["kept"] = rng.randint(1, min(16, c["drafts"]))
    else:
        form = "tree" if kind == "tree" else rng.choice(["token", "few", "prompt"])
        c.update(seqs=1 if form == "prompt" else log_uniform(1, 40), memory=rng.choice([0, 0, 1]) * log_uniform(1, 16384),
                 queries={"token": 1, "few": log_uniform(2, 64), "prompt": log_uniform(65, 4096), "tree": log_uniform(2, 64)}[form],
                 ragged=rng.random() < 0.5, lse=rng.random() < 0.5, tail=log_uniform(1, 20480))
        c["window"] = rng.choice([0, 1, 1]) * log_uniform(16, 8192)
        c["sinks"] = rng.choice([0, 1, 4, 16, 100]) if c["window"] else 0
        if form in ("prompt", "tree"):
            c["tail"] = max(c["tail"], c["queries"])
    limit_f, limit_b = 0.8 * work(listed()[5])["flops"], 6e8
    shrink = [n for n in ("seqs", "queries", "rows", "tail", "memory", "layers") if n in c]
    while work(c)["flops"] * (16 if c["dtype"] == "f32" else 1) > limit_f or work(c)["bytes"] > limit_b or plain_bytes(c) > 1.2e10:
        n = max(shrink, key=lambda k: c[k] * (64 if k in ("seqs", "layers") else 1))
        c[n] = c[n] // 2 + 1
    if kind == "tree":
        c["tail"] = max(c["tail"], c["queries"])
    return c


def plain_bytes(c):
    """Bytes of the plain form's largest tensor, about."""
    if c["kind"] == "append":
        return 4 * c["seqs"] * (c["rows"] + c["back"]) * (c["h_q"] + 2 * c["h_kv"]) * c["d"]
    if c["kind"] == "keep":
        return 16 * c["layers"] * c["seqs"] * (c["back"] + c["drafts"] + 300) * c["h_kv"] * c["d"]
    n = c["memory"] + c["tail"] + GROUP
    return 4 * c["seqs"] * max(c["h_q"] * c["queries"] * n, c["h_kv"] * n * c["d"])


def part(b, c):
    """The part of the full sizes that sequence b has: all of them, or down to a fraction where ragged."""
    return 1.0 - 0.93 * ((b * 5) % c["seqs"]) / c["seqs"] if c.get("ragged", True) else 1.0


def lengths(c):
    """(queries, memory rows, tail rows) of each sequence."""
    out = []
    for b in range(c["seqs"]):
        f = part(b, c)
        nq = max(1, int(c["queries"] * f))
        out.append((nq, int(c["memory"] * f), max(nq if c["kind"] == "tree" else 1, int(c["tail"] * f))))
    return out


def tree_of(drafts, b):
    """Each draft's mask (itself and those that it follows, first ones first): a tree with some first tokens."""
    rng = random.Random(1000 * drafts + b)
    masks = []
    for i in range(drafts):
        parent = rng.randrange(max(-1, i - 6), i)
        masks.append((masks[parent] if parent >= 0 else 0) | 1 << i)
    return masks


def path_of(c, b):
    """The drafts on the way to the one with the most before it, `kept` at most."""
    best = max(tree_of(c["drafts"], b), key=lambda m: bin(m).count("1"))
    return [i for i in range(c["drafts"]) if best >> i & 1][: c["kept"]]


def windows(c):
    """For each sequence and query (position in the tail, first row past the sinks that it sees, drafts that it sees)."""
    for b, (nq, nm, nt) in enumerate(lengths(c)):
        seen = [bin(m).count("1") for m in tree_of(nq, b)] if c["kind"] == "tree" else [1 + i for i in range(nq)]
        rows = []
        for n in seen:
            p = nt - nq + n - 1
            rows.append((p, max(0, p - c["window"] + 1) if c["window"] else 0, n))
        yield b, nq, nm, nt, rows


def work(c):
    d, elt = c["d"], ELT[c["dtype"]]
    heads = c["h_q"] + 2 * c["h_kv"]
    if c["kind"] == "append":
        n = c["seqs"] * c["rows"]
        return {"bytes": n * (2 * heads * d * elt + 4 * c["axes"]) + (2 * d * elt if c["norm"] else 0),
                "flops": (c["h_q"] + c["h_kv"]) * n * (3 * c["rot"] + (4 * d if c["norm"] else 0))}
    if c["kind"] == "keep":
        n = c["seqs"] * c["layers"] * c["drafts"]
        moved = sum(1 for b in range(c["seqs"]) for i, j in enumerate(path_of(c, b)) if i != j)
        return {"bytes": n * (2 * heads * d * elt + 4) + c["layers"] * moved * 4 * c["h_kv"] * d * elt,
                "flops": (c["h_q"] + c["h_kv"]) * n * 3 * d}
    nbytes = flops = 0
    for _, nq, nm, nt, rows in windows(c):
        first = min(lo for p, lo, _ in rows)
        some = min(first, c["sinks"]) + max(0, nt - first)             # tail rows that some query sees
        pairs = nq * nm
        for p, lo, n in rows:
            if c["kind"] == "tree":
                cached = nt - nq
                pairs += n + min(cached, lo, c["sinks"]) + max(0, cached - lo)
            else:
                pairs += min(max(p + 1, 0), lo, c["sinks"]) + max(0, p + 1 - lo)
        nbytes += (2 * c["h_q"] * nq + 2 * c["h_kv"] * some) * d * elt + c["h_kv"] * nm * (d + d // 16)
        nbytes += (4 * c["h_q"] * nq if c["lse"] else 0) + (8 * nq if c["kind"] == "tree" else 0)
        flops += 4 * d * c["h_q"] * pairs
    return {"bytes": nbytes, "flops": flops}


# --- inputs -------------------------------------------------------------------

def generator(seed, *more):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1_000_003 + sum((i + 1) * 7919 * int(m) for i, m in enumerate(more))) % (1 << 62))
    return g


def normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def pools_of(c, g, rows, seed, layers=1):
    """K and V pages [layers, pages, H_kv, page rows, d] full of rows N(0, 1) with a scale per KV head, some key channels
    larger than the rest, and each sequence's table (entries behind its rows: no page) in no order, some pages nobody's."""
    per = [-(-n // c["page"]) for n in rows]
    n_pages = sum(per) + 3
    scale = 0.5 + torch.rand((c["h_kv"], 1, 1), generator=g, device=DEV)
    wide = 1.0 + 3.0 * (torch.rand((c["h_kv"], 1, c["d"]), generator=g, device=DEV) > 0.95)
    k = normal(g, layers, n_pages, c["h_kv"], c["page"], c["d"]).mul_(scale).mul_(wide).to(TORCH[c["dtype"]])
    v = normal(g, layers, n_pages, c["h_kv"], c["page"], c["d"]).mul_(scale).to(TORCH[c["dtype"]])
    ids = list(range(n_pages))
    random.Random(int(seed) + 5).shuffle(ids)
    table, at = [], 0
    for n in per:
        table.append(ids[at: at + n] + [-1] * (max(per) - n))
        at += n
    return k, v, torch.tensor(table, dtype=torch.int32, device=DEV)


def prepare(c, seed):
    s = prepare_append(c, seed) if c["kind"] in ("append", "keep") else prepare_attend(c, seed)
    if own:
        s["calls"] = plan(s)
    return s


def prepare_append(c, seed):
    """Projections of the next rows (of every layer's drafts) and caches with `back` rows and fewer before them."""
    keep = c["kind"] == "keep"
    b, n, d, dt = c["seqs"], c["drafts"] if keep else c["rows"], c["d"], TORCH[c["dtype"]]
    axes, rot = (1, d) if keep else (c["axes"], c["rot"])
    g = generator(seed, 1, n)
    heads = c["h_q"] + 2 * c["h_kv"]
    back = [int(c["back"] * part(i, c)) for i in range(b)]
    half = rot // 2
    axis = [j * axes // half for j in range(half)]
    freq = [10000.0 ** (-j / half) for j in range(half)]
    if keep:                                     # a draft's position: its depth in the tree
        deep = [[back[i] + bin(m).count("1") - 1 for m in tree_of(n, i)] for i in range(b)]
        pos = torch.tensor(deep, dtype=torch.int32, device=DEV)[:, None]
    else:                                        # far along a stream in time, a frame's height and width
        pos = torch.stack([torch.randint(0, 2_000_000 if a == 0 else 120, (b, n), generator=g, device=DEV)
                           for a in range(axes)], 1).to(torch.int32)
    weight = (1.0 + 0.2 * normal(g, 2, d)).to(dt) if c.get("norm") else None
    layers = c["layers"] if keep else 1
    k, v, table = pools_of(c, g, [x + n for x in back], seed, layers)
    qkv = normal(g, layers, b, n, heads * d).to(dt)   # the projection's output: all heads of a token in a row
    q = torch.zeros(layers, b, c["h_q"], n, d, dtype=dt, device=DEV)
    return dict(case=c, pk=k, pv=v, q=q, layers=[dict(qkv=x, q=y, pk=z, pv=w) for x, y, z, w in zip(qkv, q, k, v)], pos=pos, freq=freq, axis=axis, weight=weight, back=back, table=table,
                back_t=torch.tensor(back, device=DEV), rot=rot, pairs="half" if keep else c["pairs"],
                freq_t=torch.tensor(freq, dtype=torch.float64, device=DEV), axis_t=torch.tensor(axis, device=DEV))


def held_blocks(c, g, b, n):
    """Memories' bytes [b, h, blocks, 34 d]: K codes by row, V codes by channel (two to a byte, the first in the low half),
    then a scale byte (exponent + 127) for each K group and each V channel."""
    shape, d = (b, c["h_kv"], -(-n // GROUP)), c["d"]
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV)
    x = normal(g, *shape, 64 * d).mul_(2.5)
    code = torch.bucketize(x.abs(), edges) + 8 * (x < 0)
    scales = torch.randint(125, 128, (*shape, 2 * d), generator=g, device=DEV)
    return torch.cat([code[..., 0::2] + 16 * code[..., 1::2], scales], -1).to(torch.uint8)


def prepare_attend(c, seed):
    b, d, dt = c["seqs"], c["d"], TORCH[c["dtype"]]
    g = generator(seed, 3, c["queries"], c["memory"])
    sizes = lengths(c)
    q = normal(g, b, c["h_q"], c["queries"], d).to(dt)
    (k,), (v,), table = pools_of(c, g, [nt for _, _, nt in sizes], seed)
    data = held_blocks(c, g, b, c["memory"]) if c["memory"] else None
    tree = torch.zeros(b, c["queries"], dtype=torch.int64, device=DEV) if c["kind"] == "tree" else None
    place = torch.zeros(b, c["queries"], dtype=torch.int64, device=DEV)          # each query's position in the tail
    for i, nq, _, nt, rows in windows(c):
        place[i, :nq] = torch.tensor([p for p, _, _ in rows], device=DEV)
        first = min(lo for _, lo, _ in rows)
        table[i, -(-c["sinks"] // c["page"]): first // c["page"]] = -1         # pages that no query sees were given back
        if tree is not None:
            tree[i, :nq] = torch.tensor([m - (m >> 63 << 64) for m in tree_of(nq, i)], device=DEV)
    scale = 1.0 / ((0.5 + 1.5 * float(torch.rand(1, generator=torch.Generator().manual_seed(int(seed) + 17)))) * math.sqrt(d))
    nq, nm, nt = (torch.tensor(x, device=DEV) for x in zip(*sizes))
    return dict(case=c, q=q, pk=k, pv=v, table=table, data=data, tree=tree, place=place, scale=scale, sizes=sizes, nq=nq, nm=nm, nt=nt,
                out=torch.zeros(b, c["queries"], c["h_q"], d, dtype=dt, device=DEV),
                lse=torch.full((b, c["h_q"], c["queries"]), -math.inf, device=DEV) if c["lse"] else None)


# --- the plain forms -----------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        for call in s["calls"]:
            call()
        return results(s)
    if kind == "append":
        return plain_append(s, s["layers"][0])
    return plain_keep(s) if kind == "keep" else plain_attend(s)


def places(s, rows):
    """Pages and rows in them of the cache's rows [seqs, n]."""
    at = s["back_t"][:, None] + rows
    return s["table"].long().gather(1, at // s["case"]["page"]), at % s["case"]["page"]


def plain_append(s, layer):
    c, rot = s["case"], s["rot"]
    qkv, d = layer["qkv"], c["d"]
    b, n = qkv.shape[:2]
    dt, half = TORCH[c["dtype"]], rot // 2
    x = qkv.view(b, n, -1, d).transpose(1, 2)                            # [b, heads, n, d]
    h_q, h_kv = c["h_q"], c["h_kv"]
    turned = x[:, : h_q + h_kv].float()
    if s["weight"] is not None:
        w = torch.cat([s["weight"][:1].expand(h_q, d), s["weight"][1:].expand(h_kv, d)])[:, None].float()
        turned = turned * torch.rsqrt((turned * turned).mean(-1, keepdim=True) + EPS) * w
    angle = s["pos"].double()[:, s["axis_t"]].transpose(1, 2) * s["freq_t"]  # [b, n, half]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if s["pairs"] == "half":
        x1, x2 = turned[..., :half], turned[..., half:rot]
        y = torch.cat([x1 * cos - x2 * sin, x1 * sin + x2 * cos], -1)
    else:
        x1, x2 = turned[..., 0:rot:2], turned[..., 1:rot:2]
        y = torch.stack([x1 * cos - x2 * sin, x1 * sin + x2 * cos], -1).flatten(-2)
    y = torch.cat([y, turned[..., rot:]], -1).to(dt)
    page, at = places(s, torch.arange(n, device=DEV)[None].expand(b, n))
    layer["pk"][page, :, at] = y[:, h_q:].transpose(1, 2)
    layer["pv"][page, :, at] = x[:, h_q + h_kv:].transpose(1, 2)
    return y[:, :h_q], layer["pk"], layer["pv"]


def plain_keep(s):
    c = s["case"]
    for layer in s["layers"]:
        layer["q"].copy_(plain_append(s, layer)[0])
    paths = [path_of(c, b) for b in range(c["seqs"])]
    b = torch.tensor([b for b, path in enumerate(paths) for _ in path], device=DEV)
    old, new = (torch.tensor([x + s["back"][b] for b, path in enumerate(paths) for x in f(path)], device=DEV)
                for f in (lambda path: path, lambda path: range(len(path))))
    old_page, new_page = s["table"].long()[b, old // c["page"]], s["table"].long()[b, new // c["page"]]
    for x in (s["pk"], s["pv"]):
        x[:, new_page, :, new % c["page"]] = x[:, old_page, :, old % c["page"]]
    return s["q"], s["pk"], s["pv"]


def value_of(code, e):
    """What codes and exponents stand for, in fp32 (exact)."""
    mag = code & 7
    x = torch.where(mag < 2, 0.5 * mag, torch.ldexp(1.0 + 0.5 * (mag & 1), (mag >> 1) - 1))
    return torch.ldexp(torch.where(code > 7, -x, x), e)


def values_of(data, d):
    """K and V rows [b, h, 32 blocks, d] of memories' bytes, in fp32."""
    b, h, n = data.shape[:3]
    two = lambda t: torch.stack([t & 15, t >> 4], -1).flatten(-2).int()
    kc = two(data[..., : 16 * d]).view(b, h, n, GROUP, d // 32, 32)
    vc = two(data[..., 16 * d: 32 * d]).view(b, h, n, d, GROUP)
    ke = data[..., 32 * d: 33 * d].int().view(b, h, n, 4, d // 32, 8).permute(0, 1, 2, 5, 3, 4).reshape(b, h, n, GROUP, d // 32, 1)
    ve = data[..., 33 * d:].int().view(b, h, n, 16, d // 16).transpose(-1, -2).reshape(b, h, n, d, 1)
    k = value_of(kc, ke - 127).reshape(b, h, n * GROUP, d)
    v = value_of(vc, ve - 127).transpose(-1, -2).reshape(b, h, n * GROUP, d)
    return k, v


def plain_attend(s):
    c = s["case"]
    b, h_q, h_kv, d, n = c["seqs"], c["h_q"], c["h_kv"], c["d"], c["queries"]
    table = s["table"].long().clamp(min=0)
    k, v = (x[table].transpose(1, 2).flatten(2, 3).float() for x in (s["pk"], s["pv"]))   # [b, h, rows, d]
    held = 0
    if s["data"] is not None:
        km, vm = values_of(s["data"], d)
        held = km.shape[2]
        k, v = torch.cat([km, k], 2), torch.cat([vm, v], 2)
    at = torch.arange(k.shape[2], device=DEV) - held                      # below 0: the memory
    i = torch.arange(n, device=DEV)[None, :, None]
    nq, nm, nt, p = s["nq"][:, None, None], s["nm"][:, None, None], s["nt"][:, None, None], s["place"][:, :, None]
    near = (at > p - c["window"]) | (at < c["sinks"]) if c["window"] else at >= 0
    if s["tree"] is None:
        near = near & (at <= p)
    else:
        first = nt - nq                                                   # row of the first draft
        draft = (s["tree"][:, :, None] >> (at - first).clamp(0, 63)) & 1 == 1
        near = torch.where(at < first, near, draft)
    seen = torch.where(at < 0, at + held < nm, near & (at < nt)) & (i < nq)
    seen = seen[:, None, None]                                            # [b, 1, 1, n, rows]
    x = torch.matmul(s["q"].float().view(b, h_kv, -1, d), k.transpose(-1, -2)).mul_(s["scale"])
    x = x.view(b, h_kv, h_q // h_kv, n, -1).masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    w = x.sub_(top.masked_fill(top == -math.inf, 0)).exp_()
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w.view(b, h_kv, -1, w.shape[-1]), v).view(b, h_q, n, d)
    total = total.view(b, h_q, n, 1)
    out = (out / total.masked_fill(total == 0, 1)).transpose(1, 2).contiguous().to(TORCH[c["dtype"]])
    return (out, (top.view(b, h_q, n) + total[..., 0].log())) if c["lse"] else (out,)


# --- the framework's calls ------------------------------------------------------

_handles = {}


def plan(s):
    """The calls of a pass, with the handle and the descriptors that a user's program keeps."""
    from paper_2606_07577_amd import omnimem as om
    c = s["case"]
    key = (c["h_q"], c["h_kv"], c["d"], c["dtype"])
    if key not in _handles:
        _handles[key] = om.Attention(*key[:3], dtype=om.BF16 if c["dtype"] == "bf16" else om.F32)
    attn, d = _handles[key], c["d"]
    if c["kind"] in ("append", "keep"):
        w = s["weight"]
        rope = om.make_rope(d, s["freq"], s["axis"], rotary_dim=s["rot"], neighbours=s["pairs"] == "neighbours",
                            q_weight=w[0] if w is not None else None, k_weight=w[1] if w is not None else None, eps=EPS)
        calls, pools = [], []
        for layer in s["layers"]:
            x = layer["qkv"].view(c["seqs"], layer["qkv"].shape[1], -1, d).transpose(1, 2)
            q, k, v = x.split([c["h_q"], c["h_kv"], c["h_kv"]], 1)
            pools.append(om.make_pages(layer["pk"], layer["pv"]))
            rows = om.array_of([om.make_paged_projection(q[b], k[b], v[b], s["pos"][b], layer["q"][b], s["table"][b], s["back"][b])
                                for b in range(c["seqs"])])
            calls.append(lambda pool=pools[-1], rows=rows: attn.omnimem_rotate_pages(rope, pool, rows))
        if c["kind"] == "keep":
            pools = om.array_of(pools)
            paths = om.array_of([om.make_path(s["table"][b], s["back"][b], path_of(c, b)) for b in range(c["seqs"])])
            calls.append(lambda: attn.omnimem_keep_pages(pools, paths))
        return calls
    pool, queries = om.make_pages(s["pk"], s["pv"]), []
    for b, (nq, nm, nt) in enumerate(s["sizes"]):
        queries.append(om.make_paged_query(s["q"][b, :, :nq], s["out"][b, :nq].transpose(0, 1), s["table"][b], nt,
                                           memory=s["data"][b] if nm else None, memory_rows=nm, sm_scale=s["scale"],
                                           tree=s["tree"][b, :nq] if s["tree"] is not None else None,
                                           lse=s["lse"][b, :, :nq] if c["lse"] else None))
    queries = om.array_of(queries)
    return [lambda: attn.omnimem_attend_pages(pool, queries, window=c["window"], sinks=c["sinks"])]


def results(s):
    c = s["case"]
    if c["kind"] in ("append", "keep"):
        return (s["q"], s["pk"], s["pv"]) if c["kind"] == "keep" else (s["q"][0], s["pk"][0], s["pv"][0])
    return (s["out"], s["lse"]) if c["lse"] else (s["out"],)


# --- the definitions in 64 bits ---------------------------------------------------

def exact(c, seed):
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    if c["kind"] in ("append", "keep"):
        out = [exact_append(s, x) for x in s["layers"]]
        return tuple(torch.stack(x) for x in zip(*out)) if c["kind"] == "keep" else out[0]
    return exact_attend(s)


def exact_append(s, layer):
    """As complex numbers: a pair turned is x_a + i x_b times exp(i angle).  Rows go to their pages one sequence after the
    other, of a drafted step the accepted ones behind the rest."""
    c = s["case"]
    b, n = layer["qkv"].shape[:2]
    x = layer["qkv"].double().view(b, n, -1, c["d"]).permute(0, 2, 1, 3)
    q, k, v = x.split([c["h_q"], c["h_kv"], c["h_kv"]], 1)
    half, out = s["rot"] // 2, []
    for which, t in enumerate((q, k)):
        if s["weight"] is not None:
            t = t / (t.pow(2).sum(-1, keepdim=True) / c["d"] + EPS).sqrt() * s["weight"][which].double()
        t = t.clone()
        turn = torch.zeros(b, 1, n, half, dtype=torch.complex128, device=DEV)
        for j in range(half):
            a = s["pos"][:, s["axis"][j]].double() * s["freq"][j]
            turn[:, 0, :, j] = torch.polar(torch.ones_like(a), a)
        one, two = (slice(0, half), slice(half, 2 * half)) if s["pairs"] == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        z = torch.complex(t[..., one].contiguous(), t[..., two].contiguous()) * turn
        t[..., one], t[..., two] = z.real, z.imag
        out.append(t)
    pools = [layer["pk"].double(), layer["pv"].double()]
    for i in range(b):
        rows = list(range(n))
        if c["kind"] == "keep":                                           # (the first rows are those of the path)
            path = path_of(c, i)
            rows = path + rows[len(path):]
        at = torch.arange(s["back"][i], s["back"][i] + n, device=DEV)
        page = s["table"][i].long()[torch.div(at, c["page"], rounding_mode="floor")]
        for pool, new in zip(pools, (out[1], v)):
            pool[page, :, at % c["page"]] = new[i][:, rows].transpose(0, 1)
    return out[0], pools[0], pools[1]


SIXTEEN = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def held_rows(data, d, n):
    """The first n K and V rows [h, n, d] of one sequence's memory in 64 bits, by a table of the sixteen values."""
    table = torch.tensor(SIXTEEN, dtype=torch.float64, device=DEV)
    row, ch = torch.arange(n, device=DEV), torch.arange(d, device=DEV)
    flat, base = data.flatten(1).long(), (row // 32 * 34 * d)[:, None]
    r = (row % 32)[:, None]
    kb, vb = flat[:, base + r * (d // 2) + ch // 2], flat[:, base + 16 * d + ch * 16 + r // 2]
    ks = flat[:, base + 32 * d + (r % 4 * (d // 32) + ch // 32) * 8 + r // 4]
    vs = flat[:, base + 33 * d + ch % 16 * (d // 16) + ch // 16]
    k = table[torch.where(ch % 2 == 0, kb % 16, kb // 16)] * torch.exp2(ks.double() - 127)
    v = table[torch.where(r % 2 == 0, vb % 16, vb // 16)] * torch.exp2(vs.double() - 127)
    return k, v


def exact_attend(s):
    c = s["case"]
    d, group = c["d"], c["h_q"] // c["h_kv"]
    if 4 * d * c["h_q"] * c["queries"] * (c["memory"] + c["tail"]) * c["seqs"] > 2e13:
        return None
    out = torch.zeros(c["seqs"], c["queries"], c["h_q"], d, dtype=torch.float64, device=DEV)
    lse = torch.full((c["seqs"], c["h_q"], c["queries"]), -math.inf, dtype=torch.float64, device=DEV)
    for b, nq, nm, nt, rows in windows(c):
        see = torch.zeros(nq, nm + nt, dtype=torch.bool, device=DEV)
        see[:, :nm] = True
        trees = tree_of(nq, b)
        for i, (p, lo, _) in enumerate(rows):                              # (row by row, as the words say it)
            end = nt - nq if c["kind"] == "tree" else p + 1
            see[i, nm + lo: nm + max(lo, end)] = True
            see[i, nm: nm + max(0, min(c["sinks"], end))] = True
            if c["kind"] == "tree":
                see[i, nm + nt - nq:] = torch.tensor([trees[i] >> j & 1 for j in range(nq)], device=DEV) == 1
        at = torch.arange(nt, device=DEV)
        page = s["table"][b].long()[torch.div(at, c["page"], rounding_mode="floor")]
        k, v = (torch.where((page >= 0)[:, None, None], x[page.clamp(min=0), :, at % c["page"]].double(), 0.0).transpose(0, 1)
                for x in (s["pk"], s["pv"]))
        if nm:
            km, vm = held_rows(s["data"][b], d, nm)
            k, v = torch.cat([km, k], 1), torch.cat([vm, v], 1)
        for h in range(c["h_q"]):
            x = (s["q"][b, h, :nq].double() @ k[h // group].T) * s["scale"]
            x = x.masked_fill(~see, -math.inf)
            lse[b, h, :nq] = torch.logsumexp(x, -1)
            out[b, :nq, h] = torch.softmax(x, -1).nan_to_num(0.0) @ v[h // group]
    return (out, lse) if c["lse"] else (out,)
