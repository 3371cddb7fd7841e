"""The operators around the compression step, as cases that can be timed and compared: the rotation that brings a
layer's projected queries, keys and values behind its cache, the memory that holds kept rows in 4 bits, and the
attention over a working set or over such a memory.

A case with `own` false is computed from the formulas with elementary torch operations in 32 bits; with `own` true it
is the calls that a user makes of omnimem.Attention.  Shapes are those of perf/cases.py: Qwen-7B-shaped layers (28
query and 4 KV heads of width 128) and the tests' narrower ones.

Formulas, for one sequence (H_q query heads, H_kv KV heads, G = H_q / H_kv, width d):
  rotate  x' = x / sqrt(mean(x^2) + eps) * w for each head's row of q and k (or x' = x), then each pair (x'_a, x'_b) of
          frequency j turns by pos[axis_j] * f_j; v is copied.
  hold    rows of K in groups of 32 channels, channels of V in groups of 32 rows.  A group with the largest magnitude
          m is held as values {0, .5, 1, 1.5, 2, 3, 4, 6} * +-2^e (nearest, ties to the even code), 2^e the smallest
          power of two of at least 2^-120 with m <= 7 * 2^e.
  attend  out_i = sum_j p_ij v_j / sum_j p_ij and lse_i = log sum_j exp(s_ij), s_ij = scale <q_i, k_j>, over the rows j
          that query i sees: every memory row, then the tail rows up to n_tail - n_queries + i (causal) or all of them.
"""
import math

import torch

own = False

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
ELT = {"bf16": 2, "f32": 4}
GROUP = 32                          # values that share a scale; rows of a memory block
EPS = 1e-6


def listed():
    qwen = dict(h_q=28, h_kv=4, d=128, dtype="bf16")
    return [
        # One answer token's projections in a 7B layer: the launch is all there is.
        dict(name="rotate-token", kind="rotate", seqs=1, rows=1, axes=3, rot=128, pairs="half", norm=False, **qwen),
        # Three streams' odd chunks in a small fp32 model, part of each head rotated, neighbours paired.
        dict(name="rotate-ragged-f32", kind="rotate", seqs=3, rows=777, axes=2, rot=48, pairs="neighbours", norm=True,
             h_q=12, h_kv=4, d=64, dtype="f32"),
        # A prefill chunk of eight streams in a 7B layer with normalised queries and keys.
        dict(name="rotate-chunks", kind="rotate", seqs=8, rows=2048, axes=3, rot=128, pairs="half", norm=True, **qwen),
        # A small fp32 model's kept rows put away and brought back: odd lengths, a last block of one row.
        dict(name="hold-small-f32", kind="hold", seqs=3, rows=1025, h_q=8, h_kv=2, d=64, dtype="f32"),
        # A 28-layer model's kept rows between two chunks of a stream.
        dict(name="hold-28layers", kind="hold", seqs=28, rows=4096, **qwen),
        # One answer token over a short memory in a small model, where latency counts.
        dict(name="token-short", kind="attend", seqs=1, queries=1, memory=219, tail=5, ragged=False, causal=True,
             lse=False, h_q=8, h_kv=2, d=128, dtype="bf16"),
        # One answer token over a long memory: one sequence has to fill the chip.
        dict(name="token-long", kind="attend", seqs=1, queries=1, memory=40256, tail=64, ragged=False, causal=True,
             lse=False, **qwen),
        # Thirty-two users' answer tokens at once, memories of all lengths.
        dict(name="token-batch", kind="attend", seqs=32, queries=1, memory=16384, tail=200, ragged=True, causal=True,
             lse=False, **qwen),
        # Short questions asked of several memories at the narrower width, everything ragged.
        dict(name="questions-ragged", kind="attend", seqs=7, queries=45, memory=4096, tail=77, ragged=True, causal=True,
             lse=False, h_q=16, h_kv=4, d=64, dtype="bf16"),
        # The next chunk's prefill over a held memory.
        dict(name="chunk-memory", kind="attend", seqs=1, queries=2048, memory=4096, tail=2048, ragged=False, causal=True,
             lse=True, **qwen),
        # A chunk's prefill over a long working set in bf16; its log-sum-exp goes to the scores.
        dict(name="chunk-working-set", kind="attend", seqs=1, queries=4096, memory=0, tail=20480, ragged=False,
             causal=True, lse=True, **qwen),
        # The same in fp32 at the narrower width, odd sizes (calibration and validation runs).
        dict(name="chunk-f32", kind="attend", seqs=2, queries=333, memory=0, tail=1501, ragged=False, causal=True,
             lse=True, h_q=16, h_kv=4, d=64, dtype="f32"),
    ]


def draw(rng):
    """One more case: sizes over the whole range, odd ones among them, below the largest listed case's cost."""
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "hold", "attend", "attend", "attend"])
    h_q, h_kv, d = rng.choice([(28, 4, 128), (8, 2, 128), (16, 4, 64), (12, 4, 64), (32, 8, 128), (5, 1, 128)])
    c = dict(kind=kind, h_q=h_q, h_kv=h_kv, d=d, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    if kind == "rotate":
        c.update(seqs=log_uniform(1, 24), rows=log_uniform(1, 4096), axes=rng.choice([1, 2, 3, 4]),
                 rot=rng.choice([d, d, d // 2, 3 * d // 4]), pairs=rng.choice(["half", "half", "neighbours"]),
                 norm=rng.random() < 0.5)
    elif kind == "hold":
        c.update(seqs=log_uniform(1, 28), rows=log_uniform(1, 16384))
    else:
        form = rng.choice(["token", "token", "few", "chunk"])
        c.update(seqs=1 if form == "chunk" else log_uniform(1, 32), memory=rng.choice([0, 1, 1, 1]) * log_uniform(1, 32768),
                 queries=1 if form == "token" else log_uniform(2, 64) if form == "few" else log_uniform(65, 4096),
                 ragged=rng.random() < 0.5, causal=rng.random() < 0.8, lse=rng.random() < 0.5)
        c["tail"] = log_uniform(1, 512) if c["memory"] and form != "chunk" else log_uniform(1, 20480)
        if form == "chunk" and rng.random() < 0.7:
            c["tail"] = max(c["tail"], c["queries"])
    limit_f, limit_b = 0.8 * work(listed()[10])["flops"], 6e8
    shrink = [n for n in ("seqs", "queries", "rows", "tail", "memory") if n in c]
    while work(c)["flops"] * (16 if c["dtype"] == "f32" else 1) > limit_f or work(c)["bytes"] > limit_b or plain_bytes(c) > 1.2e10:
        n = max(shrink, key=lambda k: c[k] * (64 if k == "seqs" else 1))
        c[n] = c[n] // 2 + 1
    return c


def plain_bytes(c):
    """Bytes of the plain form's largest tensor, about."""
    if c["kind"] != "attend":
        return 4 * c["seqs"] * c["rows"] * (c["h_q"] + 2 * c["h_kv"]) * c["d"]
    n = c["memory"] + c["tail"] + GROUP
    return 4 * c["seqs"] * max(c["h_q"] * c["queries"] * n, c["h_kv"] * n * c["d"])


def lengths(c):
    """(queries, memory rows, tail rows) of each sequence: from the full sizes down to a fraction where ragged."""
    out = []
    for b in range(c["seqs"]):
        f = 1.0 - 0.93 * ((b * 5) % c["seqs"]) / c["seqs"] if c["ragged"] else 1.0
        out.append((max(1, int(c["queries"] * f)), int(c["memory"] * f), max(1, int(c["tail"] * f))))
    return out


def work(c):
    d, elt = c["d"], ELT[c["dtype"]]
    if c["kind"] == "rotate":
        heads = c["h_q"] + 2 * c["h_kv"]
        n = c["seqs"] * c["rows"]
        turned = (c["h_q"] + c["h_kv"]) * n
        return {"bytes": n * (2 * heads * d * elt + 4 * c["axes"]) + (2 * d * elt if c["norm"] else 0),
                "flops": turned * (3 * c["rot"] + (4 * d if c["norm"] else 0))}
    if c["kind"] == "hold":
        rows = c["seqs"] * c["h_kv"] * c["rows"]
        # the rows read and the memory written, then the memory read and the rows written
        return {"bytes": rows * (4 * d * elt + 2 * (d + d // 16)), "flops": rows * 2 * d * 6}
    nbytes = flops = 0
    for nq, nm, nt in lengths(c):
        first = nt - nq + 1            # tail rows that query 0 sees under the causal rule
        if c["causal"]:
            seen = sum_clamped(first, nq, nt)
        else:
            seen = nq * nt
        pairs = c["h_q"] * (nq * nm + seen)
        nbytes += (2 * c["h_q"] * nq + 2 * c["h_kv"] * nt) * d * elt + c["h_kv"] * nm * (d + d // 16)
        nbytes += 4 * c["h_q"] * nq if c["lse"] else 0
        flops += 4 * d * pairs
    return {"bytes": nbytes, "flops": flops}


def sum_clamped(first, count, top):
    """Sum of min(max(first + i, 0), top) over i < count."""
    zeros = min(count, max(0, -first))
    a, n = first + zeros, count - zeros
    full = min(n, max(0, a + n - 1 - top))
    n -= full
    return full * top + n * a + n * (n - 1) // 2


# --- inputs -------------------------------------------------------------------

def generator(seed, *more):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1_000_003 + sum((i + 1) * 7919 * int(m) for i, m in enumerate(more))) % (1 << 62))
    return g


def normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def keys_values(g, b, c, n):
    """K and V rows in the case's type: N(0, 1) with a scale per KV head, some key channels larger than the rest."""
    scale = 0.5 + torch.rand((b, c["h_kv"], 1, 1), generator=g, device=DEV)
    wide = 1.0 + 3.0 * (torch.rand((b, c["h_kv"], 1, c["d"]), generator=g, device=DEV) > 0.95)
    k = normal(g, b, c["h_kv"], n, c["d"]).mul_(scale).mul_(wide)
    v = normal(g, b, c["h_kv"], n, c["d"]).mul_(scale)
    return k.to(TORCH[c["dtype"]]), v.to(TORCH[c["dtype"]])


def prepare(c, seed):
    s = prepare_rotate(c, seed) if c["kind"] == "rotate" else prepare_hold(c, seed) if c["kind"] == "hold" else prepare_attend(c, seed)
    if own:
        s["calls"] = plan(s)
    return s


def prepare_rotate(c, seed):
    b, n, d, dt = c["seqs"], c["rows"], c["d"], TORCH[c["dtype"]]
    g = generator(seed, 1, n)
    heads = c["h_q"] + 2 * c["h_kv"]
    qkv = normal(g, b, n, heads * d).to(dt)      # the projection's output: all heads of a token in a row
    half = c["rot"] // 2
    axis = [j * c["axes"] // half for j in range(half)]
    freq = [10000.0 ** (-j / half) for j in range(half)]
    # far along a stream in time, a frame's height and width
    pos = torch.stack([torch.randint(0, 2_000_000 if a == 0 else 120, (b, n), generator=g, device=DEV)
                       for a in range(c["axes"])], 1).to(torch.int32)
    weight = (1.0 + 0.2 * normal(g, 2, d)).to(dt) if c["norm"] else None
    back = 19 + (int(seed) % 5)                  # rows that the caches hold already
    return dict(case=c, qkv=qkv, pos=pos, freq=freq, axis=axis, weight=weight, back=back,
                freq_t=torch.tensor(freq, dtype=torch.float64, device=DEV), axis_t=torch.tensor(axis, device=DEV),
                q=torch.zeros(b, c["h_q"], n, d, dtype=dt, device=DEV),
                kc=torch.zeros(b, c["h_kv"], back + n, d, dtype=dt, device=DEV),
                vc=torch.zeros(b, c["h_kv"], back + n, d, dtype=dt, device=DEV))


def prepare_hold(c, seed):
    b, n, d = c["seqs"], c["rows"], c["d"]
    g = generator(seed, 2, n)
    k, v = keys_values(g, b, c, n)
    data = torch.zeros(b, c["h_kv"], -(-n // GROUP), 34 * d, dtype=torch.uint8, device=DEV)
    return dict(case=c, k=k, v=v, data=data, k_back=torch.zeros_like(k), v_back=torch.zeros_like(v))


def prepare_attend(c, seed):
    b, d, dt = c["seqs"], c["d"], TORCH[c["dtype"]]
    g = generator(seed, 3, c["queries"], c["memory"])
    sizes = lengths(c)
    q = normal(g, b, c["h_q"], c["queries"], d).to(dt)
    k, v = keys_values(g, b, c, c["tail"])
    scale = 1.0 / ((0.5 + 1.5 * float(torch.rand(1, generator=torch.Generator().manual_seed(int(seed) + 17)))) * math.sqrt(d))
    nq, nm, nt = (torch.tensor(x, device=DEV) for x in zip(*sizes))
    data = None
    if c["memory"]:
        km, vm = keys_values(g, b, c, c["memory"])
        keep = (torch.arange(c["memory"], device=DEV) < nm[:, None])[:, None, :, None]
        data = blocks_of(*groups_of(km * keep, vm * keep))
    return dict(case=c, q=q, k=k, v=v, data=data, scale=scale, sizes=sizes, nq=nq, nm=nm, nt=nt,
                out=torch.zeros(b, c["queries"], c["h_q"], d, dtype=dt, device=DEV),
                lse=torch.full((b, c["h_q"], c["queries"]), -math.inf, device=DEV) if c["lse"] else None)


# --- the plain forms -----------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        for call in s["calls"]:
            call()
        return results(s)
    return plain_rotate(s) if kind == "rotate" else plain_hold(s) if kind == "hold" else plain_attend(s)


def plain_rotate(s):
    c = s["case"]
    b, n, d, rot = c["seqs"], c["rows"], c["d"], c["rot"]
    dt, half = TORCH[c["dtype"]], rot // 2
    x = s["qkv"].view(b, n, -1, d).transpose(1, 2)                       # [b, heads, n, d]
    h_q, h_kv = c["h_q"], c["h_kv"]
    turned = x[:, : h_q + h_kv].float()
    if c["norm"]:
        w = torch.cat([s["weight"][:1].expand(h_q, d), s["weight"][1:].expand(h_kv, d)])[:, None].float()
        turned = turned * torch.rsqrt((turned * turned).mean(-1, keepdim=True) + EPS) * w
    angle = s["pos"].double()[:, s["axis_t"]].transpose(1, 2) * s["freq_t"]  # [b, n, half]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["pairs"] == "half":
        x1, x2 = turned[..., :half], turned[..., half:rot]
        y = torch.cat([x1 * cos - x2 * sin, x1 * sin + x2 * cos], -1)
    else:
        x1, x2 = turned[..., 0:rot:2], turned[..., 1:rot:2]
        y = torch.stack([x1 * cos - x2 * sin, x1 * sin + x2 * cos], -1).flatten(-2)
    y = torch.cat([y, turned[..., rot:]], -1).to(dt)
    return y[:, :h_q], y[:, h_q:], x[:, h_q + h_kv:].clone()


def codes_of(x):
    """4-bit codes (sign and 3 bits) and scale exponents of x [..., 32] fp32, one scale for the last axis."""
    m = x.abs().amax(-1, keepdim=True)
    e = torch.frexp(m).exponent - 3                                       # m < 2^(e + 3): m / 2^e in [4, 8)
    e = torch.where(m > 7 * torch.ldexp(torch.ones_like(m), e), e + 1, e).clamp(min=-120)
    y = torch.ldexp(x.abs(), -e)
    code = ((y > 0.25).int() + (y >= 0.75).int() + (y > 1.25).int() + (y >= 1.75).int() + (y > 2.5).int() + (y >= 3.5).int()
            + (y > 5).int())
    return code + 8 * (x < 0).int(), e


def groups_of(k, v):
    """Codes and exponents of K rows (32 channels to a group) and V channels (32 rows to a group), padded to blocks."""
    b, h, n, d = k.shape
    pad = (0, 0, 0, -n % GROUP)
    k, v = (torch.nn.functional.pad(t.float(), pad) for t in (k, v))
    kc, ke = codes_of(k.view(b, h, -1, GROUP, d // 32, 32))               # [b, h, blocks, row, part, 32]
    vc, ve = codes_of(v.view(b, h, -1, GROUP, d).transpose(-1, -2))       # [b, h, blocks, channel, row]
    return kc, ke, vc, ve


def blocks_of(kc, ke, vc, ve):
    """The memory's bytes [b, h, blocks, 34 d]: K codes by row, V codes by channel (two to a byte, the first in the low
    half), then a scale byte (exponent + 127) for each K group, at (row % 4, part, row / 4), and for each V channel, at
    (channel % 16, channel / 16)."""
    b, h, n = kc.shape[:3]
    two = lambda t: (t[..., 0::2] + 16 * t[..., 1::2]).flatten(3)
    parts, d = kc.shape[4], vc.shape[3]
    ks = (ke + 127).view(b, h, n, 8, 4, parts).permute(0, 1, 2, 4, 5, 3).flatten(3)
    vs = (ve + 127).view(b, h, n, d // 16, 16).transpose(-1, -2).flatten(3)
    return torch.cat([two(kc), two(vc), ks, vs], -1).to(torch.uint8)


def value_of(code, e):
    """What codes and exponents stand for, in fp32 (exact)."""
    mag = code & 7
    x = torch.where(mag < 2, 0.5 * mag, torch.ldexp(1.0 + 0.5 * (mag & 1), (mag >> 1) - 1))
    return torch.ldexp(torch.where(code > 7, -x, x), e)


def values_of(data, d):
    """K and V rows [b, h, 32 blocks, d] of a memory's bytes, in fp32."""
    b, h, n = data.shape[:3]
    two = lambda t: torch.stack([t & 15, t >> 4], -1).flatten(-2).int()
    kc = two(data[..., : 16 * d]).view(b, h, n, GROUP, d // 32, 32)
    vc = two(data[..., 16 * d: 32 * d]).view(b, h, n, d, GROUP)
    ke = data[..., 32 * d: 33 * d].int().view(b, h, n, 4, d // 32, 8).permute(0, 1, 2, 5, 3, 4).reshape(b, h, n, GROUP, d // 32, 1)
    ve = data[..., 33 * d:].int().view(b, h, n, 16, d // 16).transpose(-1, -2).reshape(b, h, n, d, 1)
    k = value_of(kc, ke - 127).reshape(b, h, n * GROUP, d)
    v = value_of(vc, ve - 127).transpose(-1, -2).reshape(b, h, n * GROUP, d)
    return k, v


def plain_hold(s):
    c = s["case"]
    dt = TORCH[c["dtype"]]
    s["data"].copy_(blocks_of(*groups_of(s["k"], s["v"])))
    k, v = values_of(s["data"], c["d"])
    return k[:, :, : c["rows"]].to(dt), v[:, :, : c["rows"]].to(dt)


def plain_attend(s):
    c = s["case"]
    b, h_q, h_kv, d, n = c["seqs"], c["h_q"], c["h_kv"], c["d"], c["queries"]
    k, v, held = s["k"].float(), s["v"].float(), 0
    if s["data"] is not None:
        km, vm = values_of(s["data"], d)
        held = km.shape[2]
        k, v = torch.cat([km, k], 2), torch.cat([vm, v], 2)
    at = torch.arange(k.shape[2], device=DEV) - held                      # below 0: the memory
    i = torch.arange(n, device=DEV)[None, :, None]
    nq, nm, nt = (x[:, None, None] for x in (s["nq"], s["nm"], s["nt"]))
    last = nt - nq + i if c["causal"] else nt
    seen = torch.where(at < 0, at + held < nm, (at < nt) & (at <= last)) & (i < nq)
    seen = seen[:, None, None]                                            # [b, 1, 1, n, rows]
    x = torch.matmul(s["q"].float().view(b, h_kv, -1, d), k.transpose(-1, -2)).mul_(s["scale"])
    x = x.view(b, h_kv, h_q // h_kv, n, -1).masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top.masked_fill(top == -math.inf, 0)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(b, h_kv, -1, p.shape[-1]), v).view(b, h_q, n, d)
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
    if c["kind"] == "rotate":
        w = s["weight"]
        rope = om.make_rope(d, s["freq"], s["axis"], rotary_dim=c["rot"], neighbours=c["pairs"] == "neighbours",
                            q_weight=w[0] if w is not None else None, k_weight=w[1] if w is not None else None, eps=EPS)
        x = s["qkv"].view(c["seqs"], c["rows"], -1, d).transpose(1, 2)
        q, k, v = x.split([c["h_q"], c["h_kv"], c["h_kv"]], 1)
        rows = om.array_of([om.make_projection(q[b], k[b], v[b], s["pos"][b], s["q"][b], s["kc"][b, :, s["back"]:],
                                               s["vc"][b, :, s["back"]:]) for b in range(c["seqs"])])
        return [lambda: attn.omnimem_rotate(rope, rows)]
    if c["kind"] == "hold":
        there = om.array_of([om.make_held(s["k"][b], s["v"][b], s["data"][b]) for b in range(c["seqs"])])
        back = om.array_of([om.make_held(s["k_back"][b], s["v_back"][b], s["data"][b]) for b in range(c["seqs"])])
        return [lambda: attn.omnimem_pack(there), lambda: attn.omnimem_unpack(back)]
    queries = []
    for b, (nq, nm, nt) in enumerate(s["sizes"]):
        queries.append(om.make_query(s["q"][b, :, :nq], s["out"][b, :nq].transpose(0, 1), s["k"][b, :, :nt], s["v"][b, :, :nt],
                                     memory=s["data"][b] if nm else None, memory_rows=nm, sm_scale=s["scale"],
                                     lse=s["lse"][b, :, :nq] if c["lse"] else None))
    queries = om.array_of(queries)
    return [lambda: attn.omnimem_attend(queries, causal=c["causal"])]


def results(s):
    c = s["case"]
    if c["kind"] == "rotate":
        return s["q"], s["kc"][:, :, s["back"]:], s["vc"][:, :, s["back"]:]
    if c["kind"] == "hold":
        return s["k_back"], s["v_back"]
    return (s["out"], s["lse"]) if c["lse"] else (s["out"],)


# --- the definitions in 64 bits ---------------------------------------------------

def exact(c, seed):
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    return exact_rotate(s) if c["kind"] == "rotate" else exact_hold(s) if c["kind"] == "hold" else exact_attend(s)


def exact_rotate(s):
    """As complex numbers: a pair turned is x_a + i x_b times exp(i angle)."""
    c = s["case"]
    x = s["qkv"].double().view(c["seqs"], c["rows"], -1, c["d"]).permute(0, 2, 1, 3)
    q, k, v = x.split([c["h_q"], c["h_kv"], c["h_kv"]], 1)
    out = []
    for part, t in enumerate((q, k)):
        if c["norm"]:
            t = t / (t.pow(2).sum(-1, keepdim=True) / c["d"] + EPS).sqrt() * s["weight"][part].double()
        half, t = c["rot"] // 2, t.clone()
        turn = torch.zeros(c["seqs"], 1, c["rows"], half, dtype=torch.complex128, device=DEV)
        for j in range(half):
            a = s["pos"][:, s["axis"][j]].double() * s["freq"][j]
            turn[:, 0, :, j] = torch.polar(torch.ones_like(a), a)
        a, b = (slice(0, half), slice(half, 2 * half)) if c["pairs"] == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        z = torch.complex(t[..., a].contiguous(), t[..., b].contiguous()) * turn
        t[..., a], t[..., b] = z.real, z.imag
        out.append(t)
    return out[0], out[1], v.contiguous()


SIXTEEN = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def nearest(x):
    """x [..., 32] in 64 bits, each value as its group's scale and the nearest of the eight magnitudes hold it."""
    m = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2((m / 7).clamp(min=1e-300)))
    e = torch.where(m <= 7 * torch.exp2(e - 1), e - 1, torch.where(m > 7 * torch.exp2(e), e + 1, e)).clamp(min=-120)
    mags = torch.tensor(SIXTEEN[:8], dtype=torch.float64, device=DEV)
    far = (x.abs()[..., None] * torch.exp2(-e)[..., None] - mags).abs()
    even = torch.tensor([0, 1, 0, 1, 0, 1, 0, 1], device=DEV)
    best = far.amin(-1, keepdim=True)
    code = torch.where(far == best, even, 2).argmin(-1)                    # of two as near, the even code
    return mags[code] * torch.exp2(e) * torch.sign(x)


def exact_hold(s):
    c = s["case"]
    n, d = c["rows"], c["d"]
    k_out, v_out = torch.zeros_like(s["k"], dtype=torch.float64), torch.zeros_like(s["v"], dtype=torch.float64)
    for b in range(c["seqs"]):
        for r in range(0, n, 2048):                                        # whole blocks of 32 rows
            k, v = s["k"][b, :, r: r + 2048].double(), s["v"][b, :, r: r + 2048].double()
            rows = k.shape[1]
            k_out[b, :, r: r + rows] = nearest(k.reshape(c["h_kv"], rows, d // 32, 32)).reshape(c["h_kv"], rows, d)
            v = torch.cat([v, v.new_zeros(c["h_kv"], -rows % 32, d)], 1).unflatten(1, (-1, 32)).transpose(-1, -2)
            v_out[b, :, r: r + rows] = nearest(v).transpose(-1, -2).flatten(1, 2)[:, :rows]
    return k_out, v_out


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
    for b, (nq, nm, nt) in enumerate(s["sizes"]):
        k, v = s["k"][b, :, :nt].double(), s["v"][b, :, :nt].double()
        if nm:
            km, vm = held_rows(s["data"][b], d, nm)
            k, v = torch.cat([km, k], 1), torch.cat([vm, v], 1)
        see = torch.ones(nq, nm + nt, dtype=torch.bool, device=DEV)
        if c["causal"]:
            see[:, nm:] = see[:, nm:].tril(nt - nq)                        # (the memory is seen whole)
        for h in range(c["h_q"]):
            x = (s["q"][b, h, :nq].double() @ k[h // group].T) * s["scale"]
            x = x.masked_fill(~see, -math.inf)
            lse[b, h, :nq] = torch.logsumexp(x, -1)
            out[b, :nq, h] = torch.softmax(x, -1).nan_to_num(0.0) @ v[h // group]
    return (out, lse) if c["lse"] else (out,)
