"""omnimem_attend against its definition in 64 bits.

With S the largest sum of |q||k| scale of a row's products, u = 2^-24 and N keys: a product of d terms in fp32, scaled
and turned to a power of 2, is off by at most (d + 6) u S, and so is its share of the weights, relative to them; the
maximum cancels.  Sums of N weights and of N products with v are off by at most (N + 8) u of their sizes (exp2 and the
join's factors among the 8 steps).  With A the weighted mean of |v|, out is off by at most A (2 (d + 6) u S + 2 (N + 8) u),
and with bf16 by A eps / 2 more (each weight rounded, not their sum) and eps / 2 of the value (the result rounded).
lse is off by (d + 6) u S + (N + 8) u and 2 u of its value.  A weight below 2^-126 of the largest is not an fp32 number
(the definition's 64 bits hold it): N of them times the largest |v| may be missing."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2606_07577_amd import omnimem as om

pytestmark = pytest.mark.gpu
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def host(t):
    return t.double().cpu().numpy()


class Case:
    """One sequence: random rows, a memory of them packed by the library, an output with a border that stays."""

    def __init__(self, attn, g, h_q, h_kv, d, dtype, nq, nm, nt, scale=None, lse=True):
        self.sizes, self.scale, td = (nq, nm, nt), scale or d ** -0.5, TORCH[dtype]
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.q = rnd(nq, h_q, d).to(td).transpose(0, 1)              # query-major, as a projection leaves it
        self.k, self.v = (rnd(h_kv, nt + 3, d).to(td) for _ in range(2))
        self.data, held = None, (np.zeros((h_kv, 0, d)),) * 2
        if nm:
            km, vm = (rnd(h_kv, nm, d).to(td) for _ in range(2))
            self.data = torch.zeros(om.memory_shape(h_kv, d, nm), dtype=torch.uint8, device="cuda")
            attn.omnimem_pack([om.make_held(km, vm, self.data)])
            torch.cuda.synchronize()
            held = orc.unpack(self.data.cpu().numpy(), nm)
        self.held = held
        self.k[:, nt:] = float("nan")                                # rows behind the tail
        self.v[:, nt:] = float("nan")
        self.out = torch.full((h_q, nq + 1, d), 7.0, device="cuda", dtype=td)
        self.lse = torch.full((h_q, nq + 1), 7.0, device="cuda") if lse else None

    def query(self):
        nq, nm, nt = self.sizes
        return om.make_query(self.q, self.out[:, :nq], self.k[:, :nt] if nt else None, self.v[:, :nt] if nt else None,
                             self.data, nm, self.scale, None if self.lse is None else self.lse[:, :nq])

    def check(self, causal):
        nq, nm, nt = self.sizes
        d, dt = self.q.shape[2], self.q.dtype
        k, v = (np.concatenate([m, host(t[:, :nt])], 1) for m, t in zip(self.held, (self.k, self.v)))
        out, lse, size, reach = orc.attend(host(self.q), k, v, nm, self.scale, causal)
        n, half = k.shape[1], torch.finfo(dt).eps / 2 if dt == torch.bfloat16 else 0.0
        near = 2 * (d + 6) * U * reach[..., None] + 2 * (n + 8) * U + half
        tol = size * near + (half or U) * np.abs(out) + n * 2.0 ** -126 * np.abs(v).max(initial=0.0)
        got = host(self.out[:, :nq])
        assert np.array_equal(np.isnan(got), np.isnan(out))
        fine = bool((np.abs(got - out) <= tol)[~np.isnan(out)].all())
        assert fine, (self.sizes, float(np.nanmax(np.abs(got - out) / tol)))
        assert (self.out[:, nq:] == 7).all()
        if self.lse is not None:
            got = host(self.lse[:, :nq])
            assert np.array_equal(np.isneginf(got), np.isneginf(lse)) and np.array_equal(np.isnan(got), np.isnan(lse))
            f = np.isfinite(lse)
            assert (np.abs(got[f] - lse[f]) <= (d + 6) * U * reach[f] + (n + 8) * U + 2 * U * np.abs(lse[f])).all()
            assert (self.lse[:, nq:] == 7).all()


def handle(h_q, h_kv, d, dtype):
    return om.Attention(h_q, h_kv, d, om.BF16 if dtype == "bf16" else om.F32)


SIZES = [(1, 0, 1), (1, 1, 0), (1, 219, 5), (1, 128, 128), (2, 33, 0), (3, 0, 300), (5, 700, 9), (9, 0, 4), (17, 0, 4), (40, 31, 77),
         (130, 0, 130), (70, 257, 129), (300, 100, 411)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,h_kv,d", [(7, 1, 128), (4, 2, 64), (2, 2, 128), (20, 1, 64)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("sizes", SIZES)
def test_sequences_alone(dtype, h_q, h_kv, d, causal, sizes):
    attn = handle(h_q, h_kv, d, dtype)
    c = Case(attn, torch.Generator(device="cuda").manual_seed(sum(sizes)), h_q, h_kv, d, dtype, *sizes)
    attn.omnimem_attend([c.query()], causal)
    torch.cuda.synchronize()
    c.check(causal)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_ragged_batches(dtype, d):
    """More sequences than a launch describes, of all forms, empty ones among them."""
    h_q, h_kv = 6, 2
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(d)
    sizes = [(1 + (5 * i) % 23, (37 * i) % 300, (11 * i) % 90) for i in range(18)] + [(0, 5, 5), (4, 0, 0)]
    cases = [Case(attn, g, h_q, h_kv, d, dtype, *s, lse=i % 2 == 0) for i, s in enumerate(sizes)]
    attn.omnimem_attend([c.query() for c in cases])
    torch.cuda.synchronize()
    for c in cases:
        c.check(True)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nm,nt", [(1, 9000, 70), (3, 0, 5000), (50, 2000, 1500)])
def test_keys_split_over_workgroups(dtype, nq, nm, nt):
    attn = handle(2, 1, 128, dtype)
    g = torch.Generator(device="cuda").manual_seed(nq)
    c = Case(attn, g, 2, 1, 128, dtype, nq, nm, nt)
    attn.omnimem_attend([c.query()])
    torch.cuda.synchronize()
    c.check(True)
    first = c.out.clone()
    for _ in range(3):                       # the sums' order is fixed: the same bits every time
        c.out.fill_(7.0)
        attn.omnimem_attend([c.query()])
        torch.cuda.synchronize()
        assert torch.equal(c.out, first)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-6, 30.0])
@pytest.mark.parametrize("nq", [2, 90])
def test_flat_and_sharp_weights(dtype, scale, nq):
    """Products near 0, and of several hundreds with weights that are 0 but for a few."""
    attn = handle(4, 1, 64, dtype)
    c = Case(attn, torch.Generator(device="cuda").manual_seed(5), 4, 1, 64, dtype, nq, 200, 150, scale=scale)
    attn.omnimem_attend([c.query()])
    torch.cuda.synchronize()
    c.check(True)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("nq,nm,nt", [(4, 40, 30), (9, 0, 200), (60, 100, 130), (200, 0, 333), (3, 2100, 2000)])
def test_rows_that_a_query_does_not_see_have_no_part(dtype, value, nq, nm, nt):
    """Infinities and NaN in keys and values of the last rows: the queries before them are as without them, those that
    see them get what the definition gives."""
    attn = handle(6, 2, 64, dtype)
    c = Case(attn, torch.Generator(device="cuda").manual_seed(nq), 6, 2, 64, dtype, nq, nm, nt)
    clean = Case(attn, torch.Generator(device="cuda").manual_seed(nq), 6, 2, 64, dtype, nq, nm, nt)
    at = nt - nq // 2 - 1                          # the first half of the queries does not see it
    c.v[0, at, 5:9] = value
    c.k[1, at, 0] = value
    attn.omnimem_attend([c.query()])
    attn.omnimem_attend([clean.query()])
    torch.cuda.synchronize()
    before = nq - (nt - at)                        # queries that do not see it
    assert before >= 1
    # Rows with such values are summed in another order and with weights that are not rounded: twice the bound above of
    # the sums, and in bf16 half a step for the weights of the one and for each result.
    reach = float((clean.q.float().abs().sum(-1).amax() * torch.cat([clean.k[:, :nt].float().flatten(),
                  torch.tensor(clean.held[0], device="cuda").float().flatten()]).abs().amax()) * c.scale)
    near = 2 * (2 * (64 + 6) * U * reach + 2 * (nm + nt + 8) * U) + (3 * 2.0 ** -8 if dtype == "bf16" else 0.0)
    size = torch.cat([clean.v[:, :nt].float().flatten(), torch.tensor(clean.held[1], device="cuda").float().flatten()]).abs().amax()
    assert ((c.out[:, :before].float() - clean.out[:, :before].float()).abs() <= near * size).all()
    assert torch.equal(c.lse[:, :before], clean.lse[:, :before])
    after, plain = c.out[:3, before: nq], clean.out[:3, before: nq]
    assert (~torch.isfinite(after[..., 5:9])).all()            # (heads 0 .. 2 read KV head 0)
    assert ((after[..., 9:].float() - plain[..., 9:].float()).abs() <= near * size).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [1, 40, 100])
def test_products_that_are_all_minus_infinity_count_as_none(dtype, nq):
    attn = handle(2, 1, 64, dtype)
    c = Case(attn, torch.Generator(device="cuda").manual_seed(1), 2, 1, 64, dtype, nq, 0, nq)
    c.q.fill_(1.0)
    c.k[:, :nq] = 0.0
    c.k[:, :nq, 0] = float("-inf")
    attn.omnimem_attend([c.query()])
    torch.cuda.synchronize()
    assert (c.out[:, :nq] == 0).all() and torch.isneginf(c.lse[:, :nq]).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [1, 20, 130])
def test_a_negative_scale(dtype, nq):
    attn = handle(4, 2, 64, dtype)
    c = Case(attn, torch.Generator(device="cuda").manual_seed(3), 4, 2, 64, dtype, nq, 150, 170, scale=-0.3)
    attn.omnimem_attend([c.query()])
    torch.cuda.synchronize()
    c.check(True)
    attn.close()


def by_torch(q, k, v, scale, causal):
    """out and lse of q [h_q, n, d] over k, v [h_kv, t, d] in 64 bits on the device, and the sizes of Case.check."""
    group, n, t = q.shape[0] // k.shape[0], q.shape[1], k.shape[1]
    q, k, v = q.double(), k.double().repeat_interleave(group, 0), v.double().repeat_interleave(group, 0)
    s = torch.bmm(q, k.transpose(1, 2).contiguous()) * scale
    if causal:
        s.masked_fill_(~torch.ones(n, t, dtype=torch.bool, device="cuda").tril(t - n), float("-inf"))
    p = torch.softmax(s, -1)
    reach = torch.bmm(q.abs(), k.abs().transpose(1, 2).contiguous()).amax(-1) * abs(scale)
    return torch.bmm(p, v), torch.logsumexp(s, -1), torch.bmm(p, v.abs()), reach


def check_by_torch(out, lse, ref, d, n):
    o, l, size, reach = ref
    half = torch.finfo(out.dtype).eps / 2 if out.dtype == torch.bfloat16 else 0.0
    tol = size * (2 * (d + 6) * U * reach[..., None] + 2 * (n + 8) * U + half) + (half or U) * o.abs()
    assert bool(((out.double() - o).abs() <= tol).all())
    assert bool(((lse.double() - l).abs() <= (d + 6) * U * reach + (n + 8) * U + 2 * U * l.abs()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,nq,nt,d", [(70, 1000, 1000, 64), (67, 513, 700, 128), (9, 1300, 5000, 64)])
def test_more_row_tiles_than_compute_units(dtype, h, nq, nt, d):
    """Whole row tiles for each compute unit, and the rest in shares."""
    g = torch.Generator(device="cuda").manual_seed(h)
    attn = handle(h, h, d, dtype)
    q, k, v = (torch.randn(h, n, d, generator=g, device="cuda").to(TORCH[dtype]) for n in (nq, nt, nt))
    out, lse = torch.zeros_like(q), torch.zeros(h, nq, device="cuda")
    attn.omnimem_attend([om.make_query(q, out, k, v, lse=lse)])
    torch.cuda.synchronize()
    check_by_torch(out, lse, by_torch(q, k, v, d ** -0.5, True), d, nt)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [1, 9, 40, 150])
def test_rows_interleaved_over_heads_and_far_apart(dtype, nq):
    """Keys and values [row][head][d] and query-major queries; then rows and heads whose offsets pass 32 bits."""
    h_q, h_kv, d, nt = 6, 2, 64, 700
    g = torch.Generator(device="cuda").manual_seed(nq)
    td = TORCH[dtype]
    attn = handle(h_q, h_kv, d, dtype)
    q = torch.randn(nq, h_q, d, generator=g, device="cuda").to(td).transpose(0, 1)
    k, v = (torch.randn(nt, h_kv, d, generator=g, device="cuda").to(td).transpose(0, 1) for _ in range(2))
    ref = by_torch(q, k, v, d ** -0.5, True)
    out, lse = torch.zeros(nq, h_q, d, device="cuda", dtype=td).transpose(0, 1), torch.zeros(h_q, nq, device="cuda")
    attn.omnimem_attend([om.make_query(q, out, k, v, lse=lse)])
    torch.cuda.synchronize()
    check_by_torch(out, lse, ref, d, nt)
    elt = torch.finfo(td).bits // 8
    rows, heads = (7 << 20) // elt, (5 << 30) // elt            # 700 rows of 7 MiB; heads 5 GiB apart
    buffers = [torch.empty((heads + nt * rows) * elt, dtype=torch.uint8, device="cuda").view(td) for _ in range(2)]
    far_k, far_v = (b.as_strided((h_kv, nt, d), (heads, rows, 1)) for b in buffers)
    far_k.copy_(k)
    far_v.copy_(v)
    again = torch.zeros_like(out)
    attn.omnimem_attend([om.make_query(q, again, far_k, far_v)])
    torch.cuda.synchronize()
    assert torch.equal(again, out)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,h_kv,d,nq,nm,nt", [(7, 1, 128, 1, 30000, 9), (4, 1, 64, 1, 40000, 0), (20, 1, 64, 3, 6000, 100),
                                                 (2, 2, 64, 1, 0, 2500), (16, 1, 128, 1, 2000, 0), (30, 1, 128, 1, 1500, 0)])
def test_every_way_of_joining(dtype, h_q, h_kv, d, nq, nm, nt):
    """Splits of few rows that their last unit joins, with one thread to a value or several, and that a kernel joins;
    against all keys in one share (more rows of the same keys are not split)."""
    g = torch.Generator(device="cuda").manual_seed(nm)
    attn = handle(h_q, h_kv, d, dtype)
    c = Case(attn, g, h_q, h_kv, d, dtype, nq, nm, nt)
    for _ in range(3):
        c.out.fill_(7.0)
        attn.omnimem_attend([c.query()])
        torch.cuda.synchronize()
        k, v = (torch.cat([torch.tensor(m, device="cuda"), t[:, :nt].double()], 1) for m, t in zip(c.held, (c.k, c.v)))
        o, l, size, reach = by_torch(c.q, k, v, c.scale, False)
        if nt and nq > 1:      # (the causal rule among the tail rows)
            seen = torch.ones(nq, nm + nt, dtype=torch.bool, device="cuda")
            seen[:, nm:] = seen[:, nm:].tril(nt - nq)
            s = torch.bmm(c.q.double(), k.repeat_interleave(h_q // h_kv, 0).transpose(1, 2).contiguous()) * c.scale
            s.masked_fill_(~seen, float("-inf"))
            p, l = torch.softmax(s, -1), torch.logsumexp(s, -1)
            o, size = (torch.bmm(p, x.repeat_interleave(h_q // h_kv, 0)) for x in (v, v.abs()))
        check_by_torch(c.out[:, :nq], c.lse[:, :nq], (o, l, size, reach), d, nm + nt)
        assert (c.out[:, nq:] == 7).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("chunk,others", [((2600, 0, 2600), [(1, 3000, 5), (9, 40, 0), (0, 0, 5), (200, 0, 300), (1, 0, 2700)]),
                                          ((700, 0, 2300), [(1, 2200, 3)] * 31), ((2600, 0, 2600), [(1, 100, 5), (3, 0, 7)])])
def test_chunks_and_tokens_in_one_call(dtype, chunk, others):
    """A chunk beside tokens with more keys than it, beside many tokens, and beside a few that go with it."""
    attn = handle(4, 4, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(chunk[0])
    cases = [Case(attn, g, 4, 4, 64, dtype, *s) for s in [*others[:2], chunk, *others[2:]]]
    attn.omnimem_attend([c.query() for c in cases])
    torch.cuda.synchronize()
    for c in cases:
        c.check(True)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_tokens_beside_a_chunk_with_more_keys(dtype):
    attn = handle(4, 4, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(5)
    cases = [Case(attn, g, 4, 4, 64, dtype, *s) for s in [(2600, 0, 2600)] + [(1, 2200, 3)] * 31]
    attn.omnimem_attend([c.query() for c in cases])
    torch.cuda.synchronize()
    for c in cases:
        c.check(True)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [17, 24, 25, 32, 33, 47, 48, 49])
def test_rows_about_the_limits_of_the_few_row_kernels(dtype, nq):
    """64, 96, 128 and 192 rows of a head, over a memory and over tail rows, in batches that fill the chip."""
    attn = handle(8, 2, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(nq)
    for nm, nt in ((3000, nq), (0, 3000)):
        cases = [Case(attn, g, 8, 2, 64, dtype, nq, nm, nt, lse=i == 0) for i in range(9)]
        attn.omnimem_attend([c.query() for c in cases])
        torch.cuda.synchronize()
        for c in cases:
            c.check(True)
    attn.close()


def chunk_beside(g, h_q, h_kv, d, dtype, n=2600):
    """A chunk of so much work that its call takes the kernels of many rows for all of its sequences (those of few rows
    too, as they have fewer keys)."""
    td = TORCH[dtype]
    q = torch.randn(h_q, n, d, generator=g, device="cuda").to(td)
    k, v = (torch.randn(h_kv, n, d, generator=g, device="cuda").to(td) for _ in range(2))
    out = torch.empty_like(q)
    return om.make_query(q, out, k, v), (q, k, v, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,h_kv,d", [(6, 2, 64), (14, 2, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_small_sequences_in_the_kernels_of_chunks(dtype, h_q, h_kv, d, causal):
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(d)
    chunk, keep = chunk_beside(g, h_q, h_kv, d, dtype)
    for scale in (None, -0.3):
        cases = [Case(attn, g, h_q, h_kv, d, dtype, *s, scale=scale) for s in SIZES + [(0, 5, 5), (4, 0, 0), (100, 1200, 7), (33, 1000, 1300)]]
        attn.omnimem_attend([chunk] + [c.query() for c in cases], causal)
        torch.cuda.synchronize()
        for c in cases:
            c.check(causal)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_rows_that_are_not_seen_in_the_kernels_of_chunks(dtype, value):
    """As above for few rows: queries before the last keys' infinities and NaN are as without them."""
    attn = handle(6, 2, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(8)
    chunk, keep = chunk_beside(g, 6, 2, 64, dtype)
    for nq, nm, nt in ((60, 100, 130), (200, 0, 333), (300, 70, 300), (3, 300, 200)):
        seed = lambda: torch.Generator(device="cuda").manual_seed(nq)
        c, clean = (Case(attn, seed(), 6, 2, 64, dtype, nq, nm, nt) for _ in range(2))
        at = nt - nq // 2 - 1
        c.v[0, at, 5:9] = value
        c.k[1, at, 0] = value
        attn.omnimem_attend([chunk, c.query()])
        attn.omnimem_attend([chunk, clean.query()])
        torch.cuda.synchronize()
        before = nq - (nt - at)
        reach = float((clean.q.float().abs().sum(-1).amax() * torch.cat([clean.k[:, :nt].float().flatten(),
                      torch.tensor(clean.held[0], device="cuda").float().flatten()]).abs().amax()) * c.scale)
        near = 2 * (2 * (64 + 6) * U * reach + 2 * (nm + nt + 8) * U) + (3 * 2.0 ** -8 if dtype == "bf16" else 0.0)
        size = torch.cat([clean.v[:, :nt].float().flatten(), torch.tensor(clean.held[1], device="cuda").float().flatten()]).abs().amax()
        assert ((c.out[:, :before].float() - clean.out[:, :before].float()).abs() <= near * size).all()
        assert torch.equal(c.lse[:, :before], clean.lse[:, :before])
        assert (~torch.isfinite(c.out[:3, before: nq, 5:9])).all()
        assert ((c.out[:3, before: nq, 9:].float() - clean.out[:3, before: nq, 9:].float()).abs() <= near * size).all()
    c = Case(attn, g, 6, 2, 64, dtype, 100, 0, 100)            # products that are all -inf
    c.q.fill_(1.0)
    c.k[:, :100] = 0.0
    c.k[:, :100, 0] = float("-inf")
    attn.omnimem_attend([chunk, c.query()])
    torch.cuda.synchronize()
    assert (c.out[:, :100] == 0).all() and torch.isneginf(c.lse[:, :100]).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_chunks_over_memories(dtype, d):
    """Two chunks of odd lengths over memories that end inside a block and a tile, keys split over workgroups."""
    attn = handle(4, 4, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(d)
    cases = [Case(attn, g, 4, 4, d, dtype, *s) for s in [(2101, 2001, 2177), (333, 1999, 333)]]
    attn.omnimem_attend([c.query() for c in cases])
    torch.cuda.synchronize()
    for c in cases:
        c.check(True)
    attn.close()


@pytest.mark.parametrize("dtype,nq", [("bf16", 1), ("bf16", 130), ("f32", 1), ("f32", 120)])
def test_a_memory_past_32_bits_of_bytes(dtype, nq):
    """2^26 + 5 rows of zeros, but for ones in the values of the last 37: every weight is 1, so out is 37 of the rows'
    number and lse its logarithm.  Sums of ones are exact but for the join's: a rounding for each of up to 2048 shares."""
    rows, d = (1 << 26) + 5, 64
    attn = handle(1, 1, d, dtype)
    data = torch.zeros(om.memory_shape(1, d, rows), dtype=torch.uint8, device="cuda")
    assert data.numel() > 1 << 32
    data[0, -2:, 16 * d: 32 * d] = 0x22                         # V codes of 1 ...
    last = data[0, -1, 16 * d: 32 * d].view(d, 16)
    last[:, 2], last[:, 3:] = 0x02, 0                           # ... in the last block's first five rows
    data[0, -2:, 33 * d:] = 127                                 # their scale, 2^0
    q = torch.randn(1, nq, d, device="cuda").to(TORCH[dtype])
    out, lse = torch.zeros_like(q), torch.zeros(1, nq, device="cuda")
    attn.omnimem_attend([om.make_query(q, out, memory=data, memory_rows=rows, lse=lse)])
    torch.cuda.synchronize()
    join = 2048 * U + 8 * U
    assert (np.abs(host(out) * rows / 37 - 1) <= join + (2.0 ** -8 if dtype == "bf16" else 0)).all()
    assert (np.abs(host(lse) - np.log(rows)) <= join + 2 * U * np.log(rows)).all()
    attn.close()


def infinite_last(attn, g, dtype, nq, nm, nt):
    c = Case(attn, g, 6, 2, 64, dtype, nq, nm, nt)
    c.v[0, nt - 1, 5], c.v[0, nt - 1, 6] = float("inf"), float("-inf")
    return c


def check_infinite_last(c, causal):
    """Channels 5 and 6 of heads 0 .. 2 are infinities of one sign for queries that see the last row; all else as it is
    without them."""
    nq, nm, nt = c.sizes
    seeing = slice(nq - 1, nq) if causal else slice(0, nq)
    got = c.out[:3, seeing, 5:7].float()
    assert bool((got[..., 0] == float("inf")).all()) and bool((got[..., 1] == float("-inf")).all())
    c.v[0, nt - 1, 5:7] = 0.0                      # (the others against the definition)
    c.out[:3, seeing, 5:7] = 0.0
    k, v = (np.concatenate([m, host(t[:, :nt])], 1) for m, t in zip(c.held, (c.k, c.v)))
    out, lse, size, reach = orc.attend(host(c.q), k, v, nm, c.scale, causal)
    half, n = (2.0 ** -8 if c.q.dtype == torch.bfloat16 else 0.0), nm + nt
    tol = size * (2 * (64 + 6) * U * reach[..., None] + 2 * (n + 8) * U + half) + (half or U) * np.abs(out)
    off = np.abs(host(c.out[:, :nq]) - out)
    off[:3, seeing, 5:7] = 0.0
    assert (off <= tol + n * 2.0 ** -126 * np.abs(v).max()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nm,nt", [(1, 0, 5), (5, 0, 33), (40, 31, 77), (130, 0, 131), (300, 100, 411), (3, 2100, 2001), (200, 0, 1333)])
def test_an_infinity_in_the_last_tail_row(dtype, causal, nq, nm, nt):
    """A tile that ends behind it adds nothing to it: what sees it gets an infinity and not NaN, alone and beside a chunk."""
    attn = handle(6, 2, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(nt)
    chunk, keep = chunk_beside(g, 6, 2, 64, dtype)
    for before in ([], [chunk]):
        c = infinite_last(attn, g, dtype, nq, nm, nt)
        attn.omnimem_attend(before + [c.query()], causal)
        torch.cuda.synchronize()
        check_infinite_last(c, causal)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nt", [(1, 64), (1, 3000), (40, 77), (130, 128), (200, 2500)])
def test_no_weight_at_all_is_0_whatever_the_values(dtype, nq, nt):
    """Products that are all -inf beside values that are infinite or NaN: out = 0 and lse = -inf all the same."""
    attn = handle(6, 2, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(nt)
    chunk, keep = chunk_beside(g, 6, 2, 64, dtype)
    for before in ([], [chunk]):
        c = Case(attn, g, 6, 2, 64, dtype, nq, 0, nt)
        c.q.fill_(1.0)
        c.k[:, :nt] = 0.0
        c.k[:, :nt, 0] = float("-inf")
        c.v[0, :nt:3, 5], c.v[1, :nt:5, 9] = float("inf"), float("nan")
        attn.omnimem_attend(before + [c.query()], False)
        torch.cuda.synchronize()
        assert (c.out[:, :nq] == 0).all() and torch.isneginf(c.lse[:, :nq]).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nm,nt", [(3, 0, 33), (40, 31, 77), (130, 0, 131), (300, 100, 411), (3, 2100, 2001)])
def test_nan_that_is_seen(dtype, causal, nq, nm, nt):
    """Queries that are NaN, and NaN in a key and in a value that every query sees: NaN where the definition has it, alone
    and beside a chunk."""
    attn = handle(6, 2, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(nt)
    chunk, keep = chunk_beside(g, 6, 2, 64, dtype)
    nan = float("nan")
    for before in ([], [chunk]):
        for what in ("query", "key", "value"):
            c = Case(attn, g, 6, 2, 64, dtype, nq, nm, nt)
            if what == "query":
                c.q[1, nq // 2], c.q[4, nq - 1, 7] = nan, nan
            elif what == "key":
                c.k[1, 0, 3] = nan
            else:
                c.v[1, 0, 3] = nan
            attn.omnimem_attend(before + [c.query()], causal)
            torch.cuda.synchronize()
            # (as Case.check, with the largest value that is not NaN)
            k, v = (np.concatenate([m, host(t[:, :nt])], 1) for m, t in zip(c.held, (c.k, c.v)))
            out, lse, size, reach = orc.attend(host(c.q), k, v, nm, c.scale, causal)
            half, n, got = (2.0 ** -8 if dtype == "bf16" else 0.0), nm + nt, host(c.out[:, :nq])
            nans = np.isnan(out)
            assert nans.any() and not nans.all() and np.array_equal(np.isnan(got), nans)
            tol = size * (2 * (64 + 6) * U * reach[..., None] + 2 * (n + 8) * U + half) + (half or U) * np.abs(out)
            assert (np.abs(got - out)[~nans] <= tol[~nans] + n * 2.0 ** -126 * np.nanmax(np.abs(v))).all()
            assert np.array_equal(np.isnan(host(c.lse[:, :nq])), np.isnan(lse))
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [4, 1000])
def test_nan_that_is_seen_costs_no_second_pass(dtype, nq):
    """NaN that belongs into the results takes the time of the pass, not that of forming the rows again one by one (30 to
    140 times as long at these sizes)."""
    attn = handle(8, 2, 128, dtype)
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda h, n: torch.randn(h, n, 128, generator=g, device="cuda").to(TORCH[dtype])
    q, k, v = rnd(8, nq), rnd(2, 2001), rnd(2, 2001)
    out = torch.empty_like(q)

    def least(q, v, causal):
        queries = om.array_of([om.make_query(q, out, k, v)])
        times = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            attn.omnimem_attend(queries, causal)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    bad_q, bad_v = torch.full_like(q, float("nan")), v.clone()
    bad_v[:, 0] = float("nan")
    for causal in (True, False):
        plain = least(q, v, causal)
        for args in ((bad_q, v), (q, bad_v)):
            assert least(*args, causal) < 4 * plain + 0.05
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_call_of_several_launches(dtype, d):
    """70 sequences where a launch describes 32, long ones whose keys are split and joined in each of the launches (they use
    the same partials and counters), and empty ones about the borders."""
    attn = handle(4, 2, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(d)
    sizes = [(1 + (5 * i) % 7, (337 * i) % 2900, 1 + (11 * i) % 90) for i in range(70)]
    for i in (0, 30, 31, 32, 33, 64, 69):
        sizes[i] = (0, 40, 5) if i % 2 else (2, 0, 0)
    sizes[12], sizes[45] = (1, 9000, 3), (9, 0, 6000)
    cases = [Case(attn, g, 4, 2, d, dtype, *s, lse=i % 3 == 0) for i, s in enumerate(sizes)]
    queries = om.array_of([c.query() for c in cases])
    for _ in range(2):
        for c in cases:
            c.out.fill_(7.0)
        attn.omnimem_attend(queries)
        torch.cuda.synchronize()
        for c in cases:
            c.check(True)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chunks_and_tokens_in_a_call_of_several_launches(dtype):
    """A chunk among the first 32 sequences and one behind them, tokens with more keys beside each."""
    attn = handle(4, 4, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(6)
    sizes = [(1, 20 + 3 * i, 1 + i % 5) for i in range(40)]
    sizes[3], sizes[4], sizes[36], sizes[37] = (2600, 0, 2600), (1, 3000, 5), (1, 2000, 900), (1500, 300, 1500)
    cases = [Case(attn, g, 4, 4, 64, dtype, *s) for s in sizes]
    attn.omnimem_attend([c.query() for c in cases])
    torch.cuda.synchronize()
    for c in cases:
        c.check(True)
    attn.close()
