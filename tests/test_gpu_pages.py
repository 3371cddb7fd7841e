"""The operators on caches in pages against their definitions in 64 bits.

omnimem_rotate_pages: as omnimem_rotate, with M = |x_a| + |x_b| off by 24 * 2^-24 M and the last rounding, eps / 2 of
the value.  omnimem_attend_pages: as omnimem_attend.  With S the largest sum of |q||k| scale of a row's products, u =
2^-24 and N keys: products and weights are off by at most (d + 6) u S, sums of N weights and products by (N + 8) u of
their sizes; with A the weighted mean of |v|, out is off by at most A (2 (d + 6) u S + 2 (N + 8) u), with bf16 by A eps / 2
(weights) and eps / 2 of the value (the result) more; lse by (d + 6) u S + (N + 8) u and 2 u of its value.  Weights below
2^-126 of the largest may be missing: N of them times the largest |v|.  omnimem_keep_pages moves bits."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2606_07577_amd import omnimem as om

pytestmark = pytest.mark.gpu
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
ODD = (-1, -2 ** 31, 10 ** 6, 2 ** 31 - 1)      # entries that are no page


def host(t):
    return t.double().cpu().numpy()


def handle(h_q, h_kv, d, dtype):
    return om.Attention(h_q, h_kv, d, om.BF16 if dtype == "bf16" else om.F32)


class Store:
    """Pages [pages, h, page_rows, d] in one of four layouts, all rows NaN but those that are filled."""

    def __init__(self, g, h_kv, d, dtype, page_rows, lengths, layout="pages"):
        td = TORCH[dtype]
        per = [-(-n // page_rows) for n in lengths]
        n = sum(per) + 2
        if layout == "pages":
            k, v = (torch.full((n, h_kv, page_rows, d), float("nan"), device="cuda", dtype=td) for _ in range(2))
        elif layout == "rows":                   # heads inside rows, K and V of a page side by side, rows with a gap
            both = torch.full((n, 2, page_rows, h_kv, d + 16), float("nan"), device="cuda", dtype=td)
            k, v = (both[:, i, :, :, :d].transpose(1, 2) for i in range(2))
        elif layout == "beside":                 # heads inside rows, K and V of a head of a row side by side
            both = torch.full((n, page_rows, h_kv, 2, d), float("nan"), device="cuda", dtype=td)
            k, v = (both[:, :, :, i].transpose(1, 2) for i in range(2))
        else:                                    # heads outside pages
            k, v = (torch.full((h_kv, n, page_rows, d), float("nan"), device="cuda", dtype=td).transpose(0, 1) for _ in range(2))
        self.k, self.v, self.rows = k, v, page_rows
        ids = torch.randperm(n, generator=torch.Generator().manual_seed(n)).tolist()
        self.tables = []
        for m in per:
            self.tables.append([ids.pop() for _ in range(m)])
        self.device_tables = [torch.tensor(t + [ODD[0]], dtype=torch.int32, device="cuda") for t in self.tables]
        for t, m in zip(self.tables, lengths):
            for r in range(0, m, page_rows):
                c = min(page_rows, m - r)
                for x in (self.k, self.v):
                    x[t[r // page_rows], :, :c] = torch.randn(h_kv, c, d, generator=g, device="cuda").to(td)

    def pages(self):
        return om.make_pages(self.k, self.v)

    def rows_of(self, b, n):
        """(K, V, there) of a sequence's first n rows in 64 bits."""
        table = self.device_tables[b].cpu().numpy()
        k, there = orc.paged(host(self.k), table, n, self.rows)
        return k, orc.paged(host(self.v), table, n, self.rows)[0], there


class Case:
    """One sequence's queries over a memory and its rows on the store's pages, an output with a border that stays."""

    def __init__(self, attn, g, h_q, h_kv, d, dtype, nq, nm, nt, masks=None, scale=None, lse=True):
        td = TORCH[dtype]
        self.sizes, self.masks, self.scale = (nq, nm, nt), masks, scale or d ** -0.5
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.q = rnd(nq, h_q, d).to(td).transpose(0, 1)
        self.data, self.held = None, (np.zeros((h_kv, 0, d)),) * 2
        if nm:
            km, vm = (rnd(h_kv, nm, d).to(td) for _ in range(2))
            self.data = torch.zeros(om.memory_shape(h_kv, d, nm), dtype=torch.uint8, device="cuda")
            attn.omnimem_pack([om.make_held(km, vm, self.data)])
            torch.cuda.synchronize()
            self.held = orc.unpack(self.data.cpu().numpy(), nm)
        self.tree = None if masks is None else torch.tensor([m - (m >> 63 << 64) for m in masks], dtype=torch.int64, device="cuda")
        self.out = torch.full((h_q, nq + 1, d), 7.0, device="cuda", dtype=td)
        self.lse = torch.full((h_q, nq + 1), 7.0, device="cuda") if lse else None

    def query(self, store, b):
        nq, nm, nt = self.sizes
        return om.make_paged_query(self.q, self.out[:, :nq], store.device_tables[b] if nt else None, nt, self.data, nm, self.tree, self.scale,
                                   None if self.lse is None else self.lse[:, :nq])

    def check(self, store, b, window, sinks):
        nq, nm, nt = self.sizes
        d, dt = self.q.shape[2], self.q.dtype
        k, v, there = store.rows_of(b, nt)
        see = np.concatenate([np.ones((nq, nm), bool), orc.paged_seen(nq, nt, window, sinks, self.masks) & there], 1)
        k, v = (np.concatenate([m, t], 1) for m, t in zip(self.held, (k, v)))
        out, lse, size, reach = orc.attend_seen(host(self.q), k, v, see, self.scale)
        n, half = max(1, int(see.sum(1).max(initial=0))), torch.finfo(dt).eps / 2 if dt == torch.bfloat16 else 0.0
        near = 2 * (d + 6) * U * reach[..., None] + 2 * (n + 8) * U + half
        seen_v = v[:, see.any(0)]
        tol = size * near + (half or U) * np.abs(out) + n * 2.0 ** -126 * np.abs(seen_v[np.isfinite(seen_v)]).max(initial=0.0)
        got = host(self.out[:, :nq])
        assert np.array_equal(np.isnan(got), np.isnan(out)), (self.sizes, window, sinks)
        f = np.isfinite(out)                                    # (infinities are the same ones)
        assert np.array_equal(got[np.isinf(out)], out[np.isinf(out)]), (self.sizes, window, sinks)
        assert (np.abs(got[f] - out[f]) <= tol[f]).all(), (self.sizes, window, sinks, float((np.abs(got[f] - out[f]) / tol[f]).max()))
        assert (self.out[:, nq:] == 7).all()
        if self.lse is not None:
            got = host(self.lse[:, :nq])
            assert np.array_equal(np.isneginf(got), np.isneginf(lse)) and np.array_equal(np.isnan(got), np.isnan(lse))
            f = np.isfinite(lse)
            assert (np.abs(got[f] - lse[f]) <= (d + 6) * U * reach[f] + (n + 8) * U + 2 * U * np.abs(lse[f])).all()
            assert (self.lse[:, nq:] == 7).all()


def tree_of(n, seed):
    rng = np.random.default_rng(seed)
    return [m % (1 << 64) for m in om.tree_masks([int(rng.integers(max(-1, i - 5), i)) for i in range(n)])]


class Heavy:
    """A sequence of so much work over a memory that its call takes the kernels of many rows for all of its sequences
    (those of few rows would leave for a launch of their own if they had more keys)."""

    def __init__(self, attn, g, h_q, h_kv, d, dtype, held=20000):
        n = 36000 // h_q
        self.q = torch.randn(h_q, n, d, generator=g, device="cuda").to(TORCH[dtype])
        self.out = torch.zeros_like(self.q)
        rows = [torch.randn(h_kv, held, d, generator=g, device="cuda").to(TORCH[dtype]) for _ in range(2)]
        self.data = torch.zeros(om.memory_shape(h_kv, d, held), dtype=torch.uint8, device="cuda")
        attn.omnimem_pack([om.make_held(*rows, self.data)])
        self.query = om.make_paged_query(self.q, self.out, None, 0, self.data, held)


def attend(attn, store, cases, window=0, sinks=0, beside=None, **more):
    queries = [c.query(store, b) for b, c in enumerate(cases)]
    attn.omnimem_attend_pages(store.pages(), ([beside.query] if beside else []) + queries, window, sinks, **more)
    torch.cuda.synchronize()
    for b, c in enumerate(cases):
        c.check(store, b, window, sinks)


HEADS = [(7, 1, 128), (4, 2, 64), (2, 2, 128), (20, 1, 64)]
# queries, memory rows, tail rows, window, sinks, page rows
SIZES = [(1, 0, 1, 0, 0, 16), (1, 0, 300, 100, 4, 16), (1, 219, 5, 0, 0, 16), (1, 40, 900, 1, 0, 32), (3, 0, 300, 64, 17, 128),
         (5, 70, 260, 30, 0, 256), (9, 0, 4, 2, 1, 16), (40, 31, 77, 20, 200, 64), (17, 0, 129, 0, 0, 16), (130, 0, 130, 50, 3, 16),
         (70, 257, 700, 90, 65, 32), (300, 0, 411, 64, 4, 16), (260, 33, 1500, 130, 1, 64), (2, 0, 0, 5, 5, 16), (300, 0, 100, 33, 2, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("sizes", SIZES)
def test_windows(dtype, h_q, h_kv, d, sizes):
    nq, nm, nt, window, sinks, page_rows = sizes
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(sum(sizes))
    store = Store(g, h_kv, d, dtype, page_rows, [nt], layout=["pages", "rows", "heads"][(nt + h_q) % 3])
    attend(attn, store, [Case(attn, g, h_q, h_kv, d, dtype, nq, nm, nt)], window, sinks)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("nq,nm,nt,window,sinks,page_rows", [
    (1, 0, 1, 0, 0, 16), (1, 30, 1, 7, 0, 16), (7, 219, 12, 0, 0, 16), (16, 0, 16, 0, 0, 32), (26, 100, 200, 50, 4, 32), (64, 0, 64, 0, 0, 16),
    (64, 0, 1000, 0, 0, 64), (63, 40, 333, 20, 0, 16), (64, 0, 500, 3, 70, 128), (33, 0, 159, 40, 1, 16)])
def test_trees(dtype, h_q, h_kv, d, nq, nm, nt, window, sinks, page_rows):
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(nq + nt)
    store = Store(g, h_kv, d, dtype, page_rows, [nt])
    masks = tree_of(nq, nt)
    if nq > 20:                                  # masks that are no tree's: nothing, all, bits behind the drafts
        masks[3], masks[4], masks[5] = 0, (1 << 64) - 1, 1 << 63 | 1
    attend(attn, store, [Case(attn, g, h_q, h_kv, d, dtype, nq, nm, nt, masks)], window, sinks)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_mask_that_leaves_nothing(dtype):
    """Drafts that see no draft, over no cache: 0 and -inf; a window behind which nothing lies."""
    attn = handle(4, 2, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    store = Store(g, 2, 64, dtype, 16, [5])
    c = Case(attn, g, 4, 2, 64, dtype, 5, 0, 5, [0, 1, 0, 8, 2])
    attend(attn, store, [c])
    assert (c.out[:, 0] == 0).all() and (c.out[:, 2] == 0).all() and torch.isneginf(c.lse[:, [0, 2]]).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_ragged_batches(dtype, d):
    """More sequences than a launch describes, of all forms, empty ones among them, tokens beside prompts and trees."""
    h_q, h_kv = 6, 2
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(d)
    sizes = [(1 + (5 * i) % 23, (37 * i) % 300, 24 + (11 * i) % 90) for i in range(34)] + [(0, 5, 5), (4, 0, 0), (1, 0, 2500), (200, 0, 330)]
    store = Store(g, h_kv, d, dtype, 16, [n for _, _, n in sizes])
    cases = [Case(attn, g, h_q, h_kv, d, dtype, *s, masks=tree_of(s[0], i) if i % 3 == 1 and s[0] <= min(64, s[2]) else None, lse=i % 2 == 0)
             for i, s in enumerate(sizes)]
    attend(attn, store, cases, 40, 3)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nm,nt,window,tree", [(1, 0, 9000, 0, False), (1, 9000, 70, 0, False), (3, 0, 5000, 3000, False),
                                                  (50, 2000, 1500, 0, False), (64, 0, 3000, 0, True), (40, 3000, 900, 500, True)])
def test_keys_split_over_workgroups(dtype, nq, nm, nt, window, tree):
    attn = handle(2, 1, 128, dtype)
    g = torch.Generator(device="cuda").manual_seed(nq)
    store = Store(g, 1, 128, dtype, 32, [nt])
    c = Case(attn, g, 2, 1, 128, dtype, nq, nm, nt, tree_of(nq, 3) if tree else None)
    attend(attn, store, [c], window, 4)
    first = c.out.clone()
    for _ in range(3):                       # the sums' order is fixed: the same bits every time
        c.out.fill_(7.0)
        attend(attn, store, [c], window, 4)
        assert torch.equal(c.out, first)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,h_kv,d", [(6, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 5), (1, 200)])
def test_small_sequences_in_the_kernels_of_many_rows(dtype, h_q, h_kv, d, window, sinks):
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(window)
    beside = Heavy(attn, g, h_q, h_kv, d, dtype)
    for page_rows in (16, 64, 256):
        sizes = [(1, 0, 1), (1, 219, 300), (5, 0, 64), (64, 0, 64), (33, 70, 200), (150, 0, 411), (3, 0, 2), (40, 100, 1000), (300, 40, 150)]
        store = Store(g, h_kv, d, dtype, page_rows, [n for _, _, n in sizes], ["pages", "rows", "heads"][page_rows // 64 % 3])
        cases = [Case(attn, g, h_q, h_kv, d, dtype, *s, masks=tree_of(s[0], i) if i in (3, 4, 7) else None) for i, s in enumerate(sizes)]
        attend(attn, store, cases, window, sinks, beside)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("many", [False, True])
def test_keys_beside_values(dtype, many):
    """A store whose rows hold a head's key and its value one behind the other."""
    attn = handle(4, 2, 128, dtype)
    g = torch.Generator(device="cuda").manual_seed(12)
    beside = Heavy(attn, g, 4, 2, 128, dtype) if many else None
    sizes = [(1, 0, 1), (1, 40, 300), (33, 0, 200), (150, 70, 411), (64, 0, 90)]
    store = Store(g, 2, 128, dtype, 64, [n for _, _, n in sizes], "beside")
    cases = [Case(attn, g, 4, 2, 128, dtype, *s, masks=tree_of(64, 3) if s[0] == 64 else None) for s in sizes]
    for window, sinks in ((0, 0), (70, 5)):
        attend(attn, store, cases, window, sinks, beside)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks,tail", [(0, 0, 6100), (700, 20, 9000)])
def test_prompts(dtype, window, sinks, tail):
    """Enough work for the kernels of many rows by themselves, row tiles split over workgroups."""
    attn = handle(3, 1, 128, dtype)
    g = torch.Generator(device="cuda").manual_seed(tail)
    store = Store(g, 1, 128, dtype, 64, [tail])
    beside = Heavy(attn, g, 3, 1, 128, dtype, held=8000)
    c = Case(attn, g, 3, 1, 128, dtype, 1111, 0, tail)
    attend(attn, store, [c], window, sinks, beside)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,nq,window", [(2, 1, 0), (2, 3, 100), (16, 40, 0), (8, 300, 90), (8, 300, 0)])
@pytest.mark.parametrize("many", [False, True])
def test_entries_that_are_no_page(dtype, h_q, nq, window, many):
    """Rows on them are not seen, wherever they lie; what no query's window holds is not looked at."""
    attn = handle(h_q, 2, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(nq)
    beside = Heavy(attn, g, h_q, 2, 64, dtype) if many else None
    nt = 700
    store = Store(g, 2, 64, dtype, 16, [nt])
    table = store.device_tables[0]
    for i, entry in ((0, ODD[0]), (20, ODD[1]), (37, ODD[2]), (38, ODD[3]), (43, -1)):
        table[i] = entry
    c = Case(attn, g, h_q, 2, 64, dtype, nq, 0, nt)
    attend(attn, store, [c], window, 4, beside)
    table.fill_(-1)                              # no page at all: nothing is seen
    attend(attn, store, [c], window, 4, beside)
    assert (c.out[:, :nq] == 0).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,tree", [(1, False), (20, False), (30, True), (64, True), (300, False)])
@pytest.mark.parametrize("odd", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("many", [False, True])
def test_odd_values_that_are_not_seen(dtype, nq, tree, odd, many):
    """Infinities and NaN in rows before the window, of other drafts, on other sequences' pages and behind the tail have
    no part; page 0, that entries without a page are read from, holds them too."""
    attn = handle(4, 2, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(nq)
    beside = Heavy(attn, g, 4, 2, 64, dtype) if many else None
    nt, window = 411, 100
    store = Store(g, 2, 64, dtype, 16, [nt])
    store.k[0], store.v[0] = odd, odd
    masks = tree_of(nq, 5) if tree else None
    c = Case(attn, g, 4, 2, 64, dtype, nq, 0, nt, masks)
    table = store.tables[0]
    if 0 in table:                               # (this sequence's page 0 stays out of it)
        i = table.index(0)
        free = next(p for p in range(len(store.k)) if p not in table)
        store.k[free], store.v[free] = (torch.randn(2, 16, 64, generator=g, device="cuda").to(TORCH[dtype]) for _ in range(2))
        store.device_tables[0][i] = table[i] = free
    store.device_tables[0][22] = -1              # a hole inside the window
    low = nt - nq - window                       # every query's window begins behind this row
    for j in range(max(4, low - 40), max(4, low - 5)):
        for x in (store.k, store.v):
            x[table[j // 16], :, j % 16] = odd
    if tree:                                     # a draft that only its own branch sees
        x = nt - nq + nq // 2
        store.v[table[x // 16], :, x % 16, 3] = odd
    elif nq > 1:                                 # the last row: the last query alone sees it
        store.v[table[(nt - 1) // 16], :, (nt - 1) % 16, 3] = odd
    attend(attn, store, [c], window, 4, beside)
    attn.close()


# queries, memory rows, tail rows (whole key tiles of every kernel, but for the last), page rows, entries without a page
SEEN_WHOLE = [(1, 0, 64, 16, [1]), (1, 0, 128, 16, [0, 5]), (1, 0, 384, 32, [6]), (1, 70, 384, 16, [13]), (3, 0, 8192, 64, [9, 70, 71]),
              (1, 4000, 8192, 16, [0, 300]), (20, 0, 640, 128, [2]), (90, 33, 1024, 16, [1, 20, 21]), (300, 0, 2048, 64, [7]),
              (2, 0, 256, 16, [15]), (1, 0, 32, 16, [0, 1])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,h_kv,d", [(4, 2, 64), (7, 1, 128)])
@pytest.mark.parametrize("nq,nm,nt,page_rows,lost", SEEN_WHOLE)
@pytest.mark.parametrize("many", [False, True])
def test_holes_among_rows_that_are_all_seen(dtype, h_q, h_kv, d, nq, nm, nt, page_rows, lost, many):
    """Rows without a page between rows of whole key tiles that a query sees, in one share and in several: what page 0,
    another sequence's, holds in their place has no part."""
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(nt + nq)
    beside = Heavy(attn, g, h_q, h_kv, d, dtype) if many else None
    store = Store(g, h_kv, d, dtype, page_rows, [nt])
    table = store.tables[0]
    if 0 in table:                               # (the sequence's own rows lie elsewhere)
        i, free = table.index(0), next(p for p in range(len(store.k)) if p not in table)
        store.k[free], store.v[free] = store.k[0], store.v[0]
        store.device_tables[0][i] = table[i] = free
    for i, x in enumerate(lost):
        store.device_tables[0][x] = ODD[i]
    c = Case(attn, g, h_q, h_kv, d, dtype, nq, nm, nt)
    for odd in (float("nan"), float("inf"), -float("inf")):
        store.k[0], store.v[0] = odd, odd
        c.out.fill_(7.0)
        attend(attn, store, [c], beside=beside)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_infinities_and_sharp_weights(dtype):
    attn = handle(4, 1, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(9)
    for scale in (1e-6, 30.0, -0.2):
        store = Store(g, 1, 64, dtype, 32, [350])
        for nq, masks in ((2, None), (90, None), (40, tree_of(40, 1))):
            attend(attn, store, [Case(attn, g, 4, 1, 64, dtype, nq, 200, 350, masks, scale)], 120, 2)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [1, 40, 200])
def test_whole_caches_give_what_contiguous_rows_give(dtype, nq):
    """Pages in order, no window: omnimem_attend on the rows as they lie, whose keys may be summed in another order: both
    are within the module's bound of the definition."""
    attn = handle(8, 2, 128, dtype)
    g = torch.Generator(device="cuda").manual_seed(nq)
    nt = 500
    k, v = (torch.randn(2, 512, 128, generator=g, device="cuda").to(TORCH[dtype]) for _ in range(2))
    q = torch.randn(8, nq, 128, generator=g, device="cuda").to(TORCH[dtype])
    out, paged = torch.zeros_like(q), torch.zeros_like(q)
    table = torch.arange(8, dtype=torch.int32, device="cuda")
    pages = om.make_pages(*(x.view(2, 8, 64, 128).transpose(0, 1) for x in (k, v)))
    attn.omnimem_attend([om.make_query(q, out, k[:, :nt], v[:, :nt])])
    attn.omnimem_attend_pages(pages, [om.make_paged_query(q, paged, table, nt)])
    torch.cuda.synchronize()
    want, _, size, reach = orc.attend(host(q), host(k[:, :nt]), host(v[:, :nt]), 0, 128 ** -0.5, True)
    half = torch.finfo(q.dtype).eps / 2 if dtype == "bf16" else 0.0
    tol = size * (2 * (128 + 6) * U * reach[..., None] + 2 * (nt + 8) * U + half) + (half or U) * np.abs(want) + nt * 2.0 ** -126 * 10
    for x in (out, paged):
        assert (np.abs(host(x) - want) <= tol).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sequences_that_share_pages_and_fused_rows(dtype):
    """Two sequences with the same first pages, the same sequence twice, queries and results as parts of fused rows."""
    h_q, h_kv, d = 6, 2, 64
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(5)
    store = Store(g, h_kv, d, dtype, 16, [100, 60], "rows")
    store.device_tables[1][:2] = store.device_tables[0][:2]
    store.device_tables.append(store.device_tables[0])
    cases = [Case(attn, g, h_q, h_kv, d, dtype, *s) for s in ((3, 0, 100), (20, 33, 60), (3, 0, 100))]
    cases[2].q = cases[0].q
    fused = torch.randn(20, (h_q + 2 * h_kv) * d, generator=g, device="cuda").to(TORCH[dtype])
    cases[1].q = fused.view(20, h_q + 2 * h_kv, d).transpose(0, 1)[:h_q]
    rows = torch.full((21, h_q, d + 8), 7.0, device="cuda", dtype=TORCH[dtype])
    cases[1].out = rows[:, :, :d].transpose(0, 1)
    attend(attn, store, cases, 50, 3)
    assert torch.equal(cases[0].out, cases[2].out) and (rows[:, :, d:] == 7).all()
    attn.close()


def test_pages_far_apart():
    """Pages past 2^32 bytes from the first."""
    attn = handle(4, 2, 128, "bf16")
    g = torch.Generator(device="cuda").manual_seed(2)
    far = (5 << 30) // 2                         # elements
    flat = torch.zeros(2 * far + 2 * 16 * 128, device="cuda", dtype=torch.bfloat16)
    k, v = (flat[i * 2 * 16 * 128:][: far + 2 * 16 * 128].as_strided((2, 2, 16, 128), (far, 16 * 128, 128, 1)) for i in (0, 1))
    k.copy_(torch.randn(2, 2, 16, 128, generator=g, device="cuda"))
    v.copy_(torch.randn(2, 2, 16, 128, generator=g, device="cuda"))
    store = Store.__new__(Store)
    store.k, store.v, store.rows = k, v, 16
    store.device_tables = [torch.tensor([1, 0], dtype=torch.int32, device="cuda")]
    for nq in (1, 31):
        attend(attn, store, [Case(attn, g, 4, 2, 128, "bf16", nq, 0, 31)])
    new = [torch.randn(h, 1, 128, generator=g, device="cuda").bfloat16() for h in (4, 2, 2)]
    rope = om.make_rope(128, [0.0] * 64)
    pos = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    row = om.make_paged_projection(*new, pos, torch.zeros_like(new[0]), store.device_tables[0], 15)
    attn.omnimem_rotate_pages(rope, store.pages(), [row])
    attn.omnimem_keep_pages([store.pages()], [om.make_path(store.device_tables[0], 5, [10])])
    torch.cuda.synchronize()
    assert torch.equal(k[1, :, 15], new[1][:, 0]) and torch.equal(k[1, :, 5], new[1][:, 0]) and torch.equal(v[1, :, 5], new[2][:, 0])
    attn.close()


# --- rotation into pages -------------------------------------------------------

def size_of(x, rot, neighbours):
    """|x_a| + |x_b| of each channel's pair (|x| of one that does not turn)."""
    a, half = np.abs(x), rot // 2
    out = a.copy()
    if neighbours:
        out[..., :rot] = np.repeat(a[..., 0:rot:2] + a[..., 1:rot:2], 2, -1)
    else:
        out[..., :rot] = np.tile(a[..., :half] + a[..., half:rot], 2)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,neighbours", [(128, 128, False), (128, 96, True), (64, 64, False), (64, 48, True), (64, 0, False)])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("page_rows,layout,lengths", [(16, "pages", [1, 0, 7, 130]), (64, "rows", [1] * 35), (32, "heads", [4000, 300, 1]), (128, "beside", [70, 300, 1])])
def test_rows_go_to_their_pages(dtype, d, rot, neighbours, norm, page_rows, layout, lengths):
    h_q, h_kv, axes = 5, 1, 3
    g = torch.Generator(device="cuda").manual_seed(rot + d)
    attn = handle(h_q, h_kv, d, dtype)
    freq = [10000.0 ** (-j / max(1, rot // 2)) for j in range(rot // 2)]
    axis = [(j * 7) % axes for j in range(rot // 2)]
    w = (1 + 0.3 * torch.randn(2, d, generator=g, device="cuda")).to(TORCH[dtype])
    rope = om.make_rope(d, freq, axis, axes, rot, neighbours, w[0] if norm else None, w[1] if norm else None, eps=1e-5)
    back = [(13 * i) % 50 for i in range(len(lengths))]
    store = Store(g, h_kv, d, dtype, page_rows, [n + b for n, b in zip(lengths, back)], layout)
    before = store.k.clone(), store.v.clone()
    keep, seqs = [], []
    for i, n in enumerate(lengths):
        fused = torch.randn(n, (h_q + 2 * h_kv) * d, generator=g, device="cuda").to(TORCH[dtype])
        q, k, v = fused.view(n, h_q + 2 * h_kv, d).transpose(0, 1).split([h_q, h_kv, h_kv])
        pos = torch.randint(-2_000_000, 2_000_000, (axes, n), generator=g, device="cuda").to(torch.int32)
        q_out = torch.full((h_q, n + 2, d), 7.0, device="cuda", dtype=TORCH[dtype])
        keep.append((q, k, v, pos, q_out))
        seqs.append(om.make_paged_projection(q, k, v, pos, q_out[:, :n], store.device_tables[i], back[i]))
    attn.omnimem_rotate_pages(rope, store.pages(), seqs)
    torch.cuda.synchronize()
    same = torch.ones(store.k.shape[:3], dtype=torch.bool, device="cuda")        # rows that nobody writes
    for i, (n, (q, k, v, pos, q_out)) in enumerate(zip(lengths, keep)):
        p = pos.cpu().numpy()
        at = torch.arange(back[i], back[i] + n, device="cuda")
        page, row = store.device_tables[i].long()[at // page_rows], at % page_rows
        same[page, :, row] = False
        for x, y, weight in ((q, q_out[:, :n], w[0]), (k, store.k[page, :, row].transpose(0, 1), w[1])):
            weight = host(weight) if norm else None
            ref = orc.rotate(host(x), p, freq, axis, rot, neighbours, weight, 1e-5)
            flat = orc.rotate(host(x), p, freq, axis, 0, neighbours, weight, 1e-5)
            tol = torch.finfo(TORCH[dtype]).eps / 2 * np.abs(ref) + 24 * U * size_of(flat, rot, neighbours)
            assert (np.abs(host(y) - ref) <= tol).all()
        assert torch.equal(store.v[page, :, row].transpose(0, 1), v)
        assert (q_out[:, n:] == 7).all()
    for x, y in zip((store.k, store.v), before):
        assert torch.equal(x[same].nan_to_num(9.0), y[same].nan_to_num(9.0))
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,h_kv,d", [(120, 30, 128), (31, 31, 64), (1, 1, 64)])
def test_more_heads_than_a_workgroup_has_lanes_for(dtype, h_q, h_kv, d):
    """As omnimem_rotate in rows of their own, within twice its bound (the norm's squares are summed in another order)."""
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(h_q)
    n = 9
    store = Store(g, h_kv, d, dtype, 16, [n + 3])
    q, k, v = (torch.randn(h, n, d, generator=g, device="cuda").to(TORCH[dtype]) for h in (h_q, h_kv, h_kv))
    w = (1 + 0.3 * torch.randn(2, d, generator=g, device="cuda")).to(TORCH[dtype])
    pos = torch.randint(0, 9000, (2, n), generator=g, device="cuda").to(torch.int32)
    rope = om.make_rope(d, [0.9 ** j for j in range(d // 2)], [j % 2 for j in range(d // 2)], q_weight=w[0], k_weight=w[1])
    out, outs = torch.zeros_like(q), [torch.zeros_like(x) for x in (q, k, v)]
    attn.omnimem_rotate_pages(rope, store.pages(), [om.make_paged_projection(q, k, v, pos, out, store.device_tables[0], 3)])
    attn.omnimem_rotate(rope, [om.make_projection(q, k, v, pos, *outs)])
    torch.cuda.synchronize()
    at = torch.arange(3, 3 + n, device="cuda")
    page = store.device_tables[0].long()[at // 16]
    keys = store.k[page, :, at % 16].transpose(0, 1)
    for x, y, raw, weight in ((out, outs[0], q, w[0]), (keys, outs[1], k, w[1])):
        flat = orc.rotate(host(raw), pos.cpu().numpy(), [0.0] * (d // 2), [0] * (d // 2), 0, False, host(weight), 1e-6)
        tol = 2 * (torch.finfo(x.dtype).eps / 2 * np.abs(host(y)) * (1 + 2.0 ** -7) + 24 * U * size_of(flat, d, False))
        assert (np.abs(host(x) - host(y)) <= tol).all()
    assert torch.equal(store.v[page, :, at % 16].transpose(0, 1), v)
    attn.close()


@pytest.mark.parametrize("rows", [5, 5000])
def test_rows_without_a_page_are_dropped(rows):
    attn = handle(2, 2, 64, "bf16")
    g = torch.Generator(device="cuda").manual_seed(rows)
    store = Store(g, 2, 64, "bf16", 16, [rows + 20])
    before = store.k.clone()
    lost = store.device_tables[0].clone()
    for i, entry in enumerate(ODD[: 1 if rows < 100 else 4]):
        lost[1 + i * max(1, rows // 100)] = entry
    q, k, v = (torch.randn(2, rows, 64, generator=g, device="cuda").bfloat16() for _ in range(3))
    pos = torch.zeros(1, rows, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    attn.omnimem_rotate_pages(om.make_rope(64, []), store.pages(), [om.make_paged_projection(q, k, v, pos, out, lost, 20)])
    torch.cuda.synchronize()
    assert torch.equal(out, q)
    at = torch.arange(20, 20 + rows, device="cuda")
    page, there = lost.long()[at // 16], (lost[at // 16] >= 0) & (lost[at // 16] < len(store.k))
    want = before.clone()
    want[page[there], :, (at % 16)[there]] = k.transpose(0, 1)[there]
    assert torch.equal(store.k.nan_to_num(9.0), want.nan_to_num(9.0))
    attn.close()


# --- accepted drafts -----------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_kv,d,layout", [(1, 64, "pages"), (4, 128, "rows"), (3, 64, "heads"), (2, 128, "beside")])
@pytest.mark.parametrize("layers", [1, 35])
def test_accepted_drafts_move_up(dtype, h_kv, d, layout, layers):
    attn = handle(2 * h_kv, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(d)
    paths = [[0, 1, 2], [3], [1, 2, 5, 9], list(range(64)), list(range(1, 64)), [], [63], [0, 2, 4, 60, 61], [7, 8, 9, 10, 11, 12, 13, 14, 15, 40]]
    paths = paths * 5 if layers == 1 else paths
    lengths = [64 + 5 * i for i in range(len(paths))]
    stores = [Store(g, h_kv, d, dtype, 16, lengths, layout) for _ in range(layers)]
    wants = [(s.k.clone(), s.v.clone()) for s in stores]
    descs = [om.make_path(stores[0].device_tables[i], 5 * i, p) for i, p in enumerate(paths)]
    attn.omnimem_keep_pages([s.pages() for s in stores], descs)
    torch.cuda.synchronize()
    for s, want in zip(stores, wants):
        for x, y in zip((s.k, s.v), want):
            for i, path in enumerate(paths):
                rows = [y[s.tables[i][(5 * i + r) // 16], :, (5 * i + r) % 16].clone() for r in path]
                for j, row in enumerate(rows):
                    y[s.tables[i][(5 * i + j) // 16], :, (5 * i + j) % 16] = row
            assert torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0))
    attn.close()


def test_accepted_drafts_without_a_page_stay():
    attn = handle(2, 2, 64, "bf16")
    store = Store(torch.Generator(device="cuda").manual_seed(4), 2, 64, "bf16", 16, [80])
    before, table = store.k.clone(), store.tables[0]
    lost = store.device_tables[0].clone()
    lost[1], lost[3] = -1, 10 ** 6
    attn.omnimem_keep_pages([store.pages()], [om.make_path(lost, 10, [2, 3, 10, 30, 40, 50])])   # rows 12, 13, 20, 40, 50, 60 to 10 ..
    torch.cuda.synchronize()
    want = before.clone()
    for old, new in ((12, 10), (13, 11), (40, 13)):            # (20, 50 and 60 have no page)
        want[table[new // 16], :, new % 16] = before[table[old // 16], :, old % 16]
    assert torch.equal(store.k.nan_to_num(9.0), want.nan_to_num(9.0))
    attn.close()


# --- together --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_handles_and_layouts_are_compared(dtype):
    attn = handle(4, 2, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    store = Store(g, 2, 64, dtype, 16, [20])
    other = Store(g, 2, 128, dtype, 16, [20])
    c = Case(attn, g, 4, 2, 64, dtype, 3, 0, 20)
    with pytest.raises(ValueError):
        attn.omnimem_attend_pages(other.pages(), [c.query(store, 0)])
    with pytest.raises(ValueError):                             # a table of 3 entries holds 20 rows of pages of 16, not of 8 ..
        om.make_paged_query(c.q, c.out[:, :3], store.device_tables[0], 3 * 256 + 1)
    short = om.make_paged_query(c.q, c.out[:, :3], store.device_tables[0][:1], 20)     # one page of 32 or more
    with pytest.raises(ValueError):
        attn.omnimem_attend_pages(store.pages(), [short])
    with pytest.raises(om.OmnimemError):
        attn.omnimem_attend_pages(store.pages(), [c.query(store, 0)], window=-1)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [1, 30])
def test_captured_calls_take_the_tables_of_their_replay(dtype, nq):
    """A step captured once: replays see other pages, masks and rows, eager calls and waits between them."""
    h_q, h_kv, d, nt = 8, 2, 64, 300
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(nq)
    store = Store(g, h_kv, d, dtype, 16, [nt, nt])
    table, other = (t.clone() for t in store.device_tables)
    store.device_tables = [table]
    c = Case(attn, g, h_q, h_kv, d, dtype, nq, 100, nt, tree_of(nq, 1) if nq > 1 else None)
    k, v = (torch.randn(h_kv, nq, d, generator=g, device="cuda").to(TORCH[dtype]) for _ in range(2))
    pos = torch.arange(nq, device="cuda", dtype=torch.int32)[None].contiguous()
    rope = om.make_rope(d, [0.1 * j for j in range(d // 2)])
    pages, raw = store.pages(), c.q.clone()
    rows = om.array_of([om.make_paged_projection(raw, k, v, pos, c.q, table, nt - nq)])
    queries = om.array_of([c.query(store, 0)])
    paths = om.array_of([om.make_path(table, nt - nq, [0] if nq == 1 else [1, 4, 20])])

    def step():
        attn.omnimem_rotate_pages(rope, pages, rows)
        attn.omnimem_attend_pages(pages, queries, 90, 4)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        step()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
            attn.omnimem_keep_pages([pages], paths)
    for turn in range(4):
        table.copy_(other if turn % 2 else store_table(store, 0))
        raw.copy_(torch.randn(raw.shape, generator=g, device="cuda"))
        k.copy_(torch.randn(k.shape, generator=g, device="cuda"))
        if c.tree is not None:
            c.masks = tree_of(nq, 10 + turn)
            c.tree.copy_(torch.tensor(om_signed(c.masks), device="cuda"))
        c.out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        after = store.k.clone(), store.v.clone(), c.out.clone()
        step()                                   # the same eagerly, and its result against the definition
        torch.cuda.synchronize()
        c.check(store, 0, 90, 4)
        assert torch.equal(c.out, after[2])
        attn.omnimem_keep_pages([pages], paths)
        torch.cuda.synchronize()
        assert torch.equal(store.k.nan_to_num(9.0), after[0].nan_to_num(9.0)) and torch.equal(store.v.nan_to_num(9.0), after[1].nan_to_num(9.0))
    attn.close()


def store_table(store, b):
    return torch.tensor(store.tables[b] + [-1], dtype=torch.int32, device="cuda")


def om_signed(masks):
    return [m - (m >> 63 << 64) for m in masks]


def test_calls_on_another_stream():
    attn = handle(8, 2, 128, "bf16")
    g = torch.Generator(device="cuda").manual_seed(3)
    store = Store(g, 2, 128, "bf16", 64, [2000])
    c = Case(attn, g, 8, 2, 128, "bf16", 5, 0, 2000)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    attend(attn, store, [c], 0, 0, stream=stream)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_handles_at_once(dtype):
    """Handles have workspaces of their own: their calls may run side by side, keys split over workgroups in both."""
    g = torch.Generator(device="cuda").manual_seed(8)
    store = Store(g, 2, 128, dtype, 64, [4000, 3500])
    handles, streams = [handle(8, 2, 128, dtype) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    cases = [[Case(attn, g, 8, 2, 128, dtype, nq, 0, nt) for nq, nt in sizes]
             for attn, sizes in zip(handles, ([(1, 4000), (3, 3500)], [(40, 4000), (64, 3500)]))]
    torch.cuda.synchronize()
    for _ in range(20):
        for attn, stream, cs in zip(handles, streams, cases):
            attn.omnimem_attend_pages(store.pages(), [c.query(store, b) for b, c in enumerate(cs)], 3000, 7, stream=stream)
    torch.cuda.synchronize()
    for cs in cases:
        for b, c in enumerate(cs):
            c.check(store, b, 3000, 7)
    for attn in handles:
        attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,tree", [(1, False), (40, True), (300, False)])
def test_the_last_rows_of_the_longest_cache(dtype, nq, tree):
    """2^30 rows on a few pages' repetitions: the last ones are written, seen through a window and moved as those of a short
    cache on the same pages are (the same key tiles, so the same bits)."""
    h_q, h_kv, d, rows, short = 4, 2, 64, 256, 1024
    attn = handle(h_q, h_kv, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(nq)
    rope = om.make_rope(d, [0.1 ** j for j in range(d // 2)])
    table = torch.full((2 ** 30 // rows,), -1, dtype=torch.int32, device="cuda")
    table[-short // rows:] = torch.arange(short // rows, device="cuda", dtype=torch.int32)
    q, k, v, start = (torch.randn(h, n, d, generator=g, device="cuda").to(TORCH[dtype])
                      for h, n in ((h_q, nq), (h_kv, nq), (h_kv, nq), (short // rows * h_kv, rows)))
    pos = torch.arange(nq, dtype=torch.int32, device="cuda")[None]
    masks = torch.tensor(om_signed(tree_of(nq, 2)), dtype=torch.int64, device="cuda") if tree else None
    results = []
    for t, n in ((table, 2 ** 30), (table[-short // rows:].clone(), short)):
        kp, vp = (x.clone().view(short // rows, h_kv, rows, d) for x in (start, -start))
        pages, turned, out = om.make_pages(kp, vp), torch.empty_like(q), torch.zeros_like(q)
        lse = torch.zeros(h_q, nq, device="cuda")
        attn.omnimem_rotate_pages(rope, pages, [om.make_paged_projection(q, k, v, pos, turned, t, n - nq)])
        attn.omnimem_attend_pages(pages, [om.make_paged_query(turned, out, t, n, tree=masks, lse=lse)], 150)
        attn.omnimem_keep_pages([pages], [om.make_path(t, n - 64, [1, 5, 63])])
        torch.cuda.synchronize()
        assert torch.isfinite(out).all() and (out != 0).any(2).all()
        results.append((turned, out, lse, kp, vp))
    for long, little in zip(*results):
        assert torch.equal(long, little)
    attn.close()
