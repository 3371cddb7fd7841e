"""What the operators on caches in pages refuse, and that nothing is launched then (CPU).  The library's argument checks
(csrc/pages_api.hip) are built for the host with stand-ins for the runtime and the launches, which count."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2606_07577_amd import build, omnimem as om

CSRC = build.CSRC
STANDINS = r"""
#include "%s/attn.h"
static int launches = 0, sequences = 0, moved = 0;
static omnimem::KeptSeq kept;
extern "C" {
int standin_launches() { int n = launches; launches = 0; return n; }
int standin_sequences() { int n = sequences; sequences = 0; return n; }
int standin_moved() { int n = moved; moved = 0; return n; }
int standin_skip() { return kept.skip; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipMalloc(void** p, size_t) { *p = (void*)4096; return hipSuccess; }
hipError_t hipMemset(void*, int, size_t) { return hipSuccess; }
hipError_t hipFree(void*) { return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return ""; }
}
namespace omnimem {
hipError_t prepare_attend(const AttnDims&) { return hipSuccess; }
hipError_t launch_rotate(const AttnDims&, const RotateArgs<kRotatesPerLaunch>&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_hold(const AttnDims&, const HeldArgs&, int, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_attend(const AttnDims&, AttendArgs<kQueriesPerLaunch>&, int, int, void*, hipStream_t) { return hipSuccess; }
hipError_t launch_rotate_pages(const AttnDims&, const PagedRotateArgs<kPagedRotatesPerLaunch>&, int n, hipStream_t) { ++launches; sequences += n; return hipSuccess; }
hipError_t launch_attend_pages(const AttnDims&, PagedArgs<kQueriesPerLaunch>&, int n, int, void*, hipStream_t) { ++launches; sequences += n; return hipSuccess; }
hipError_t launch_keep(const AttnDims&, const KeepArgs& a, int n, int stores, hipStream_t) {
  ++launches; sequences += n; moved += n * stores; kept = a.seq[n - 1];
  return hipSuccess;
}
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("standins")
    (d / "standins.hip").write_text(STANDINS % CSRC)
    out = str(d / "checks.so")
    flags = [f for f in build.FLAGS if f.startswith(("-std", "-f"))] + ["-O1", "-I", os.path.join(build.ROOT, "include")]
    res = subprocess.run([hipcc, "--cuda-host-only", *flags, "-shared", "-Wl,-Bsymbolic", "-o", out, os.path.join(CSRC, "attn_api.hip"),
                          os.path.join(CSRC, "pages_api.hip"), str(d / "standins.hip")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    lib = ctypes.CDLL(out)
    real = om.load_library()
    for name in om.EXPORTED:
        if name.startswith("omnimem_attn") or name.endswith("_pages"):
            getattr(lib, name).argtypes, getattr(lib, name).restype = getattr(real, name).argtypes, getattr(real, name).restype
    return lib


@pytest.fixture(params=[om.BF16, om.F32], ids=["bf16", "f32"])
def attn(lib, request):
    h = ctypes.c_void_p()
    assert lib.omnimem_attn_create(ctypes.byref(om.AttnConfig(4, 2, 64, request.param)), ctypes.byref(h)) == om.OK
    h.elt = 2 if request.param == om.BF16 else 4
    yield h
    assert lib.omnimem_attn_destroy(h) == om.OK


BASE, FAR = 1 << 32, 1 << 36
D, H, P = 64, 2, 32
PAGE = H * P * D
POOL = dict(k=FAR, v=2 * FAR, page_stride=PAGE, head_stride=P * D, row_stride=D, n_pages=100, page_rows=P)
ROPE = om.Rope(n_axes=1, eps=1e-6)
N = 40
PROJECTION = dict(q=BASE, q_head_stride=N * D, q_row_stride=D, k=BASE + (1 << 20), v=BASE + (2 << 20), kv_head_stride=N * D, kv_row_stride=D,
                  pos=BASE + (3 << 20), pos_stride=N, n_rows=N, q_out=BASE + (4 << 20), q_out_head_stride=N * D, q_out_row_stride=D,
                  table=BASE + (5 << 20), first_row=7)
QUERY = dict(q=BASE, q_head_stride=N * D, q_row_stride=D, n_queries=N, memory=BASE + (1 << 20), memory_head_stride=34 * D * 4, memory_rows=100,
             table=BASE + (2 << 20), n_tail=300, tree=None, sm_scale=0.1, out=BASE + (3 << 20), out_head_stride=N * D, out_row_stride=D,
             lse=BASE + (4 << 20), lse_head_stride=N)


def rotate(lib, attn, n=1, pool=POOL, rope=ROPE, **change):
    seqs = (om.PagedProjection * max(1, n))(*[om.PagedProjection(**PROJECTION) for _ in range(max(1, n))])
    for key, value in change.items():
        setattr(seqs[n - 1], key, value)
    return lib.omnimem_rotate_pages(attn, ctypes.byref(rope), ctypes.byref(om.Pages(**pool)), seqs, n, None)


def attend(lib, attn, n=1, pool=POOL, window=0, sinks=0, **change):
    seqs = (om.PagedQuery * max(1, n))(*[om.PagedQuery(**QUERY) for _ in range(max(1, n))])
    for key, value in change.items():
        setattr(seqs[n - 1], key, value)
    return lib.omnimem_attend_pages(attn, ctypes.byref(om.Pages(**pool)), seqs, n, window, sinks, None)


def keep(lib, attn, n=1, pools=(POOL,), path=(1, 4, 9), **change):
    host = (ctypes.c_uint8 * max(1, len(path)))(*path)
    seqs = (om.Path * max(1, n))(*[om.Path(BASE, 5, host, len(path)) for _ in range(max(1, n))])
    for key, value in change.items():
        setattr(seqs[n - 1], key, value)
    layers = (om.Pages * len(pools))(*[om.Pages(**p) for p in pools])
    return lib.omnimem_keep_pages(attn, layers, len(pools), seqs, n, None)


def refused(lib, attn, call, changes, status=om.ERR_INVALID_ARG, n=2, text=b"sequence 1"):
    lib.standin_launches()
    for change in changes:
        assert call(lib, attn, n=n, **change) == status, change
        assert text in lib.omnimem_attn_last_error(attn), (change, lib.omnimem_attn_last_error(attn))
        assert lib.standin_launches() == 0


def taken(lib, attn, call, changes):
    for change in changes:
        assert call(lib, attn, **change) == om.OK, (change, lib.omnimem_attn_last_error(attn))
        assert lib.standin_launches() == 1, change


CALLS = [rotate, attend, keep]


@pytest.mark.parametrize("call", CALLS, ids=lambda f: f.__name__)
def test_handles_counts_and_long_calls(lib, attn, call):
    lib.standin_launches()
    assert call(lib, None) == om.ERR_INVALID_ARG and call(lib, attn, n=-1) == om.ERR_INVALID_ARG
    assert call(lib, attn, n=0) == om.OK and lib.standin_launches() == 0
    lib.standin_sequences()
    assert call(lib, attn, n=100) == om.OK
    assert lib.standin_sequences() == 100 and 2 <= lib.standin_launches() <= 4
    name = f"omnimem_{call.__name__}_pages"
    more = (ctypes.byref(ROPE),) if call is rotate else ()
    pool, after = ctypes.byref(om.Pages(**POOL)), (0, 0) if call is attend else ()
    layers = (1,) if call is keep else ()
    assert getattr(lib, name)(attn, *more, pool, *layers, None, 1, *after, None) == om.ERR_INVALID_ARG
    assert getattr(lib, name)(attn, *more, None, *layers, None, 0, *after, None) == om.ERR_INVALID_ARG
    if call is rotate:
        assert lib.omnimem_rotate_pages(attn, None, pool, None, 0, None) == om.ERR_INVALID_ARG


@pytest.mark.parametrize("call", CALLS, ids=lambda f: f.__name__)
def test_stores(lib, attn, call):
    run = (lambda p, n=1: keep(lib, attn, n, (p,))) if call is keep else lambda p, n=1: call(lib, attn, n, pool=p)
    unit = 16 // attn.elt
    lib.standin_launches()
    good = [dict(page_rows=16), dict(page_stride=PAGE + unit), dict(n_pages=1, page_stride=0), dict(n_pages=2 ** 31 - 1, v=1 << 50),
            dict(page_stride=2 * PAGE, v=FAR + PAGE * attn.elt),                      # K and V of a page side by side
            dict(head_stride=D, row_stride=H * D),                                   # heads inside rows
            dict(head_stride=100 * P * D, page_stride=P * D),                        # heads outside pages
            dict(row_stride=D + unit, head_stride=P * (D + unit), page_stride=2 * PAGE)]
    for change in good:
        assert run({**POOL, **change}) == om.OK and lib.standin_launches() == 1, change
    bad = [dict(k=None), dict(v=None), dict(k=FAR + 8), dict(v=FAR), dict(v=FAR + PAGE * attn.elt), dict(n_pages=0), dict(n_pages=-1),
           dict(page_stride=PAGE - unit), dict(page_stride=0), dict(page_stride=PAGE + 1), dict(page_stride=-PAGE), dict(head_stride=P * D - unit),
           dict(head_stride=0), dict(row_stride=D - unit), dict(row_stride=0), dict(row_stride=-D),
           dict(row_stride=(1 << 24) // attn.elt, head_stride=1 << 30, page_stride=1 << 32), dict(page_stride=1 << 45),
           dict(n_pages=2 ** 31 - 1, page_stride=1 << 20, v=1 << 60), dict(n_pages=2 ** 31 - 1)]   # (the last: K reaches V)
    for change in bad:
        assert run({**POOL, **change}) == om.ERR_INVALID_ARG, change
        assert b"pages" in lib.omnimem_attn_last_error(attn) and lib.standin_launches() == 0
    for rows in (0, 8, 24, 48, 512, -16):
        assert run({**POOL, "page_rows": rows, "head_stride": 1024 * D, "page_stride": 4096 * D}) == om.ERR_UNSUPPORTED
        assert lib.standin_launches() == 0


def test_rotate_pages(lib, attn):
    unit = 16 // attn.elt
    taken(lib, attn, rotate, [{}, dict(first_row=0), dict(first_row=(1 << 30) - N), dict(q_out=BASE), dict(pos_stride=0),
                              dict(q_row_stride=4 * D, q_head_stride=D, kv_row_stride=4 * D, kv_head_stride=D)])
    lib.standin_launches()
    assert rotate(lib, attn, n_rows=0, q=None, table=None) == om.OK and lib.standin_launches() == 0
    refused(lib, attn, rotate, [dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(first_row=-1), dict(first_row=(1 << 30) - N + 1), dict(q=None),
                                dict(k=None), dict(v=None), dict(k=BASE + (1 << 20) + 8), dict(kv_row_stride=D - unit), dict(kv_row_stride=D + 1),
                                dict(pos=None), dict(pos=BASE + 2), dict(pos_stride=-1), dict(q_out=None), dict(q_out_row_stride=0),
                                dict(q_out_head_stride=D), dict(table=None), dict(table=BASE + 6), dict(q_out=BASE + 16), dict(q_out=FAR),
                                dict(k=FAR), dict(v=2 * FAR + 64), dict(q=FAR + PAGE * attn.elt * 99), dict(q_out=BASE + (1 << 20)),
                                dict(table=2 * FAR), dict(table=BASE + (4 << 20) + 16)])
    bad = om.Rope(n_axes=1, eps=-1.0)
    assert rotate(lib, attn, rope=bad) == om.ERR_INVALID_ARG
    assert rotate(lib, attn, rope=om.Rope(n_axes=1, rotary_dim=8, inv_freq=(ctypes.c_double * 4)())) == om.ERR_UNSUPPORTED


def test_rotate_pages_over_its_positions_or_weights(lib, attn):
    """Rotated queries and the pages share no byte with the positions (of the last axis too) or with a norm's weights."""
    out, end = BASE + (4 << 20), BASE + (4 << 20) + 4 * N * D * attn.elt          # (q_out is [4][N][D])
    rope = lambda **weights: om.Rope(n_axes=3, eps=1e-6, **weights)
    last = 4 * (2 * 1000 + N)                                                   # bytes of three axes, 1000 positions apart
    lib.standin_launches()
    for pos in (end, out - last, FAR - last, BASE + (3 << 20)):
        assert rotate(lib, attn, rope=rope(), pos=pos, pos_stride=1000) == om.OK and lib.standin_launches() == 1
    pool = FAR + 100 * PAGE * attn.elt
    refused(lib, attn, rotate, [dict(rope=rope(), pos=p, pos_stride=1000)
                                for p in (out, end - 4, out - last + 4, FAR - last + 4, pool - 4, 2 * FAR, 2 * FAR + 64)])
    bytes = D * attn.elt
    for name in ("q_weight", "k_weight"):
        for w in (end, out - bytes, pool, FAR - bytes, BASE):
            assert rotate(lib, attn, rope=rope(**{name: w})) == om.OK and lib.standin_launches() == 1
        refused(lib, attn, rotate, [dict(rope=rope(**{name: w})) for w in (out, end - 16, out - bytes + 16, FAR, pool - 16, 2 * FAR + 4096)], n=1,
                text=b"sequence 0")
    assert rotate(lib, attn, rope=rope(q_weight=out, k_weight=FAR), n_rows=0) == om.OK and lib.standin_launches() == 0


def test_attend_pages(lib, attn):
    unit = 16 // attn.elt
    tree = BASE + (6 << 20)
    taken(lib, attn, attend, [{}, dict(window=1), dict(window=2 ** 62, sinks=2 ** 62), dict(sinks=5), dict(tree=tree), dict(tree=tree, n_tail=N),
                              dict(memory=None, memory_rows=0), dict(n_tail=0, table=None), dict(lse=None), dict(n_tail=1 << 30, table=BASE + (1 << 30)),
                              dict(out_head_stride=D, out_row_stride=4 * D)])
    lib.standin_launches()
    assert attend(lib, attn, n_queries=0, q=None, table=None) == om.OK and lib.standin_launches() == 0
    refused(lib, attn, attend, [dict(n_queries=-1), dict(n_tail=-1), dict(n_tail=(1 << 30) + 1), dict(memory_rows=-1), dict(q=None), dict(out=None),
                                dict(table=None), dict(table=BASE + (2 << 20) + 2), dict(tree=tree + 4), dict(tree=tree, n_tail=N - 1),
                                dict(tree=tree, n_queries=65, q_head_stride=65 * D, out_head_stride=65 * D, lse=None), dict(memory=None),
                                dict(memory_head_stride=34 * D * 3), dict(memory=BASE + (1 << 20) + 4), dict(sm_scale=float("inf")),
                                dict(sm_scale=float("nan")), dict(sm_scale=3e38), dict(out_row_stride=D - unit), dict(out_row_stride=0),
                                dict(lse=BASE + (4 << 20) + 2), dict(lse_head_stride=N - 1), dict(out=BASE), dict(out=FAR), dict(lse=2 * FAR + 4),
                                dict(out=BASE + (1 << 20)), dict(lse=BASE + (3 << 20)), dict(table=BASE + (3 << 20)), dict(table=BASE + (4 << 20) + 4),
                                dict(tree=BASE + (3 << 20) + 8)])
    for change in (dict(window=-1), dict(sinks=-1)):
        assert attend(lib, attn, **change) == om.ERR_INVALID_ARG and b"window" in lib.omnimem_attn_last_error(attn)
        assert lib.standin_launches() == 0


def test_keep_pages(lib, attn):
    taken(lib, attn, keep, [{}, dict(path=(63,)), dict(path=tuple(range(1, 64))), dict(first_row=(1 << 30) - 64)])
    assert keep(lib, attn, path=(0, 1, 3)) == om.OK and lib.standin_skip() == 2
    lib.standin_launches()
    for path in ((), (0,), (0, 1, 2, 3)):                       # nothing moves
        assert keep(lib, attn, path=path) == om.OK and lib.standin_launches() == 0
    refused(lib, attn, keep, [dict(n_kept=-1), dict(n_kept=65), dict(first_row=-1), dict(first_row=1 << 30), dict(table=None),
                              dict(table=BASE + 1), dict(table=FAR + 4)])
    refused(lib, attn, keep, [dict(path=(1, 1)), dict(path=(3, 2)), dict(path=(64,)), dict(path=(1, 255))], text=b"sequence 0")
    seqs = (om.Path * 1)(om.Path(BASE, 5, None, 2))
    assert lib.omnimem_keep_pages(attn, ctypes.byref(om.Pages(**POOL)), 1, seqs, 1, None) == om.ERR_INVALID_ARG
    assert keep(lib, attn, pools=()) == om.OK and lib.standin_launches() == 0
    # layers: alike but for k and v, in launches of some
    many = [{**POOL, "k": FAR * (2 * i + 1), "v": FAR * (2 * i + 2)} for i in range(70)]
    lib.standin_moved()
    assert keep(lib, attn, pools=many, table=many[60]["v"] + 8) == om.ERR_INVALID_ARG and lib.standin_launches() == 0
    assert keep(lib, attn, pools=many) == om.OK and lib.standin_moved() == 70 and 2 <= lib.standin_launches() <= 4
    for change in (dict(n_pages=99), dict(page_stride=2 * PAGE), dict(head_stride=D, row_stride=H * D)):
        assert keep(lib, attn, pools=(POOL, {**POOL, **change})) == om.ERR_INVALID_ARG
        assert b"layer 1" in lib.omnimem_attn_last_error(attn) and lib.standin_launches() == 0


def rows_of(start, pool, elt):
    """The first bytes of a small store's rows, in units of 16."""
    return {(start + elt * (p * pool["page_stride"] + h * pool["head_stride"] + r * pool["row_stride"])) // 16
            for p in range(pool["n_pages"]) for h in range(H) for r in range(pool["page_rows"])}


def test_stores_inside_one_another(lib, attn):
    """K and V, and the stores of several layers, may lie between one another's rows, heads and pages, but share no row: against
    all rows of small stores, at every distance of their width and some others."""
    e, width, pages = attn.elt, D * attn.elt, 3
    layouts = [dict(row_stride=2 * H * D, head_stride=D, page_stride=32 * H * D),              # K and V of a row side by side
               dict(row_stride=2 * H * D, head_stride=2 * D, page_stride=32 * H * D),          # of a head of a row
               dict(row_stride=D, head_stride=32 * D, page_stride=32 * H * D),                 # of a head
               dict(row_stride=2 * D, head_stride=16 * 2 * D * pages, page_stride=16 * 2 * D),  # heads outside pages
               dict(row_stride=D + 16, head_stride=40 * D, page_stride=90 * D)]                # gaps that no row fits
    lib.standin_launches()
    met = 0
    for layout in layouts:
        pool = dict(k=FAR, v=2 * FAR, n_pages=pages, page_rows=16, **layout)
        k = rows_of(FAR, pool, e)
        assert len(k) == pages * H * 16
        for off in [i * width for i in range(400)] + [i * width + 16 for i in range(0, 400, 7)] + [i * width - 32 for i in range(1, 400, 9)]:
            share = any(x + j in k for x in rows_of(FAR + off, pool, e) for j in range(1 - width // 16, width // 16))
            met += share
            status = om.ERR_INVALID_ARG if share else om.OK
            assert keep(lib, attn, pools=({**pool, "v": FAR + off},)) == status, (layout, off)
            if off % (5 * width) == 0:
                assert keep(lib, attn, pools=({**pool, "v": FAR + off} if not share else pool,)) == om.OK
                for second in (dict(k=FAR + off, v=3 * FAR), dict(k=3 * FAR, v=FAR + off), dict(k=3 * FAR, v=2 * FAR + off),
                               dict(k=2 * FAR + off, v=3 * FAR)):
                    assert keep(lib, attn, pools=(pool, {**pool, "k": 4 * FAR, "v": 5 * FAR}, {**pool, **second})) == status
                    assert status == om.OK or b"layer 2" in lib.omnimem_attn_last_error(attn)
    assert met > 500
    lib.standin_launches()
    assert keep(lib, attn, pools=(POOL, POOL)) == om.ERR_INVALID_ARG and lib.standin_launches() == 0


def test_binding():
    """Tensors that do not fit are refused before the library is called; tables as long as their rows need."""
    assert om.tree_masks([-1, 0, 0, 2, -1]) == [1, 3, 5, 13, 16]
    assert om.tree_masks([-1] * 64)[63] == -2 ** 63
    for bad in ([0], [-1, 1], [-2], [-1] * 65):
        with pytest.raises(ValueError):
            om.tree_masks(bad)
    t = torch.zeros(5, dtype=torch.int32)
    assert om._table(t, 80) == 16 and om._table(t, 81) == 32 and om._table(t, 0) == 16 and om._table(t, 5 * 256) == 256
    for bad in (t.long(), t[None], torch.zeros(10, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            om._table(bad, 1)
    with pytest.raises(ValueError):
        om._table(t, 5 * 256 + 1)
    for path in ([1, 1], [2, 1], [64], [-1]):
        with pytest.raises(ValueError):
            om.make_path(t, 0, path)
    k = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    for a, b in ((k, k.float()), (k, k[:2]), (k[..., ::2], k[..., ::2]), (k[0], k[0]), (k.half(), k.half())):
        with pytest.raises(ValueError):
            om.make_pages(a, b)
