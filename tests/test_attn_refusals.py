"""What the operators around the step refuse, and that nothing is launched then (CPU).  The library's argument checks
(csrc/attn_api.hip) are built for the host with stand-ins for the runtime and the launches, which count."""
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
static int launches = 0, sequences = 0, queries = 0;
extern "C" {
int standin_launches() { int n = launches; launches = 0; return n; }
int standin_sequences() { int n = sequences; sequences = 0; return n; }
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
hipError_t launch_rotate(const AttnDims&, const RotateArgs<kRotatesPerLaunch>&, int n, hipStream_t) { ++launches; sequences += n; return hipSuccess; }
hipError_t launch_hold(const AttnDims&, const HeldArgs&, int n, bool, hipStream_t) { ++launches; sequences += n; return hipSuccess; }
hipError_t launch_attend(const AttnDims&, AttendArgs<kQueriesPerLaunch>&, int n, int, void*, hipStream_t) { ++launches; sequences += n; return hipSuccess; }
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
                          str(d / "standins.hip")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    lib = ctypes.CDLL(out)
    real = om.load_library()
    for name in om.EXPORTED:
        if name.startswith("omnimem_attn") or name in ("omnimem_rotate", "omnimem_pack", "omnimem_unpack", "omnimem_attend",
                                                       "omnimem_memory_bytes"):
            getattr(lib, name).argtypes, getattr(lib, name).restype = getattr(real, name).argtypes, getattr(real, name).restype
    return lib


def create(lib, h_q=4, h_kv=2, d=64, dtype=om.BF16):
    h = ctypes.c_void_p()
    st = lib.omnimem_attn_create(ctypes.byref(om.AttnConfig(h_q, h_kv, d, dtype)), ctypes.byref(h))
    return st, h


@pytest.fixture(params=[om.BF16, om.F32], ids=["bf16", "f32"])
def attn(lib, request):
    st, h = create(lib, dtype=request.param)
    assert st == om.OK
    h.elt = 2 if request.param == om.BF16 else 4
    yield h
    assert lib.omnimem_attn_destroy(h) == om.OK


BASE = 1 << 32


def call(lib, attn, name, kind, fields, n=1, more=(), **change):
    """Status of a call with n descriptors of these fields, the last one changed."""
    seqs = (kind * max(1, n))(*[kind(**fields) for _ in range(max(1, n))])
    for key, value in change.items():
        setattr(seqs[n - 1], key, value)
    before, after = (more[:1], more[1:]) if kind is om.Projection else ((), more)
    return getattr(lib, name)(attn, *before, seqs, n, *after, None)


def check(lib, attn, name, kind, fields, more, good, bad):
    lib.standin_launches()
    assert call(lib, attn, name, kind, fields, more=more) == om.OK and lib.standin_launches() == 1
    for change in good:
        assert call(lib, attn, name, kind, fields, more=more, **change) == om.OK, change
    lib.standin_launches()
    for change in bad:
        assert call(lib, attn, name, kind, fields, n=2, more=more, **change) == om.ERR_INVALID_ARG, change
        assert b"sequence 1" in lib.omnimem_attn_last_error(attn), change
        assert lib.standin_launches() == 0
    assert getattr(lib, name)(attn, *(more[:1] if kind is om.Projection else ()), None, 1,
                              *(more[1:] if kind is om.Projection else more), None) == om.ERR_INVALID_ARG
    assert call(lib, attn, name, kind, fields, n=-1, more=more) == om.ERR_INVALID_ARG
    assert call(lib, None, name, kind, fields, more=more) == om.ERR_INVALID_ARG
    assert call(lib, attn, name, kind, fields, n=0, more=more) == om.OK and lib.standin_launches() == 0
    lib.standin_sequences()
    assert call(lib, attn, name, kind, fields, n=70, more=more) == om.OK
    assert lib.standin_sequences() == 70 and 2 <= lib.standin_launches() <= 5


def test_handles(lib):
    assert create(lib, 4, 3)[0] == om.ERR_INVALID_ARG and b"H_kv" in lib.omnimem_attn_last_error(None)
    assert create(lib, 0, 1)[0] == om.ERR_INVALID_ARG
    assert create(lib, 2048, 1)[0] == om.ERR_INVALID_ARG
    assert create(lib, d=96)[0] == om.ERR_UNSUPPORTED
    assert create(lib, dtype=2)[0] == om.ERR_UNSUPPORTED
    assert lib.omnimem_attn_create(None, None) == om.ERR_INVALID_ARG
    assert lib.omnimem_attn_destroy(None) == om.OK


def test_memory_bytes(lib):
    assert [lib.omnimem_memory_bytes(128, n) for n in (0, 1, 32, 33)] == [0, 4352, 4352, 8704]
    assert lib.omnimem_memory_bytes(64, 64) == 4352
    assert lib.omnimem_memory_bytes(96, 5) == 0 and lib.omnimem_memory_bytes(64, -1) == 0


def held():
    return dict(k=BASE, v=BASE + (1 << 24), kv_head_stride=64 * 100, kv_row_stride=64, data=BASE + (1 << 28),
                data_head_stride=34 * 64 * 4, n_rows=100)


@pytest.mark.parametrize("name", ["omnimem_pack", "omnimem_unpack"])
def test_hold(lib, attn, name):
    f = held()
    check(lib, attn, name, om.Held, f, (),
          good=[dict(n_rows=0, k=None, v=None, data=None), dict(kv_head_stride=64, kv_row_stride=128)],
          bad=[dict(n_rows=-1), dict(n_rows=1 << 31), dict(k=None), dict(v=None), dict(data=None), dict(k=f["k"] + 4), dict(v=f["v"] + 2),
               dict(data=f["data"] + 8), dict(data_head_stride=34 * 64 * 4 - 16), dict(data_head_stride=34 * 64 * 4 + 8),
               dict(data_head_stride=-16), dict(kv_row_stride=56), dict(kv_row_stride=66), dict(kv_head_stride=-64),
               dict(data=f["k"] + 64), dict(data=f["v"])] +
              ([dict(kv_head_stride=64 * 50), dict(v=f["k"]), dict(v=f["k"] + 128)] if name == "omnimem_unpack" else []))


def rope(**change):
    r = om.Rope(rotary_dim=32, neighbours=0, n_axes=2, eps=1e-6)
    r._freq, r._axis = (ctypes.c_double * 32)(*([0.5] * 32)), (ctypes.c_uint8 * 32)(*([1] * 32))
    r.inv_freq, r.axis = r._freq, r._axis
    for key, value in change.items():
        setattr(r, key, value)
    return r


def projection(elt):
    # a fused projection [100][4 + 2 + 2 heads][64], outputs apart
    return dict(q=BASE, q_head_stride=64, q_row_stride=512, k=BASE + 4 * 64 * elt, v=BASE + 6 * 64 * elt, kv_head_stride=64, kv_row_stride=512,
                pos=BASE + (1 << 30), pos_stride=100, n_rows=100, q_out=BASE + (1 << 24), q_out_head_stride=6400, q_out_row_stride=64,
                k_out=BASE + (1 << 25), v_out=BASE + (1 << 26), out_head_stride=64 * 200, out_row_stride=64)


def test_rotate(lib, attn):
    f = projection(attn.elt)
    check(lib, attn, "omnimem_rotate", om.Projection, f, (rope(),),
          good=[dict(n_rows=0, q=None, k=None, v=None, pos=None, q_out=None, k_out=None, v_out=None),
                dict(modality=BASE + (1 << 31), modality_out=BASE + (1 << 31) + 100),
                dict(modality=BASE + (1 << 31), modality_out=BASE + (1 << 31)),
                dict(q_out=f["q"], q_out_head_stride=64, q_out_row_stride=512),            # in place, each alone or all
                dict(pos_stride=0)],
          bad=[dict(n_rows=-1), dict(n_rows=1 << 31), dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(q_out=None),
               dict(k_out=None), dict(v_out=None), dict(q=f["q"] + 8), dict(pos=f["pos"] + 2), dict(pos_stride=-1),
               dict(q_row_stride=60), dict(q_head_stride=65), dict(out_row_stride=32), dict(q_out_head_stride=64 * 50),
               dict(modality=BASE + (1 << 31)), dict(modality_out=BASE + (1 << 31)),
               dict(modality=BASE + (1 << 31), modality_out=BASE + (1 << 31) + 50),
               dict(q_out=f["k_out"]), dict(v_out=f["k_out"]), dict(v_out=f["k_out"] + 256), dict(q_out=f["q"] + 64),
               dict(k_out=f["k"]), dict(q_out=f["q"])])
    for change, status in [(dict(rotary_dim=-16), om.ERR_INVALID_ARG), (dict(rotary_dim=80), om.ERR_INVALID_ARG),
                           (dict(rotary_dim=24), om.ERR_UNSUPPORTED), (dict(n_axes=0), om.ERR_INVALID_ARG),
                           (dict(n_axes=5), om.ERR_INVALID_ARG), (dict(n_axes=1), om.ERR_INVALID_ARG),
                           (dict(inv_freq=None), om.ERR_INVALID_ARG), (dict(eps=-1.0), om.ERR_INVALID_ARG),
                           (dict(eps=float("nan")), om.ERR_INVALID_ARG), (dict(q_weight=BASE + 8), om.ERR_INVALID_ARG)]:
        assert call(lib, attn, "omnimem_rotate", om.Projection, f, more=(rope(**change),)) == status, change
    odd = rope()
    odd._freq[3] = float("inf")
    assert call(lib, attn, "omnimem_rotate", om.Projection, f, more=(odd,)) == om.ERR_INVALID_ARG
    assert lib.omnimem_rotate(attn, None, (om.Projection * 1)(om.Projection(**f)), 1, None) == om.ERR_INVALID_ARG
    assert call(lib, attn, "omnimem_rotate", om.Projection, f, more=(rope(rotary_dim=0, inv_freq=None, axis=None),)) == om.OK
    assert call(lib, attn, "omnimem_rotate", om.Projection, f, more=(rope(axis=None),)) == om.OK


def query():
    return dict(q=BASE, q_head_stride=64, q_row_stride=256, n_queries=10, memory=BASE + (1 << 28), memory_head_stride=34 * 64 * 4,
                memory_rows=100, k=BASE + (1 << 24), v=BASE + (1 << 25), kv_head_stride=64 * 50, kv_row_stride=64, n_tail=50, sm_scale=0.1,
                out=BASE + (1 << 26), out_head_stride=64, out_row_stride=256, lse=BASE + (1 << 27), lse_head_stride=10)


def test_attend(lib, attn):
    f = query()
    check(lib, attn, "omnimem_attend", om.Query, f, (1,),
          good=[dict(memory=None, memory_rows=0), dict(k=None, v=None, n_tail=0), dict(memory=None, memory_rows=0, k=None, v=None, n_tail=0),
                dict(lse=None), dict(sm_scale=0.0), dict(sm_scale=-2.0), dict(out=f["q"] + (1 << 20))],
          bad=[dict(n_queries=-1), dict(n_queries=1 << 30), dict(memory_rows=-1), dict(memory_rows=1 << 31), dict(n_tail=-1),
               dict(n_tail=1 << 31), dict(q=None), dict(k=None), dict(v=None), dict(memory=None), dict(out=None), dict(q=f["q"] + 4),
               dict(k=f["k"] + 8), dict(memory=f["memory"] + 4), dict(memory_head_stride=34 * 64 * 4 - 16),
               dict(memory_head_stride=34 * 64 * 4 + 4), dict(memory_head_stride=1 << 37), dict(out=f["out"] + 4),
               dict(q_row_stride=60), dict(kv_row_stride=62), dict(kv_row_stride=1 << 23), dict(kv_head_stride=-64),
               dict(out_head_stride=32), dict(out_row_stride=64), dict(lse=f["lse"] + 2), dict(lse_head_stride=9),
               dict(lse_head_stride=1 << 32), dict(sm_scale=float("nan")), dict(sm_scale=float("inf")), dict(out=f["q"]),
               dict(out=f["q"] + 128), dict(out=f["k"]), dict(out=f["v"] + 64 * 4), dict(out=f["memory"])])
    lib.standin_launches()
    assert call(lib, attn, "omnimem_attend", om.Query, f, more=(1,), n_queries=0) == om.OK and lib.standin_launches() == 0


def test_descriptors_refuse_tensors_that_do_not_fit():
    """The binding's own checks, before any pointer is taken."""
    t = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)
    q, k, v = t(4, 5, 64), t(2, 5, 64), t(2, 5, 64)
    pos, data = t(3, 5, dtype=torch.int32), t(*om.memory_shape(2, 64, 40), dtype=torch.uint8)
    assert data.shape == (2, 2, 34 * 64)
    for args in [(q, k, v[:, :4], pos, q, k, v), (q, k, v, pos.long(), q, k, v), (q, k, v, pos[:, :4], q, k, v),
                 (q, k, v, pos, q[:, :4], k, v), (q.float(), k, v, pos, q, k, v), (q[:, :, ::2], k, v, pos, q, k, v)]:
        with pytest.raises((ValueError, TypeError)):
            om.make_projection(*args)
    for args in [(k, v.float(), data), (k, v, data.int()), (t(2, 65, 64), t(2, 65, 64), data), (t(3, 5, 64), t(3, 5, 64), data),
                 (t(2, 5, 128), t(2, 5, 128), data), (k, v, data[:, :, :-1])]:
        with pytest.raises(ValueError):
            om.make_held(*args)
    for args, more in [((q, q[:, :4]), {}), ((q, q, k), {}), ((q, q, t(2, 5, 128), t(2, 5, 128)), {}), ((q, q, k.float(), v.float()), {}),
                       ((q, q.float()), {})]:
        with pytest.raises(ValueError):
            om.make_query(*args, **more)
    for args in [dict(inv_freq=[1.0] * 16, rotary_dim=30), dict(inv_freq=[1.0] * 40), dict(inv_freq=[1.0] * 16, axis=[4] * 16),
                 dict(inv_freq=[1.0] * 16, axis=[0] * 8), dict(inv_freq=[1.0] * 16, q_weight=t(32))]:
        with pytest.raises(ValueError):
            om.make_rope(64, **args)
    with pytest.raises(TypeError):                 # (fits, but lies in host memory)
        om.make_held(k, v, data)


def test_handles_refuse_descriptors_of_another_layout():
    """Head counts, width, type, device and position axes are compared before the call (a handle made without a device)."""
    attn = object.__new__(om.Attention)
    attn.handle, attn._fits = None, set()
    attn._layout = om._Layout(4, 2, 64, torch.bfloat16, 0)
    fine = om._Layout(4, 2, 64, torch.bfloat16, 0, 3)
    attn._check_layouts({fine, om._Layout(None, 2, 64, torch.bfloat16, 0), om._Layout(head_dim=64)})
    for change in (dict(n_q_heads=8), dict(n_kv_heads=4), dict(head_dim=128), dict(dtype=torch.float32), dict(device=1)):
        with pytest.raises(ValueError, match=next(iter(change))):
            attn._check_layouts({fine, fine._replace(**change)})
    p = om.Projection()
    p._layout = fine._replace(axes=1)
    with pytest.raises(ValueError, match="axes"):
        attn.omnimem_rotate(om.make_rope(64, [0.5] * 8, axis=[0, 1] * 4), [p])


def refused(lib, attn, name, kind, fields, more, changes):
    for change in changes:
        lib.standin_launches()
        assert call(lib, attn, name, kind, fields, more=more, **change) == om.ERR_INVALID_ARG, change
        assert b"sequence 0" in lib.omnimem_attn_last_error(attn) and lib.standin_launches() == 0, change


def test_one_row_of_several_heads_needs_a_place_for_each(lib, attn):
    refused(lib, attn, "omnimem_rotate", om.Projection, dict(projection(attn.elt), n_rows=1), (rope(),),
            [dict(q_out_head_stride=0), dict(out_head_stride=0), dict(out_head_stride=32)])
    refused(lib, attn, "omnimem_unpack", om.Held, dict(held(), n_rows=1), (), [dict(kv_head_stride=0)])
    refused(lib, attn, "omnimem_attend", om.Query, dict(query(), n_queries=1), (1,), [dict(out_head_stride=0)])


def test_strides_that_pass_any_address(lib, attn):
    far = 1 << 34
    refused(lib, attn, "omnimem_rotate", om.Projection, dict(projection(attn.elt), n_rows=1 << 30), (rope(),),
            [dict(q_row_stride=far), dict(kv_row_stride=far), dict(q_out_row_stride=far), dict(out_row_stride=far)])
    refused(lib, attn, "omnimem_rotate", om.Projection, projection(attn.elt), (rope(),), [dict(pos_stride=1 << 62)])
    for name in ("omnimem_pack", "omnimem_unpack"):
        refused(lib, attn, name, om.Held, held(), (), [dict(data_head_stride=1 << 62), dict(kv_row_stride=far, n_rows=1 << 30)])
    refused(lib, attn, "omnimem_attend", om.Query, query(), (1,),
            [dict(n_queries=1 << 29, q_row_stride=far), dict(n_queries=1 << 29, out_row_stride=far), dict(n_queries=(1 << 62) + 1),
             dict(n_tail=1 << 30, kv_head_stride=1 << 50)])


def test_lse_that_lies_in_another_array(lib, attn):
    f = query()
    refused(lib, attn, "omnimem_attend", om.Query, f, (1,),
            [dict(lse=f["out"]), dict(lse=f["out"] + 64), dict(lse=f["q"] + 4), dict(lse=f["k"]), dict(lse=f["v"] + 128),
             dict(lse=f["memory"] + 34 * 64 * 4)])


def test_a_scale_that_is_no_fp32_in_log2_units(lib, attn):
    refused(lib, attn, "omnimem_attend", om.Query, query(), (1,), [dict(sm_scale=3.0e38), dict(sm_scale=-3.0e38)])


def test_descriptors_refuse_tensors_of_several_devices():
    t = lambda *s, dtype=torch.bfloat16, device="cpu": torch.zeros(*s, dtype=dtype, device=device)
    rows = [t(h, 5, 64) for h in (4, 2, 2)]
    far = [t(h, 5, 64, device="meta") for h in (4, 2, 2)]
    pos = t(1, 5, dtype=torch.int32)
    with pytest.raises(ValueError, match="one device"):
        om.make_projection(*rows, pos, *far)
    with pytest.raises(ValueError, match="one device"):
        om.make_held(rows[1], rows[2], t(*om.memory_shape(2, 64, 5), dtype=torch.uint8, device="meta"))
    with pytest.raises(ValueError, match="one device"):
        om.make_query(rows[0], rows[0], far[1], far[2])
