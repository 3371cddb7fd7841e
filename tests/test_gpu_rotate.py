"""omnimem_rotate against its definition in 64 bits.

An output is y = x_a cos - x_b sin (or its like) of normalised values, computed in fp32 and rounded once.  With M =
|x_a| + |x_b| the fp32 steps are off by at most: the angle's rounding as a fraction of a turn in [-1/2, 1/2], 2^-25
turns or 3.2 * 2^-24 radians, times M; the sine and cosine, 2 steps of 2^-24 each; the norm's sum of d squares, square
root, reciprocal and products, together below (log2(d) + d / 16 + 6) / 2 + 3 steps, 10.5 at d = 128; the two products
and their sum, 3 steps: below 24 * 2^-24 * M.  The last rounding is half a step of the type, eps / 2 of the value."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2606_07577_amd import omnimem as om

pytestmark = pytest.mark.gpu
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def rows(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda").to(TORCH[dtype])


def host(t):
    return t.double().cpu().numpy()


def check(y, ref, size, dtype):
    tol = torch.finfo(TORCH[dtype]).eps / 2 * np.abs(ref) + 24 * 2.0 ** -24 * size
    assert (np.abs(host(y) - ref) <= tol).all(), float((np.abs(host(y) - ref) / tol).max())


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
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 96), (128, 0), (64, 64), (64, 48), (64, 16)])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("norm", ["none", "both", "keys"])
def test_rows_go_behind_the_cache(dtype, d, rot, neighbours, norm):
    h_q, h_kv, axes, back = 5, 1, 3, 3
    g = torch.Generator(device="cuda").manual_seed(rot + d)
    attn = om.Attention(h_q, h_kv, d, om.BF16 if dtype == "bf16" else om.F32)
    freq = [10000.0 ** (-j / max(1, rot // 2)) for j in range(rot // 2)]
    axis = [(j * 7) % axes for j in range(rot // 2)]
    w = (1 + 0.3 * torch.randn(2, d, generator=g, device="cuda")).to(TORCH[dtype])
    qw, kw = (w[0] if norm == "both" else None), (w[1] if norm != "none" else None)
    rope = om.make_rope(d, freq, axis, axes, rot, neighbours, qw, kw, eps=1e-5)
    lengths = [1, 0, 7, 130]
    keep, seqs = [], []
    for n in lengths:
        fused = rows(g, (n, (h_q + 2 * h_kv) * d), dtype)
        q, k, v = fused.view(n, h_q + 2 * h_kv, d).transpose(0, 1).split([h_q, h_kv, h_kv])
        pos = torch.randint(-2_000_000, 2_000_000, (axes, n), generator=g, device="cuda").to(torch.int32)
        mod = torch.randint(0, 2, (n,), generator=g, device="cuda").to(torch.uint8)
        q_out = torch.full((h_q, n + 2, d), 7.0, device="cuda", dtype=TORCH[dtype])
        k_out, v_out = (torch.full((h_kv, back + n + 2, d), 7.0, device="cuda", dtype=TORCH[dtype]) for _ in range(2))
        m_out = torch.full((back + n + 2,), 9, device="cuda", dtype=torch.uint8)
        keep.append((q, k, v, pos, mod, q_out, k_out, v_out, m_out))
        seqs.append(om.make_projection(q, k, v, pos, q_out[:, :n], k_out[:, back: back + n], v_out[:, back: back + n], mod,
                                       m_out[back:]))
    attn.omnimem_rotate(rope, seqs)
    torch.cuda.synchronize()
    for n, (q, k, v, pos, mod, q_out, k_out, v_out, m_out) in zip(lengths, keep):
        p = pos.cpu().numpy()
        for x, y, weight in ((q, q_out[:, :n], qw), (k, k_out[:, back: back + n], kw)):
            weight = None if weight is None else host(weight)
            flat = orc.rotate(host(x), p, freq, axis, 0, neighbours, weight, 1e-5)
            check(y, orc.rotate(host(x), p, freq, axis, rot, neighbours, weight, 1e-5), size_of(flat, rot, neighbours), dtype)
        assert torch.equal(v_out[:, back: back + n], v) and torch.equal(m_out[back: back + n], mod)
        # nothing else is written
        assert (q_out[:, n:] == 7).all() and (m_out[:back] == 9).all() and (m_out[back + n:] == 9).all()
        for t in (k_out, v_out):
            assert (t[:, :back] == 7).all() and (t[:, back + n:] == 7).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_in_a_fused_projection(dtype):
    """Queries, keys and values that are windows of one buffer turn where they are, as they do out of place."""
    h_q, h_kv, d, n = 6, 2, 64, 33
    g = torch.Generator(device="cuda").manual_seed(2)
    attn = om.Attention(h_q, h_kv, d, om.BF16 if dtype == "bf16" else om.F32)
    rope = om.make_rope(d, [0.7 ** j for j in range(32)])
    fused = rows(g, (n, (h_q + 2 * h_kv) * d), dtype)
    pos = torch.arange(n, device="cuda", dtype=torch.int32)[None]
    outs = [torch.zeros(h, n, d, device="cuda", dtype=TORCH[dtype]) for h in (h_q, h_kv, h_kv)]
    split = lambda t: t.view(n, -1, d).transpose(0, 1).split([h_q, h_kv, h_kv])
    attn.omnimem_rotate(rope, [om.make_projection(*split(fused), pos, *outs)])
    here = fused.clone()
    attn.omnimem_rotate(rope, [om.make_projection(*split(here), pos, *split(here))])
    torch.cuda.synchronize()
    for x, y in zip(split(here), outs):
        assert torch.equal(x, y)
    attn.close()


def test_more_sequences_than_a_launch_describes():
    h_q, h_kv, d = 2, 1, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    attn = om.Attention(h_q, h_kv, d)
    rope = om.make_rope(d, [0.5 ** j for j in range(32)])
    x = rows(g, (37, 4, 3, d), "bf16")
    out = torch.zeros_like(x)
    pos = torch.arange(3, device="cuda", dtype=torch.int32)[None]
    part = lambda t, b: (t[b, :2], t[b, 2:3], t[b, 3:])
    attn.omnimem_rotate(rope, [om.make_projection(*part(x, b), pos, *part(out, b)) for b in range(37)])
    one = torch.zeros_like(x)
    for b in range(37):
        attn.omnimem_rotate(rope, [om.make_projection(*part(x, b), pos, *part(one, b))])
    torch.cuda.synchronize()
    assert torch.equal(out, one) and out.abs().sum(-1).gt(0).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,neighbours", [(128, False), (64, True)])
def test_many_tokens_turn_as_few_do(dtype, d, neighbours):
    """More tokens than go by a workgroup each: against calls of a part of them (fp32 sums in the same order)."""
    h_q, h_kv, lengths = 5, 1, [2500, 1, 1700, 33]
    g = torch.Generator(device="cuda").manual_seed(4)
    attn = om.Attention(h_q, h_kv, d, om.BF16 if dtype == "bf16" else om.F32)
    w = rows(g, (2, d), dtype)
    rope = om.make_rope(d, [0.9 ** j for j in range(d // 2 - 8)], axis=[j % 2 for j in range(d // 2 - 8)], neighbours=neighbours,
                        q_weight=w[0], k_weight=w[1])
    x = [rows(g, (h_q + 2 * h_kv, n, d), dtype) for n in lengths]
    pos = [torch.randint(0, 10000, (2, n), generator=g, device="cuda").to(torch.int32) for n in lengths]
    mod = [torch.randint(0, 2, (n,), generator=g, device="cuda").to(torch.uint8) for n in lengths]
    many, few = ([torch.full_like(t, 7.0) for t in x] for _ in range(2))
    m_many, m_few = ([torch.full((n,), 9, dtype=torch.uint8, device="cuda") for n in lengths] for _ in range(2))
    split = lambda t, a=0, b=None: (t[:h_q, a:b], t[h_q: h_q + h_kv, a:b], t[h_q + h_kv:, a:b])
    attn.omnimem_rotate(rope, [om.make_projection(*split(t), p, *split(o), m, mo) for t, p, o, m, mo in zip(x, pos, many, mod, m_many)])
    for t, p, o, m, mo in zip(x, pos, few, mod, m_few):
        for a in range(0, t.shape[1], 1000):
            b = min(a + 1000, t.shape[1])
            attn.omnimem_rotate(rope, [om.make_projection(*split(t, a, b), p[:, a:b], *split(o, a, b), m[a:b], mo[a:b])])
    torch.cuda.synchronize()
    for a, b in zip(many + m_many, few + m_few):
        assert torch.equal(a, b)
    attn.close()
