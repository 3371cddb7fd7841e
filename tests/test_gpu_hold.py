"""omnimem_pack and omnimem_unpack: a memory's bytes and the values that come back are exactly those of the definition."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2606_07577_amd import omnimem as om

pytestmark = pytest.mark.gpu
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def odd_rows(g, h, n, d, dtype):
    """Rows over many magnitudes, with values at and next to the borders between codes and between scales."""
    x = torch.randn(h, n, d, generator=g, device="cuda") * torch.exp2(torch.randint(-30, 30, (h, n, 1), generator=g, device="cuda").float())
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 0.0, -0.25, -0.75, -2.5, -5.0, 7.0, 0.24999999, 2.5000002,
                           6.9999995, -0.0, 1e-38], device="cuda")
    pick = torch.randint(0, len(border), (h, n, d), generator=g, device="cuda")
    exact = border[pick] * torch.exp2(torch.randint(-3, 4, (h, n, 1), generator=g, device="cuda").float())
    return torch.where(torch.rand(h, n, 1, generator=g, device="cuda") < 0.5, exact, x).to(TORCH[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 31, 32, 33, 129])
def test_bytes_and_values(dtype, d, n):
    h = 2
    g = torch.Generator(device="cuda").manual_seed(n + d)
    attn = om.Attention(2 * h, h, d, om.BF16 if dtype == "bf16" else om.F32)
    k, v = odd_rows(g, h, n, d, dtype), odd_rows(g, h, n, d, dtype)
    blocks = -(-n // 32)
    data = torch.full((h, blocks + 1, 34 * d), 0xA5, dtype=torch.uint8, device="cuda")
    attn.omnimem_pack([om.make_held(k, v, data)])
    kb, vb = (torch.full((h, n + 1, d), 7.0, device="cuda", dtype=TORCH[dtype]) for _ in range(2))
    attn.omnimem_unpack([om.make_held(kb[:, :n], vb[:, :n], data)])
    torch.cuda.synchronize()
    want = orc.pack(k.double().cpu().numpy(), v.double().cpu().numpy())
    assert np.array_equal(data[:, :blocks].cpu().numpy(), want)
    assert (data[:, blocks:] == 0xA5).all()                     # the block behind is left as it was
    for back, x in zip((kb, vb), orc.unpack(want, n)):
        assert np.array_equal(back[:, :n].double().cpu().numpy(), x)
        assert (back[:, n:] == 7).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_a_group_with_no_finite_largest_comes_back_as_nan(dtype, value):
    h, n, d = 1, 40, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    attn = om.Attention(1, h, d, om.BF16 if dtype == "bf16" else om.F32)
    k, v = (torch.randn(h, n, d, generator=g, device="cuda").to(TORCH[dtype]) for _ in range(2))
    k[0, 3, 40] = value
    v[0, 35, 9] = value
    data = torch.zeros(om.memory_shape(h, d, n), dtype=torch.uint8, device="cuda")
    attn.omnimem_pack([om.make_held(k, v, data)])
    kb, vb = torch.zeros_like(k), torch.zeros_like(v)
    attn.omnimem_unpack([om.make_held(kb, vb, data)])
    torch.cuda.synchronize()
    bad_k, bad_v = torch.zeros(h, n, d, dtype=torch.bool), torch.zeros(h, n, d, dtype=torch.bool)
    bad_k[0, 3, 32:] = True
    bad_v[0, 32:, 9] = True
    assert torch.equal(kb.isnan().cpu(), bad_k) and torch.equal(vb.isnan().cpu(), bad_v)
    attn.close()


def test_many_sequences_strides_and_a_block_at_a_time():
    """Rows interleaved over heads; more sequences than a launch describes; a memory filled in two calls."""
    h, d, b = 3, 128, 19
    g = torch.Generator(device="cuda").manual_seed(4)
    attn = om.Attention(h, h, d)
    lengths = [(7 * i) % 100 for i in range(b)]                 # 0 among them
    k, v = (torch.randn(b, 100, h, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    part = lambda t, i: t[i, : lengths[i]].transpose(0, 1)
    data = torch.zeros(b, h, 4, 34 * d, dtype=torch.uint8, device="cuda")
    attn.omnimem_pack([om.make_held(part(k, i), part(v, i), data[i]) for i in range(b)])
    two = torch.zeros_like(data)
    for i in range(b):
        first = min(lengths[i], 64)
        attn.omnimem_pack([om.make_held(part(k, i)[:, :first], part(v, i)[:, :first], two[i])])
        attn.omnimem_pack([om.make_held(part(k, i)[:, first:], part(v, i)[:, first:], two[i][:, 2:])])
    back_k, back_v = torch.zeros_like(k), torch.zeros_like(v)
    attn.omnimem_unpack([om.make_held(part(back_k, i), part(back_v, i), data[i]) for i in range(b)])
    torch.cuda.synchronize()
    assert torch.equal(data, two)
    for i in range(b):
        want = orc.pack(part(k, i).double().cpu().numpy(), part(v, i).double().cpu().numpy())
        assert np.array_equal(data[i, :, : want.shape[1]].cpu().numpy(), want)
        for t, x in zip((back_k, back_v), orc.unpack(want, lengths[i])):
            assert np.array_equal(part(t, i).double().cpu().numpy(), x) and (t[i, lengths[i]:] == 0).all()
    attn.close()


def test_offsets_past_32_bits():
    """Rows and heads whose offsets pass 32 bits, in the rows and in the memory."""
    h, d, n = 2, 64, 700
    g = torch.Generator(device="cuda").manual_seed(7)
    attn = om.Attention(h, h, d)
    k, v = (torch.randn(h, n, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    near, near_k, near_v = torch.zeros(om.memory_shape(h, d, n), dtype=torch.uint8, device="cuda"), torch.zeros_like(k), torch.zeros_like(v)
    attn.omnimem_pack([om.make_held(k, v, near)])
    attn.omnimem_unpack([om.make_held(near_k, near_v, near)])
    rows, heads = 7 << 19, 5 << 29                 # 7 MiB, 5 GiB
    far = [torch.empty(heads + n * rows, dtype=torch.bfloat16, device="cuda").as_strided((h, n, d), (heads, rows, 1)) for _ in range(2)]
    data = torch.empty((5 << 30) + near.numel(), dtype=torch.uint8, device="cuda").as_strided(near.shape, (5 << 30, near.shape[2], 1))
    far[0].copy_(k)
    far[1].copy_(v)
    attn.omnimem_pack([om.make_held(*far, data)])
    torch.cuda.synchronize()
    assert torch.equal(data, near)
    for t in far:
        t.zero_()
    attn.omnimem_unpack([om.make_held(*far, data)])
    torch.cuda.synchronize()
    assert torch.equal(far[0], near_k) and torch.equal(far[1], near_v)
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_finite_values_come_back_finite(dtype, d):
    """Groups up to the type's largest value: bytes and values of the definition, off by at most 2^126 (4 * 2^126, the code
    nearest to the largest value at the next scale, is no fp32 or bf16 number)."""
    td, n = TORCH[dtype], 64
    top = torch.finfo(td).max
    attn = om.Attention(1, 1, d, om.BF16 if dtype == "bf16" else om.F32)
    g = torch.Generator(device="cuda").manual_seed(d)
    k, v = ((torch.rand(1, n, d, generator=g, device="cuda", dtype=torch.float64) * 2 - 1).mul_(top).to(td) for _ in range(2))
    k[0, 0, :8] = torch.tensor([top, -top, 7 * 2.0 ** 125, 7.0625 * 2.0 ** 125, 6 * 2.0 ** 125, 2.0 ** 127, 3.5 * 2.0 ** 125, 1.0])
    v[0, :8, 0] = k[0, 0, :8]
    k[0, 1] = 7 * 2.0 ** 125                       # the largest group of the scale 2^125 that is not cut off
    data = torch.zeros(om.memory_shape(1, d, n), dtype=torch.uint8, device="cuda")
    attn.omnimem_pack([om.make_held(k, v, data)])
    back = [torch.zeros_like(k) for _ in range(2)]
    attn.omnimem_unpack([om.make_held(*back, data)])
    torch.cuda.synchronize()
    want = orc.pack(k.double().cpu().numpy(), v.double().cpu().numpy())
    assert np.array_equal(data.cpu().numpy(), want)
    for t, x, y in zip(back, orc.unpack(want, n), (k, v)):
        got, was = t.double().cpu().numpy(), y.double().cpu().numpy()
        assert np.isfinite(got).all() and np.array_equal(got, x)
        assert (np.abs(got - was) <= 2.0 ** 126).all()
        assert (np.abs(got) <= 6 * 2.0 ** 125).all() and (np.sign(got[was != 1]) * np.sign(was[was != 1]) >= 0).all()
    attn.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_call_of_several_launches(dtype):
    """150 sequences where a launch describes 64, empty ones about the borders: each as in a call of its own."""
    h, d, b, td = 2, 64, 150, TORCH[dtype]
    g = torch.Generator(device="cuda").manual_seed(9)
    attn = om.Attention(h, h, d, om.BF16 if dtype == "bf16" else om.F32)
    lengths = [1 + (13 * i) % 70 for i in range(b)]
    for i in (0, 62, 63, 64, 65, 128, 149):
        lengths[i] = 0
    k, v = (torch.randn(b, h, 70, d, generator=g, device="cuda").to(td) for _ in range(2))
    data, one = (torch.zeros(b, h, 3, 34 * d, dtype=torch.uint8, device="cuda") for _ in range(2))
    attn.omnimem_pack([om.make_held(k[i, :, :n], v[i, :, :n], data[i]) for i, n in enumerate(lengths)])
    for i, n in enumerate(lengths):
        attn.omnimem_pack([om.make_held(k[i, :, :n], v[i, :, :n], one[i])])
    back, alone = ([torch.full_like(t, 7.0) for t in (k, v)] for _ in range(2))
    attn.omnimem_unpack([om.make_held(back[0][i, :, :n], back[1][i, :, :n], data[i]) for i, n in enumerate(lengths)])
    for i, n in enumerate(lengths):
        attn.omnimem_unpack([om.make_held(alone[0][i, :, :n], alone[1][i, :, :n], data[i])])
    torch.cuda.synchronize()
    assert torch.equal(data, one)
    for i, n in enumerate(lengths):
        want = orc.pack(k[i, :, :n].double().cpu().numpy(), v[i, :, :n].double().cpu().numpy())
        assert np.array_equal(data[i, :, : want.shape[1]].cpu().numpy(), want)
        for x, y, z in zip(back, alone, orc.unpack(want, n)):
            assert torch.equal(x[i], y[i]) and (x[i, :, n:] == 7).all()
            assert np.array_equal(x[i, :, :n].double().cpu().numpy(), z)
    attn.close()
