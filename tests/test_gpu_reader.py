"""The operators around the step as they are used together: a chunk's attention and the scores that take its
log-sum-exp, a stream's caches held in 4 bits and brought back, answers read from held memories, and a token's calls
captured into a graph."""
import copy
import pickle

import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2606_07577_amd import omnimem as om
from paper_2606_07577_amd import synth
from paper_2606_07577_amd.step import DeviceStep, HeldMemory, Reader, StreamRunner

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def host(t):
    return t.double().cpu().numpy()


def stream_chunk(g, layers, h_q, h_kv, d, n, dtype=torch.bfloat16):
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)
    mod = (torch.arange(n, device="cuda") % 4 == 3).to(torch.uint8)
    return [dict(q=rnd(h_q, n, d), k=rnd(h_kv, n, d), v=rnd(h_kv, n, d), modality=mod, sm_scale=d ** -0.5)
            for _ in range(layers)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_chunks_attention_gives_the_scores_their_lse(dtype):
    """Scores that take attend()'s log-sum-exp are those that compute it.  Both are sums of exp(s - lse) over the chunk's
    queries: a difference of the two lse is a relative one of their terms.  Each is off by at most (d + 6) u S + (N + 8) u
    + 2 u |lse| (S: the largest sum of |q||k| scale), below 2^-12 here; the sums themselves add (C + 8) u each."""
    layer = synth.make_layer([3, 1], h_q=8, h_kv=2, d=128, n_cache_v=301, n_cache_a=77, n_frames=3, frame_v=41, frame_a=13,
                             dup_frac=0.3, head_scale=(0.5, 2.0), dtype=dtype)
    plain, step = DeviceStep([layer], 250), DeviceStep([layer], 250)
    plain.score()
    step.attend()
    step.score()
    torch.cuda.synchronize()
    n, c = step.n[0], step.n[0] - step.n_cache[0]
    q, k, v = host(step.q[0]), host(step.k[0]), host(step.v[0])
    _, lse, _, reach = orc.attend(q, k, v, 0, step.sm_scale[0], True)
    bound = float(((128 + 6) * U * reach + (n + 8) * U + 2 * U * np.abs(lse)).max())
    assert bound < 2.0 ** -12
    a, b = plain.host("a", 0), step.host("a", 0)
    assert (np.abs(a - b) <= (2 * bound + 2 * (4 * c + 8) * U) * np.abs(a) + 1e-30).all()
    assert np.array_equal(step.host("lse", 0), step.lse_in[0].cpu().numpy())
    step.run()                                     # and the whole step goes on from there
    torch.cuda.synchronize()
    assert int(step.budgets.sum()) == 250
    plain.close()
    step.close()


def test_a_streams_caches_held_and_brought_back():
    layers, h_q, h_kv, d, n = 3, 4, 2, 64, 160
    g = torch.Generator(device="cuda").manual_seed(6)
    run = StreamRunner(layers, h_q, h_kv, d, n, 300)
    for _ in range(3):
        budgets = run.push(stream_chunk(g, layers, h_q, h_kv, d, n))
    held = run.hold()
    again = run.hold()                             # (no step in between: the rows' modality says what is visual)
    torch.cuda.synchronize()
    assert held.rows == again.rows == [int(b.sum()) for b in budgets] and held.visual == again.visual == [int(b[0]) for b in budgets]
    other = StreamRunner(layers, h_q, h_kv, d, n, 300)
    other.restore(held)
    torch.cuda.synchronize()
    for l in range(layers):
        want = orc.pack(host(run.cache_k(l)), host(run.cache_v(l)))
        assert np.array_equal(held.data[l].cpu().numpy(), want) and torch.equal(held.data[l], again.data[l])
        k, v = orc.unpack(want, held.rows[l])
        assert np.array_equal(host(other.cache_k(l)), k) and np.array_equal(host(other.cache_v(l)), v)
        assert torch.equal(other.cache_modality(l), run.cache_modality(l))
    other.push(stream_chunk(g, layers, h_q, h_kv, d, n))   # the stream goes on
    assert sum(other.n_cache) == 300
    with pytest.raises(ValueError):
        StreamRunner(layers, h_q, h_kv, d, n, 30).restore(held)
    run.close()
    other.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_answers_from_held_memories(dtype):
    """Prompts of different lengths over three memories (one empty), then single tokens: each layer's result against the
    definition on the memories' values and the rotated rows as the library wrote them (their own bounds are tested with
    the rotation)."""
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    layers, h_q, h_kv, d, cap = 2, 6, 2, 64, 40
    g = torch.Generator(device="cuda").manual_seed(8)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(td)
    attn = om.Attention(h_q, h_kv, d, om.BF16 if dtype == "bf16" else om.F32)
    memories = []
    for rows in (77, 0, 300):
        data = [torch.zeros(om.memory_shape(h_kv, d, rows), dtype=torch.uint8, device="cuda") for _ in range(layers)]
        if rows:
            attn.omnimem_pack([om.make_held(rnd(h_kv, rows, d), rnd(h_kv, rows, d), x) for x in data])
        memories.append(HeldMemory(data, [rows] * layers, [rows // 2] * layers))
    freq = [1000.0 ** (-j / 16) for j in range(16)]
    axis = [j % 3 for j in range(16)]
    weight = rnd(2, d)
    rope = om.make_rope(d, freq, axis, q_weight=weight[0], k_weight=weight[1])
    reader = Reader(memories, h_q, h_kv, d, rope, cap, dtype=dtype)
    tails = [[([], []) for _ in memories] for _ in range(layers)]
    for lengths in ([5, 17, 1], [1, 1, 1], [1, 1, 1]):
        for l in range(layers):
            q, k, v = ([rnd(h, n, d) for n in lengths] for h in (h_q, h_kv, h_kv))
            pos = [torch.randint(0, 5000, (3, n), generator=g, device="cuda").to(torch.int32) for n in lengths]
            outs = reader.layer(l, q, k, v, pos)
            torch.cuda.synchronize()
            for b, n in enumerate(lengths):
                t = reader.tail[b]
                p = pos[b].cpu().numpy()
                kr = orc.rotate(host(k[b]), p, freq, axis, 32, False, host(weight[1]), 1e-6)
                got = host(reader.k[l, b, :, t: t + n])
                assert np.abs(got - kr).max() <= torch.finfo(td).eps * np.abs(kr).max() + 64 * U * np.abs(kr).max()
                assert torch.equal(reader.v[l, b, :, t: t + n], v[b])
                qr = torch.zeros(h_q, n, d, device="cuda", dtype=td)
                kv = torch.zeros(2, h_kv, n, d, device="cuda", dtype=td)
                attn.omnimem_rotate(rope, [om.make_projection(q[b], k[b], v[b], pos[b], qr, kv[0], kv[1])])
                torch.cuda.synchronize()
                mk, mv = orc.unpack(memories[b].data[l].cpu().numpy(), memories[b].rows[l])
                kk = np.concatenate([mk, host(reader.k[l, b, :, : t + n])], 1)
                vv = np.concatenate([mv, host(reader.v[l, b, :, : t + n])], 1)
                out, _, size, reach = orc.attend(host(qr), kk, vv, memories[b].rows[l], d ** -0.5, True)
                half = torch.finfo(td).eps / 2 if dtype == "bf16" else 0.0
                near = 2 * (d + 6) * U * reach[..., None] + 2 * (kk.shape[1] + 8) * U + half
                off = np.abs(host(outs[b]) - out) / (size * near + (half or U) * np.abs(out))
                assert off.max() <= 1, (l, b, lengths, off.max((1, 2)), off.max((0, 2)))
        reader.next()
    assert reader.tail == [7, 19, 3]
    with pytest.raises(ValueError):
        reader.layer(0, [rnd(h_q, 40, d)] * 3, [rnd(h_kv, 40, d)] * 3, [rnd(h_kv, 40, d)] * 3, [pos[0]] * 3)
    reader.close()
    attn.close()


def test_a_tokens_calls_captured_and_replayed():
    """Rotation, packing and attention of a token in one graph: every replay gives what the calls give on the same
    buffers, with eager work and other graphs' replays between."""
    h_q, h_kv, d, rows, tail = 7, 1, 128, 1500, 40
    g = torch.Generator(device="cuda").manual_seed(9)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    attn, eager = om.Attention(h_q, h_kv, d), om.Attention(h_q, h_kv, d)
    rope = om.make_rope(d, [0.8 ** j for j in range(64)])
    k, v, kc, vc = rnd(h_kv, rows, d), rnd(h_kv, rows, d), rnd(h_kv, tail, d), rnd(h_kv, tail, d)
    q, kn, vn = rnd(h_q, 1, d), rnd(h_kv, 1, d), rnd(h_kv, 1, d)
    pos = torch.tensor([[12345]], dtype=torch.int32, device="cuda")
    data = torch.zeros(om.memory_shape(h_kv, d, rows), dtype=torch.uint8, device="cuda")
    q_rot, out = torch.zeros_like(q), torch.zeros(2, h_q, 1, d, device="cuda", dtype=torch.bfloat16)

    def calls(a, to, stream=None):
        a.omnimem_pack([om.make_held(k, v, data)], stream)
        a.omnimem_rotate(rope, [om.make_projection(q, kn, vn, pos, q_rot, kc[:, -1:], vc[:, -1:])], stream)
        a.omnimem_attend([om.make_query(q_rot, to, kc, vc, data, rows)], True, stream)

    calls(attn, out[0])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graphs = []
    for _ in range(2):                             # two graphs of one handle, replayed one after the other
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            calls(attn, out[0], stream)
        graphs.append(graph)
    for i in range(6):
        for t in (k, v, q, kn, vn):
            t.copy_(rnd(*t.shape))
        pos.fill_(1000 * i)
        out.fill_(7.0)
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got, memory, rotated = out[0].clone(), data.clone(), kc.clone()
        calls(eager, out[1])
        torch.cuda.synchronize()
        assert torch.equal(got, out[1]) and torch.equal(memory, data) and torch.equal(rotated, kc)
    attn.close()
    eager.close()


def test_handles_on_two_streams_at_once():
    """Two handles on two streams: results are those of one after the other."""
    h_q, h_kv, d, rows = 7, 1, 128, 6000
    g = torch.Generator(device="cuda").manual_seed(10)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    handles = [om.Attention(h_q, h_kv, d) for _ in range(2)]
    q, k, v = rnd(2, h_q, 3, d), rnd(2, h_kv, rows, d), rnd(2, h_kv, rows, d)
    out, ref = torch.zeros_like(q), torch.zeros_like(q)
    for b in range(2):
        handles[b].omnimem_attend([om.make_query(q[b], ref[b], k[b], v[b])])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for b in range(2):
            handles[b].omnimem_attend([om.make_query(q[b], out[b], k[b], v[b])], stream=streams[b])
    torch.cuda.synchronize()
    assert torch.equal(out, ref)
    for h in handles:
        h.close()


def test_a_chunks_attention_first_run_on_another_stream():
    """What attend() makes at its first call is made on its stream: the current one is behind."""
    layer = synth.make_layer([5, 2], h_q=4, h_kv=2, d=64, n_cache_v=90, n_cache_a=30, n_frames=2, frame_v=20, frame_a=5,
                             dup_frac=0.3, head_scale=(0.5, 2.0), dtype="bf16")
    plain, step = DeviceStep([layer], 80), DeviceStep([layer], 80)
    plain.attend()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)
    step.attend(side)
    torch.cuda.synchronize()
    assert torch.equal(step.attn_out[0], plain.attn_out[0]) and torch.equal(step.lse_in[0], plain.lse_in[0])
    plain.close()
    step.close()


def test_caches_held_behind_a_step_on_another_stream():
    layers, h_q, h_kv, d, n = 2, 4, 2, 64, 160
    g = torch.Generator(device="cuda").manual_seed(7)
    run = StreamRunner(layers, h_q, h_kv, d, n, 200)
    side, third = torch.cuda.Stream(), torch.cuda.Stream()
    chunks = [stream_chunk(g, layers, h_q, h_kv, d, n) for _ in range(3)]
    torch.cuda.synchronize()
    run.push(chunks[0], side)
    run.push(chunks[1], side)
    held = run.hold(third)                         # (the step's compaction is on the side stream)
    torch.cuda.synchronize()
    again = run.hold()
    torch.cuda.synchronize()
    assert held.visual == again.visual and all(torch.equal(a, b) for a, b in zip(held.data, again.data))
    run.push(chunks[2], side)
    run.restore(held, third)
    torch.cuda.synchronize()
    assert run.n_cache == held.rows
    for l in range(layers):
        k, v = orc.unpack(held.data[l].cpu().numpy(), held.rows[l])
        assert np.array_equal(host(run.cache_k(l)), k) and np.array_equal(host(run.cache_v(l)), v)
    small = HeldMemory([x[:1] for x in held.data], held.rows, held.visual)      # (one KV head instead of two)
    run.push(chunks[0], side)
    before = list(run.n_cache)
    with pytest.raises(ValueError):
        run.restore(small)
    assert run.n_cache == before
    run.close()


def test_a_reader_refuses_other_numbers_of_streams():
    h_q, h_kv, d, n = 2, 1, 64, 3
    rnd = lambda h: torch.randn(h, n, d, device="cuda").bfloat16()
    memory = HeldMemory([torch.zeros(om.memory_shape(h_kv, d, 0), dtype=torch.uint8, device="cuda")], [0], [0])
    rope = om.make_rope(d, [0.5 ** j for j in range(32)])
    pos = torch.zeros(1, n, dtype=torch.int32, device="cuda")
    reader = Reader([memory, memory], h_q, h_kv, d, rope, 8)
    for streams in (0, 1, 3):
        with pytest.raises(ValueError, match="2 streams"):
            reader.layer(0, [rnd(h_q)] * streams, [rnd(h_kv)] * streams, [rnd(h_kv)] * streams, [pos] * streams)
    outs = reader.layer(0, [rnd(h_q)] * 2, [rnd(h_kv)] * 2, [rnd(h_kv)] * 2, [pos] * 2)
    torch.cuda.synchronize()
    assert len(outs) == 2 and all(torch.isfinite(o.float()).all() for o in outs)
    reader.close()
    for memories in ([], [memory, HeldMemory(memory.data * 2, [0, 0], [0, 0])]):
        with pytest.raises(ValueError):
            Reader(memories, h_q, h_kv, d, rope, 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_reader_takes_the_streams_stacked(dtype):
    """A fused projection's heads of all streams, stacked, give what the streams' tensors in lists give, bit by bit."""
    h_q, h_kv, d, streams, layers, td = 4, 2, 64, 3, 2, torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(11)
    attn = om.Attention(h_q, h_kv, d, om.BF16 if dtype == "bf16" else om.F32)
    memories = []
    for rows in ([100, 0], [33, 64], [0, 7]):
        data = [torch.zeros(om.memory_shape(h_kv, d, n), dtype=torch.uint8, device="cuda") for n in rows]
        kv = [torch.randn(2, h_kv, n, d, generator=g, device="cuda").to(td) for n in rows]
        attn.omnimem_pack([om.make_held(x[0], x[1], m) for x, m, n in zip(kv, data, rows) if n])
        torch.cuda.synchronize()
        memories.append(HeldMemory(data, rows, rows))
    rope = om.make_rope(d, [0.7 ** j for j in range(16)], axis=[j % 2 for j in range(16)])
    lists, stacked = (Reader(memories, h_q, h_kv, d, rope, 16, dtype=dtype) for _ in range(2))
    side = torch.cuda.Stream()
    for n in (5, 1, 1):
        for l in range(layers):
            x = torch.randn(streams, n, h_q + 2 * h_kv, d, generator=g, device="cuda").to(td).transpose(1, 2)
            q, k, v = x[:, :h_q], x[:, h_q: h_q + h_kv], x[:, h_q + h_kv:]
            pos = torch.randint(0, 900, (streams, 2, n), generator=g, device="cuda").to(torch.int32)
            torch.cuda.synchronize()
            want = lists.layer(l, list(q), list(k), list(v), list(pos))
            got = stacked.layer(l, q, k, v, pos, side)
            torch.cuda.synchronize()
            assert got.shape == (streams, h_q, n, d) and all(torch.equal(a, b) for a, b in zip(want, got))
        lists.next()
        stacked.next()
    assert torch.equal(lists.k, stacked.k) and torch.equal(lists.v, stacked.v) and lists.tail == stacked.tail == [7] * 3
    good = dict(q=q, k=k, v=v, pos=pos)
    for change in (dict(q=q[:2]), dict(q=q[:, :3]), dict(q=q.double()), dict(q=q[0]), dict(k=k.cpu()), dict(v=v[..., :32]),
                   dict(pos=pos[:, :1]), dict(pos=pos.long()), dict(q=torch.cat([q, q], 2)), dict(v=v.contiguous()),
                   dict(q=q.transpose(2, 3).contiguous().transpose(2, 3).expand(-1, -1, 5, -1))):
        with pytest.raises(ValueError):
            stacked.layer(0, **{**good, **change})
    lists.close()
    stacked.close()
    attn.close()


def test_a_readers_first_layer_on_another_stream(monkeypatch):
    """What the constructor fills is filled before a call on any stream, whatever its own stream has to do before."""
    class Slow(om.Attention):
        def __init__(self, *args):
            super().__init__(*args)
            torch.cuda._sleep(20_000_000)          # (what follows on the constructor's stream comes late)

    h_q, h_kv, d, n = 4, 2, 64, 6
    g = torch.Generator(device="cuda").manual_seed(12)
    rnd = lambda h: torch.randn(h, n, d, generator=g, device="cuda").bfloat16()
    memory = HeldMemory([torch.zeros(om.memory_shape(h_kv, d, 0), dtype=torch.uint8, device="cuda")], [0], [0])
    rope = om.make_rope(d, [0.5 ** j for j in range(32)])
    pos, q, k, v = torch.arange(n, dtype=torch.int32, device="cuda")[None], rnd(h_q), rnd(h_kv), rnd(h_kv)
    plain = Reader([memory], h_q, h_kv, d, rope, 8)
    [want] = plain.layer(0, [q], [k], [v], [pos])
    torch.cuda.synchronize()
    monkeypatch.setattr(om, "Attention", Slow)
    side = torch.cuda.Stream()
    late = Reader([memory], h_q, h_kv, d, rope, 8)
    [got] = late.layer(0, [q], [k], [v], [pos], side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(late.k, plain.k) and torch.equal(late.v, plain.v)
    assert late.v[0, 0, :, :n].abs().sum() > 0
    plain.close()
    late.close()


def test_steps_behind_held_and_restored_caches_on_another_stream():
    """No synchronization between hold() or restore() on one stream, late as they are, and the step on another: budgets,
    caches and memories are those of one stream."""
    layers, h_q, h_kv, d, n = 2, 4, 2, 64, 160
    g = torch.Generator(device="cuda").manual_seed(13)
    chunks = [stream_chunk(g, layers, h_q, h_kv, d, n) for _ in range(6)]
    side, third = torch.cuda.Stream(), torch.cuda.Stream()

    def late():
        with torch.cuda.stream(third):
            torch.cuda._sleep(20_000_000)

    runs = []
    for step, other in ((None, None), (side, third)):
        run = StreamRunner(layers, h_q, h_kv, d, n, 200)
        run.push(chunks[0], step)
        run.hold(other)                            # (makes the handle, which waits for the device)
        torch.cuda.synchronize()
        run.push(chunks[1], step, wait=False)
        if other is not None:
            late()
        held = run.hold(other)
        budgets = [run.push(chunks[2], step)]      # compacts the rows that are held
        run.push(chunks[3], step, wait=False)
        if other is not None:
            late()
        run.restore(held, other)
        budgets.append(run.push(chunks[4], step))  # scores the rows that come back
        run.push(chunks[5], step, wait=False)
        if other is not None:
            late()
        again = run.hold(other)
        for l in range(layers):
            run.set_cache(l, chunks[0][l]["k"][:, :30], chunks[0][l]["v"][:, :30], 20, 10)
        budgets.append(run.push(chunks[0], step))
        views = [t.clone() for l in range(layers) for t in (run.cache_k(l), run.cache_v(l), run.cache_modality(l))]
        torch.cuda.synchronize()
        runs.append((budgets, held.data + again.data + views))
        run.close()
    for a, b in zip(*[r[0] for r in runs]):
        assert np.array_equal(a, b)
    for a, b in zip(*[r[1] for r in runs]):
        assert torch.equal(a, b)


def test_a_runners_first_step_on_another_stream(monkeypatch):
    """The caches' fill on the constructor's stream, late as it is, lies before the rows of a step on another."""
    class Slow(om.Context):
        def __init__(self, *args, **options):
            super().__init__(*args, **options)
            torch.cuda._sleep(20_000_000)          # (what follows on the constructor's stream comes late)

    layers, h_q, h_kv, d, n = 2, 4, 2, 64, 160
    g = torch.Generator(device="cuda").manual_seed(14)
    chunk = stream_chunk(g, layers, h_q, h_kv, d, n)
    plain = StreamRunner(layers, h_q, h_kv, d, n, 200)
    want = plain.push(chunk)
    torch.cuda.synchronize()
    monkeypatch.setattr(om, "Context", Slow)
    late = StreamRunner(layers, h_q, h_kv, d, n, 200)
    got = late.push(chunk, torch.cuda.Stream())
    torch.cuda.synchronize()
    assert np.array_equal(got, want)
    for l in range(layers):
        assert torch.equal(late.cache_k(l), plain.cache_k(l)) and torch.equal(late.cache_v(l), plain.cache_v(l))
        assert torch.equal(late.cache_modality(l), plain.cache_modality(l))
    plain.close()
    late.close()


def test_a_refused_layer_leaves_the_reader_as_it_was():
    """A call that the library refuses sets no number of tokens: next() adds none, and other numbers are taken."""
    h_q, h_kv, d = 2, 1, 64
    g = torch.Generator(device="cuda").manual_seed(15)
    rnd = lambda h, n: torch.randn(h, n, d, generator=g, device="cuda").bfloat16()
    pos = lambda n: torch.arange(n, dtype=torch.int32, device="cuda")[None]
    memory = HeldMemory([torch.zeros(om.memory_shape(h_kv, d, 0), dtype=torch.uint8, device="cuda")] * 2, [0, 0], [0, 0])
    reader = Reader([memory], h_q, h_kv, d, om.make_rope(d, [0.5 ** j for j in range(32)]), 16)
    off = torch.zeros(h_q * 5 * d + 1, device="cuda", dtype=torch.bfloat16)[1:].view(h_q, 5, d)      # (2 bytes past 16)
    with pytest.raises(om.OmnimemError):
        reader.layer(0, [off], [rnd(h_kv, 5)], [rnd(h_kv, 5)], [pos(5)])
    reader.next()
    assert reader.tail == [0]
    with pytest.raises(om.OmnimemError):
        reader.layer(0, [off], [rnd(h_kv, 5)], [rnd(h_kv, 5)], [pos(5)])
    for l in range(2):
        reader.layer(l, [rnd(h_q, 3)], [rnd(h_kv, 3)], [rnd(h_kv, 3)], [pos(3)])
    with pytest.raises(om.OmnimemError):           # (a layer before it was taken: its numbers stay)
        reader.layer(1, [off[:, :3]], [rnd(h_kv, 3)], [rnd(h_kv, 3)], [pos(3)])
    with pytest.raises(ValueError, match="same numbers"):
        reader.layer(1, [rnd(h_q, 4)], [rnd(h_kv, 4)], [rnd(h_kv, 4)], [pos(4)])
    reader.next()
    assert reader.tail == [3]
    torch.cuda.synchronize()
    reader.close()


def test_a_chunks_attention_after_other_lse_inputs():
    """attend() again behind set_lse_inputs(): its log-sum-exp goes to arrays of its own (which the caller's inputs do not
    free), and the scores take it again."""
    layer = synth.make_layer([7, 1], h_q=4, h_kv=2, d=64, n_cache_v=90, n_cache_a=30, n_frames=2, frame_v=20, frame_a=5,
                             dup_frac=0.3, head_scale=(0.5, 2.0), dtype="bf16")
    step = DeviceStep([layer], 80)
    step.attend()
    step.score()
    torch.cuda.synchronize()
    want, lse, c = step.host("a", 0), step.lse_in[0].clone(), step.n[0] - step.n_cache[0]
    step.set_lse_inputs([None])
    others = [torch.full((4, c), 3.0, device="cuda") for _ in range(20)]   # (freed arrays would be among these)
    step.set_lse_inputs([others[0]])
    step.attend()
    step.score()
    torch.cuda.synchronize()
    assert all((t == 3.0).all() for t in others)
    assert torch.equal(step.lse_in[0], lse) and np.array_equal(step.host("a", 0), want)
    step.close()


def test_a_steps_first_stage_on_another_stream(monkeypatch):
    """What the constructor fills, late as it is, is filled before a stage on another stream writes there."""
    layer = synth.make_layer([8, 1], h_q=4, h_kv=2, d=64, n_cache_v=90, n_cache_a=30, n_frames=2, frame_v=20, frame_a=5,
                             dup_frac=0.3, head_scale=(0.5, 2.0), dtype="bf16")
    plain = DeviceStep([layer], 80)
    plain.score()
    torch.cuda.synchronize()
    zeros_like, side = torch.zeros_like, torch.cuda.Stream()

    def slow(t):
        torch.cuda._sleep(20_000_000)              # (what follows on the constructor's stream comes late)
        return zeros_like(t)

    monkeypatch.setattr(torch, "zeros_like", slow)
    late = DeviceStep([layer], 80)
    late.score(side)
    torch.cuda.synchronize()
    assert np.array_equal(late.host("a", 0), plain.host("a", 0)) and plain.host("a", 0).sum() > 0
    assert np.array_equal(late.host("lse", 0), plain.host("lse", 0))
    plain.close()
    late.close()


def test_a_memory_that_is_still_being_held():
    """Another stream's caches are brought back from a memory that is packed late, and dropped before they are; and an
    answer is read from such a memory."""
    layers, h_q, h_kv, d, n = 2, 4, 2, 64, 160
    g = torch.Generator(device="cuda").manual_seed(16)
    run, other = (StreamRunner(layers, h_q, h_kv, d, n, 200) for _ in range(2))
    run.hold()
    other.hold()                                   # (make the handles, which wait for the device)
    side, third = torch.cuda.Stream(), torch.cuda.Stream()

    def late():
        run.push(stream_chunk(g, layers, h_q, h_kv, d, n), wait=False)
        with torch.cuda.stream(third):
            torch.cuda._sleep(20_000_000)
        return run.hold(third)

    held = late()
    other.restore(held, side)
    del held
    with torch.cuda.stream(third):                 # (would take the memory's place)
        noise = [torch.full((1 << i,), 0xA5, dtype=torch.uint8, device="cuda") for i in range(8, 20) for _ in range(4)]
    want = run.hold()
    torch.cuda.synchronize()
    assert other.n_cache == want.rows
    for l in range(layers):
        kv = orc.unpack(want.data[l].cpu().numpy(), want.rows[l])
        assert np.array_equal(host(other.cache_k(l)), kv[0]) and np.array_equal(host(other.cache_v(l)), kv[1])
    rope = om.make_rope(d, [0.5 ** j for j in range(32)])
    q, k, v = (torch.randn(h, 3, d, generator=g, device="cuda").bfloat16() for h in (h_q, h_kv, h_kv))
    pos = torch.arange(3, dtype=torch.int32, device="cuda")[None]
    torch.cuda.synchronize()
    outs, held = [], late()
    for memory in (held, None):
        reader = Reader([memory or run.hold()], h_q, h_kv, d, rope, 8)
        outs.append(reader.layer(0, [q], [k], [v], [pos], side)[0])
        torch.cuda.synchronize()
        reader.close()
    assert torch.equal(*outs)
    run.close()
    other.close()


def test_a_chunk_that_is_copied_for_a_step_on_another_stream():
    """Rows that push() makes contiguous are made so on the step's stream, whatever the current one has to do before."""
    layers, h_q, h_kv, d, n = 2, 4, 2, 64, 160
    g = torch.Generator(device="cuda").manual_seed(17)
    chunk = stream_chunk(g, layers, h_q, h_kv, d, n)
    spread = [dict(ch, **{x: torch.stack([ch[x]] * 2, -1)[..., 0] for x in ("q", "k", "v")}) for ch in chunk]
    plain, late = (StreamRunner(layers, h_q, h_kv, d, n, 200) for _ in range(2))
    want = plain.push(chunk)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    got = late.push(spread, side)
    torch.cuda.synchronize()
    assert np.array_equal(got, want)
    for l in range(layers):
        assert torch.equal(late.cache_k(l), plain.cache_k(l)) and torch.equal(late.cache_v(l), plain.cache_v(l))
    plain.close()
    late.close()


def test_a_memory_is_copied_and_one_in_host_memory_refused():
    """A copy of a memory (or a saved one) waits for its packing and needs no event; rows in host memory are refused as
    other tensors that do not fit, and the caches stay."""
    layers, h_q, h_kv, d, n = 2, 4, 2, 64, 160
    g = torch.Generator(device="cuda").manual_seed(18)
    run = StreamRunner(layers, h_q, h_kv, d, n, 200)
    run.push(stream_chunk(g, layers, h_q, h_kv, d, n))
    held = run.hold()
    for other in (copy.deepcopy(held), pickle.loads(pickle.dumps(held))):
        assert other.ready is None and other.rows == held.rows and other.visual == held.visual
        assert all(torch.equal(a, b) for a, b in zip(other.data, held.data))
        run.restore(other)
        assert run.n_cache == held.rows
    before = [run.cache_k(l).clone() for l in range(layers)]
    with pytest.raises(ValueError, match="one device"):
        run.restore(HeldMemory([x.cpu() for x in held.data], held.rows, held.visual))
    assert run.n_cache == held.rows and all(torch.equal(run.cache_k(l), before[l]) for l in range(layers))
    run.close()


def test_a_memory_brought_back_in_a_graph():
    """restore() captured behind steps on another stream, and replayed with eager work between."""
    layers, h_q, h_kv, d, n = 2, 4, 2, 64, 160
    g = torch.Generator(device="cuda").manual_seed(19)
    run = StreamRunner(layers, h_q, h_kv, d, n, 200)
    run.push(stream_chunk(g, layers, h_q, h_kv, d, n))
    held = run.hold()
    run.restore(held)
    want = [t.clone() for l in range(layers) for t in (run.cache_k(l), run.cache_v(l), run.cache_modality(l))]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run.restore(held)
        views = [t for l in range(layers) for t in (run.cache_k(l), run.cache_v(l), run.cache_modality(l))]
    for i in range(3):
        for t in views:
            t.fill_(1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(views, want))
    run.push(stream_chunk(g, layers, h_q, h_kv, d, n))
    assert sum(run.n_cache) == 200
    run.close()


def test_a_readers_and_a_steps_calls_in_graphs():
    """A token's layer, and a chunk's attention with the scores behind it, captured once and replayed on new inputs."""
    h_q, h_kv, d, layers = 4, 2, 64, 2
    g = torch.Generator(device="cuda").manual_seed(20)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    attn = om.Attention(h_q, h_kv, d)
    data = [torch.zeros(om.memory_shape(h_kv, d, 700), dtype=torch.uint8, device="cuda") for _ in range(layers)]
    attn.omnimem_pack([om.make_held(rnd(h_kv, 700, d), rnd(h_kv, 700, d), x) for x in data])
    memory = HeldMemory(data, [700] * layers, [350] * layers)
    rope = om.make_rope(d, [0.5 ** j for j in range(32)])
    captured, eager = (Reader([memory], h_q, h_kv, d, rope, 8) for _ in range(2))
    q, k, v = rnd(layers, h_q, 1, d), rnd(layers, h_kv, 1, d), rnd(layers, h_kv, 1, d)
    pos = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    token = lambda r: [r.layer(l, [q[l]], [k[l]], [v[l]], [pos])[0] for l in range(layers)]
    layer = synth.make_layer([9, 1], h_q=h_q, h_kv=h_kv, d=d, n_cache_v=300, n_cache_a=30, n_frames=2, frame_v=60, frame_a=5,
                             dup_frac=0.3, head_scale=(0.5, 2.0), dtype="bf16")
    steps = [DeviceStep([layer], 80) for _ in range(2)]
    for s in steps:
        s.attend()
        s.score()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = token(captured)
        steps[0].attend()
        steps[0].score()
    for i in range(4):
        for t in (q, k, v):
            t.copy_(rnd(*t.shape))
        pos.fill_(700 + 11 * i)
        fresh = rnd(*steps[0].q[0].shape)
        for s in steps:
            s.q[0].copy_(fresh)
            s.a.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        want = token(eager)
        steps[1].attend()
        steps[1].score()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)) and torch.equal(captured.k, eager.k)
        assert torch.equal(steps[0].attn_out[0], steps[1].attn_out[0]) and torch.equal(steps[0].a, steps[1].a)
    for x in (captured, eager, attn, *steps):
        x.close()
