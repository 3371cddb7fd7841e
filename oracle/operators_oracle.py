"""Plain float64 forms of the operators around the compression step, from their definitions (test infrastructure
only).  Arrays are [heads, rows, d] numpy float64; a memory is the uint8 array [H_kv, blocks, 34 d]."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rotate(x, pos, inv_freq, axis, rotary_dim, neighbours, weight=None, eps=0.0):
    """Rows x [h, n, d], positions pos [axes, n]: normalised with `weight` if given, then each frequency's pair turned."""
    x = x.copy()
    if weight is not None:
        x = x * weight / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    half, out = rotary_dim // 2, x.copy()
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if neighbours else (j, j + half)
        t = pos[axis[j]].astype(np.float64) * inv_freq[j]
        out[..., a] = x[..., a] * np.cos(t) - x[..., b] * np.sin(t)
        out[..., b] = x[..., a] * np.sin(t) + x[..., b] * np.cos(t)
    return out


def hold_group(x):
    """(codes, scale byte) of one group of at most 32 values."""
    m = np.abs(x).max() if len(x) else 0.0
    if not np.isfinite(x).all():
        return np.zeros(len(x), np.int64), 255
    e = -120
    while m > 7 * 2.0 ** e and e < 125:
        e += 1
    codes = []
    for v in x:
        far = np.abs(abs(v) / 2.0 ** e - MAGNITUDES)
        near = np.flatnonzero(far == far.min())
        codes.append(int(min(near, key=lambda c: c % 2)) + 8 * int(np.signbit(v)))   # of two as near, the even one
    return np.array(codes), e + 127


def held_value(code, byte):
    if byte == 255:
        return np.nan
    return (-1.0 if code & 8 else 1.0) * MAGNITUDES[code & 7] * 2.0 ** (byte - 127)


def pack(k, v):
    """The memory of rows k, v [h, n, d]."""
    h, n, d = k.shape
    blocks = -(-n // 32)
    data = np.zeros((h, blocks, 34 * d), np.uint8)
    for g in range(h):
        for b in range(blocks):
            kb, vb = k[g, 32 * b: 32 * b + 32], v[g, 32 * b: 32 * b + 32]
            out = data[g, b]
            for t in range(32):
                for p in range(d // 32):
                    c, byte = hold_group(kb[t, 32 * p: 32 * p + 32]) if t < len(kb) else (np.zeros(32, np.int64), 7)
                    out[d // 2 * t + 16 * p: d // 2 * t + 16 * p + 16] = c[0::2] + 16 * c[1::2]
                    out[32 * d + (t % 4 * (d // 32) + p) * 8 + t // 4] = byte
            for ch in range(d):
                c, byte = hold_group(vb[:, ch])
                c = np.concatenate([c, np.zeros(32 - len(c), np.int64)])
                out[16 * d + 16 * ch: 16 * d + 16 * ch + 16] = c[0::2] + 16 * c[1::2]
                out[33 * d + ch % 16 * (d // 16) + ch // 16] = byte
    return data


def unpack(data, n):
    """Rows k, v [h, n, d] of a memory."""
    h, _, bytes_ = data.shape
    d = bytes_ // 34
    table = np.array([[held_value(c, b) for c in range(16)] for b in range(256)])
    row, ch = np.arange(n)[:, None], np.arange(d)
    blk, t = row // 32, row % 32
    kb, vb = data[:, blk, t * (d // 2) + ch // 2], data[:, blk, 16 * d + 16 * ch + t // 2]
    kc = np.where(ch % 2 == 0, kb & 15, kb >> 4)
    vc = np.where(t % 2 == 0, vb & 15, vb >> 4)
    ks = data[:, blk, 32 * d + (t % 4 * (d // 32) + ch // 32) * 8 + t // 4]
    vs = data[:, blk, 33 * d + ch % 16 * (d // 16) + ch // 16 + 0 * t]
    return table[ks, kc], table[vs, vc]


def attend(q, k, v, held, scale, causal):
    """Queries q [h_q, n, d] over rows k, v [h_kv, held + tail, d], the first `held` a memory's: (out, lse, weighted
    |v|, largest sum of |q||k| scale that a query sees, per query)."""
    h_q, n, d = q.shape
    group, tail = h_q // k.shape[0], k.shape[1] - held
    out, lse = np.zeros((h_q, n, d)), np.full((h_q, n), -np.inf)
    size, reach = np.zeros((h_q, n, d)), np.zeros((h_q, n))
    for h in range(h_q):
        kk, vv = k[h // group], v[h // group]
        for i in range(n):
            rows = held + (min(max(tail - n + i + 1, 0), tail) if causal else tail)
            if rows == 0:
                continue
            s = kk[:rows] @ q[h, i] * scale
            m = s.max()
            if m == -np.inf:
                continue
            p = np.exp(s - m)
            lse[h, i] = m + np.log(p.sum())
            p /= p.sum()
            out[h, i] = p @ vv[:rows]
            size[h, i] = p @ np.abs(vv[:rows])
            reach[h, i] = (np.abs(kk[:rows]) @ np.abs(q[h, i])).max() * abs(scale)
    return out, lse, size, reach
