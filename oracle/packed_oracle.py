"""CPU oracle of the packed-batch operators (layout, rotary positions, attention), numpy in float64."""
import numpy as np


def packed_layout(shapes, capacity, text_after=False):
    """(offsets, request, positions) of the packed rows; request and positions only of rows that fit the capacity."""
    offsets, request, positions = [0], [], []
    for s, row in enumerate(shapes):
        f, h, w, t = (max(int(x), 0) for x in row)
        length = min(f * h * w + t, capacity - offsets[-1])
        for i in range(length):
            if i < f * h * w:
                p = (i // (h * w), i % (h * w) // w, i % w)
            else:
                p = (max(f, h, w) + i - f * h * w,) * 3 if text_after else (0, 0, 0)
            request.append(s)
            positions.append(p)
        offsets.append(offsets[-1] + length)
    return np.array(offsets), np.array(request, dtype=np.int64), np.array(positions, dtype=np.int64).reshape(-1, 3)


def rotary(x, positions, axis_dims, theta=10000.0, halves=False, axis_scale=None, inverse=False, scale=1.0):
    """x: [tokens, heads, head_dim]; positions: [tokens, axes]."""
    x = np.asarray(x, dtype=np.float64) * scale
    out, width, p = x.copy(), sum(axis_dims), 0
    for a, n in enumerate(axis_dims):
        for j in range(n // 2):
            angle = np.asarray(positions)[:, a].astype(np.float64) * (axis_scale[a] if axis_scale is not None else 1.0) * float(theta) ** (-2.0 * j / n)
            c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1.0 if inverse else 1.0)
            i, k = (p, p + width // 2) if halves else (2 * p, 2 * p + 1)
            out[..., i], out[..., k] = x[..., i] * c - x[..., k] * s, x[..., i] * s + x[..., k] * c
            p += 1
    return out


def rotary_bound(x, half_step, scale=1.0, axis_dims=(), halves=False):
    """How far a rotated value may be from rotary(): half a step of the type of the value itself, and 2^-21 of |x| + |y| of its pair for what is done in fp32.
    (Sine and cosine to 2^-22: the angle's conversion, product and constant are off by 3 roundings of at most pi / 4, the polynomial by 1.5 of 1;
    scaling, product and sum add 3 roundings of 2^-24.)"""
    x = np.abs(np.asarray(x, dtype=np.float64) * scale)
    pair, width = x.copy(), sum(axis_dims)
    i = np.arange(0, width // 2) if halves else np.arange(0, width, 2)
    k = i + width // 2 if halves else i + 1
    pair[..., i] = pair[..., k] = x[..., i] + x[..., k]
    return lambda exact: half_step * np.abs(exact) + 2.0 ** -21 * pair


def packed_attention(q, k, v, offsets_q, offsets_k, causal=False, scale=None, o=None):
    """q: [rows, q_heads, d]; k, v: [rows, k_heads, d]; o: what the rows of no sequence hold."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    out = np.zeros_like(q) if o is None else np.array(o, dtype=np.float64)
    group, scale = q.shape[1] // k.shape[1], q.shape[2] ** -0.5 if scale is None else scale
    for s in range(len(offsets_q) - 1):
        q0, q1 = (min(max(int(x), 0), q.shape[0]) for x in offsets_q[s:s + 2])
        k0, k1 = (min(max(int(x), 0), k.shape[0]) for x in offsets_k[s:s + 2])
        nq, nk = q1 - q0, max(k1 - k0, 0)
        for t in range(max(nq, 0)):
            last = min(nk, t + nk - nq + 1) if causal else nk
            for h in range(q.shape[1]):
                if last <= 0:
                    out[q0 + t, h] = 0.0
                    continue
                z = k[k0:k0 + last, h // group] @ q[q0 + t, h] * scale
                e = np.exp(z - z.max())
                out[q0 + t, h] = (e / e.sum()) @ v[k0:k0 + last, h // group]
    return out


def packed_attention_bound(q, k, v, offsets_q, offsets_k, bf16, causal=False, scale=None):
    """How far a value may be from packed_attention(), to first order.  With u = 2^-24 and scores off by at most d = (head_dim + 2) u scale sum |q k| (their sums in
    fp32), every probability is off by a factor of at most 1 + 2 d + 8 u and sums over n keys by n u, so the output by (2 d + (n + 8) u) sum p |v|; bf16 rounds every
    probability once more (2^-8, and the normaliser by as much) and the output (2^-8)."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    u, group, scale = 2.0 ** -24, q.shape[1] // k.shape[1], q.shape[2] ** -0.5 if scale is None else scale
    mag = packed_attention(q, k, np.abs(v), offsets_q, offsets_k, causal, scale)
    worst = (q.shape[2] + 2) * u * scale * np.linalg.norm(q, axis=2).max(initial=0.0) * np.linalg.norm(k, axis=2).max(initial=0.0)
    n = k.shape[0]
    return mag * (2 * worst + (n + 8) * u + (3 * 2.0 ** -8 if bf16 else 0.0)) + 1e-30
