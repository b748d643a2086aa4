"""The 4-bit cache row in plain 64-bit numpy, for the tests: from the format's definition, without the library."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
ROW = 400


def bf16_bits_to_f64(u):
    return (u.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def pack(bits):
    """bits: uint16 [.., 576] (bf16) -> uint8 [.., 400]."""
    lead = bits.shape[:-1]
    bits = np.ascontiguousarray(bits).reshape(-1, 576)
    out = np.zeros((bits.shape[0], ROW), dtype=np.uint8)
    x = bf16_bits_to_f64(bits[:, :512]).reshape(-1, 4, 128)
    with np.errstate(all="ignore"):
        top = np.abs(x).max(-1)
    finite = np.isfinite(top)
    e = np.full(top.shape, -100, dtype=np.int64)
    for c in range(-100, 101):                                   # the least that holds the largest value
        e = np.where((top > 6.0 * 2.0 ** (c - 1)) & finite, c, e) if c > -100 else e
    y = np.where(finite[..., None], np.abs(np.where(finite[..., None], x, 0.0)) / 2.0 ** e[..., None], 0.0)
    y = np.minimum(y, 6.0)
    d = np.abs(y[..., None] - LEVELS)
    best = d.min(-1, keepdims=True)
    near = d == best                                             # one level, or two at a tie: the even code
    code = np.where(near.sum(-1) == 1, near.argmax(-1), np.where(near.argmax(-1) % 2 == 0, near.argmax(-1), near.argmax(-1) + 1))
    sign = (bits[:, :512] >> 15).reshape(-1, 4, 128)
    code = np.where(finite[..., None], code | (sign << 3), 0).reshape(-1, 512).astype(np.uint8)
    out[:, :256] = code[:, 0::2] | (code[:, 1::2] << 4)
    out[:, 256:384] = np.ascontiguousarray(bits[:, 512:]).view(np.uint8)
    out[:, 384:388] = np.where(finite, e + 127, 255).astype(np.uint8)
    return out.reshape(*lead, ROW)


def unpack(rows):
    """uint8 [.., 400] -> float64 [.., 576]"""
    lead = rows.shape[:-1]
    rows = np.ascontiguousarray(rows).reshape(-1, ROW)
    code = np.stack([rows[:, :256] & 15, rows[:, :256] >> 4], -1).reshape(-1, 512)
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    b = rows[:, 384:388].astype(np.float64)
    s = np.where(b == 255, np.nan, 2.0 ** (b - 127)).repeat(128, axis=1)
    rope = bf16_bits_to_f64(np.ascontiguousarray(rows[:, 256:384]).view(np.uint16))
    return np.concatenate([v * s, rope], -1).reshape(*lead, 576)


def attention(Q, rows, valid, scale):
    """One query: Q [H,576] float64, rows [k,576] float64, valid [k] -> O [H,512], lse [H], p [H,k], zerr [H]: what a
    32-bit sum of the 576 products may be off in the exponent, and sum p |v| [H,512]."""
    H = Q.shape[0]
    if not valid.any():
        return np.zeros((H, 512)), np.full(H, -np.inf), np.zeros((H, len(valid))), np.zeros(H), np.zeros((H, 512))
    kv = rows[valid]
    z = scale * (Q @ kv.T)
    zerr = scale * (np.abs(Q) @ np.abs(kv).T).max(-1) * 576 * 2.0 ** -24
    m = z.max(-1, keepdims=True)
    w = np.exp(z - m)
    l = w.sum(-1, keepdims=True)
    p = np.zeros((H, len(valid)))
    p[:, valid] = w / l
    return (w / l) @ kv[:, :512], (m + np.log(l))[:, 0], p, zerr, (w / l) @ np.abs(kv[:, :512])
