"""fp64 restatements (numpy) of the residual block's parts: the dropout masks, the residual join
and its gradients.  Shares no code with the library."""
import numpy as np


def philox4x32(block, key, rounds=10):
    """Philox4x32 (Salmon et al., SC 2011): block counters (uint64 array; the upper two counter
    words are 0) and a 64-bit key -> uint32 [len, 4]."""
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    block = np.asarray(block, dtype=np.uint64)
    x = [block & low, block >> sh, np.zeros_like(block), np.zeros_like(block)]
    for r in range(rounds):
        k0 = np.uint64((key + 0x9E3779B9 * r) & 0xFFFFFFFF)
        k1 = np.uint64(((key >> 32) + 0xBB67AE85 * r) & 0xFFFFFFFF)
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> sh) ^ x[1] ^ k0, b & low, (a >> sh) ^ x[3] ^ k1, a & low]
    return np.stack(x, axis=1).astype(np.uint32)


def dropout_factor(n, p, seed, offset=0):
    """[n] fp64: 0 where an element is dropped, 1 / (1 - p) (p in steps of 2^-16) elsewhere."""
    t = int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))
    if t == 0:
        return np.ones(n)
    blocks = (offset + np.arange(-(-n // 8), dtype=object)) % (1 << 64)
    w = philox4x32(blocks.astype(np.uint64), seed)
    bits = np.stack([w & 0xFFFF, w >> 16], axis=2).reshape(-1)[:n]
    return np.where(bits >= t, 65536.0 / (65536.0 - t) if t < 65536 else 0.0, 0.0)


def _rms(v, groups, eps):
    """rms of each row's groups, spread over the row."""
    g = v.reshape(v.shape[0], groups, -1)
    r = np.sqrt((g * g).mean(axis=2, keepdims=True) + eps)
    return np.broadcast_to(r, g.shape).reshape(v.shape)


def _gate_rows(gate, rows, C):
    if gate is None:
        return np.ones((rows, C))
    g = np.asarray(gate, dtype=np.float64).reshape(-1, C)
    return np.repeat(g, rows // g.shape[0], axis=0) if rows else np.ones((0, C))


def join(x, h=None, post=None, gate=None, pre=None, alpha=1.0, groups=1, eps=1e-5, factor=None):
    """(y, n) of rows x, h [rows, C]; factor is dropout_factor's, shaped like x, or None."""
    rows, C = x.shape
    y = x
    if h is not None:
        u = h if post is None else h / _rms(h, groups, eps) * post
        d = u if factor is None else np.where(factor == 0.0, 0.0, u * factor)
        y = x + alpha * _gate_rows(gate, rows, C) * d
    return y, (None if pre is None else y / _rms(y, groups, eps) * pre)


def join_backward(dy, dn, y, h=None, post=None, gate=None, pre=None, alpha=1.0, groups=1,
                  eps=1e-5, factor=None):
    """(dx, dh, dpost, dgate, dpre) of rows; None for what is absent."""
    def back(t, v, r):  # gradient through v / rms(v)
        a = (t * v).reshape(v.shape[0], groups, -1).mean(axis=2, keepdims=True)
        a = np.broadcast_to(a, (v.shape[0], groups, v.shape[1] // groups)).reshape(v.shape)
        return t / r - v * a / r ** 3

    like = dy if dy is not None else dn
    rows, C = like.shape
    dx = np.zeros_like(like) if dy is None else dy
    dh = dpost = dgate = dpre = None
    if pre is not None:
        r = _rms(y, groups, eps)
        dx = dx + back(dn * pre, y, r)
        dpre = (dn * y / r).sum(axis=0)
    if h is not None:
        s = alpha * dx * (1.0 if factor is None else factor)
        r = None if post is None else _rms(h, groups, eps)
        hn = h if post is None else h / r
        u = hn if post is None else hn * post
        if gate is not None:
            g = np.asarray(gate)
            dgate = (s * u).reshape(g.reshape(-1, C).shape[0], -1, C).sum(axis=1).reshape(g.shape)
        v = s * _gate_rows(gate, rows, C)
        if post is None:
            dh = v
        else:
            dpost = (v * hn).sum(axis=0)
            dh = back(v * post, h, r)
    return dx, dh, dpost, dgate, dpre
