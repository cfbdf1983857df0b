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
            kept = u if factor is None else np.where(factor == 0.0, 0.0, u)
            dgate = (s * kept).reshape(g.reshape(-1, C).shape[0], -1, C).sum(axis=1).reshape(g.shape)
        v = s * _gate_rows(gate, rows, C)
        if post is None:
            dh = v
        else:
            dpost = (v * hn).sum(axis=0)
            dh = back(v * post, h, r)
    return dx, dh, dpost, dgate, dpre


def round_e4m3(v):
    """|v| <= 448 to the nearest e4m3 value (three mantissa bits, smallest step 2^-9), ties to
    even."""
    v = np.asarray(v, dtype=np.float64)
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    return np.rint(v / step) * step


def f8_scale(amax):
    """The smallest 2^e with amax / 2^e <= 448, e >= -126; 1 for 0, NaN for inf or NaN."""
    amax = np.asarray(amax, dtype=np.float64)
    ok = np.isfinite(amax) & (amax > 0)
    m, e = np.frexp(np.where(ok, amax, 1.0))  # 448 = 0.875 2^9
    s = np.ldexp(1.0, np.maximum(e - 9 + (m > 0.875), -126))
    return np.where(ok, s, np.where(amax == 0, 1.0, np.nan))


def _amax(v, axis):
    a = np.abs(v).max(axis=axis, initial=0.0)
    return np.where(np.isnan(v).any(axis=axis), np.nan, a)


def f8_rows(x):
    """The values that rows [rows, C] stand for after quantisation: 128 channels of one component
    a block."""
    out = np.array(x, dtype=np.float64)
    Q = out.shape[1] // 4
    for c in range(4):
        for k in range(0, Q, 128):
            part = out[:, c * Q + k:c * Q + min(k + 128, Q)]
            s = f8_scale(_amax(part, 1))[:, None]
            ok = np.isfinite(s)
            q = round_e4m3(np.where(ok, part, 0.0) / np.where(ok, s, 1.0))
            part[:] = np.where(ok, q * np.where(ok, s, 1.0), np.nan)
    return out


def f8_letter(w):
    """(values, scales) of one letter [Qout, Qin]: 128 x 128 blocks."""
    w = np.array(w, dtype=np.float64)
    Qo, Qi = w.shape
    scales = np.empty((-(-Qo // 128), -(-Qi // 128)))
    for a in range(scales.shape[0]):
        for b in range(scales.shape[1]):
            part = w[128 * a:128 * a + 128, 128 * b:128 * b + 128]
            s = f8_scale(_amax(part, (0, 1)))
            scales[a, b] = s
            part[:] = round_e4m3(part / s) * s if np.isfinite(s) else np.nan
    return w, scales


def w4_letter(w, group):
    """(values, whole numbers, scales [Qout, groups]) of one letter [Qout, Qin] in 4 bits: `group`
    inputs of an output share max / 7 in bf16 (1 for 0; NaN for an infinity or a NaN)."""
    w = np.array(w, dtype=np.float64)
    Qo, Qi = w.shape
    q, scales = np.zeros_like(w), np.empty((Qo, -(-Qi // group)))
    for b in range(scales.shape[1]):
        part = w[:, b * group:(b + 1) * group]
        a = _amax(part, 1)
        ok = np.isfinite(a)
        m, e = np.frexp(np.where(ok, a, 0.0) / 7.0)  # bf16: 8 significant bits, steps of 2^-133
        unit = np.maximum(e - 8, -133)
        s = np.ldexp(np.rint(np.ldexp(m, e - unit)), unit)
        s = np.where(ok, np.where(s > 0, s, 1.0), np.nan)
        scales[:, b] = s
        good = np.where(ok, s, 1.0)[:, None]
        v = np.clip(np.rint(np.where(ok[:, None], part, 0.0) / good), -7, 7)
        q[:, b * group:(b + 1) * group] = v
        part[:] = np.where(ok[:, None], v * good, np.nan)
    return w, q, scales


# Eq. 3: output component co takes input component ci through letter co xor ci.
_SIGN = np.array([[1, -1, -1, -1], [1, 1, -1, 1], [1, 1, 1, -1], [1, -1, 1, 1]], dtype=np.float64)


def qpoint(rows, letters, transpose=False):
    """Rows times the real block matrix of the letters (values), or with transpose times its
    transpose's counterpart, the input gradient: (result, sum of the terms' magnitudes)."""
    n_out, n_in = letters[0].shape
    k = n_out if transpose else n_in
    out, mag = [], []
    for a in range(4):
        acc, m = 0.0, 0.0
        for b in range(4):
            part = rows[:, b * k:(b + 1) * k]
            w = letters[a ^ b] if transpose else letters[a ^ b].T
            acc = acc + (_SIGN[b, a] if transpose else _SIGN[a, b]) * (part @ w)
            m = m + np.abs(part) @ np.abs(w)
        out.append(acc)
        mag.append(m)
    return np.concatenate(out, axis=1), np.concatenate(mag, axis=1)
