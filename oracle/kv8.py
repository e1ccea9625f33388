"""Plain statement of the 8-bit KV cache operators, in float64 on the CPU (test infrastructure).

e4m3: sign, 4 exponent bits (bias 7), 3 mantissa bits; normal values from 2^-6, spacing 2^-9 below; largest
448; no infinities.  A block (page of 16 tokens, KV head; K and V apart) holds codes and one scale 2^e.
"""
import numpy as np

PAGE = 16
E_MIN, E_MAX = -32, 24


def e4m3(x):
    """Nearest e4m3 value, ties to even, saturating at +-448; NaN stays NaN."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.minimum(np.abs(x), 448.0)
    _, p = np.frexp(np.where(mag > 0, mag, 1.0))
    step = np.exp2(np.maximum(p - 1, -6) - 3.0)
    return np.copysign(np.minimum(np.round(mag / step) * step, 448.0), x)


def e4m3_half_step(x):
    """Half the distance between the e4m3 values around x."""
    mag = np.minimum(np.abs(np.asarray(x, dtype=np.float64)), 448.0)
    _, p = np.frexp(np.where(mag > 0, mag, 1.0))
    return 0.5 * np.exp2(np.where(mag > 0, np.maximum(p - 1, -6), -6) - 3.0)


def exponent(amax):
    """Smallest e in [E_MIN, E_MAX] with amax <= 448 * 2^e (E_MAX if there is none)."""
    for e in range(E_MIN, E_MAX):
        if amax <= 448.0 * 2.0 ** e:
            return e
    return E_MAX


def rmsnorm_head(x, gain, eps):
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * gain


def rotate(x, cos, sin, halves):
    """x [..., Dh]; cos, sin [rot / 2]: the first rot dimensions turn, in pairs (2i, 2i+1) or (i, i + rot/2)."""
    y = np.array(x, dtype=np.float64)
    half = len(cos)
    for i in range(half):
        a, b = (i, i + half) if halves else (2 * i, 2 * i + 1)
        y[..., a] = x[..., a] * cos[i] - x[..., b] * sin[i]
        y[..., b] = x[..., b] * cos[i] + x[..., a] * sin[i]
    return y


class Cache:
    """Code values [page, head, 16, Dh] and exponents [page, head] of K (0) and V (1) of one layer."""

    def __init__(self, codes, exps):
        self.codes, self.exps = codes, exps

    def append(self, which, page, slot0, rows):
        """rows [n, head, Dh], n <= 16 - slot0: appended to `page` from slot0 on."""
        c, e = self.codes[which], self.exps[which]
        for h in range(rows.shape[1]):
            x = rows[:, h]
            finite = np.abs(x[~np.isnan(x)])
            new = exponent(np.max(finite, initial=0.0))
            if slot0 == 0:
                c[page, h] = 0.0
                e[page, h] = new
            elif new > e[page, h]:
                c[page, h] = e4m3(c[page, h] * 2.0 ** (int(e[page, h]) - new))
                e[page, h] = new
            c[page, h, slot0:slot0 + len(x)] = e4m3(x * 2.0 ** -int(e[page, h]))

    def rows(self, which, pages, n):
        """The first n tokens of a page list, dequantised: [n, head, Dh]."""
        v = self.codes[which][pages] * np.exp2(self.exps[which][pages].astype(np.float64))[:, :, None, None]
        return v.transpose(0, 2, 1, 3).reshape(-1, v.shape[1], v.shape[3])[:n]


def attend(q, K, V, pos_start, scale):
    """q [n, Hq, Dh] at positions pos_start + j over K, V [keys, Hkv, Dh]: (out, sum of p |v|), both [n, Hq, Dh]."""
    n, Hq, _ = q.shape
    Hkv = K.shape[1]
    out, mass = np.empty_like(q), np.empty_like(q)
    for h in range(Hq):
        k, v = K[:, h * Hkv // Hq], V[:, h * Hkv // Hq]
        s = q[:, h] @ k.T * scale
        s[np.arange(K.shape[0])[None, :] > pos_start + np.arange(n)[:, None]] = -np.inf
        p = np.exp(s - s.max(axis=1, keepdims=True))
        p /= p.sum(axis=1, keepdims=True)
        with np.errstate(invalid="ignore"):
            out[:, h] = p @ v
            mass[:, h] = p @ np.abs(v)
    return out, mass


# ---- the arena's byte order ----


def k_byte(t, d):
    return d // 64 * 1024 + t * 64 + d % 64


def v_byte(t, d):
    return d // 32 * 512 + (d % 8 * 4 + t % 8 // 2) * 16 + d % 32 // 8 * 4 + t // 8 * 2 + t % 2


def code_value(byte):
    """Value of an e4m3 byte (NaN for 0x7f / 0xff)."""
    b = np.asarray(byte, dtype=np.int64)
    sign, ex, man = np.where(b & 0x80, -1.0, 1.0), (b >> 3) & 15, b & 7
    v = np.where(ex > 0, (1.0 + man / 8.0) * np.exp2(ex - 7.0), man / 8.0 * 2.0 ** -6)
    return np.where((b & 0x7f) == 0x7f, np.nan, sign * v)


def read_layer(arena, dh):
    """uint8 [page, head, 32 * dh + 32] -> Cache (codes and exponents as stored)."""
    t, d = np.arange(PAGE)[:, None], np.arange(dh)[None, :]
    val = code_value(arena[..., :32 * dh])
    codes = [val[..., k_byte(t, d)], val[..., 16 * dh + v_byte(t, d)]]
    sc = np.ascontiguousarray(arena[..., 32 * dh:32 * dh + 8]).view(np.float32).astype(np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        ex = np.where(sc > 0, np.round(np.log2(np.where(sc > 0, sc, 1.0))), E_MIN).astype(np.int64)
    return Cache(codes, [ex[..., 0].copy(), ex[..., 1].copy()])
