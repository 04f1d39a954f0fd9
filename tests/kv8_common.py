"""Plain 64-bit forms of the operators over an 8-bit cache and of the adjustment of head outputs, and the batches that
their tests run.  Imports nothing of the product."""
import numpy as np

from tests.decode_common import rotate

RUN = 16
TOP = 1.875 * 2.0 ** 127


def e4m3_values():
    """Value of each code: sign, 4 exponent bits of bias 7, 3 mantissa bits, no infinities."""
    b = np.arange(256)
    m, e = b & 7, (b >> 3) & 15
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b > 127, -v, v)


VALUES = e4m3_values()


def to_codes(y):
    """The e4m3 code nearest to each y (magnitudes up to 448), ties to the even one; NaN: 0x7F."""
    pos = VALUES[:127]
    a = np.abs(y)
    hi = np.clip(np.searchsorted(pos, a, "left"), 1, 126)
    lo = hi - 1
    dl, dh = a - pos[lo], pos[hi] - a
    code = np.where(dl < dh, lo, np.where(dl > dh, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.isnan(y), 127, code)
    return (code | np.where(np.signbit(y) & ~np.isnan(y), 128, 0)).astype(np.uint8)


def exponent_of(a):
    """The least e >= 1 with a <= 448 2^(e - 127)."""
    limits = 448.0 * 2.0 ** np.arange(-126, 121)
    return int(np.searchsorted(limits, a, "left")) + 1


def append(codes, exps, rows, pos, ctx):
    """One head's cache of one request, codes [positions, dh] uint8 and exps [runs]: rows [m, dh] (64 bits, rotated) at
    positions pos .. are written, in place."""
    y = np.where(np.isfinite(rows), np.clip(rows, -TOP, TOP), np.nan)
    for run in range(pos[0] // RUN, pos[-1] // RUN + 1):
        new = (pos // RUN) == run
        a = np.abs(y[new])
        e = exponent_of(np.max(np.where(np.isnan(a), 0.0, a)))
        if ctx > run * RUN:
            e = max(e, int(exps[run]))
            old = slice(run * RUN, ctx)
            codes[old] = to_codes(VALUES[codes[old]] * 2.0 ** (int(exps[run]) - e))
        exps[run] = e
        codes[pos[new]] = to_codes(y[new] * 2.0 ** (127 - e))


def rotated(rows, H, KH, pos, theta):
    """(q, k, v) of rows [m, H + 2 KH, dh]."""
    qk = rotate(rows[:, :H + KH], pos, theta)
    return qk[:, :H], qk[:, H:], rows[:, H + KH:]


def adjust(l, r=1.0, p=0.0, f=0.0, hist=(), n_prompt=0, bias=(), allowed=None):
    """Head outputs l of one request (64 bits) after penalties, biases [(id, value)] and a mask of allowed outputs."""
    l, n = np.array(l, np.float64), len(l)
    hist = np.asarray(hist, np.int64)
    inside = (hist >= 0) & (hist < n)
    count = np.zeros(n, np.int64)
    np.add.at(count, hist[inside & (np.arange(len(hist)) >= n_prompt)], 1)
    seen = np.zeros(n, bool)
    seen[hist[inside]] = True
    r = r if r > 0 else 1.0
    p, f = (0.0 if np.isnan(x) else x for x in (p, f))
    with np.errstate(invalid="ignore", over="ignore"):
        l[seen] = np.where(l[seen] > 0, l[seen] / r, l[seen] * r)
        l[count > 0] -= f * count[count > 0] + p
        for j, v in dict(bias).items():                  # the last one of an output
            if 0 <= j < n:
                l[j] += v
    if allowed is not None:
        l[~allowed] = -np.inf if allowed.any() else np.nan
    return l


def mask_words(allowed, words):
    """uint32 words (as int32) of a mask's row: bit j % 32 of word j / 32."""
    bits = np.zeros(words * 32, np.uint64)
    n = min(len(allowed), words * 32)
    bits[:n] = allowed[:n]
    w = (bits.reshape(words, 32) << np.arange(32, dtype=np.uint64)).sum(1)
    return w.astype(np.uint32).view(np.int32)
