"""The rows of the 4-bit KV cache from whole numbers: every difference,
quotient and comparison exact, whatever the sizes of a row's values (the
definition in include/wide.h; tests/_kvq.py forms differences in fp64, which
holds 53 bits of them)."""
import numpy as np

from tests import _kvq

HD = 128
UNIT = 149                                  # values are multiples of 2^-149


def _int(x):
    n, d = float(x).as_integer_ratio()
    assert (1 << UNIT) % d == 0
    return n * ((1 << UNIT) // d)


def _bf16_floor(v):
    step = max(abs(v).bit_length() - 8, UNIT - 133)            # (2^-133: the step of the smallest bf16 values)
    return v >> step << step


def _scale(w):
    """w / 15 to 8 bits, ties to even; 0 below 2^-126."""
    step = max(0, (w // 15).bit_length() - 8)
    k, r = divmod(w, 15 << step)
    k += 2 * r > 15 << step or (2 * r == 15 << step and k & 1)
    return k << step if k << step >= 1 << (UNIT - 126) else 0


def quantize(x, qg):
    """Rows [n][128] of values that are exact in fp32 -> uint8 [n][row bytes]."""
    x = np.asarray(x, np.float64)
    ng = HD // qg
    out = np.zeros((len(x), _kvq.row_bytes(qg)), np.uint8)
    for r, row in enumerate(x):
        scales, lows, codes = [0] * ng, [np.nan] * ng, [0] * HD
        if (np.abs(row) < 2.0 ** 127).all():
            for g in range(ng):
                v = [_int(t) for t in row[g * qg:(g + 1) * qg]]
                low = _bf16_floor(min(v))
                s = _scale(max(v) - low)
                scales[g], lows[g] = s, low / (1 << UNIT)
                for i, t in enumerate(v if s else ()):
                    c, rest = divmod(t - low, s)
                    c += 2 * rest > s or (2 * rest == s and c & 1)
                    codes[g * qg + i] = min(c, 15)
        for dim, c in enumerate(codes):
            n = dim // 32 + 4 * (dim % 2)
            out[r, 4 * (dim % 32 // 2) + n // 2] |= c << (4 * (n % 2))
        meta = np.array([s / (1 << UNIT) for s in scales] + lows, np.float32)
        out[r, 64:] = (meta.view(np.uint32) >> 16).astype(np.uint16).view(np.uint8)
    return out


def border_rows():
    """Rows with values 2^-45 to 2^-129 off the border of two codes, or (the last 100, in fp32 only)
    ranges as far off the border of two scales: differences that 53 bits do not hold.  Returns (bf16
    rows, fp32 rows), fp64."""
    g = np.random.default_rng(11)
    rows = np.zeros((500, HD))
    for n in range(500):
        s = 2.0 ** int(g.integers(-3, 4))
        tiny = float(g.choice([-1, 1]) * g.integers(1, 16)) * 2.0 ** -int(g.integers(49, 130))
        if n >= 400:                        # from tiny to 15 times a value between two bf16 ones
            low, s = tiny, s * float(2 * g.integers(128, 256) + 1)
            row = g.integers(1, 15, HD) * s
        elif n % 2:                         # tiny values, the low c + 1/2 scales under zero
            c = int(g.integers(0, 15))
            low = -(c + 0.5) * s
            row = np.where(g.random(HD) < 0.5, tiny, g.integers(-c, 15 - c, HD) * s)
        else:                               # the low is tiny, halves of scales above zero
            low, row = tiny, g.integers(1, 30, HD) * (0.5 * s)
        row[::32], row[31::32] = low, (low if n % 2 and n < 400 else 0.0) + 15 * s
        rows[n] = row
    return rows[:400], rows
