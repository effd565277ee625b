"""Plain float64 statement of a cache held in 4 bits: rows of groups of 16 channels, a scale byte and 16
codes each. numpy only, one group at a time."""
import numpy as np

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
GROUP = 16


def scale_of(byte):
    """What a scale's byte stands for: the fp16 number with it in bits 14 to 7; 226 for larger ones."""
    byte = min(int(byte), 226)
    e, f = byte >> 3, byte & 7
    return (8 + f) * 2.0 ** (e - 18) if e else f * 2.0 ** -17


def scale_byte(top):
    """Byte of the scale next to top / 6, ties to the even significand, within 2^-14 .. 10240."""
    want = min(max(top / 6, 2.0 ** -14), 10240.0)    # (far beyond, all distances would round to one)
    ok = range(8, 227)
    near = min(abs(scale_of(b) - want) for b in ok)
    best = [b for b in ok if abs(scale_of(b) - want) == near]
    return best[0] if len(best) == 1 else [b for b in best if b % 2 == 0][0]


def code_of(x, s):
    """Code of the value next to x (a sign bit over the magnitude's index), ties to the even index."""
    r = min(abs(x) / s, 6.0)
    near = min(abs(r - v) for v in GRID)
    best = [i for i, v in enumerate(GRID) if abs(r - v) == near]
    i = best[0] if len(best) == 1 else [i for i in best if i % 2 == 0][0]
    return i | (8 if np.signbit(x) else 0)


def store(x):
    """codes [.., D / 2] and scales [.., 4 or 8] (uint8) of rows x [.., D]; NaN as 0, infinities as the largest
    number of their sign."""
    x = np.asarray(x, dtype=np.float64)
    D = x.shape[-1]
    rows = np.where(np.isnan(x), 0.0, np.clip(x, -3.4e38, 3.4e38)).reshape(-1, D)
    codes = np.zeros((rows.shape[0], D // 2), np.uint8)
    scales = np.zeros((rows.shape[0], 4 if D <= 64 else 8), np.uint8)
    for r, row in enumerate(rows):
        for g in range(D // GROUP):
            part = row[g * GROUP:(g + 1) * GROUP]
            b = scale_byte(np.abs(part).max())
            scales[r, g] = b
            for i, v in enumerate(part):
                at = g * GROUP + i
                codes[r, at // 2] |= code_of(v, scale_of(b)) << (4 * (at % 2))
    return tuple(y.reshape(*x.shape[:-1], y.shape[1]) for y in (codes, scales))


def values(codes, scales):
    """The numbers [.., D] that codes and scales stand for."""
    D = codes.shape[-1] * 2
    c, s = codes.reshape(-1, D // 2), scales.reshape(-1, scales.shape[-1])
    by = np.array([scale_of(b) for b in range(256)])[s[:, :D // GROUP]].repeat(GROUP, axis=1)
    index = np.stack((c & 15, c >> 4), -1).reshape(-1, D)
    x = np.array(GRID)[index & 7] * np.where(index & 8, -1.0, 1.0) * by
    return x.reshape(*codes.shape[:-1], D)
