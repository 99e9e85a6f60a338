"""The 4-bit formats in 64 bits on the CPU: decisions, packed layout, what packed arrays stand for."""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
BORDERS = (E2M1[1:] + E2M1[:-1]) / 2
BLOCK = {"mxf4": 32, "nvf4": 16}


def e4m3_values():
    """All 127 finite non-negative E4M3 numbers, by their byte."""
    b = np.arange(127)
    e, f = b >> 3, b & 7
    return np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e.astype(np.float64) - 10))


def nearest(y, grid):
    """Place in the increasing grid of the number nearest to y >= 0, ties to the even place, the last beyond the end."""
    y = np.minimum(y, grid[-1])
    hi = np.clip(np.searchsorted(grid, y), 1, len(grid) - 1)
    lo = hi - 1
    down, up = y - grid[lo], grid[hi] - y
    return np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)


def padded(length):
    return (length + 63) // 64 * 64


def quantise(x, fmt, t=1.0):
    """Of the rows of x (float64 [outer][length]): codes [outer][padded], scale bytes [outer][blocks], and how far each quotient is from the
    nearest border, as a share of it."""
    b = BLOCK[fmt]
    outer, length = x.shape
    full = np.zeros((outer, (padded(length) + b - 1) // b * b))
    full[:, :length] = x
    z = full.reshape(outer, -1, b)
    with np.errstate(all="ignore"):
        m = np.abs(z).max(2) if z.size else np.zeros(z.shape[:2])      # (NaN where there is one)
        bad = ~np.isfinite(m)
        if fmt == "mxf4":
            e = np.frexp(np.where(bad, 1.0, m))[1] - 3
            byte = np.where(m > 0, np.clip(e + 127, 0, 254), 0)
            unit = 2.0 ** (byte.astype(np.float64) - 127)
            byte = np.where(bad, 255, byte)
        else:
            bad |= not (0 < t < np.inf)
            byte = np.where(bad, 127, nearest(np.where(bad, 0, m / (6 * t)), e4m3_values()))
            unit = e4m3_values()[np.where(bad, 0, byte)] * t
        q = np.where((unit > 0)[..., None] & ~bad[..., None], np.abs(z) / np.where(unit > 0, unit, 1)[..., None], 0)
        code = nearest(q, E2M1) | np.where(np.signbit(z), 8, 0)
        code = np.where(bad[..., None], 0, code)
        near = np.abs(q[..., None] - BORDERS).min(-1)
    codes = code.reshape(outer, -1)[:, :padded(length)].astype(np.uint8)
    # blocks that begin behind the end have scale 0
    nb = (length + b - 1) // b
    byte[:, nb:] = 0
    return codes, byte.astype(np.uint8), near.reshape(outer, -1)[:, :padded(length)]


def values(codes, bytes_, fmt, t=1.0, length=None):
    b = BLOCK[fmt]
    if fmt == "mxf4":
        s = np.where(bytes_ == 255, np.nan, 2.0 ** (bytes_.astype(np.float64) - 127))
    else:
        s = np.where(bytes_ == 127, np.nan, e4m3_values()[np.minimum(bytes_, 126)]) * t
    e = np.where(codes & 8, -1.0, 1.0) * E2M1[codes & 7]
    v = e * np.repeat(s, b, axis=1)[:, :e.shape[1]]
    return v if length is None else v[:, :length]


def unpack_data(data, outer, length):
    """Codes [outer][padded] of packed bytes; the two zeros alike."""
    d = np.asarray(data).reshape(outer, padded(length) // 2)
    c = np.empty((outer, padded(length)), dtype=np.uint8)
    c[:, 0::2], c[:, 1::2] = d & 15, d >> 4
    return one_zero(c)


def one_zero(codes):
    return np.where(codes == 8, 0, codes)


def tiles_of(length, fmt):
    return -(-padded(length) // (4 * BLOCK[fmt]))


def unpack_scales(scales, rows_at, length, fmt):
    """Scale bytes [rows][blocks] of the rows that lie at `rows_at` (places counted over the tiles of 128)."""
    C = tiles_of(length, fmt)
    t = np.asarray(scales).reshape(-1, C, 32, 4, 4)           # tile, column tile, r % 32, r / 32, c
    t = t.transpose(0, 3, 2, 1, 4).reshape(-1, C * 4)         # (tile, r / 32, r % 32), (column tile, c)
    return t[rows_at][:, : -(-padded(length) // BLOCK[fmt])]


def group_places(offsets):
    """For the rows of every group in turn: its number and its place over the tiles of scales."""
    rows, at = [], []
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        rows += range(lo, hi)
        at += range((lo // 128 + g) * 128, (lo // 128 + g) * 128 + hi - lo)
    return np.array(rows, dtype=np.int64), np.array(at, dtype=np.int64)


def tensor_scale(x):
    m = float(np.abs(x).max()) if x.size else 0.0
    t = max(m / 2688, 2.0 ** -60)
    step = 2.0 ** (np.frexp(t)[1] - 8)
    return float(np.ceil(t / step) * step)


def one_groups_tiles(rows, N, K, pairs, cut=True):
    """Which tiles a plan without groups takes on `pairs` pairs of SMs (csrc/nk_mx.cu): rows of a tile, parts of those of the last wave."""
    best, width, parts = 1e300, 0, 1
    tiles_i, kbs = -(-N // 256), -(-K // 256)
    w = 32 if rows <= 32 else 64
    while w <= 256:
        n = -(-rows // w) * tiles_i
        waves, rest = divmod(n, pairs)

        def block(active):
            return 460 + (450 + w + w // 2 - 460) * min(1.0, active / pairs)
        c = 1
        while c == 1 or (cut and rest and c <= 8 and c <= kbs and c * rest <= pairs):
            t = waves * (kbs * block(pairs) + 300) + (-(-kbs // c) * block(rest * c) if rest else 0) + 300 + 8 * w
            t += 2900 + 700 * c + rest * c * w * (2048 / 3500) if c > 1 else 0
            if t < best * 0.999 or (t <= best * 1.001 and c == 1 and parts == 1):
                best, width, parts = min(best, t), w, c
            c += 1
        if w >= rows:
            break
        w += 32 if w < 64 else 64
    return width, parts


def groups_width(sizes, N, K, pairs):
    """Rows of a tile where the rows are grouped, as the kernel's scheduler chooses them (csrc/mx.cuh)."""
    most = max(sizes)
    if most <= 64:
        return 32 if most <= 32 else 64
    found = []
    for w in (64, 128, 192, 256):
        w = min(w, (most + 63) // 64 * 64)
        waves = -(-sum(-(-n // w) for n in sizes) * -(-N // 256) // pairs)
        found.append((waves * (-(-K // 256) * (450 + w + w // 2) + 300) + 8 * w, -w))
    return -min(found)[1]
