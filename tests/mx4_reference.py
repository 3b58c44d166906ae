"""4-bit images (include/brgemm.h) in numpy and 64 bits, written from their definition."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([GRID, -GRID])
ORDER = [0, 4, 1, 5, 2, 6, 3, 7]         # block of 32 whose power stands at each of the 8 places


def padded(K):
    return (K + 255) // 256 * 256


def nbytes(rows, K):
    return rows * (padded(K) // 2 + padded(K) // 32)


def quantise(x):
    """codes (rows x Kp) and power bytes (rows x Kp / 32) of rows of numbers."""
    rows, K = x.shape
    full = np.zeros((rows, padded(K)))
    full[:, :K] = x
    codes = np.zeros(full.shape, np.uint8)
    powers = np.zeros((rows, padded(K) // 32), np.uint8)
    for b in range(padded(K) // 32):
        block = full[:, 32 * b:32 * b + 32]
        with np.errstate(invalid="ignore", divide="ignore"):
            largest = np.abs(block).max(1)
            e = np.where(largest > 0, np.floor(np.log2(np.where(largest > 0, largest, 1.0))), -1000.0)
            e = np.where(np.ldexp(1.0, e.clip(-1000, 1000).astype(int)) > largest, e - 1, e)
            e = np.maximum(e - 2, -127.0)
            finite = np.isfinite(largest)
            e = np.where(finite, e, 0.0).astype(int)
            y = np.abs(block) / np.ldexp(1.0, e)[:, None]
            off = np.abs(y[:, :, None] - GRID)
            # the nearest; of two the one with an even code
            best = np.argmin(off + np.where(np.arange(8) % 2, 1e-9, 0.0), axis=2)
            best[y >= 6.0] = 7
            code = best + 8 * np.signbit(block)
        codes[:, 32 * b:32 * b + 32] = np.where(finite[:, None], code, 0)
        powers[:, b] = np.where(finite, e + 127, 255)
    return codes, powers


def image(x):
    codes, powers = quantise(np.asarray(x, dtype=np.float64))
    rows = codes.shape[0]
    planes = powers.reshape(rows, -1, 8)[:, :, ORDER].transpose(1, 0, 2)
    return np.concatenate([(codes[:, 0::2] | codes[:, 1::2] << 4).reshape(-1), planes.reshape(-1)])


def values(img, rows, K):
    """What an image stands for."""
    Kp = padded(K)
    raw = img[:rows * Kp // 2].reshape(rows, Kp // 2)
    code = np.empty((rows, Kp), np.uint8)
    code[:, 0::2], code[:, 1::2] = raw & 15, raw >> 4
    planes = img[rows * Kp // 2:].reshape(Kp // 256, rows, 8)
    powers = np.empty((rows, Kp // 256, 8), np.int64)
    powers[:, :, ORDER] = planes.transpose(1, 0, 2)
    scale = np.where(powers == 255, np.nan, np.ldexp(1.0, powers.astype(int) - 127)).reshape(rows, Kp // 32)
    return (VALUES[code] * np.repeat(scale, 32, axis=1))[:, :K]


def most_off(a, b, deep):
    """How far sums of a x b^T in fp32 may be off.  `deep`: the 128-deep instruction, whose sum is off by up to 2^-19 of its products'
    magnitudes (it cuts them off below the largest), and one rounding per instruction and per adding of partial sums (16 at most);
    else a rounding per product."""
    K = a.shape[1]
    magnitude = np.abs(a) @ np.abs(b).T
    return magnitude * (2.0 ** -19 + (K / 128 + 18) * 2.0 ** -24 if deep else (K + 18) * 2.0 ** -24)
