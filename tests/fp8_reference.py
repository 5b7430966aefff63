"""Plain definitions of the 8-bit and sorted-row operators in 64 bits (numpy), and how far fp32 arithmetic may be from them.

A rounding to a type is off by at most half a step: 2^-24 of the value in fp32, 2^-8 in bf16, 2^-4 in e4m3 (2^-10 absolute where e4m3
values are subnormal, below 2^-6)."""
import numpy as np

BLOCK = 128
U32, UBF16 = 2.0 ** -24, 2.0 ** -8


def blocks(n):
    return -(-n // BLOCK)


def e4m3(v):
    """Nearest e4m3 value, ties to even: four significant bits, steps no finer than 2^-9, at most 448."""
    v = np.asarray(v, np.float64)
    with np.errstate(invalid="ignore"):
        step = np.ldexp(1.0, np.maximum(np.frexp(v)[1] - 4, -9))
        return np.clip(np.round(v / step) * step, -448.0, 448.0)


def block_max(x, rows_a_block=1):
    """Largest magnitude of every block [.., blocks of rows, blocks of K], NaN where there is one."""
    R, K = x.shape[-2:]
    pad = [(0, 0)] * (x.ndim - 2) + [(0, -R % rows_a_block), (0, -K % BLOCK)]
    b = np.pad(np.abs(x), pad)
    b = b.reshape(*x.shape[:-2], -1, rows_a_block, blocks(K), BLOCK)
    return b.max(axis=(-3, -1))


def spread(scale, R, K, rows_a_block=1):
    """A scale for every value."""
    return np.repeat(np.repeat(scale, rows_a_block, axis=-2)[..., :R, :], BLOCK, axis=-1)[..., :K]


def quantize32(x, rows_a_block=1):
    """The definition with its fp32 roundings: (values, fp32 scales), to be matched bit for bit."""
    x = np.asarray(x, np.float32)
    m = np.maximum(block_max(x, rows_a_block), np.float32(1e-30))
    with np.errstate(invalid="ignore"):
        v = x * spread(np.float32(448) / m, *x.shape[-2:], rows_a_block)
    return e4m3(v), m / np.float32(448)


def values(q, scale, rows_a_block=1):
    return np.asarray(q, np.float64) * spread(np.asarray(scale, np.float64), *q.shape[-2:], rows_a_block)


def product(x, w):
    """x [R,K] . w [N,K]^T in 64 bits, and how far fp32 may be off: a block's 128 exact products, summed and then scaled and added to
    the other blocks, pass fewer than 128 + 4 * blocks roundings."""
    bound = (BLOCK + 4 * blocks(x.shape[1]) + 8) * U32
    return x @ w.T, bound * (np.abs(x) @ np.abs(w).T)


def product_many(x, w):
    """As `product` where the matrix cores multiply e4m3 values themselves (16-bit results of many rows): they align the 128 products of a
    block to the largest and drop what lies more than 13 binary places below it, so each is off by at most 2^-13 of the largest."""
    y, err = product(x, w)
    for k in range(0, x.shape[1], BLOCK):
        # the largest product of a pair of rows is at most that of their largest values
        most = np.abs(x[:, k:k + BLOCK]).max(axis=1)[:, None] * np.abs(w[:, k:k + BLOCK]).max(axis=1)[None]
        err = err + BLOCK * 2.0 ** -13 * most
    return y, err


def ffn(x, w13, w2, product=product):
    """One expert on rows x [R,H] (values): (y [R,H], how far it may be off before y itself is rounded).

    The activation is requantized.  Its fp32 error moves a value by at most `da`, and the block's maximum likewise, so its e4m3 value
    lies between those of the two ends, which are two neighbours where the value is near a rounding border."""
    I = w13.shape[0] // 2
    gate, eg = product(x, w13[:I])
    up, eu = product(x, w13[I:])
    sig = 1 / (1 + np.exp(-gate))
    a = gate * sig * up
    # |silu'| < 1.1; exponential, sum, quotient and product: fewer than 8 roundings
    da = 1.1 * eg * (np.abs(up) + eu) + np.abs(gate * sig) * eu + 8 * U32 * np.abs(a)
    m = np.maximum(block_max(a), 1e-30)
    dm = spread(block_max(da) / m, *a.shape) + 4 * U32
    scale = spread(m / 448, *a.shape)
    q = e4m3(a / scale)
    lo, hi = (e4m3(np.clip((a + s * (da + np.abs(a) * dm)) / scale, -448, 448)) for s in (-1, 1))
    dq = np.maximum(np.abs(hi - q), np.abs(q - lo)) * scale + np.abs(q * scale) * dm
    y, ey = product(q * scale, w2)
    return y, ey + dq @ np.abs(w2).T


def rounded(y, err, bf16):
    """What a result off by `err` may be off after its own rounding (a float32 sum is rounded already)."""
    return err + UBF16 * (np.abs(y) + err) if bf16 else err + U32 * np.abs(y)
