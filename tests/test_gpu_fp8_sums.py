"""Sums of the 8-bit products and of the 8-bit FFN where large products cancel, in batches of few rows and of many: every product counts,
whatever the largest of its block, and the fp32 bounds of fp8_reference.py hold without any allowance."""
import numpy as np
import pytest

import fp8_reference as ref
from test_gpu_fp8 import dev, e4m3_rows, offsets_of, wide

pytestmark = pytest.mark.gpu

K, N = 256, 512


def cancelling(rng, rows, cols, at, sign=1):
    """[rows, cols] of +-1, +-2 and +-3 with 448 in column at[0] and +-448 in column at[1] of every row."""
    v = rng.integers(1, 4, (rows, cols)) * rng.choice([-1.0, 1.0], (rows, cols))
    v[:, at[0]], v[:, at[1]] = 448, 448 * sign
    return v


def run_product(xv, xs, wv, dtype):
    """y of rows xv * xs (a scale for each row) with one group of weights wv, scales 1, against 64 bits; y on the host."""
    import torch

    from paper_2512_09277_amd import api

    rows, k = xv.shape
    n = wv.shape[0]
    print(f"rows={rows} K={k} N={n} {dtype}", flush=True)
    s = np.repeat(xs[:, None], ref.blocks(k), axis=1).astype(np.float32)
    y = torch.full((rows, n), -7.0, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    api.moe_grouped_mm_fp8(e4m3_rows(xv), dev(s), dev(offsets_of([rows])), e4m3_rows(wv[None]),
                           torch.ones((1, ref.blocks(n), ref.blocks(k)), device="cuda"), y=y)
    got = wide(y)
    want, err = ref.product(xv * xs[:, None], wv)
    off_by = np.abs(got - want) - ref.rounded(want, err, dtype == "bf16")
    assert (off_by <= 0).all(), off_by.max()
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [24, 16384])
@pytest.mark.parametrize("at", [(0, 1), (0, 127), (5, 70), (31, 32), (130, 255)])
def test_large_products_that_cancel(at, rows, dtype):
    """448 * 448 - 448 * 448 + 126 small products: what remains is 2^-17 of the largest."""
    rng = np.random.default_rng(sum(at) + rows)
    run_product(cancelling(rng, rows, K, at), 2.0 ** rng.integers(-6, 7, rows), cancelling(rng, N, K, at, -1), dtype)


@pytest.mark.parametrize("times", [20, 400])
def test_outlier_channels_in_a_small_and_a_large_batch(times):
    """A few channels `times` as large as the others, in pairs whose weights are opposite; the same rows beside few others and beside
    many differ by the rounding of their results only."""
    rng = np.random.default_rng(times)
    x = rng.standard_normal((16384, K))
    w = rng.standard_normal((N, K))
    for a, b in ((3, 90), (140, 141), (200, 129)):
        x[:, a] *= times
        x[:, b] = x[:, a]
        w[:, b] = -w[:, a]
    xv, s = ref.quantize32(x)
    wv = ref.e4m3(64 * w)
    one = np.ones(16384)
    few, many = run_product(xv[:24], one[:24], wv, "bf16"), run_product(xv, one, wv, "bf16")
    _, err = ref.product(xv[:24], wv)
    assert (np.abs(few - many[:24]) <= 2 * ref.rounded(few, err, True)).all()


def run_ffn(x, w13, w2, T, k):
    import torch

    from paper_2512_09277_amd import api

    print(f"ffn T={T} k={k}", flush=True)
    H, I = x.shape[1], w2.shape[1]
    n = T * k - 3
    rng = np.random.default_rng(T)
    perm = np.full(T * k, -1, np.int32)
    perm[:n] = rng.permutation(T * k)[:n]
    one = lambda *s: torch.ones(s, device="cuda")  # noqa: E731
    y = api.moe_grouped_ffn_fp8(e4m3_rows(x), one(T, ref.blocks(H)), dev(perm), dev(offsets_of([n])), k, e4m3_rows(w13[None]),
                                one(1, 2 * ref.blocks(I), ref.blocks(H)), e4m3_rows(w2[None]), one(1, ref.blocks(H), ref.blocks(I)))
    want, err = ref.ffn(x[perm[:n] // k], w13, w2)
    off_by = np.abs(wide(y)[:n] - want) - ref.rounded(want, err, True)
    assert (off_by <= 0).all(), off_by.max()
    assert np.abs(want).min() > 4 * ref.rounded(want, err, True).max()      # far from the zero that is left when small products are lost


@pytest.mark.parametrize("T,k", [(12, 2), (2500, 2)])
def test_ffn_gate_of_products_that_cancel(T, k):
    """gate = 448 * 448 - 448 * 448 + 126, up = 1."""
    H, I = 128, 128
    x = np.ones((T, H))
    x[:, [7, 99]] = 448
    w13 = np.zeros((2 * I, H))
    w13[:I] = 1
    w13[:I, 7], w13[:I, 99] = 448, -448
    w13[I:, 0] = 1
    run_ffn(x, w13, np.ones((H, I)), T, k)


@pytest.mark.parametrize("T,k", [(12, 2), (2500, 2)])
def test_ffn_output_of_products_that_cancel(T, k):
    """act = 126 * (448, 448, 1, 1, ..), whose products with 448, -448, 1, 1, .. leave 126 * 126."""
    H, I = 256, 128
    x = np.ones((T, H))
    w13 = np.zeros((2 * I, H))
    w13[:I, :126] = 1
    w13[I:, 0] = 1
    w13[[I + 20, I + 100], 0] = 448
    w2 = np.ones((H, I))
    w2[:, 20], w2[:, 100] = 448, -448
    run_ffn(x, w13, w2, T, k)
