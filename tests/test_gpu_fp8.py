"""8-bit experts with block scales against plain definitions in 64 bits (fp8_reference.py): quantization bit for bit, the grouped product
and the FFN element by element within what fp32 arithmetic and the result's rounding allow."""
import numpy as np
import pytest

import fp8_reference as ref

pytestmark = pytest.mark.gpu


def dev(a):
    import torch

    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def wide(t):
    import torch

    return (t.float() if t.dtype == torch.float8_e4m3fn else t).double().cpu().numpy()


def bf16(a):
    """numpy values rounded to bf16, as float32"""
    import torch

    return torch.from_numpy(np.asarray(a, np.float32)).bfloat16().float().numpy()


def e4m3_rows(v, fill=0x7f, extra=0):
    """e4m3 tensor of the values `v` [.., R, K] on the device, rows padded with NaN bytes."""
    import torch

    K = v.shape[-1]
    buf = torch.full((*v.shape[:-1], (K + 15) // 16 * 16 + extra), fill, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    out = buf[..., :K]
    out.copy_(torch.from_numpy(np.asarray(v, np.float32)).cuda().to(torch.float8_e4m3fn))
    return out


def quantized(rng, shape, rows_a_block=1, size=1.0):
    """Random values: (e4m3 device tensor, scales on the device, the values they stand for)"""
    q, s = ref.quantize32(size * rng.standard_normal(shape), rows_a_block)
    return e4m3_rows(q, extra=16 * int(rng.integers(0, 3))), dev(s), ref.values(q, s, rows_a_block)


# ------------------------------------------------------------------------------------------ quantization
def awkward(rng, R, K):
    """Normal values with blocks of zeros, tiny, huge and tied values among them."""
    x = rng.standard_normal((R, K)).astype(np.float32)
    x[R // 2] *= 1e30
    x[R // 3, : K // 2] = 0
    x[R - 1] = 1e-38
    x[0, ::3] *= 448
    if R > 4:
        x[1] = np.float32(2.0) ** rng.integers(-12, 9, K)          # exact powers: ties and subnormals once scaled
        x[2] = np.round(x[2] * 8) / 8
        x[3] *= 3e-31                                               # around the smallest maximum
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,K", [(1, 1), (1, 128), (3, 127), (5, 136), (7, 2048), (64, 7168), (129, 1001), (33, 264), (300, 4096)])
def test_rows(R, K, dtype):
    import torch

    from paper_2512_09277_amd import api

    x = awkward(np.random.default_rng(R + K), R, K)
    if dtype == "bf16":
        x = bf16(x)
    buf = torch.zeros((R, K + (8 if K % 8 == 0 else 3)), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    for t in (buf[:, :K], buf[:, :K].clone()):                      # strided rows, whole ones
        t.copy_(dev(x))
        out = api.moe_quantize_fp8(t)
        q, s = ref.quantize32(x)
        assert np.array_equal(wide(out["scale"]), s.astype(np.float64))
        assert np.array_equal(wide(out["q"]), q)
        assert (np.abs(ref.values(q, s) - x) <= (2.0 ** -4 + 4 * ref.U32) * np.abs(x) + 2.0 ** -10 * ref.spread(s, R, K)).all()


def test_rows_up_to_a_count_on_the_device():
    import torch

    from paper_2512_09277_amd import api

    x = np.random.default_rng(3).standard_normal((40, 200)).astype(np.float32)
    q, s = ref.quantize32(x)
    for n, valid in ((0, 0), (1, 1), (17, 17), (40, 40), (99, 40), (-3, 0)):
        out = api.quantize_buffers(40, 200, "cuda")
        out["q"].view(torch.uint8).fill_(0x35)
        out["scale"].fill_(-2)
        api.moe_quantize_fp8(dev(x), n_rows=dev(np.array([n], np.int32)), out=out)
        assert np.array_equal(wide(out["q"])[:valid], q[:valid]) and np.array_equal(wide(out["scale"])[:valid], s[:valid])
        assert (out["q"].view(torch.uint8)[valid:] == 0x35).all() and (out["scale"][valid:] == -2).all()
    assert api.moe_quantize_fp8(torch.empty((0, 200), device="cuda"))["q"].shape == (0, 200)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_not_finite(dtype):
    import torch

    from paper_2512_09277_amd import api

    x = torch.ones((4, 384), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    x[0, 5] = float("nan")
    x[1, 130] = float("-inf")
    x[2, 0], x[2, 1] = float("inf"), float("nan")
    out = api.moe_quantize_fp8(x)
    q, s = wide(out["q"]), wide(out["scale"])
    assert np.isnan(s[0, 0]) and np.isnan(q[0, :128]).all() and np.isinf(s[1, 1]) and np.isnan(q[1, 130]) and np.isnan(s[2, 0])
    assert not q[1, 128:130].any() and not q[1, 131:256].any()
    fine = np.ones((4, 3), bool)
    fine[0, 0] = fine[1, 1] = fine[2, 0] = False
    assert (s[fine] == np.float32(1) / np.float32(448)).all() and (q.reshape(4, 3, 128)[fine] == 448).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,R,K", [(1, 1, 1), (2, 128, 128), (3, 130, 264), (2, 71, 1001), (1, 300, 4096), (5, 256, 136)])
def test_weights(S, R, K, dtype):
    import torch

    from paper_2512_09277_amd import api

    rng = np.random.default_rng(S * R + K)
    x = np.stack([awkward(rng, R, K) for _ in range(S)])
    if dtype == "bf16":
        x = bf16(x)
    buf = torch.zeros((S, R, K + 8), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    for t in (buf[:, :, :K], buf[:, :, :K].clone(memory_format=torch.contiguous_format)):
        t.copy_(dev(x))
        out = api.moe_quantize_weights_fp8(t)
        q, s = ref.quantize32(x, 128)
        assert np.array_equal(wide(out["scale"]), s.astype(np.float64)) and np.array_equal(wide(out["q"]), q)


# ------------------------------------------------------------------------------------------ products
def offsets_of(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)


def run_mm(sizes, K, N, dtype, rows=None, seed=0, product=ref.product):
    import torch

    from paper_2512_09277_amd import api

    print(f"mm sizes={sizes} K={K} N={N} {dtype}", flush=True)
    rng = np.random.default_rng(seed + K * 3 + N)
    n = int(sum(sizes))
    rows = n + 3 if rows is None else rows
    x, xs, xv = quantized(rng, (rows, K))
    w, ws, wv = quantized(rng, (len(sizes), N, K), 128, 0.02)
    off = offsets_of(sizes)
    y = torch.full((rows, N), -7.0, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    assert api.moe_grouped_mm_fp8(x, xs, dev(off), w, ws, y=y) is y
    got = wide(y)
    assert (got[n:] == -7).all()                                    # rows past the last group stay as they were
    for l, (a, b) in enumerate(zip(off, off[1:])):
        if b > a:
            want, err = product(xv[a:b], wv[l])
            off_by = np.abs(got[a:b] - want) - ref.rounded(want, err, dtype == "bf16")
            assert (off_by <= 0).all(), (l, off_by.max())
            # half a step of the result's type, and a hundredth of that for the sums
            assert np.linalg.norm(got[a:b] - want) <= 1.01 * (ref.UBF16 if dtype == "bf16" else 64 * ref.U32) * np.linalg.norm(want)
    return y


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes,K,N", [
    ([1], 128, 128), ([1], 1, 1), ([3, 0, 1], 16, 5), ([0, 0], 128, 128), ([16, 17, 15], 256, 128), ([31, 32, 33, 1], 384, 256),
    ([5, 0, 70, 2], 1024, 384), ([40, 9], 200, 72), ([2, 18], 127, 130), ([7], 129, 1001), ([64, 65, 63], 640, 128),
    ([128, 129, 127, 97], 896, 256), ([300, 1], 512, 640), ([1, 1, 1, 1, 1], 2048, 256), ([20], 4096, 128), ([9, 33], 1336, 1000)])
def test_product(sizes, K, N, dtype):
    run_mm(sizes, K, N, dtype)


def test_product_of_more_rows_than_a_launch_has_workgroups():
    run_mm([700, 0, 1300, 41], 256, 1024, "bf16")
    run_mm([64, 64] + [30] * 62, 128, 2048, "f32")


def many(sizes, N):
    """Rows of a batch that takes the tiles for many rows."""
    return max(sum(sizes), 32 * len(sizes) + 1, -(-(1 << 21) // N))


@pytest.mark.parametrize("sizes,K,N", [
    ([1], 128, 128), ([0, 5, 0, 17], 256, 384), ([32, 33, 31], 384, 256), ([64, 65, 63], 512, 640), ([128, 129, 127], 640, 128), ([97, 96], 768, 256),
    ([300, 0, 1, 513], 896, 384), ([40], 1024, 2176), ([200], 2048, 256), ([1100, 1000], 128, 256), ([20] * 64, 1152, 128)])
def test_product_of_many_rows(sizes, K, N):
    run_mm(sizes, K, N, "bf16", rows=many(sizes, N), product=ref.product_many)
    if N >= 384:                                                    # fp32 results: from four times as many on
        run_mm(sizes, K, N, "f32", rows=4 * many(sizes, N))


@pytest.mark.parametrize("K", [128, 256, 384, 512, 640, 1152])
def test_product_of_more_tiles_than_workgroups(K):
    """A workgroup's next tile is loaded by the last steps of the one before: steps fewer than the stages of the ring, as many, more; big
    tiles of both kinds and small ones, a change from the ones to the others, fewer columns than XCDs and more."""
    run_mm([7000, 1500, 70, 1, 20, 45, 8, 300], K, 1024, "bf16", product=ref.product_many)
    run_mm([2900, 40, 1, 129, 31], K, 2304, "bf16", product=ref.product_many)
    run_mm([2900, 40, 1, 129, 31], K, 2304, "f32", rows=3700)
    run_mm([20, 3, 31, 0] * 16, K, 2176, "bf16", rows=many([20, 3, 31, 0] * 16, 2176), product=ref.product_many)


def test_product_of_token_rows():
    """perm_pair names the token of a row; entries out of range are clamped, offsets that are no partition too."""
    import torch

    from paper_2512_09277_amd import api

    T, k, K, N = 13, 3, 256, 128
    rng = np.random.default_rng(4)
    x, xs, xv = quantized(rng, (T, K))
    w, ws, wv = quantized(rng, (2, N, K), 128)
    perm = rng.permutation(T * k).astype(np.int32)
    off = offsets_of([20, 11])
    y = api.moe_grouped_mm_fp8(x, xs, dev(off), w, ws, dtype=torch.float32, perm_pair=dev(perm), k=k)
    for l in (0, 1):
        rows = slice(off[l], off[l + 1])
        want, err = ref.product(xv[perm[rows] // k], wv[l])
        assert (np.abs(wide(y)[rows] - want) <= ref.rounded(want, err, False)).all()
    bad = perm.copy()
    bad[3], bad[7] = -9, T * k + 5
    guard = torch.full((T * k + 64, N), -7.0, device="cuda")
    z = api.moe_grouped_mm_fp8(x, xs, dev(np.array([-4, 20, 500], np.int32)), w, ws, y=guard[32:32 + T * k], perm_pair=dev(bad), k=k)
    assert (guard[:32] == -7).all() and (guard[32 + T * k:] == -7).all()
    same = np.setdiff1d(np.arange(31), [3, 7])
    assert torch.equal(z[same], y[same])


@pytest.mark.parametrize("offsets", [[-4, 900, 100000], [700, 300, 20000], [0, 16000, 16384], [16384, 16384, 16384]])
def test_offsets_that_are_no_partition(offsets):
    """Batches of many rows: what offsets past the batch name is left out, and nothing outside y is written."""
    import torch

    from paper_2512_09277_amd import api

    rng = np.random.default_rng(9)
    K, N, rows = 256, 128, 16384
    x, xs, _ = quantized(rng, (rows, K))
    w, ws, _ = quantized(rng, (2, N, K), 128)
    clean = [max(0, min(o, rows)) for o in offsets]
    for l in (1, 2):
        clean[l] = max(clean[l - 1], clean[l]) if offsets[l] >= offsets[l - 1] else clean[l]
    guard = torch.full((rows + 256, N), -7.0, dtype=torch.bfloat16, device="cuda")
    api.moe_grouped_mm_fp8(x, xs, dev(np.array(offsets, np.int32)), w, ws, y=guard[128:128 + rows])
    assert (guard[:128] == -7).all() and (guard[128 + rows:] == -7).all() and torch.isfinite(guard.float()).all()
    if sorted(offsets) == offsets:
        want = torch.full((rows, N), -7.0, dtype=torch.bfloat16, device="cuda")
        api.moe_grouped_mm_fp8(x, xs, dev(np.array(clean, np.int32)), w, ws, y=want)
        assert torch.equal(guard[128:128 + rows], want)


def test_offsets_past_32_bits():
    """Rows of x and weights of a group that start more than 4 GiB behind their first."""
    import torch

    from paper_2512_09277_amd import api

    rng = np.random.default_rng(10)
    K, N, T = 8192, 128, (1 << 19) + 40
    far, fs, fv = quantized(rng, (40, K))
    w, ws, wv = quantized(rng, (1, N, K), 128, 0.02)
    x = torch.zeros((T, K), dtype=torch.uint8, device="cuda").view(api.FP8)
    x[T - 40:].copy_(far)
    xs = torch.zeros((T, K // 128), device="cuda")
    xs[T - 40:] = fs
    perm = torch.full((T,), T - 1, dtype=torch.int32, device="cuda")
    perm[:40] = torch.arange(T - 40, T, dtype=torch.int32)
    off = dev(np.array([0, 40], np.int32))
    y = api.moe_grouped_mm_fp8(x, xs, off, w, ws, dtype=torch.float32, perm_pair=perm)
    want, err = ref.product(fv, wv[0])
    assert (np.abs(wide(y[:40]) - want) <= ref.rounded(want, err, False)).all()
    del x, xs, perm, y
    G, M = 65 - 1, 8200
    big = torch.zeros((G, M, K), dtype=torch.uint8, device="cuda").view(api.FP8)       # 4.3 GB; the last group's last rows count
    big[G - 1, M - N:].copy_(w[0])
    scale = torch.zeros((G, (M + 127) // 128, K // 128), device="cuda")
    scale[G - 1, (M - N) // 128:] = 1
    off = torch.zeros(G + 1, dtype=torch.int32, device="cuda")
    off[G] = 40
    y = api.moe_grouped_mm_fp8(far, fs, off, big, scale, dtype=torch.float32)
    want, err = ref.product(fv, wide(w[0]))
    assert (np.abs(wide(y[:, M - N:]) - want) <= ref.rounded(want, err, False)).all() and not y[:, :M - N].any()


def test_values_that_are_not_finite_stay_in_their_rows_and_columns():
    import torch

    from paper_2512_09277_amd import api

    rng = np.random.default_rng(5)
    K, N = 384, 256
    x, xs, xv = quantized(rng, (12, K))
    w, ws, wv = quantized(rng, (2, N, K), 128)
    off = dev(offsets_of([5, 7]))
    clean = api.moe_grouped_mm_fp8(x, xs, off, w, ws, dtype=torch.float32)
    x2, w2 = x.clone(), w.clone()
    x2.view(torch.uint8)[3, 100] = 0x7f
    w2.view(torch.uint8)[1, 200, 380] = 0xff
    bad = api.moe_grouped_mm_fp8(x2, xs, off, w2, ws, dtype=torch.float32)
    nan = torch.zeros((12, N), dtype=torch.bool, device="cuda")
    nan[3] = True
    nan[5:, 200] = True
    assert torch.equal(torch.isnan(bad), nan) and torch.equal(bad[~nan], clean[~nan])
    xs2 = xs.clone()
    xs2[6, 1] = float("inf")
    assert not torch.isfinite(api.moe_grouped_mm_fp8(x, xs2, off, w, ws, dtype=torch.float32)[6]).any()


def test_the_input_gradient_is_the_same_call():
    """dx = dy . W: transposed weights and scales; blocks of 128 x 128 stay blocks."""
    import torch

    from paper_2512_09277_amd import api

    rng = np.random.default_rng(6)
    K, N, sizes = 384, 256, [9, 0, 23]
    w, ws, wv = quantized(rng, (3, N, K), 128, 0.02)
    dy = torch.from_numpy(rng.standard_normal((sum(sizes), N)).astype(np.float32)).cuda()
    g = api.moe_quantize_fp8(dy)
    wt = w.transpose(1, 2).contiguous()
    dx = api.moe_grouped_mm_fp8(g["q"], g["scale"], dev(offsets_of(sizes)), wt, ws.transpose(1, 2).contiguous(), dtype=torch.float32)
    gv = ref.values(wide(g["q"]), wide(g["scale"]))
    off = offsets_of(sizes)
    for l in range(3):
        rows = slice(off[l], off[l + 1])
        want, err = ref.product(gv[rows], wv[l].T)
        assert (np.abs(wide(dx)[rows] - want) <= ref.rounded(want, err, False)).all()


# ------------------------------------------------------------------------------------------ FFN
def ffn_case(T, k, H, I, sizes, dtype, seed=0):
    import torch

    rng = np.random.default_rng(seed + H + 5 * I)
    spr, n = len(sizes), int(sum(sizes))
    x, xs, xv = quantized(rng, (T, H))
    w13 = (0.05 * rng.standard_normal((spr, 2, I, H))).astype(np.float32)
    q13, s13 = ref.quantize32(w13, 128)                             # gate and up have blocks of their own
    w2, s2, w2v = quantized(rng, (spr, H, I), 128, 0.05)
    v13 = ref.values(q13, s13, 128).reshape(spr, 2 * I, H)
    perm = np.full(T * k, -1, np.int32)
    perm[:n] = rng.permutation(T * k)[:n]
    y = torch.full((T * k, H), -7.0, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    args = dict(x=x, xs=xs, perm_pair=dev(perm), group_offsets=dev(offsets_of(sizes)), k=k, w13=e4m3_rows(q13.reshape(spr, 2 * I, H)),
                s13=dev(s13.reshape(spr, -1, s13.shape[-1])), w2=w2, s2=s2, y_perm=y)
    return args, xv, v13, w2v, perm


def check_ffn(got, xv, v13, w2v, perm, k, sizes, dtype):
    off = offsets_of(sizes)
    assert (got[off[-1]:] == -7).all()
    for l, (a, b) in enumerate(zip(off, off[1:])):
        if b > a:
            want, err = ref.ffn(xv[perm[a:b] // k], v13[l], w2v[l])
            off_by = np.abs(got[a:b] - want) - ref.rounded(want, err, dtype == "bf16")
            assert (off_by <= 0).all(), (l, off_by.max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,H,I,sizes", [
    (1, 1, 128, 128, [1]), (1, 2, 64, 8, [0, 1, 1]), (8, 2, 256, 128, [3, 0, 5]), (16, 2, 384, 256, [16, 15, 1]), (40, 2, 512, 384, [17, 33, 0, 30]),
    (9, 3, 200, 72, [4, 9, 1]), (12, 2, 127, 130, [7, 12]), (33, 2, 1000, 356, [40, 2, 20]), (100, 4, 256, 256, [130, 128, 65, 1, 60]),
    (6, 1, 2048, 768, [1, 2, 3]), (5, 2, 96, 5, [6]), (300, 2, 256, 128, [300, 290])])
def test_ffn(T, k, H, I, sizes, dtype):
    from paper_2512_09277_amd import api

    print(f"ffn T={T} k={k} H={H} I={I} sizes={sizes} {dtype}", flush=True)
    args, xv, v13, w2v, perm = ffn_case(T, k, H, I, sizes, dtype)
    y = api.moe_grouped_ffn_fp8(**args)
    check_ffn(wide(y), xv, v13, w2v, perm, k, sizes, dtype)


@pytest.mark.parametrize("T,k,H,I,sizes", [
    (2100, 2, 128, 128, [1]), (2100, 2, 256, 384, [3, 0, 32, 33]), (2100, 2, 512, 256, [64, 65, 0, 1]), (2100, 2, 640, 128, [128, 129, 127]),
    (2100, 2, 896, 640, [300, 20, 513, 60]), (1500, 4, 256, 1152, [2000, 1000, 40, 7, 33, 900, 20]), (2200, 2, 256, 256, [4300, 0, 100]),
    (1100, 4, 384, 1152, [30] * 20), (4200, 1, 2048, 256, [90, 7])])
def test_ffn_of_many_rows(T, k, H, I, sizes):
    """Products of e4m3 values (see ref.product_many).  Element by element, what that bound lets happen to the activation: at worst most
    values move over an e4m3 border, a step of up to 2^-3 of themselves.  Over the rows of a group the norm tells more: sums of 128
    products of normal values are off by 1.5e-5 rms (the instruction's, measured), which moves a value over a border with a probability of
    about 1.5e-5 / 2^-4 by 2^-4 of itself, sqrt(2.4e-4) * 2^-4 = 1e-3 of the norm, beside 2^-8 at most for the rounding to bf16.  A single
    row can be off by more: one of its largest activations moved is 2^-3 of that one."""
    from paper_2512_09277_amd import api

    print(f"ffn of many rows T={T} k={k} H={H} I={I} sizes={sizes}", flush=True)
    args, xv, v13, w2v, perm = ffn_case(T, k, H, I, sizes, "bf16")
    got = wide(api.moe_grouped_ffn_fp8(**args))
    off = offsets_of(sizes)
    assert (got[off[-1]:] == -7).all()
    for l, (a, b) in enumerate(zip(off, off[1:])):
        if b > a:
            want, err = ref.ffn(xv[perm[a:b] // k], v13[l], w2v[l], product=ref.product_many)
            off_by = np.abs(got[a:b] - want) - ref.rounded(want, err, True)
            assert (off_by <= 0).all(), (l, off_by.max())
            if b - a >= 30:
                assert np.linalg.norm(got[a:b] - want) <= (ref.UBF16 + 1e-3) * np.linalg.norm(want)


@pytest.mark.parametrize("T,k,H,I,sizes,dtype", [
    (2100, 2, 256, 128, [40, 0, 150, 3], "f32"), (4200, 1, 200, 128, [17, 33], "bf16"), (2100, 2, 128, 72, [20, 5], "bf16")])
def test_ffn_of_many_rows_in_other_forms(T, k, H, I, sizes, dtype):
    """fp32 results and odd sizes keep the tiles for few rows, whose activation between the products is fp32; so does a full batch."""
    from paper_2512_09277_amd import api

    args, xv, v13, w2v, perm = ffn_case(T, k, H, I, sizes, dtype)
    check_ffn(wide(api.moe_grouped_ffn_fp8(**args)), xv, v13, w2v, perm, k, sizes, dtype)
    sizes = [T * k]
    args, xv, v13, w2v, perm = ffn_case(T, k, H, I, sizes, dtype)
    import torch

    need = api.moe_grouped_ffn_fp8_workspace_bytes(T, k, 1, H, I)
    guard = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    check_ffn(wide(api.moe_grouped_ffn_fp8(**args, ws=guard[:need])), xv, v13, w2v, perm, k, sizes, dtype)
    assert (guard[need:] == 0x5a).all()


def test_ffn_without_rows():
    import torch

    from paper_2512_09277_amd import api

    args, *_ = ffn_case(4, 2, 128, 128, [0, 0], "bf16")
    assert (api.moe_grouped_ffn_fp8(**args) == -7).all()
    args.update(x=args["x"][:0], xs=args["xs"][:0], perm_pair=args["perm_pair"][:0], y_perm=torch.empty((0, 128), device="cuda"))
    assert api.moe_grouped_ffn_fp8(**args).shape == (0, 128)


def test_a_later_call_leaves_no_trace():
    """A workspace that a larger batch has used, full of NaN beside: the same result as a clean one."""
    import torch

    from paper_2512_09277_amd import api

    args, *_ = ffn_case(40, 2, 200, 72, [17, 33, 0, 30], "f32")
    need = api.moe_grouped_ffn_fp8_workspace_bytes(40, 2, 4, 200, 72)
    a = api.moe_grouped_ffn_fp8(**args, ws=torch.zeros(need, dtype=torch.uint8, device="cuda")).clone()
    b = api.moe_grouped_ffn_fp8(**args, ws=torch.full((need + 512,), 0xff, dtype=torch.uint8, device="cuda"))
    assert torch.equal(a, b)
