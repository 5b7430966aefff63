"""8-bit products and FFN in batches that take the tiles for many rows: token lists, entries and offsets out of range, values that are not
finite, workspaces of the exact size and with old contents, captured graphs, other streams, addresses next to 4 GiB."""
import numpy as np
import pytest

import fp8_reference as ref
from test_gpu_fp8 import check_ffn, dev, e4m3_rows, ffn_case, offsets_of, quantized, run_mm, wide

pytestmark = pytest.mark.gpu

TYPES = ["bf16", "f32"]


def torch_type(dtype):
    import torch

    return torch.bfloat16 if dtype == "bf16" else torch.float32


def many(sizes, N):
    """Rows of a batch that takes the tiles for many rows: more than 32 a group, 2^22 results."""
    return max(sum(sizes), 32 * len(sizes) + 1, -(-(1 << 22) // N))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,K,N", [
    ([1], 128, 1024), ([0, 5, 0, 17], 256, 1152), ([32, 33, 31], 384, 2176), ([64, 65, 63], 512, 640), ([128, 129, 127], 640, 1024), ([97, 96], 768, 896),
    ([300, 0, 1, 513], 896, 2304), ([40], 1024, 2176), ([1100, 1000], 128, 1024), ([20] * 64, 1152, 1920), ([2000, 1, 33], 2048, 2048)])
def test_product(sizes, K, N, dtype):
    run_mm(sizes, K, N, dtype, rows=many(sizes, N))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,N", [(128, 128), (640, 384)])
def test_product_of_token_rows(K, N, dtype):
    """perm_pair names the token of a row; entries out of range are clamped to the first and the last token, offsets that are no partition
    to the batch, and nothing outside y is written."""
    import torch

    from paper_2512_09277_amd import api

    T, k = 2100, 2
    rng = np.random.default_rng(K)
    x, xs, xv = quantized(rng, (T, K))
    w, ws, wv = quantized(rng, (3, N, K), 128)
    perm = rng.permutation(T * k).astype(np.int32)
    off = np.array([0, 700, 761, T * k - 5], np.int32)
    guard = torch.full((T * k + 64, N), -7.0, dtype=torch_type(dtype), device="cuda")
    y = api.moe_grouped_mm_fp8(x, xs, dev(off), w, ws, y=guard[32:32 + T * k], perm_pair=dev(perm), k=k).clone()
    for l in range(3):
        rows = slice(off[l], off[l + 1])
        want, err = ref.product(xv[perm[rows] // k], wv[l])
        assert (np.abs(wide(y)[rows] - want) <= ref.rounded(want, err, dtype == "bf16")).all()
    assert (y[T * k - 5:] == -7).all() and (guard[:32] == -7).all() and (guard[32 + T * k:] == -7).all()
    bad, same = perm.copy(), perm.copy()
    bad[[3, 800]], same[[3, 800]] = [-9, -1 << 30], 0
    bad[[7, 4000]], same[[7, 4000]] = [T * k + 5, (1 << 31) - 1], T * k - 1
    guard.fill_(-7)
    got = api.moe_grouped_mm_fp8(x, xs, dev(np.array([-4, 700, 761, 1 << 20], np.int32)), w, ws, y=guard[32:32 + T * k], perm_pair=dev(bad), k=k)
    want = api.moe_grouped_mm_fp8(x, xs, dev(np.array([0, 700, 761, T * k], np.int32)), w, ws, dtype=torch_type(dtype), perm_pair=dev(same), k=k)
    assert torch.equal(got, want) and (guard[:32] == -7).all() and (guard[32 + T * k:] == -7).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_values_that_are_not_finite_stay_in_their_rows_and_columns(dtype):
    """Also where rows and columns past a tile's end are loaded again: remainders of every class, half a tile of columns."""
    import torch

    from paper_2512_09277_amd import api

    rng = np.random.default_rng(5)
    K, N, sizes = 384, 640, [129, 50, 3, 7000]
    rows = many(sizes, N)
    x, xs, _ = quantized(rng, (rows, K))
    w, ws, _ = quantized(rng, (len(sizes), N, K), 128)
    off = dev(offsets_of(sizes))
    n = int(off[-1])
    call = lambda *a: api.moe_grouped_mm_fp8(*a, dtype=torch_type(dtype))[:n]  # noqa: E731
    clean = call(x, xs, off, w, ws)
    assert torch.isfinite(clean.float()).all()
    x2, w2 = x.clone(), w.clone()
    nan = torch.zeros((n, N), dtype=torch.bool, device="cuda")
    for r, c in ((128, 0), (178, 383), (181, 127), (182, 128), (7181, 200)):            # last rows of their groups, a first one
        x2.view(torch.uint8)[r, c] = 0x7f
        nan[r] = True
    for l, c, i in ((0, 639, 5), (1, 0, 383), (2, 512, 256), (3, 300, 130)):
        w2.view(torch.uint8)[l, c, i] = 0xff
        nan[int(off[l]):int(off[l + 1]), c] = True
    bad = call(x2, xs, off, w2, ws)
    assert torch.equal(torch.isnan(bad), nan) and torch.equal(bad[~nan], clean[~nan])
    xs2 = xs.clone()
    xs2[[60, 7000], [1, 2]] = torch.tensor([float("inf"), float("nan")], device="cuda")
    bad = call(x, xs2, off, w, ws)
    fine = torch.ones(n, dtype=torch.bool, device="cuda")
    fine[[60, 7000]] = False
    assert not torch.isfinite(bad[~fine].float()).any() and torch.equal(bad[fine], clean[fine])


@pytest.mark.parametrize("T,k,H,I,sizes", [(2100, 2, 256, 384, [4200]), (600, 8, 384, 128, [1000, 64, 0, 31, 3705]), (4097, 1, 128, 1152, [97, 4000])])
def test_ffn_workspace_of_the_exact_size(T, k, H, I, sizes):
    """The e4m3 activation and its scales lie inside the workspace; what an earlier call left there does not matter."""
    import torch

    from paper_2512_09277_amd import api

    args, xv, v13, w2v, perm = ffn_case(T, k, H, I, sizes, "bf16")
    need = api.moe_grouped_ffn_fp8_workspace_bytes(T, k, len(sizes), H, I)
    guard = torch.full((need + 4096,), 0xff, dtype=torch.uint8, device="cuda")
    y = api.moe_grouped_ffn_fp8(**args, ws=guard[:need]).clone()
    assert (guard[need:] == 0xff).all()
    check_ffn(wide(y), xv, v13, w2v, perm, k, sizes, "bf16")
    args["y_perm"].fill_(-7)
    assert torch.equal(api.moe_grouped_ffn_fp8(**args, ws=torch.zeros(need, dtype=torch.uint8, device="cuda")), y)


def test_ffn_values_that_are_not_finite_stay_in_their_rows():
    import torch

    from paper_2512_09277_amd import api

    sizes = [129, 50, 3, 4000]
    args, *_, perm = ffn_case(2100, 2, 256, 384, sizes, "bf16")
    n = sum(sizes)
    clean = api.moe_grouped_ffn_fp8(**args).clone()
    token = perm[128] // 2
    args["x"].view(torch.uint8)[token, 200] = 0x7f
    bad = api.moe_grouped_ffn_fp8(**args)
    nan = dev(perm[:n] // 2 == token)
    assert torch.isnan(bad[:n][nan].float()).all() and torch.equal(bad[:n][~nan], clean[:n][~nan]) and torch.equal(bad[n:], clean[n:])


def test_ffn_of_lists_out_of_range():
    """Tokens and offsets that are clamped, and groups that overlap, stay inside y and the workspace."""
    import torch

    from paper_2512_09277_amd import api

    T, k, H, I = 2100, 2, 256, 128
    args, *_ = ffn_case(T, k, H, I, [2000, 100, 2100], "bf16")
    clean = api.moe_grouped_ffn_fp8(**args).clone()
    need = api.moe_grouped_ffn_fp8_workspace_bytes(T, k, 3, H, I)
    ws = torch.full((need + 4096,), 0xff, dtype=torch.uint8, device="cuda")
    guard = torch.full((T * k + 64, H), -7.0, dtype=torch.bfloat16, device="cuda")
    args["perm_pair"][50], args["perm_pair"][3000] = -5, 1 << 30
    for off in ([0, 2000, 2100, 4200], [-9, 2000, 2100, 1 << 20], [0, 4200, 100, 4200]):
        args.update(group_offsets=dev(np.array(off, np.int32)), y_perm=guard[32:32 + T * k])
        guard.fill_(-7)
        y = api.moe_grouped_ffn_fp8(**args, ws=ws[:need])
        torch.cuda.synchronize()
        assert (guard[:32] == -7).all() and (guard[32 + T * k:] == -7).all() and (ws[need:] == 0xff).all()
        if off[2] == 2100:
            same = torch.ones(T * k, dtype=torch.bool, device="cuda")
            same[[50, 3000]] = False
            assert torch.equal(y[same], clean[same])


def test_captured_and_replayed():
    """The FFN and a product in one graph on other rows, lists and group sizes each time, beside eager calls on the same workspace."""
    import torch

    from paper_2512_09277_amd import api

    T, k, H, I = 2100, 2, 256, 128
    args, *_ = ffn_case(T, k, H, I, [2000, 100, 2100], "bf16")
    ws = torch.empty(api.moe_grouped_ffn_fp8_workspace_bytes(T, k, 3, H, I), dtype=torch.uint8, device="cuda")
    h = torch.empty((T * k, 2 * I), dtype=torch.float32, device="cuda")

    def step():
        api.moe_grouped_mm_fp8(args["x"], args["xs"], args["group_offsets"], args["w13"], args["s13"], y=h, perm_pair=args["perm_pair"], k=k)
        return api.moe_grouped_ffn_fp8(**args, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    rng = np.random.default_rng(3)
    for off in ([0, 2000, 2100, 4200], [0, 0, 3, 4100], [0, 1400, 2800, 4200], [0, 0, 0, 0], [0, 65, 4097, 4200]):
        q, s = ref.quantize32(rng.standard_normal((T, H)))
        args["x"].copy_(e4m3_rows(q))
        args["xs"].copy_(dev(s))
        args["perm_pair"].copy_(dev(rng.permutation(T * k).astype(np.int32)))
        args["group_offsets"].copy_(dev(np.array(off, np.int32)))
        args["y_perm"].fill_(-7)
        h.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        y, h1 = args["y_perm"].clone(), h.clone()
        args["y_perm"].fill_(-7)
        h.fill_(-7)
        step()
        torch.cuda.synchronize()
        assert torch.equal(args["y_perm"], y) and torch.equal(h, h1) and (y[off[-1]:] == -7).all()


def test_two_calls_at_once():
    """Two batches on two streams, each with a workspace of its own."""
    import torch

    from paper_2512_09277_amd import api

    calls = [ffn_case(2100, 2, 256, 384, [2000, 100, 2100], "bf16", seed=s)[0] for s in (1, 2)]
    want = [api.moe_grouped_ffn_fp8(**c).clone() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for c, s in zip(calls, streams):
        c["y_perm"].fill_(-7)
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                api.moe_grouped_ffn_fp8(**c)
    torch.cuda.synchronize()
    assert all(torch.equal(c["y_perm"], w) for c, w in zip(calls, want))


def test_addresses_next_to_4_gib():
    """Rows of x, and weight rows of a group, up to just below 2^32 bytes behind the first: what these tiles address in 32 bits."""
    import torch

    from paper_2512_09277_amd import api

    rng = np.random.default_rng(12)
    K, pitch, far = 128, 1 << 16, (1 << 16) - 1
    w, ws, wv = quantized(rng, (1, 128, K), 128)
    q, s = ref.quantize32(rng.standard_normal((300, K)))
    x = torch.zeros((far, pitch), dtype=torch.uint8, device="cuda").view(api.FP8)[:, :K]
    x[far - 300:].copy_(e4m3_rows(q))
    xs = torch.zeros((far, 1), device="cuda")
    xs[far - 300:] = dev(s)
    y = api.moe_grouped_mm_fp8(x, xs, dev(np.array([0, far], np.int32)), w, ws, dtype=torch.float32)
    want, err = ref.product(ref.values(q, s), wv[0])
    assert (np.abs(wide(y[far - 300:]) - want) <= ref.rounded(want, err, False)).all() and not y[:far - 300].any()
    del x, xs, y
    N = (1 << 16) - 128
    big = torch.zeros((1, N, pitch), dtype=torch.uint8, device="cuda").view(api.FP8)[:, :, :K]
    big[0, N - 128:].copy_(w[0])
    scale = torch.ones((1, N // 128, 1), device="cuda")
    scale[0, -1] = ws[0, 0]
    y = api.moe_grouped_mm_fp8(e4m3_rows(q), dev(s), dev(np.array([0, 300], np.int32)), big, scale, dtype=torch.float32)
    assert (np.abs(wide(y[:, N - 128:]) - want) <= ref.rounded(want, err, False)).all() and not y[:, :N - 128].any()


@pytest.mark.parametrize("T,k,H,I,sizes", [(20, 2, 4096, 256, [17, 0, 20]), (2100, 2, 4096, 128, [130, 0, 70]), (12, 2, 200, 72, [9, 8, 3])])
def test_weights_as_they_are_quantized(T, k, H, I, sizes):
    """moe_quantize_weights_fp8 on the halves of w13 as matrices of their own, its padded output taken as [spr, 2I, H] by the FFN."""
    import torch

    from paper_2512_09277_amd import api

    rng = np.random.default_rng(T)
    spr = len(sizes)
    w13, w2 = (torch.from_numpy((0.05 * rng.standard_normal(s)).astype(np.float32)).cuda().bfloat16() for s in ((spr, 2 * I, H), (spr, H, I)))
    x = torch.from_numpy(rng.standard_normal((T, H)).astype(np.float32)).cuda().bfloat16()
    a, b, c = api.moe_quantize_weights_fp8(w13.view(2 * spr, I, H)), api.moe_quantize_weights_fp8(w2), api.moe_quantize_fp8(x)
    q13, s13 = a["q"].view(spr, 2 * I, H), a["scale"].view(spr, -1, ref.blocks(H))
    assert q13.data_ptr() == a["q"].data_ptr()
    perm = np.full(T * k, -1, np.int32)
    perm[:sum(sizes)] = rng.permutation(T * k)[:sum(sizes)]
    y = torch.full((T * k, H), -7.0, dtype=torch.bfloat16, device="cuda")
    api.moe_grouped_ffn_fp8(c["q"], c["scale"], dev(perm), dev(offsets_of(sizes)), k, q13, s13, b["q"], b["scale"], y_perm=y)
    v13 = ref.values(wide(a["q"]), wide(a["scale"]), 128).reshape(spr, 2 * I, H)
    check_ffn(wide(y), ref.values(wide(c["q"]), wide(c["scale"])), v13, ref.values(wide(b["q"]), wide(b["scale"]), 128), perm, k, sizes, "bf16")
