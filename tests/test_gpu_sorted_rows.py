"""moe_permute_rows, its gradient and the gradient of moe_unpermute against plain definitions in 64 bits, at the sizes where the kernels
change path: rows of whole vectors and odd ones, a wave or a workgroup per token, more pairs than a token keeps in registers, tokens
without a pair, one token, none."""
import numpy as np
import pytest

import fp8_reference as ref

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 8), (1, 2, 7), (5, 2, 1), (33, 3, 40), (64, 8, 256), (37, 8, 2048), (19, 9, 2056), (12, 17, 1001), (130, 6, 7168), (7, 2, 4100)]


def inputs(T, k, H, dtype, seed, absent=0.4):
    """Random rows for a part of the pairs, as a rank's lists give them: (pair_row, rows in use, tensors by name)."""
    import torch

    rng = np.random.default_rng(seed)
    here = np.flatnonzero(rng.random(T * k) >= absent)
    row = np.full(T * k, -1, np.int32)
    row[here] = rng.permutation(here.size)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rnd = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(dt).cuda()  # noqa: E731
    t = dict(x=rnd(T, H), y=rnd(T * k, H), w=torch.from_numpy(rng.random((T, k)).astype(np.float32)).cuda())
    return row.reshape(T, k), here.size, t


def wide(t):
    return t.double().cpu().numpy()


def dev(a):
    import torch

    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def filled(shape, dtype):
    import torch

    return torch.full(shape, -7.0, dtype=dtype, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,H", SIZES)
def test_rows_and_gradient(T, k, H, dtype):
    from paper_2512_09277_amd import api

    row, n, t = inputs(T, k, H, dtype, T * 31 + H)
    x_perm = api.moe_permute_rows(t["x"], dev(row), x_perm=filled((T * k, H), t["x"].dtype))
    want = np.full((T * k, H), -7.0)
    pair = np.flatnonzero(row.reshape(-1) >= 0)
    want[row.reshape(-1)[pair]] = wide(t["x"])[pair // k]
    assert np.array_equal(wide(x_perm), want)                       # rows are copied; those that no pair names stay as they were
    dx = api.moe_permute_rows_backward(t["y"], dev(row), dx=filled((T, H), t["x"].dtype))
    y, size = np.zeros((T, H)), np.zeros((T, H))
    np.add.at(y, pair // k, wide(t["y"])[row.reshape(-1)[pair]])
    np.add.at(size, pair // k, np.abs(wide(t["y"]))[row.reshape(-1)[pair]])
    assert (np.abs(wide(dx) - y) <= ref.rounded(y, k * ref.U32 * size, dtype == "bf16")).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,H", SIZES)
def test_combine_gradient(T, k, H, dtype):
    import torch

    from paper_2512_09277_amd import api

    row, n, t = inputs(T, k, H, dtype, T * 37 + H)
    dy, dw = api.moe_unpermute_backward(t["x"], t["y"], dev(row), t["w"], dy_perm=filled((T * k, H), t["x"].dtype),
                                        dtopk_w=filled((T, k), torch.float32))
    flat = row.reshape(-1)
    pair = np.flatnonzero(flat >= 0)
    g, y, w = wide(t["x"]), wide(t["y"]), wide(t["w"]).reshape(-1)
    want = np.full((T * k, H), -7.0)
    want[flat[pair]] = g[pair // k] * w[pair][:, None]
    assert (np.abs(wide(dy) - want) <= ref.rounded(want, 0 * want, dtype == "bf16") + ref.U32 * np.abs(want)).all()
    dots, size = np.zeros(T * k), np.zeros(T * k)
    dots[pair] = (g[pair // k] * y[flat[pair]]).sum(axis=1)
    size[pair] = np.abs(g[pair // k] * y[flat[pair]]).sum(axis=1)
    assert (np.abs(wide(dw).reshape(-1) - dots) <= (H + 8) * ref.U32 * size).all()      # pairs of other ranks: exactly 0


def test_gradients_are_those_of_the_forward_calls():
    """Central differences of the forward kernels: the combine is linear in the rows and in the weights, the sort in the tokens, so a
    difference over any step is the derivative, up to fp32 sums of T * H terms."""
    import torch

    from paper_2512_09277_amd import api

    T, k, H = 9, 3, 52
    row, n, t = inputs(T, k, H, "f32", 5)
    r, c = dev(row), torch.randn((T, H), generator=torch.Generator().manual_seed(1)).cuda()
    out = lambda y, w: (api.moe_unpermute(y, r, w).double() * c.double()).sum().item()  # noqa: E731
    dy, dw = api.moe_unpermute_backward(c, t["y"], r, t["w"], dy_perm=torch.zeros_like(t["y"]))
    size = float((t["y"].abs().double().sum()))
    for i, j in ((0, 0), (3, 1), (8, 2), (5, 0)):
        step = torch.zeros_like(t["w"])
        step[i, j] = 1
        diff = (out(t["y"], t["w"] + step) - out(t["y"], t["w"] - step)) / 2
        assert abs(diff - dw[i, j].item()) <= 16 * ref.U32 * size
    for i in range(n):
        step = torch.zeros_like(t["y"])
        step[i, i % H] = 1
        diff = (out(t["y"] + step, t["w"]) - out(t["y"] - step, t["w"])) / 2
        assert abs(diff - dy[i, i % H].item()) <= 16 * ref.U32 * size
    cp = torch.randn((T * k, H), generator=torch.Generator().manual_seed(2)).cuda()
    dx = api.moe_permute_rows_backward(cp, r)
    sort = lambda x: (api.moe_permute_rows(x, r, x_perm=torch.zeros_like(cp)).double() * cp.double()).sum().item()  # noqa: E731
    for i in range(T):
        step = torch.zeros_like(t["x"])
        step[i, i % H] = 1
        diff = (sort(t["x"] + step) - sort(t["x"] - step)) / 2
        assert abs(diff - dx[i, i % H].item()) <= 16 * ref.U32 * size


def test_rows_out_of_range_and_unaligned_memory():
    """Entries outside [0, T*k) count as pairs of other ranks; tensors that start off a 16-byte border take the element-wise kernels."""
    import torch

    from paper_2512_09277_amd import api

    T, k, H = 11, 2, 64
    row, n, t = inputs(T, k, H, "f32", 8)
    bad = row.copy()
    bad.reshape(-1)[np.flatnonzero(row.reshape(-1) < 0)] = [T * k, -5, 1 << 30, T * k + 7][0]
    a = api.moe_permute_rows(t["x"], dev(row), x_perm=filled((T * k, H), torch.float32))
    b = api.moe_permute_rows(t["x"], dev(bad), x_perm=filled((T * k, H), torch.float32))
    assert torch.equal(a, b)
    off = lambda s: torch.empty(s.numel() + 1, dtype=s.dtype, device="cuda")[1:].view(s.shape).copy_(s)  # noqa: E731
    assert torch.equal(api.moe_permute_rows(off(t["x"]), dev(row), x_perm=filled((T * k, H), torch.float32)), a)
    dy, dw = api.moe_unpermute_backward(t["x"], t["y"], dev(row), t["w"], dy_perm=filled((T * k, H), torch.float32))
    dy2, dw2 = api.moe_unpermute_backward(off(t["x"]), off(t["y"]), dev(bad), t["w"], dy_perm=filled((T * k, H), torch.float32))
    assert torch.equal(dy, dy2) and torch.allclose(dw, dw2, rtol=0, atol=(H + 8) * 2 * ref.U32 * H)
    assert torch.equal(api.moe_permute_rows_backward(off(t["y"]), dev(bad)), api.moe_permute_rows_backward(t["y"], dev(row)))


def test_nothing_to_do():
    import torch

    from paper_2512_09277_amd import api

    e = torch.empty((0, 16), device="cuda")
    r = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    assert api.moe_permute_rows(e, r).shape == (0, 16) and api.moe_permute_rows_backward(e, r).shape == (0, 16)
    dy, dw = api.moe_unpermute_backward(e, e, r, torch.empty((0, 2), device="cuda"))
    assert dy.shape == (0, 16) and dw.shape == (0, 2)
    row, n, t = inputs(6, 2, 16, "f32", 3, absent=2.0)              # no pair here at all
    dx = api.moe_permute_rows_backward(t["y"], dev(row), dx=filled((6, 16), torch.float32))
    dy, dw = api.moe_unpermute_backward(t["x"], t["y"], dev(row), t["w"], dy_perm=filled((12, 16), torch.float32))
    assert n == 0 and not dx.any() and not dw.any() and (dy == -7).all()


def test_non_finite_rows_stay_where_they_are():
    import torch

    from paper_2512_09277_amd import api

    T, k, H = 8, 2, 32
    row, n, t = inputs(T, k, H, "bf16", 9, absent=0.0)
    t["y"][row[2, 1]] = float("inf")
    t["y"][row[3, 0], 5] = float("nan")
    dy, dw = api.moe_unpermute_backward(t["x"], t["y"], dev(row), t["w"], dy_perm=torch.zeros_like(t["y"]))
    assert torch.isfinite(dy.float()).all() and not torch.isfinite(dw[2, 1]) and torch.isnan(dw[3, 0]) and int((~torch.isfinite(dw)).sum()) == 2
    dx = api.moe_permute_rows_backward(t["y"], dev(row))
    bad = ~torch.isfinite(dx.float())
    assert bad[2].all() and bad[3, 5] and int(bad.sum()) == H + 1
