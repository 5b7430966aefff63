"""What the calls for sorted rows, their gradients and 8-bit experts refuse, without a GPU: the C ABI returns before any launch, the
binding raises."""
import ctypes

import numpy as np
import pytest
import torch

from test_abi import lib  # noqa: F401  (the built library)

import fp8_reference as ref  # beside this file

P, ODD, NONE = ctypes.c_void_p(4096), ctypes.c_void_p(4100), None      # never dereferenced: the checks fail first


def refusals(fn, good, wrong):
    """Every (position, value, status) of `wrong` in turn in place of the good argument."""
    for at, value, status in wrong:
        args = list(good)
        args[at] = value
        assert fn(*args) == status, (fn.__name__, at, value)


def test_sorted_rows(lib):  # noqa: F811
    for fn in (lib.moe_permute_rows, lib.moe_permute_rows_backward):
        refusals(fn, [P, P, 4, 2, 64, 1, P, NONE], [(0, NONE, -1), (1, NONE, -1), (2, -1, -1), (3, 0, -1), (4, 0, -1), (5, 2, -2), (5, -1, -2),
                                                    (6, NONE, -1), (2, 1 << 23, -2)])
    assert lib.moe_permute_rows(P, P, 0, 2, 64, 1, P, NONE) == 0
    assert lib.moe_permute_rows_backward(P, P, 0, 2, 64, 1, P, NONE) == 0
    refusals(lib.moe_unpermute_backward, [P, P, P, P, 4, 2, 64, 0, P, P, NONE],
             [(i, NONE, -1) for i in (0, 1, 2, 3, 8, 9)] + [(4, -1, -1), (5, 0, -1), (6, 0, -1), (7, 7, -2), (4, 1 << 23, -2)])
    assert lib.moe_unpermute_backward(P, P, P, P, 0, 2, 64, 0, P, P, NONE) == 0


def test_quantize(lib):  # noqa: F811
    refusals(lib.moe_quantize_fp8, [P, 200, 4, 200, 1, NONE, P, 208, P, NONE],
             [(0, NONE, -1), (1, 199, -1), (2, -1, -1), (3, 0, -1), (4, 3, -2), (6, NONE, -1), (6, ODD, -1), (7, 192, -1), (7, 201, -1), (8, NONE, -1),
              (3, (1 << 30) + 1, -2)])
    assert lib.moe_quantize_fp8(P, 200, 0, 200, 1, NONE, P, 208, P, NONE) == 0
    refusals(lib.moe_quantize_weights_fp8, [P, 200, 2, 50, 200, 0, P, 208, P, NONE],
             [(0, NONE, -1), (1, 199, -1), (2, -1, -1), (3, 0, -1), (4, 0, -1), (5, 3, -2), (6, NONE, -1), (6, ODD, -1), (7, 192, -1), (7, 201, -1),
              (8, NONE, -1), (2, 1 << 23, -2), (3, (1 << 31) - 1, -2), (4, (1 << 31) - 1, -2)])
    assert lib.moe_quantize_weights_fp8(P, 200, 0, 50, 200, 0, P, 208, P, NONE) == 0


def test_products(lib):  # noqa: F811
    good = [P, 208, P, P, P, 4, 2, 3, 200, 72, P, 208, P, 1, P, NONE]
    refusals(lib.moe_grouped_mm_fp8, good,
             [(i, NONE, -1) for i in (0, 2, 4, 10, 12, 14)] + [(i, ODD, -1) for i in (0, 10, 14)] +
             [(1, 192, -1), (1, 201, -1), (5, -1, -1), (6, 0, -1), (7, 0, -1), (7, 65, -2), (8, 0, -1), (8, (1 << 20) + 16, -2), (9, 0, -1),
              (9, (1 << 20) + 1, -2), (11, 192, -1), (11, 204, -1), (11, 1 << 29, -1), (13, 2, -2), (5, 1 << 23, -2)])
    good[5] = 0
    assert lib.moe_grouped_mm_fp8(*good) == 0
    need = lib.moe_grouped_ffn_fp8_workspace_bytes(4, 2, 3, 200, 72)
    assert need >= 4 * 2 * 72 * 4
    good = [P, 208, P, P, P, 4, 2, 3, 200, 72, P, 208, P, P, 80, P, 1, P, P, need, NONE]
    refusals(lib.moe_grouped_ffn_fp8, good,
             [(i, NONE, -1) for i in (0, 2, 3, 4, 10, 12, 13, 15, 17, 18)] + [(i, ODD, -1) for i in (0, 10, 13, 17)] +
             [(1, 192, -1), (5, -1, -1), (6, 0, -1), (7, 0, -1), (7, 65, -2), (8, 0, -1), (9, 0, -1), (9, (1 << 20) + 1, -2), (11, 204, -1),
              (14, 72, -1), (16, 5, -2), (18, ctypes.c_void_p(4096 + 16), -1), (19, need - 1, -3), (5, 1 << 23, -2)])
    good[5] = 0
    assert lib.moe_grouped_ffn_fp8(*good) == 0


def test_workspace_query(lib):  # noqa: F811
    """Plain host arithmetic; the figure for a batch is enough for every smaller one."""
    q = lib.moe_grouped_ffn_fp8_workspace_bytes
    assert q(-1, 2, 3, 256, 128) == 0 and q(4, 0, 3, 256, 128) == 0 and q(4, 2, 3, 256, 0) == 0
    for spr, H, I, k in ((18, 2048, 768, 8), (36, 7168, 2048, 8), (5, 200, 72, 2), (64, 96, 2000, 1)):
        need = [q(T, k, spr, H, I) for T in range(0, 9000, 7)]
        assert need == sorted(need) and need[0] >= 0


def test_binding_refuses_host_tensors_and_wrong_shapes(lib):  # noqa: F811
    from paper_2512_09277_amd import api

    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    f8 = lambda *s: torch.zeros(s, dtype=torch.uint8).view(api.FP8)  # noqa: E731
    x, row = torch.zeros(4, 64), i32(4, 2)
    wrong = [
        lambda: api.moe_permute_rows(x, row), lambda: api.moe_permute_rows_backward(torch.zeros(8, 64), row),
        lambda: api.moe_unpermute_backward(x, torch.zeros(8, 64), row, torch.zeros(4, 2)), lambda: api.moe_quantize_fp8(x),
        lambda: api.moe_quantize_weights_fp8(torch.zeros(2, 4, 64)),
        lambda: api.moe_grouped_mm_fp8(f8(4, 64), torch.zeros(4, 1), i32(3), f8(2, 16, 64), torch.zeros(2, 1, 1)),
        lambda: api.moe_grouped_ffn_fp8(f8(4, 64), torch.zeros(4, 1), i32(8), i32(3), 2, f8(2, 32, 64), torch.zeros(2, 2, 1), f8(2, 64, 16),
                                        torch.zeros(2, 1, 1), ws=torch.zeros(1 << 16, dtype=torch.uint8)),
    ]
    for call in wrong:
        with pytest.raises(TypeError, match="device tensor"):
            call()
    for call in (lambda: api.moe_permute_rows(x, i32(5, 2)), lambda: api.moe_permute_rows_backward(torch.zeros(7, 64), row),
                 lambda: api.moe_permute_rows(x.half(), row),
                 lambda: api.moe_grouped_mm_fp8(f8(4, 64), torch.zeros(4, 1), i32(3), f8(2, 16, 64), torch.zeros(2, 1, 1), k=2)):
        with pytest.raises((ValueError, TypeError)):
            call()


def test_the_reference_rounding():
    """e4m3 of the reference against torch's conversion on the host, over every border between two values."""
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    every = np.unique(every[np.isfinite(every)])
    assert every.max() == 448
    mid = (every[1:] + every[:-1]) / 2
    x = np.concatenate([every, mid, np.nextafter(mid.astype(np.float32), np.float32(-1e9)), np.nextafter(mid.astype(np.float32), np.float32(1e9))])
    assert np.array_equal(ref.e4m3(x), torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).float().numpy())
