"""Sorted rows and their gradients on rows of 2^31 - 1 elements, the longest that the calls take: the elements behind the last whole vector
are those of the row, and nothing is read or written past it."""
import pytest

pytestmark = pytest.mark.gpu

H = (1 << 31) - 1


@pytest.fixture()
def row():
    """[1, H] of bf16 with memory behind it, (the row, all of the memory)."""
    import torch

    memory = torch.full((H + 513,), 1.5, dtype=torch.bfloat16, device="cuda")
    memory[:H].view(torch.int16).random_(1 << 10, 1 << 14)          # normal values below 2
    yield memory[:H].view(1, H), memory
    del memory
    torch.cuda.empty_cache()


def guarded():
    import torch

    memory = torch.full((H + 513,), -7.0, dtype=torch.bfloat16, device="cuda")
    return memory[:H].view(1, H), memory


def test_sort_and_its_gradient(row):
    import torch

    from paper_2512_09277_amd import api

    x, _ = row
    here = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    for call in (api.moe_permute_rows, api.moe_permute_rows_backward):
        print(call.__name__, flush=True)
        y, memory = guarded()
        call(x, here, y)
        torch.cuda.synchronize()
        assert torch.equal(y, x) and (memory[H:] == -7).all()
        del y, memory


def test_gradient_of_the_combine(row):
    import torch

    from paper_2512_09277_amd import api

    g, _ = row
    here, half = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.full((1, 1), 0.5, device="cuda")
    y = torch.zeros((1, H), dtype=torch.bfloat16, device="cuda")
    y[0, [0, H - 9, H - 7, H - 1]] = 1
    dy, memory = guarded()
    _, dw = api.moe_unpermute_backward(g, y, here, half, dy_perm=dy)
    torch.cuda.synchronize()
    want = g[0, [0, H - 9, H - 7, H - 1]].double().sum()
    assert abs(dw.double() - want) <= 4 * 2.0 ** -24 * want
    assert torch.equal(dy, g * 0.5) and (memory[H:] == -7).all()


def test_combine(row):
    """Rows that are no whole vectors are combined element by element."""
    import torch

    from paper_2512_09277_amd import api

    y, _ = row
    here, half = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.full((1, 1), 0.5, device="cuda")
    out, memory = guarded()
    api.moe_unpermute(y, here, half, out)
    torch.cuda.synchronize()
    assert torch.equal(out, y * 0.5) and (memory[H:] == -7).all()
