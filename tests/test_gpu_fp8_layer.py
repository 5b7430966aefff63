"""The operators together, as a serving step and a training step use them, and the ways they are called: captured graphs, side streams,
the native and the Python marshalling."""
import numpy as np
import pytest

import fp8_reference as ref
from paper_2512_09277_amd import workloads as W
from test_gpu_fp8 import dev, e4m3_rows, ffn_case, wide

pytestmark = pytest.mark.gpu

T, K, N, G, SPR, H, I = 24, 2, 16, 4, 5, 256, 128


def experts(rng):
    w13, s13 = ref.quantize32((0.1 * rng.standard_normal((N, 2, I, H))).astype(np.float32), 128)
    w2, s2 = ref.quantize32((0.1 * rng.standard_normal((N, H, I))).astype(np.float32), 128)
    return w13.reshape(N, 2 * I, H), s13.reshape(N, -1, s13.shape[-1]), w2, s2


def placed(a, s2e, rank):
    return a[np.maximum(s2e[rank * SPR:(rank + 1) * SPR], 0)]


def serving_step(api, st, rank):
    gate = api.moe_gate_topk(st["x"], st["wg"], K, out=st["gate"], ws=st["gws"], n_valid=st["n_valid"])
    _, lists = api.metro_route_permute(gate["topk_ids"], st["s2e"], N, G, SPR, rank, out=st["routing"], lists=st["lists"])
    q = api.moe_quantize_fp8(st["x"], n_rows=st["n_valid"], out=st["q"])
    y = api.moe_grouped_ffn_fp8(q["q"], q["scale"], lists["perm_pair"], lists["group_offsets"], K, *st["experts"], y_perm=st["y"], ws=st["ws"])
    return api.moe_unpermute(y, lists["pair_row"], gate["topk_w"], out=st["out"])


def serving_state(api, rng, rank, w):
    import torch

    p = W.popularity(N, 1.0, 1)
    s2e = W.placement(p, G, SPR)
    w13, s13, w2, s2 = (placed(a, s2e, rank) for a in w)
    e = lambda *s, **kw: torch.empty(s, device="cuda", **kw)  # noqa: E731
    return dict(x=e(T, H, dtype=torch.bfloat16), wg=dev(W.gate_weights(N, H, 2, "f32")).bfloat16(), s2e=dev(s2e), n_valid=dev(np.array([T], np.int32)),
                gate=dict(topk_ids=e(T, K, dtype=torch.int32), topk_w=e(T, K), expert_count=e(N, dtype=torch.int32)),
                gws=e(1 << 20, dtype=torch.uint8), routing=api.route_buffers(1, T, K, N, G, "cuda"), lists=api.permute_buffers(T, K, SPR, "cuda"),
                q=api.quantize_buffers(T, H, "cuda"), y=e(T * K, H, dtype=torch.bfloat16), out=e(T, H, dtype=torch.bfloat16),
                ws=e(api.moe_grouped_ffn_fp8_workspace_bytes(T, K, SPR, H, I), dtype=torch.uint8),
                experts=(e4m3_rows(w13), dev(s13), e4m3_rows(w2), dev(s2)), host=(ref.values(w13, s13, 128), ref.values(w2, s2, 128), s2e))


def expected(st, x, n, rank):
    """out [n, H] of this rank and how far it may be off, from the kernels' own ids and weights."""
    v13, v2, s2e = st["host"]
    ids, tw, slot = (st["gate"][m].cpu().numpy() for m in ("topk_ids", "topk_w")) if False else \
        (st["gate"]["topk_ids"].cpu().numpy(), wide(st["gate"]["topk_w"]), st["routing"]["pair_slot"][0].cpu().numpy())
    xv = ref.values(*ref.quantize32(x))
    out, err = np.zeros((n, H)), np.zeros((n, H))
    for t in range(n):
        for j in range(K):
            l = slot[t, j] - rank * SPR
            if 0 <= l < SPR:
                assert s2e[slot[t, j]] == ids[t, j]
                y, e = ref.ffn(xv[t:t + 1], v13[l], v2[l])
                out[t] += tw[t, j] * y[0]
                err[t] += tw[t, j] * ref.rounded(y, e, True)[0]
    return out, ref.rounded(out, err + K * ref.U32 * np.abs(out), True)


def test_serving_step_captured_and_replayed():
    """gate, routing, quantization, FFN and combine in one graph, on other inputs and numbers of real tokens each time."""
    import torch

    from paper_2512_09277_amd import api

    rng = np.random.default_rng(11)
    rank, w = 1, experts(rng)
    st = serving_state(api, rng, rank, w)
    st["x"].normal_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serving_step(api, st, rank)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        serving_step(api, st, rank)
    for n in (T, 5, 17, 1, T):
        x = rng.standard_normal((T, H)).astype(np.float32)
        st["x"].copy_(dev(x))
        st["n_valid"].fill_(n)
        graph.replay()
        torch.cuda.synchronize()
        got = wide(st["out"])
        want, err = expected(st, wide(st["x"]), n, rank)
        assert (np.abs(got[:n] - want) <= err).all() and not got[n:].any()
        replayed = st["out"].clone()
        st["out"].fill_(-7)
        serving_step(api, st, rank)
        assert torch.equal(st["out"], replayed)


def test_two_graphs_share_a_workspace():
    """Two captured layers on one workspace, replayed one after the other on one stream."""
    import torch

    from paper_2512_09277_amd import api

    calls = [ffn_case(30, 2, 256, 128, [17, 3, 0, 35], "bf16", seed=s)[0] for s in (1, 2)]
    ws = torch.empty(api.moe_grouped_ffn_fp8_workspace_bytes(30, 2, 4, 256, 128), dtype=torch.uint8, device="cuda")
    want = [api.moe_grouped_ffn_fp8(**c).clone() for c in calls]
    graphs = []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            api.moe_grouped_ffn_fp8(**c, ws=ws)
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 1)):
        for c in calls:
            c["y_perm"].fill_(-7)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(c["y_perm"], w) for c, w in zip(calls, want))


def test_on_a_side_stream():
    import torch

    from paper_2512_09277_amd import api

    args, *_ = ffn_case(30, 2, 256, 128, [17, 3, 0, 35], "bf16")
    want = api.moe_grouped_ffn_fp8(**args).clone()
    x = torch.randn((64, 256), device="cuda")
    q = api.moe_quantize_fp8(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        args["y_perm"].fill_(-7)
        got = api.moe_grouped_ffn_fp8(**args)
        q2 = api.moe_quantize_fp8(x)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(q["q"].view(torch.uint8), q2["q"].view(torch.uint8)) and torch.equal(q["scale"], q2["scale"])


def training_step(api, x, pair_row, lists, tw, w13, s13, w2, s2, dout):
    """Forward and backward of the layer around fixed 8-bit experts, in the framework's calls and torch's elementwise ones:
    (out, dx, dtopk_w)."""
    import torch

    off = lists["group_offsets"]
    quant = lambda t: api.moe_quantize_fp8(t, n_rows=lists["n_pairs"])  # noqa: E731
    mm = lambda t, w, s: api.moe_grouped_mm_fp8(t["q"], t["scale"], off, w, s, dtype=torch.float32)  # noqa: E731
    n = off[-1]
    inside = (torch.arange(T * K, device="cuda") < n).unsqueeze(1)
    x_perm = api.moe_permute_rows(x, pair_row, x_perm=torch.zeros((T * K, H), dtype=x.dtype, device="cuda"))
    h = mm(quant(x_perm), w13, s13)
    gate, up = h[:, :I], h[:, I:]
    sig = torch.sigmoid(gate)
    act = torch.where(inside, gate * sig * up, 0.0)
    y = torch.where(inside, mm(quant(act), w2, s2), 0.0)
    out = api.moe_unpermute(y, pair_row, tw)
    dy, dw = api.moe_unpermute_backward(dout, y, pair_row, tw, dy_perm=torch.zeros_like(y))
    turned = lambda w, s: (e4m3_rows(wide(w).transpose(0, 2, 1)), s.transpose(1, 2).contiguous())  # noqa: E731
    da = mm(quant(dy), *turned(w2, s2))
    dgate, dup = da * up * (sig * (1 + gate * (1 - sig))), da * gate * sig
    dh = torch.where(inside, torch.cat([dgate, dup], dim=1), 0.0)
    dx_perm = mm(quant(dh), *turned(w13, s13))
    return out, api.moe_permute_rows_backward(dx_perm, pair_row), dw


def test_training_step():
    """Against the formulas in 64 bits with the same quantizations.  fp32 sums of a few hundred terms are off by about 1e-6, which moves
    about one value in 10^4 over an e4m3 border, by 2^-3 of itself: sqrt(1e-4) * 2^-3 = 1.3e-3 of the norm for each of the four
    quantizations in a chain, 5e-3 together."""
    import torch

    from paper_2512_09277_amd import api

    rng = np.random.default_rng(21)
    rank = 2
    p = W.popularity(N, 0.6, 1)
    s2e, ids = W.placement(p, G, SPR), W.topk_trace(p, T, K, 3)
    w13, s13, w2, s2 = (placed(a, s2e, rank) for a in experts(rng))
    _, lists = api.metro_route_permute(dev(ids), dev(s2e), N, G, SPR, rank)
    x, dout = rng.standard_normal((2, T, H)).astype(np.float32)
    tw = rng.random((T, K)).astype(np.float32)
    got = training_step(api, dev(x), lists["pair_row"], lists, dev(tw), e4m3_rows(w13), dev(s13), e4m3_rows(w2), dev(s2), dev(dout))
    v13, v2 = ref.values(w13, s13, 128), ref.values(w2, s2, 128)
    row = lists["pair_row"].cpu().numpy()
    off = lists["group_offsets"].cpu().numpy()
    assert off[-1] > 8
    out, dx, dw = np.zeros((T, H)), np.zeros((T, H)), np.zeros((T, K))

    def q64(a):
        m = np.maximum(ref.block_max(a), 1e-30)
        s = ref.spread(m / 448, *a.shape)
        return ref.e4m3(a / s) * s

    for t in range(T):
        for j in range(K):
            if row[t, j] < 0:
                continue
            l = int(np.searchsorted(off[1:], row[t, j], side="right"))
            g, u = np.split(q64(x[t:t + 1].astype(np.float64)) @ v13[l].T, 2, axis=1)
            sig = 1 / (1 + np.exp(-g))
            y = q64(g * sig * u) @ v2[l].T
            out[t] += tw[t, j] * y[0]
            dw[t, j] = dout[t].astype(np.float64) @ y[0]
            da = q64(tw[t, j].astype(np.float64) * dout[t:t + 1]) @ v2[l]
            dh = np.concatenate([da * u * (sig * (1 + g * (1 - sig))), da * g * sig], axis=1)
            dx[t] += (q64(dh) @ v13[l])[0]
    for a, b in zip(got, (out, dx, dw)):
        assert np.linalg.norm(wide(a) - b) <= 5e-3 * np.linalg.norm(b)
    assert (wide(got[2])[row < 0] == 0).all()


# ------------------------------------------------------------------------------------------ marshalling
class OnlyPython:
    """Stands in for the native module: nothing is its plain case."""

    def __getattr__(self, name):
        return lambda *a: 1


def forms():
    """name -> (call, arguments by name); arguments are then replaced one at a time."""
    import torch

    from paper_2512_09277_amd import api

    f, *_ = ffn_case(12, 2, 128, 128, [7, 0, 9], "bf16")
    f["ws"] = torch.zeros(api.moe_grouped_ffn_fp8_workspace_bytes(12, 2, 3, 128, 128), dtype=torch.uint8, device="cuda")
    rnd = lambda *s: torch.randn(s, generator=torch.Generator().manual_seed(1)).cuda()  # noqa: E731
    row = torch.full((12, 2), -1, dtype=torch.int32)
    row.view(-1)[f["perm_pair"].cpu()[:16].long()] = torch.arange(16, dtype=torch.int32)
    m = dict(x=f["x"], xs=f["xs"], group_offsets=f["group_offsets"], w=f["w13"][:, :128].contiguous(), ws=f["s13"][:, :1].contiguous(),
             y=torch.zeros((24, 128), device="cuda"), perm_pair=f["perm_pair"], k=2)
    qb = {n: t.zero_() if n == "scale" else t for n, t in api.quantize_buffers(12, 200, "cuda").items()}
    qb["q"].view(torch.uint8).zero_()
    return {
        "ffn": (api.moe_grouped_ffn_fp8, f),
        "mm": (api.moe_grouped_mm_fp8, m),
        "quantize": (api.moe_quantize_fp8, dict(x=rnd(12, 200), n_rows=dev(np.array([9], np.int32)), out=qb)),
        "rows": (api.moe_permute_rows, dict(x=rnd(12, 64), pair_row=row.cuda(), x_perm=torch.zeros((24, 64), device="cuda"))),
        "rows_grad": (api.moe_permute_rows_backward, dict(dx_perm=rnd(24, 64), pair_row=row.cuda(), dx=torch.zeros((12, 64), device="cuda"))),
        "combine_grad": (api.moe_unpermute_backward, dict(dout=rnd(12, 64), y_perm=rnd(24, 64), pair_row=row.cuda(), topk_w=rnd(12, 2),
                                                          dy_perm=torch.zeros((24, 64), device="cuda"), dtopk_w=torch.zeros((12, 2), device="cuda"))),
    }


def outcome(call, args):
    import torch

    try:
        r = call(**args)
        torch.cuda.synchronize()
    except Exception as e:
        return type(e).__name__, str(e)
    r = [r[n] for n in sorted(r)] if isinstance(r, dict) else list(r) if isinstance(r, tuple) else [r]
    return [t.cpu().float() for t in r]


def same(a, b):
    import torch

    return a == b if isinstance(a, tuple) or isinstance(b, tuple) else len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("name", ["ffn", "mm", "quantize", "rows", "rows_grad", "combine_grad"])
def test_native_and_python_marshalling_agree(monkeypatch, name):
    """Every tensor in turn on the host, of another type, one row short, transposed, missing; and the plain call."""
    import torch

    from paper_2512_09277_amd import api

    call, good = forms()[name]
    swaps = [{}]
    for n, v in good.items():
        if isinstance(v, torch.Tensor):
            swaps += [{n: v.cpu()}, {n: v.to(torch.float64) if v.dtype != api.FP8 else v.view(torch.uint8)}, {n: v[:-1]}]
            if v.dim() == 2:
                swaps.append({n: v.t()})
        elif isinstance(v, dict):
            swaps += [{n: {**v, m: v[m][:-1]}} for m in v] + [{n: {**v, m: v[m].cpu()}} for m in v]
        else:
            swaps += [{n: 0}, {n: v + 1}]
    natively = 0
    for swap in swaps:
        native = outcome(call, {**good, **swap})
        with monkeypatch.context() as m:
            m.setattr(api, "_native", OnlyPython())
            python = outcome(call, {**good, **swap})
        assert same(native, python), (name, list(swap), native, python)
        natively += not isinstance(native, tuple)
    assert natively >= 1
