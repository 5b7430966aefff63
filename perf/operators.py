"""Operators of a mixture-of-experts layer in 8-bit floating point and in training, and what they are measured on.

  quantize       rows of activations (or of a gradient) to e4m3 with a scale for each 128 values of a row
  quantize_w     expert weights to e4m3 with a scale for each block of 128 x 128
  mm             product of rows sorted by expert with their expert's e4m3 weights, both with a scale for each block of 128
  ffn            the SwiGLU experts on e4m3 weights over one rank's token lists, the activation between the products requantized
  rows           tokens sorted by expert: the row of every (token, expert) pair on this rank
  rows_grad      its gradient: the rows of a token added up
  combine_grad   the gradient of the weighted sum of a token's rows: of the rows and of the weights

`own` False: plain definitions in elementary torch operations, 32 bits whatever the storage.  `own` True: the package's calls.
Expert popularity is skewed (Zipf), tokens choose distinct experts; a rank holds some of the experts.
"""
import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda"
BLOCK = 128
E4M3_MAX = 448.0
SMALLEST = 1e-30                                      # a block's largest magnitude counts as at least this
F8 = torch.float8_e4m3fn
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _experts(N, k, spr, T, s):
    return dict(N=N, k=k, spr=spr, T=T, s=s)


_30B = dict(N=128, k=8, spr=18)                       # the shapes of the package's workloads: experts, top-k, experts of a rank
_235B = dict(N=128, k=8, spr=18)
_DSV3 = dict(N=256, k=8, spr=36)


def listed():
    return [
        # activations of a decode batch on their way to the experts: launch latency
        dict(name="quantize_t64", kind="quantize", dtype="bf16", rows=64, valid=64, K=7168),
        # one layer's experts of a rank after a weight update (or once, when a 16-bit checkpoint is loaded)
        dict(name="quantize_w_30b", kind="quantize_w", dtype="bf16", slots=18, rows=1536, K=2048),
        # a few sorted rows against eight experts: a small decode batch, bound by latency and the weights
        dict(name="mm_few_rows", kind="mm", out="bf16", groups=8, rows=24, s=0.8, K=2048, N=4096),
        # a training or prefill batch: thousands of rows an expert, bound by the matrix cores
        dict(name="mm_many_rows", kind="mm", out="bf16", groups=16, rows=16384, s=0.6, K=4096, N=4096),
        # sizes that fit no tile or block, fp32 result
        dict(name="mm_ragged_f32", kind="mm", out="f32", groups=5, rows=301, s=1.0, K=1336, N=1000),
        # interactive serving: eight tokens in flight, a few rows per activated expert
        dict(_30B, name="ffn_30b_t8", kind="ffn", out="bf16", T=8, s=0.8, H=2048, I=768),
        # the ordinary decode batch of the largest shape: weights stream from HBM
        dict(_DSV3, name="ffn_dsv3_t1024", kind="ffn", out="bf16", T=1024, s=1.0, H=7168, I=2048),
        # a prefill chunk, not a power of two
        dict(_30B, name="ffn_30b_t4000", kind="ffn", out="bf16", T=4000, s=0.8, H=2048, I=768),
        # training, one rank of eight: the forward sort of a batch
        dict(_DSV3, name="rows_dsv3_t4096", kind="rows", dtype="bf16", T=4096, s=1.0, H=7168),
        # its gradient in fp32 at odd sizes
        dict(name="rows_grad_f32_t1500", kind="rows_grad", dtype="f32", H=2000, **_experts(64, 6, 16, 1500, 0.8)),
        # every expert on one GPU, a training batch: the gradient of the combine
        dict(name="combine_grad_t8192", kind="combine_grad", dtype="bf16", H=2048, **_experts(64, 8, 64, 8192, 0.6)),
        # a test-sized layer: launch latency
        dict(name="combine_grad_f32_t33", kind="combine_grad", dtype="f32", H=1000, **_experts(16, 2, 16, 33, 1.0)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    what = rng.choice(["quantize", "quantize_w", "mm", "mm", "ffn", "ffn", "ffn", "rows", "rows_grad", "combine_grad"])
    s = round(rng.uniform(0.5, 1.3), 2)
    dtype = rng.choice(["bf16", "f32"])
    if what == "quantize":
        rows = _log_int(rng, 1, 16384)
        K = rng.choice([2048, 4096, 7168, _log_int(rng, 64, 7168)])
        return dict(kind=what, dtype=dtype, rows=rows, valid=rows - rng.choice([0, rng.randint(0, rows - 1)]), K=K)
    if what == "quantize_w":
        rows, K = rng.choice([(1536, 2048), (4096, 7168), (7168, 2048), (_log_int(rng, 64, 4096), _log_int(rng, 64, 4096))])
        return dict(kind=what, dtype=dtype, slots=rng.randint(1, 12), rows=rows, K=K)
    if what == "mm":
        K, N = (rng.choice([2048, 4096, 7168, _log_int(rng, 64, 7168)]) for _ in range(2))
        groups = max(1, min(_log_int(rng, 1, 36), int(6e8 / (K * N))))
        rows = max(1, min(_log_int(rng, 1, 16384), int(2.7e11 / (K * N))))
        return dict(kind=what, out=rng.choice(["bf16", "f32"]), groups=groups, rows=rows, s=min(s, 1.0), K=K, N=N)
    if what == "ffn":
        if rng.random() < 0.75:                       # a model's layer, any batch it is served at
            shape, H, I, most = rng.choice([(_30B, 2048, 768, 4096), (_235B, 4096, 1536, 1024), (_DSV3, 7168, 2048, 1024)])
            return dict(shape, kind=what, out="bf16", T=_log_int(rng, 1, most), s=s, H=H, I=I)
        return dict(kind=what, out="bf16", H=_log_int(rng, 64, 2048), I=_log_int(rng, 64, 768),
                    **_experts(32, 4, 16, _log_int(rng, 1, 256), s))
    N, k, spr = rng.choice([(256, 8, 36), (128, 8, 18), (64, 6, 64), (16, 2, 16), (32, 12, 8)])
    H = rng.choice([2048, 4096, 7168, _log_int(rng, 64, 7168)])
    most = max(64, min(8192, int(1.3e8 * N / (k * spr * H))))
    return dict(kind=what, dtype=dtype, H=H, **_experts(N, k, spr, _log_int(rng, 1, most), s))


# ------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) % (1 << 62))
    return g


def _popularity(n, s, rng):
    p = 1.0 / np.power(rng.permutation(n) + 1.0, s)
    return p / p.sum()


def _lists(case, seed):
    """(group_offsets, perm_pair, pair_row) of one rank that holds experts 0 .. spr - 1: pairs by expert, then by token."""
    N, k, spr, T = (case[n] for n in ("N", "k", "spr", "T"))
    rng = np.random.default_rng(int(seed) % (1 << 62))
    key = rng.exponential(size=(T, N)) / _popularity(N, case["s"], rng)
    flat = np.argsort(key, axis=1, kind="stable")[:, :k].reshape(-1)
    here = np.flatnonzero(flat < spr)
    order = here[np.argsort(flat[here], kind="stable")]
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[here], minlength=spr))]).astype(np.int32)
    perm = np.full(T * k, -1, np.int32)
    perm[:order.size] = order
    row = np.full(T * k, -1, np.int32)
    row[order] = np.arange(order.size)
    return offsets, perm, row.reshape(T, k)


def _groups(case, seed):
    """group_offsets of rows that were sorted by expert."""
    rng = np.random.default_rng(int(seed) % (1 << 62))
    count = rng.multinomial(case["rows"], _popularity(case["groups"], case["s"], rng))
    return np.concatenate([[0], np.cumsum(count)]).astype(np.int32)


def _up(n, to):
    return (n + to - 1) // to * to


def _pitch(K):
    """Bytes between the rows of e4m3 weights, as the package recommends: a multiple of 16, rows not a multiple of 4096 apart."""
    return K + 128 if K % 4096 == 0 else _up(K, 16)


def _padded(rows, K, pitch, lead=()):
    """An e4m3 matrix whose rows are `pitch` bytes apart."""
    return torch.zeros((*lead, rows, pitch), dtype=torch.uint8, device=DEV).view(F8)[..., :K]


def _scale_of(largest):
    return torch.div(largest, torch.full((), E4M3_MAX, dtype=largest.dtype, device=largest.device))


def _inverse(largest):
    return torch.div(torch.full((), E4M3_MAX, dtype=largest.dtype, device=largest.device), largest)


def _plain_quantize(x):
    """x [R, K] in fp32 -> e4m3 values and a scale for each 128 of a row."""
    R, K = x.shape
    b = torch.nn.functional.pad(x, (0, _up(K, BLOCK) - K)).reshape(R, -1, BLOCK)
    largest = b.abs().amax(dim=2).clamp(min=SMALLEST)
    q = (b * _inverse(largest).unsqueeze(2)).to(F8)
    return q.reshape(R, -1)[:, :K], _scale_of(largest)


def _plain_quantize_weights(w):
    """w [slots, R, K] in fp32 -> e4m3 values and a scale for each 128 x 128."""
    S, R, K = w.shape
    b = torch.nn.functional.pad(w, (0, _up(K, BLOCK) - K, 0, _up(R, BLOCK) - R)).reshape(S, _up(R, BLOCK) // BLOCK, BLOCK, -1, BLOCK)
    largest = b.abs().amax(dim=(2, 4)).clamp(min=SMALLEST)
    q = (b * _inverse(largest)[:, :, None, :, None]).to(F8)
    return q.reshape(S, _up(R, BLOCK), -1)[:, :R, :K], _scale_of(largest)


def _expert_weights(gen, slots, halves, rows, K):
    """e4m3 weights [slots, halves * rows, K] from N(0, 0.02), each half with blocks of its own; scales."""
    out = _padded(halves * rows, K, _pitch(K), (slots,))
    scale = torch.empty((slots, halves * _up(rows, BLOCK) // BLOCK, _up(K, BLOCK) // BLOCK), device=DEV)
    for l in range(slots):                            # per expert: the fp32 staging stays small
        q, sc = _plain_quantize_weights(0.02 * torch.randn((halves, rows, K), generator=gen, device=DEV))
        out[l] = q.reshape(halves * rows, K)
        scale[l] = sc.reshape(scale.shape[1:])
    return out, scale


def _rows_e4m3(gen, rows, K):
    q = _padded(rows, K, _up(K, 16))
    v, scale = _plain_quantize(torch.randn((rows, K), generator=gen, device=DEV).to(torch.bfloat16).float())
    q.copy_(v)
    return q, scale


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def prepare(case, seed):
    g = _generator(seed)
    c = case
    st = dict(case=c)
    rnd = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    if c["kind"] == "quantize":
        st["x"] = rnd(c["rows"], c["K"]).to(_TYPES[c["dtype"]])
        # one channel in a few hundred is much larger, as activations have them
        st["x"][:, torch.randint(0, c["K"], (1 + c["K"] // 500,), generator=g, device=DEV)] *= 20
        st["n_rows"] = _i32(np.array([c["valid"]], np.int32))
        st["out"] = dict(q=_padded(c["rows"], c["K"], _up(c["K"], 16)), scale=torch.zeros((c["rows"], _up(c["K"], BLOCK) // BLOCK), device=DEV))
    elif c["kind"] == "quantize_w":
        st["w"] = (0.02 * rnd(c["slots"], c["rows"], c["K"])).to(_TYPES[c["dtype"]])
        st["out"] = dict(q=_padded(c["rows"], c["K"], _pitch(c["K"]), (c["slots"],)),
                         scale=torch.zeros((c["slots"], _up(c["rows"], BLOCK) // BLOCK, _up(c["K"], BLOCK) // BLOCK), device=DEV))
    elif c["kind"] == "mm":
        offsets = _groups(c, seed)
        st["most"] = int(np.diff(offsets).max())
        st["offsets"] = _i32(offsets)
        st["x"], st["xs"] = _rows_e4m3(g, c["rows"], c["K"])
        st["w"], st["ws"] = _expert_weights(g, c["groups"], 1, c["N"], c["K"])
        st["y"] = torch.zeros((c["rows"], c["N"]), dtype=_TYPES[c["out"]], device=DEV)
    else:
        T, k, H = c["T"], c["k"], c["H"]
        offsets, perm, row = _lists(c, seed)
        st.update(offsets=_i32(offsets), perm=_i32(perm), row=_i32(row))
        if c["kind"] == "ffn":
            st["most"] = int(np.diff(offsets).max())
            st["x"], st["xs"] = _rows_e4m3(g, T, H)
            st["w13"], st["s13"] = _expert_weights(g, c["spr"], 2, c["I"], H)
            st["w2"], st["s2"] = _expert_weights(g, c["spr"], 1, H, c["I"])
            st["y"] = torch.zeros((T * k, H), dtype=_TYPES[c["out"]], device=DEV)
            # between the two products: an fp32 activation of every pair, its e4m3 form and scales
            st["ws"] = torch.zeros((T * k * (5 * _up(c["I"], 16) + 4 * _up(c["I"], BLOCK) // BLOCK) + (1 << 20),), dtype=torch.uint8, device=DEV)
        else:
            dt = _TYPES[c["dtype"]]
            if c["kind"] == "rows":
                st["x"], st["out"] = rnd(T, H).to(dt), torch.zeros((T * k, H), dtype=dt, device=DEV)
            elif c["kind"] == "rows_grad":
                st["dx_perm"], st["out"] = rnd(T * k, H).to(dt), torch.zeros((T, H), dtype=dt, device=DEV)
            else:
                st["dout"], st["y"] = rnd(T, H).to(dt), rnd(T * k, H).to(dt)
                st["topk_w"] = torch.softmax(rnd(T, k), dim=1)
                st["dy"], st["dw"] = torch.zeros((T * k, H), dtype=dt, device=DEV), torch.zeros((T, k), device=DEV)
    return st


# ------------------------------------------------------------------------------------------ plain forms
def _blocks(v, scale, rows_a_block):
    """The values that e4m3 `v` [..., R, K] with `scale` stands for, in fp32."""
    R, K = v.shape[-2:]
    at = torch.arange(max(R, K), device=DEV)
    out = v.float()
    return out * (scale if rows_a_block == 1 else scale[..., at[:R] // rows_a_block, :])[..., at[:K] // BLOCK]


def _grouped(x, offsets, most):
    """Rows of every group, padded to the largest one with zeros: [groups, most, K]."""
    at = offsets[:-1, None].long() + torch.arange(most, device=DEV)
    inside = at < offsets[1:, None]
    return x[at.clamp(max=x.shape[0] - 1)] * inside.unsqueeze(2)


def _ungrouped(y, offsets, into):
    """The rows of _grouped back in order; rows behind the last group as they are in `into`."""
    at = torch.arange(into.shape[0], device=DEV)
    group = torch.searchsorted(offsets[1:].contiguous(), at, right=True).clamp(max=y.shape[0] - 1)
    rows = y[group, (at - offsets[group]).clamp(min=0, max=y.shape[1] - 1)]
    return torch.where((at < offsets[-1]).unsqueeze(1), rows.to(into.dtype), into)


def _products(x, w):
    """x [groups, rows, K], w [groups, N, K] -> [groups, rows, N]."""
    return torch.bmm(w, x.transpose(1, 2).contiguous()).transpose(1, 2).contiguous()


def _plain(st):
    c = st["case"]
    kind = c["kind"]
    if kind == "quantize":
        q, scale = _plain_quantize(st["x"].float())
        inside = (torch.arange(c["rows"], device=DEV) < st["n_rows"]).unsqueeze(1)
        return dict(q=torch.where(inside, q.float(), 0.0).to(F8), scale=torch.where(inside, scale, 0.0))
    if kind == "quantize_w":
        q, scale = _plain_quantize_weights(st["w"].float())
        return dict(q=q, scale=scale)
    if kind == "mm":
        x = _grouped(_blocks(st["x"], st["xs"], 1), st["offsets"], st["most"])
        return dict(y=_ungrouped(_products(x, _blocks(st["w"], st["ws"], BLOCK)), st["offsets"], st["y"]))
    if kind == "ffn":
        H, I, B = c["H"], c["I"], _up(c["I"], BLOCK) // BLOCK
        token = (st["perm"].clamp(min=0) // c["k"]).long()
        x = _grouped(_blocks(st["x"], st["xs"], 1)[token], st["offsets"], st["most"])
        w13, s13 = st["w13"], st["s13"]
        gate = _products(x, _blocks(w13[:, :I], s13[:, :B], BLOCK))
        up = _products(x, _blocks(w13[:, I:], s13[:, B:], BLOCK))
        act = (gate / (1 + torch.exp(-gate)) * up).reshape(-1, I)
        act = _blocks(*_plain_quantize(act), 1).reshape(gate.shape)
        return dict(y=_ungrouped(_products(act, _blocks(st["w2"], st["s2"], BLOCK)), st["offsets"], st["y"]))
    row = st["row"].long()
    here, at = (row >= 0).unsqueeze(2), row.clamp(min=0)
    if kind == "rows":
        token = (st["perm"].clamp(min=0) // c["k"]).long()
        inside = (torch.arange(token.numel(), device=DEV) < st["offsets"][-1]).unsqueeze(1)
        return dict(x_perm=torch.where(inside, st["x"][token], st["out"]))
    if kind == "rows_grad":
        return dict(dx=torch.where(here, st["dx_perm"][at].float(), 0.0).sum(dim=1).to(st["out"].dtype))
    pair = st["perm"].clamp(min=0).long()
    inside = (torch.arange(pair.numel(), device=DEV) < st["offsets"][-1]).unsqueeze(1)
    dout = st["dout"].float()
    dy = dout[pair // c["k"]] * st["topk_w"].reshape(-1)[pair].unsqueeze(1)
    dw = torch.where(here, st["y"][at].float() * dout.unsqueeze(1), 0.0).sum(dim=2)
    return dict(dy_perm=torch.where(inside, dy.to(st["dy"].dtype), st["dy"]), dtopk_w=dw)


def run(state):
    if not own:
        return _plain(state)
    from paper_2512_09277_amd import api

    st, c = state, state["case"]
    kind = c["kind"]
    if kind == "quantize":
        return api.moe_quantize_fp8(st["x"], n_rows=st["n_rows"], out=st["out"])
    if kind == "quantize_w":
        return api.moe_quantize_weights_fp8(st["w"], out=st["out"])
    if kind == "mm":
        return dict(y=api.moe_grouped_mm_fp8(st["x"], st["xs"], st["offsets"], st["w"], st["ws"], y=st["y"]))
    if kind == "ffn":
        return dict(y=api.moe_grouped_ffn_fp8(st["x"], st["xs"], st["perm"], st["offsets"], c["k"], st["w13"], st["s13"], st["w2"],
                                              st["s2"], y_perm=st["y"], ws=st["ws"]))
    if kind == "rows":
        return dict(x_perm=api.moe_permute_rows(st["x"], st["row"], x_perm=st["out"]))
    if kind == "rows_grad":
        return dict(dx=api.moe_permute_rows_backward(st["dx_perm"], st["row"], dx=st["out"]))
    dy, dw = api.moe_unpermute_backward(st["dout"], st["y"], st["row"], st["topk_w"], dy_perm=st["dy"], dtopk_w=st["dw"])
    return dict(dy_perm=dy, dtopk_w=dw)


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def _e4m3(v):
    """Nearest e4m3 value, ties to even, in 64 bits: three bits behind the leading one, steps no finer than 2^-9."""
    step = torch.ldexp(torch.ones_like(v), (torch.frexp(v).exponent - 4).clamp(min=-9))
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_quantize(x, block_rows):
    """x [R, K] in 64 bits -> values, scales."""
    R, K = x.shape
    nr, nk = -(-R // block_rows), -(-K // BLOCK)
    full = torch.zeros((nr * block_rows, nk * BLOCK), dtype=torch.float64, device=DEV)
    full[:R, :K] = x
    b = full.reshape(nr, block_rows, nk, BLOCK)
    largest = torch.maximum(b.abs().amax(dim=3).amax(dim=1), torch.full((), SMALLEST, dtype=torch.float64, device=DEV))
    q = _e4m3(b * (E4M3_MAX / largest)[:, None, :, None])
    return q.reshape(full.shape)[:R, :K], largest / E4M3_MAX


def exact(case, seed):
    c, st = case, prepare(case, seed)
    kind = c["kind"]

    def wide(v, scale, block_rows):                   # one matrix of stored values times their scales
        s = scale.double().repeat_interleave(block_rows, 0)[:v.shape[0]]
        return v.double() * s.repeat_interleave(BLOCK, 1)[:, :v.shape[1]]

    if kind == "quantize":
        q, scale = _exact_quantize(st["x"].double(), 1)
        q[c["valid"]:], scale[c["valid"]:] = 0, 0
        return dict(q=q, scale=scale)
    if kind == "quantize_w":
        each = [_exact_quantize(w.double(), BLOCK) for w in st["w"]]
        return dict(q=torch.stack([a for a, _ in each]), scale=torch.stack([b for _, b in each]))
    if kind in ("mm", "ffn"):
        offsets = st["offsets"].tolist()
        y = torch.zeros(st["y"].shape, dtype=torch.float64, device=DEV)
        x = wide(st["x"], st["xs"], 1)
        for l, (a, b) in enumerate(zip(offsets, offsets[1:])):
            if a == b:
                continue
            if kind == "mm":
                y[a:b] = torch.mm(x[a:b], wide(st["w"][l], st["ws"][l], BLOCK).t().contiguous())
                continue
            I, B = c["I"], -(-c["I"] // BLOCK)
            t = x[st["perm"][a:b].long() // c["k"]]
            gate = torch.mm(t, wide(st["w13"][l, :I], st["s13"][l, :B], BLOCK).t().contiguous())
            up = torch.mm(t, wide(st["w13"][l, I:], st["s13"][l, B:], BLOCK).t().contiguous())
            q, scale = _exact_quantize(gate * torch.sigmoid(gate) * up, 1)
            act = q * scale.repeat_interleave(BLOCK, 1)[:, :I]
            y[a:b] = torch.mm(act, wide(st["w2"][l], st["s2"][l], BLOCK).t().contiguous())
        return dict(y=y)
    T, k, H = c["T"], c["k"], c["H"]
    _, _, row = _lists(c, seed)
    pair = np.flatnonzero(row.reshape(-1) >= 0)
    pair, at = _i32(pair).long(), _i32(row.reshape(-1)[pair]).long()
    if kind == "rows":
        out = torch.zeros((T * k, H), dtype=torch.float64, device=DEV)
        out[at] = st["x"].double()[pair // k]
        return dict(x_perm=out)
    if kind == "rows_grad":
        dx = torch.zeros((T, H), dtype=torch.float64, device=DEV)
        return dict(dx=dx.index_add_(0, pair // k, st["dx_perm"].double()[at]))
    dout, w = st["dout"].double()[pair // k], st["topk_w"].double().reshape(-1)[pair]
    dy = torch.zeros((T * k, H), dtype=torch.float64, device=DEV)
    dy[at] = dout * w[:, None]
    dw = torch.zeros(T * k, dtype=torch.float64, device=DEV)
    dw[pair] = (dout * st["y"].double()[at]).sum(dim=1)
    return dict(dy_perm=dy, dtopk_w=dw.reshape(T, k))


# ------------------------------------------------------------------------------------------ what a pass cannot do without
@functools.lru_cache(maxsize=64)
def _share(items):
    """(rows, experts with a row, tokens with a row) of one drawn instance."""
    case = dict(items)
    if case["kind"] == "mm":
        n = np.diff(_groups(case, 1))
        return int(n.sum()), int((n > 0).sum()), 0
    offsets, _, row = _lists(case, 1)
    return int(offsets[-1]), int((np.diff(offsets) > 0).sum()), int((row >= 0).any(axis=1).sum())


def work(case):
    c = case
    kind = c["kind"]
    blocks = lambda r, K, h: 4 * (-(-r // h)) * (-(-K // BLOCK))  # noqa: E731  bytes of the scales
    if kind == "quantize":
        elt = 2 if c["dtype"] == "bf16" else 4
        return dict(bytes=c["valid"] * c["K"] * (elt + 1) + blocks(c["valid"], c["K"], 1) + 4, flops=3 * c["valid"] * c["K"])
    if kind == "quantize_w":
        elt = 2 if c["dtype"] == "bf16" else 4
        n = c["rows"] * c["K"]
        return dict(bytes=c["slots"] * (n * (elt + 1) + blocks(c["rows"], c["K"], BLOCK)), flops=3 * c["slots"] * n)
    rows, active, tokens = _share(tuple(sorted((n, v) for n, v in c.items() if n != "name")))
    if kind == "mm":
        K, N, elt = c["K"], c["N"], 2 if c["out"] == "bf16" else 4
        return dict(bytes=active * (N * K + blocks(N, K, BLOCK)) + rows * (K + N * elt) + blocks(rows, K, 1) + 4 * (c["groups"] + 1),
                    flops=2 * rows * N * K)
    if kind == "ffn":
        H, I, elt = c["H"], c["I"], 2 if c["out"] == "bf16" else 4
        weights = 3 * H * I + 2 * blocks(I, H, BLOCK) + blocks(H, I, BLOCK)
        return dict(bytes=active * weights + tokens * H + blocks(tokens, H, 1) + rows * (H * elt + 4) + 4 * (c["spr"] + 1),
                    flops=6 * rows * H * I)
    T, k, H, elt = c["T"], c["k"], c["H"], 2 if c["dtype"] == "bf16" else 4
    if kind == "rows":
        return dict(bytes=elt * H * (tokens + rows) + 4 * T * k, flops=0)
    if kind == "rows_grad":
        return dict(bytes=elt * H * (T + rows) + 4 * T * k, flops=rows * H)
    return dict(bytes=elt * H * (tokens + 2 * rows) + 12 * T * k, flops=3 * rows * H)
