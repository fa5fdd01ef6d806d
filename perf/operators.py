"""What stands between and beside the structured-binary linears of a decoder block, as cases to time and to compare: the matrix product in
8-bit integers with scales for each token and channel, the quantizer that makes its operands, and the norms before and after a block with
its gate, residual scale and residual sum.

Sizes are those of the LLaMA-2 7B / 13B / 70B linears the repository is configured for, with ragged ones between them.  Weights and
activations follow the repository's recipe (weights N(0, 0.02), 1 % of the columns x 10; activations N(0, 1), 0.5 % of the channels x 20).
"""
import math
import types

import torch

own = False
DEV = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # -- the product.  The smallest call: a grouped-query k/v projection of 70B kept in 8 bits, one token
        dict(name="gemm_i8_1024x8192_t1", kind="gemm_i8", n=1024, m=8192, T=1, out="f16", bias=False),
        # sizes of no model: no row tile, no 16 bytes of a row is full, three sequences, a bias
        dict(name="gemm_i8_5003x2813_t3_bias", kind="gemm_i8", n=5003, m=2813, T=3, out="f32", bias=True),
        # the down projection of 7B for 64 sequences in decode
        dict(name="gemm_i8_4096x11008_t64", kind="gemm_i8", n=4096, m=11008, T=64, out="f16", bias=False),
        # a short prompt of odd length through the down projection of 13B, fp32 out
        dict(name="gemm_i8_5120x13824_t333", kind="gemm_i8", n=5120, m=13824, T=333, out="f32", bias=False),
        # the largest: gate / up of 70B for a prompt of 2048 tokens
        dict(name="gemm_i8_28672x8192_t2048", kind="gemm_i8", n=28672, m=8192, T=2048, out="bf16", bias=False),
        # -- its operands.  One token's activations before q / k / v of 7B
        dict(name="quantize_i8_1x4096", kind="quantize_i8", rows=1, m=4096, dt="f16", gated=False),
        # converting a checkpoint: the gate projection of 7B, a scale for each output channel
        dict(name="quantize_i8_weights_11008x4096", kind="quantize_i8", rows=11008, m=4096, dt="f16", gated=False),
        # what the down projection of 70B reads in prefill: silu(gate) * up, quantized on the way
        dict(name="quantize_i8_gated_2048x28672", kind="quantize_i8", rows=2048, m=28672, dt="bf16", gated=True),
        # -- norms around a block.  Decode of one token, 7B: residual sum and the norm before the next block
        dict(name="norm_1x4096", kind="norm", T=1, h=4096, norm="rms", x="f32", r="f16", w="f16", y="f16", post=False, gate=0, bias=False, alpha=1.0),
        # decode of 37 sequences with layer norms and their biases, straight into the 8-bit product; an odd width
        dict(name="norm_layer_37x5111_i8", kind="norm", T=37, h=5111, norm="layer", x="f16", r="f32", w="f32", y="i8", post=False, gate=0, bias=True, alpha=1.0),
        # prefill of 70B width without a residual sum: the norm before the head, into the 8-bit product
        dict(name="norm_333x8192_i8", kind="norm", T=333, h=8192, norm="rms", x="bf16", r=None, w="bf16", y="i8", post=False, gate=0, bias=False, alpha=1.0),
        # prefill of 70B width, norms on both sides of the block, a gate per sequence (four of 512 tokens) and a residual scale
        dict(name="norm_sandwich_2048x8192", kind="norm", T=2048, h=8192, norm="rms", x="bf16", r="bf16", w="bf16", y="bf16", post=True, gate=4, bias=False, alpha=0.25),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("gemm_i8", "gemm_i8", "gemm_i8", "quantize_i8", "quantize_i8", "norm", "norm", "norm"))
    if kind == "gemm_i8":
        while True:
            n, m, T = _log(rng, 64, 28672), _log(rng, 64, 28672), rng.choice((1, _log(rng, 1, 16), _log(rng, 16, 256), _log(rng, 256, 4096)))
            if n * m <= 28672 * 8192 and n * m * T <= 28672 * 8192 * 2048:
                return dict(kind=kind, n=n, m=m, T=T, out=rng.choice(("f32", "f16", "bf16")), bias=rng.random() < 0.3)
    if kind == "quantize_i8":
        while True:
            rows, m = _log(rng, 1, 16384), _log(rng, 64, 28672)
            if rows * m <= 2048 * 28672:
                gated = rng.random() < 0.4
                return dict(kind=kind, rows=rows, m=m, dt=rng.choice(("f16", "bf16") if gated else ("f16", "bf16", "f32")), gated=gated)
    while True:
        T, h = rng.choice((1, _log(rng, 1, 64), _log(rng, 64, 4096))), _log(rng, 64, 16384)
        if T * h <= 2048 * 8192:
            break
    sixteen = rng.choice(("f16", "bf16"))
    either = lambda: rng.choice((sixteen, sixteen, "f32"))  # noqa: E731
    # a gate of the whole width, one per sequence, or one per token
    gate = rng.choice((0, 0, 1, T, rng.choice([g for g in range(1, min(T, 64) + 1) if T % g == 0])))
    norm = rng.choice(("rms", "rms", "layer"))
    return dict(kind=kind, T=T, h=h, norm=norm, x=either(), r=rng.choice((None, either(), either())), w=either(), y=rng.choice((sixteen, "f32", "i8")),
                post=rng.random() < 0.4, gate=gate, bias=norm == "layer" and rng.random() < 0.7, alpha=rng.choice((1.0, 0.25, 0.7071)))


# ---------------------------------------------------------------------------------------------------------------------
def _randn(rows, m, g, columns, factor):
    x = torch.randn(rows, m, generator=g, device=DEV, dtype=torch.float32)
    x[:, torch.randperm(m, generator=g, device=DEV)[: round(columns * m)]] *= factor
    return x


def _activations(rows, m, g):
    return _randn(rows, m, g, 0.005, 20.0)


def _eight(x):
    """Rows in 8 bits, on a stride of whole 16 bytes; what is behind a row's end is not part of it and can hold anything."""
    rows, m = x.shape
    buf = torch.full((rows, -(-m // 16) * 16), 77, dtype=torch.int8, device=DEV)
    largest = x.abs().amax(1)
    buf[:, :m] = torch.round(x * (127.0 / largest)[:, None]).to(torch.int8)
    return buf[:, :m], largest / 127.0


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    st = types.SimpleNamespace(**case)
    if case["kind"] == "gemm_i8":
        n, m, T = case["n"], case["m"], case["T"]
        st.wq, st.w_scale = _eight(_randn(n, m, g, 0.01, 10.0).mul_(0.02))
        st.xq, st.x_scale = _eight(_activations(T, m, g))
        st.b = torch.randn(n, generator=g, device=DEV) if case["bias"] else None
        return st
    if case["kind"] == "quantize_i8":
        rows, m, dt = case["rows"], case["m"], DTYPES[case["dt"]]
        st.x = _activations(rows, m, g).to(dt)
        st.x2 = _activations(rows, m, g).to(dt) if case["gated"] else None
        if rows > 8:                    # a padded batch: a row of nothing
            st.x[rows // 2] = 0
        return st
    T, h, wdt = case["T"], case["h"], DTYPES[case["w"]]
    vector = lambda: torch.randn(h, generator=g, device=DEV).mul_(0.1)  # noqa: E731
    st.x = _activations(T, h, g).to(DTYPES[case["x"]])
    st.r = _activations(T, h, g).mul_(4.0).to(DTYPES[case["r"]]) if case["r"] else None
    st.w = (1.0 + vector()).to(wdt)
    st.b = vector().to(wdt) if case["bias"] else None
    st.post_w = (1.0 + vector()).to(wdt) if case["post"] else None
    st.gates = torch.randn(case["gate"], h, generator=g, device=DEV).to(wdt) if case["gate"] else None
    return st


# -- plain forms: 32 bits, rounded once at the end ---------------------------------------------------------------------------------------
def _plain_rows(v):
    """Rows of fp32 values in 8 bits: (whole numbers, scale of each row).  The nearest whole number to v * 127 / max|v|, in 64 bits: 16-bit
    values lie on the borders between two of them now and then."""
    largest = v.abs().amax(1, keepdim=True)
    live, broken = largest >= 2.0 ** -118, ~torch.isfinite(largest)
    q = torch.round(v.double() * 127.0 / largest.double()).float()
    q = torch.where(live & ~broken, q, torch.zeros_like(q))
    scale = torch.where(live, largest / 127.0, torch.zeros_like(largest))
    return q, torch.where(broken, torch.full_like(scale, math.nan), scale)


def _plain_norm(v, kind, eps):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)


def _values(q, scale, dtype):
    """What numbers in 8 bits stand for."""
    return torch.mul(q, scale[:, None], out=torch.empty(q.shape, dtype=dtype, device=q.device))


def _formula_norm(st, up, eps=1e-5):
    """(norm of the new residual, new residual) in the type that `up` brings its argument to."""
    v = up(st.x)
    if st.post_w is not None:
        v = _plain_norm(v, st.norm, eps) * up(st.post_w)
    if st.gates is not None:
        v = v * up(st.gates).repeat_interleave(st.T // st.gate, 0)
    v = st.alpha * v
    if st.r is not None:
        v = up(st.r) + v
    y = _plain_norm(v, st.norm, eps) * up(st.w)
    return (y if st.b is None else y + up(st.b)), v


def run(st):
    if own:
        import paper_2408_01803_b200 as stb
    if st.kind == "gemm_i8":
        if own:
            return stb.gemm_i8(st.xq, st.x_scale, st.wq, st.w_scale, bias=st.b, out_dtype=DTYPES[st.out])
        y = (st.xq.float() @ st.wq.float().t()) * st.x_scale[:, None] * st.w_scale
        return (y if st.b is None else y + st.b).to(DTYPES[st.out])
    if st.kind == "quantize_i8":
        if own:
            q, scale = stb.quantize_i8(st.x, st.x2)
            return {"values": _values(q, scale, st.x.dtype), "scale": scale}
        v = st.x.float()
        if st.gated:
            # the definition rounds the gated activation to 32 bits and then to its 16-bit type: 64 bits say which way, next to a border
            d = st.x.double()
            v = (d / (1.0 + torch.exp(-d)) * st.x2.double()).float().to(st.x.dtype).float()
        q, scale = _plain_rows(v)
        return {"values": _values(q, scale[:, 0], st.x.dtype), "scale": scale[:, 0]}
    if own:
        y, r = stb.block_norm(st.x, st.w, residual=st.r, bias=st.b, post_weight=st.post_w, gate=st.gates, alpha=st.alpha, kind=st.norm,
                              out_dtype=torch.int8 if st.y == "i8" else DTYPES[st.y])
        if st.y == "i8":
            return {"values": _values(*y, torch.float16), "scale": y[1], "residual": r}
        return {"y": y, "residual": r}
    y, r = _formula_norm(st, lambda t: t.float())
    r = None if st.r is None else r.to(st.r.dtype)
    if st.y == "i8":
        q, scale = _plain_rows(y)
        return {"values": _values(q, scale[:, 0], torch.float16), "scale": scale[:, 0], "residual": r}
    return {"y": y.to(DTYPES[st.y]), "residual": r}


# -- the definitions in 64 bits ----------------------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "gemm_i8":
        y = torch.mm(st.xq.double(), st.wq.double().T)
        y.mul_(st.x_scale.double()[:, None]).mul_(st.w_scale.double()[None, :])
        return y if st.b is None else y.add_(st.b.double())
    if case["kind"] == "quantize_i8":
        v = st.x.double()
        if case["gated"]:
            v = (v * torch.sigmoid(v) * st.x2.double()).float().to(st.x.dtype).double()
        return _exact_rows(v)
    x = st.x.double()
    center = (lambda v: v - v.sum(1, keepdim=True) / v.shape[1]) if case["norm"] == "layer" else (lambda v: v)
    unit = lambda v: center(v) * torch.rsqrt(center(v).square().sum(1, keepdim=True) / v.shape[1] + 1e-5)  # noqa: E731
    if case["post"]:
        x = unit(x) * st.post_w.double()
    if case["gate"]:
        x = (x.view(case["gate"], -1, case["h"]) * st.gates.double()[:, None, :]).view_as(x)
    x = case["alpha"] * x + (0.0 if st.r is None else st.r.double())
    y = unit(x) * st.w.double() + (0.0 if st.b is None else st.b.double())
    residual = None if st.r is None else x
    return {"y": y, "residual": residual} if case["y"] != "i8" else dict(_exact_rows(y), residual=residual)


def _exact_rows(v):
    top = torch.linalg.vector_norm(v, math.inf, dim=1)
    steps = torch.where(top > 0, v.T * 127.0 / top, 0.0).T.round()
    return {"values": steps * (top / 127.0)[:, None], "scale": top / 127.0}


def work(case):
    if case["kind"] == "gemm_i8":
        n, m, T = case["n"], case["m"], case["T"]
        return {"bytes": n * m + T * m + 4 * (n + T) + T * n * SIZES[case["out"]] + (4 * n if case["bias"] else 0), "flops": 2.0 * n * m * T}
    if case["kind"] == "quantize_i8":
        values = case["rows"] * case["m"]
        return {"bytes": values * (SIZES[case["dt"]] * (2 if case["gated"] else 1) + 1) + 4 * case["rows"], "flops": 0.0}
    T, h = case["T"], case["h"]
    a_value = SIZES[case["x"]] + (2 * SIZES[case["r"]] if case["r"] else 0) + (1 if case["y"] == "i8" else SIZES[case["y"]])
    vectors = 1 + case["bias"] + case["post"] + case["gate"]
    return {"bytes": T * h * a_value + vectors * h * SIZES[case["w"]] + (4 * T if case["y"] == "i8" else 0), "flops": 0.0}
