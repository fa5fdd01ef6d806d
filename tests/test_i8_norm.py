"""The operators beside and between the structured-binary layers -- rows in 8 bits, the 8-bit product, the norms of a block -- against plain
forms in 64 bits.  Whole numbers and everything that is defined by a fixed sequence of roundings is compared bit for bit; the norms, whose
sums are rounded in an order of the kernel's own, within bounds that are derived where they are used."""
import ctypes as C
import math

import pytest
import torch

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U32 = 2.0 ** -24                                    # half a step of fp32, relative


@pytest.fixture(scope="module")
def stb():
    from paper_2408_01803_b200 import build
    build.build()
    import paper_2408_01803_b200 as stb
    return stb


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _values(rows, m, seed, dtype="f32", size=1.0):
    x = torch.randn(rows, m, generator=_gen(seed)) * size
    x[:, ::97] *= 20.0
    return x.to(DTYPES[dtype])


def _place(t, pad, shift):
    """The same matrix on the GPU inside a larger buffer: rows `pad` values longer, starting `shift` values in; what surrounds it is no number."""
    rows, m = t.shape
    fill = 99 if t.dtype == torch.int8 else math.nan
    buf = torch.full((rows * (m + pad) + shift,), fill, dtype=t.dtype, device="cuda")
    view = buf[shift:].view(rows, m + pad)[:, :m]
    view.copy_(t)
    return view


def _rows64(v):
    """Rows of exact values in 8 bits by the definition: (q, scale) in 64 bits."""
    v = v.double()
    top = v.abs().amax(1, keepdim=True)
    live = top >= 2.0 ** -118
    broken = ~torch.isfinite(top)
    q = torch.where(live & ~broken, torch.round(v * 127.0 / top), torch.zeros_like(v))
    scale = torch.where(live, top / 127.0, torch.zeros_like(top))
    return q, torch.where(broken, torch.full_like(scale, math.nan), scale)[:, 0]


def _gated64(a, b):
    """silu(a) b, rounded to fp32 and then to the 16-bit type."""
    d = a.double()
    return (d / (1.0 + torch.exp(-d)) * b.double()).float().to(a.dtype)


def _same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=-1e30), torch.nan_to_num(b, nan=-1e30))


def _check_rows(q, scale, v):
    want_q, want_s = _rows64(v.cuda())
    assert torch.equal(q.double(), want_q)
    assert _same(scale.cpu(), want_s.float().cpu())


# ---- without a GPU: what is refused ---------------------------------------------------------------------------------------------------
def test_quantize_i8_refuses(stb):
    f, one, odd = stb._lib.stb_quantize_i8, C.c_void_p(256), C.c_void_p(257)
    ok = dict(x=one, ldx=64, x2=None, ldx2=0, dt=stb.STB_F16, rows=2, m=64, q=one, ldq=64, scale=one)
    call = lambda **kw: f(*[dict(ok, **kw)[k] for k in ok], None)  # noqa: E731
    for kw, code in ((dict(x=None), stb.STB_ERR_ARG), (dict(q=None), stb.STB_ERR_ARG), (dict(scale=None), stb.STB_ERR_ARG), (dict(rows=0), stb.STB_ERR_SHAPE),
                     (dict(m=0), stb.STB_ERR_SHAPE), (dict(rows=-1), stb.STB_ERR_SHAPE), (dict(dt=3), stb.STB_ERR_UNSUPPORTED),
                     (dict(x2=one, ldx2=64, dt=stb.STB_F32), stb.STB_ERR_UNSUPPORTED), (dict(ldx=63), stb.STB_ERR_ARG), (dict(ldq=63), stb.STB_ERR_ARG),
                     (dict(x2=one, ldx2=63), stb.STB_ERR_ARG), (dict(x=odd), stb.STB_ERR_ARG), (dict(x2=odd, ldx2=64), stb.STB_ERR_ARG), (dict(scale=odd), stb.STB_ERR_ARG)):
        assert call(**kw) == code, kw


def test_gemm_i8_refuses(stb):
    f, one = stb._lib.stb_gemm_i8, C.c_void_p(256)
    ok = dict(W=one, ldw=64, ws=one, bias=None, n=8, m=64, X=one, ldx=64, xs=one, T=2, Y=one, dt=stb.STB_F32, ldy=8)
    call = lambda **kw: f(*[dict(ok, **kw)[k] for k in ok], None, None)  # noqa: E731
    for kw, code in ((dict(W=None), stb.STB_ERR_ARG), (dict(ws=None), stb.STB_ERR_ARG), (dict(X=None), stb.STB_ERR_ARG), (dict(xs=None), stb.STB_ERR_ARG),
                     (dict(Y=None), stb.STB_ERR_ARG), (dict(n=0), stb.STB_ERR_SHAPE), (dict(m=0), stb.STB_ERR_SHAPE), (dict(T=0), stb.STB_ERR_SHAPE),
                     (dict(m=131072, ldw=131072, ldx=131072), stb.STB_ERR_SHAPE), (dict(dt=3), stb.STB_ERR_UNSUPPORTED), (dict(ldw=48), stb.STB_ERR_ARG),
                     (dict(ldx=48), stb.STB_ERR_ARG), (dict(ldw=72), stb.STB_ERR_ARG), (dict(ldx=72), stb.STB_ERR_ARG), (dict(ldy=7), stb.STB_ERR_ARG),
                     (dict(W=C.c_void_p(264)), stb.STB_ERR_ARG), (dict(X=C.c_void_p(264)), stb.STB_ERR_ARG), (dict(Y=C.c_void_p(258)), stb.STB_ERR_ARG),
                     (dict(bias=C.c_void_p(257)), stb.STB_ERR_ARG), (dict(ws=C.c_void_p(258)), stb.STB_ERR_ARG), (dict(Y=C.c_void_p(257), dt=stb.STB_F16), stb.STB_ERR_ARG)):
        assert call(**kw) == code, kw


def test_block_norm_refuses(stb):
    ok = dict(tokens=2, h=64, kind=0, post=0, eps=1e-5, alpha=1.0, x=256, xdt=0, ldx=64, y=256, ydt=0, ldy=64)

    def call(**kw):
        return stb._lib.stb_block_norm(C.byref(stb._Norm(**dict(ok, **kw))), None)

    assert stb._lib.stb_block_norm(None, None) == stb.STB_ERR_ARG
    for kw, code in ((dict(x=None), stb.STB_ERR_ARG), (dict(y=None), stb.STB_ERR_ARG), (dict(tokens=0), stb.STB_ERR_SHAPE), (dict(h=0), stb.STB_ERR_SHAPE),
                     (dict(h=32769, ldx=32769, ldy=32769), stb.STB_ERR_SIZE), (dict(kind=2), stb.STB_ERR_UNSUPPORTED), (dict(xdt=3), stb.STB_ERR_UNSUPPORTED),
                     (dict(ydt=3), stb.STB_ERR_UNSUPPORTED), (dict(ldx=63), stb.STB_ERR_ARG), (dict(ldy=63), stb.STB_ERR_ARG), (dict(eps=-1.0), stb.STB_ERR_ARG),
                     (dict(eps=math.nan), stb.STB_ERR_ARG), (dict(eps=math.inf), stb.STB_ERR_ARG), (dict(alpha=math.nan), stb.STB_ERR_ARG), (dict(alpha=math.inf), stb.STB_ERR_ARG),
                     (dict(q=256, ldq=64), stb.STB_ERR_ARG), (dict(q=256, ldq=63, q_scale=256), stb.STB_ERR_ARG), (dict(weight=256, wdt=3), stb.STB_ERR_UNSUPPORTED),
                     (dict(post_weight=256), stb.STB_ERR_ARG), (dict(resid=256, ldr=63), stb.STB_ERR_ARG), (dict(resid=256, ldr=64, rdt=3), stb.STB_ERR_UNSUPPORTED),
                     (dict(resid_out=256, ldro=63), stb.STB_ERR_ARG), (dict(gate=256, ldgate=64), stb.STB_ERR_ARG), (dict(gate=256, ldgate=63, tokens_per_gate=1), stb.STB_ERR_ARG),
                     (dict(x=257), stb.STB_ERR_ARG), (dict(weight=257), stb.STB_ERR_ARG), (dict(y=None, resid_out=256, ldro=64, weight=256), stb.STB_ERR_ARG)):
        assert call(**kw) == code, kw


def test_python_calls_refuse_what_is_not_on_one_device(stb):
    x, q, s = torch.zeros(2, 64, dtype=torch.float16), torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2)
    for call in (lambda: stb.quantize_i8(x), lambda: stb.gemm_i8(q, s, q, s), lambda: stb.block_norm(x)):
        with pytest.raises(stb.StbError) as e:
            call()
        assert e.value.status == stb.STB_ERR_ARG


def test_gemm_i8_refuses_sides_beyond_its_range(stb):
    """n and T of more than 2^30: what lies behind the last tile would pass 32 bits."""
    one, top = C.c_void_p(256), (1 << 31) - 1
    for n, T in ((top, 1), ((1 << 30) + 1, 8), (64, (1 << 30) + 1), (1, top)):
        assert stb._lib.stb_gemm_i8(one, 64, one, None, n, 64, one, 64, one, T, one, stb.STB_F32, n, None, None) == stb.STB_ERR_SHAPE, (n, T)


def test_python_calls_refuse_sides_beyond_32_bits(stb):
    """Sizes that the library's int cannot hold are refused, not cut to their low 32 bits."""
    class Matrix:
        is_cuda, device, dtype = True, torch.device("cuda", 0), torch.int8

        def __init__(self, *shape):
            self.shape = shape

        def dim(self):
            return 2

        def stride(self, i):
            return (self.shape[1], 1)[i]

    for shape in (((1 << 32) + 5, 1), (3, (1 << 32) + 16), (1 << 31, 1)):
        with pytest.raises(stb.StbError) as e:
            stb._rows(Matrix(*shape), Matrix(1, 1), "x")
        assert e.value.status == stb.STB_ERR_SHAPE
    assert stb._rows(Matrix((1 << 31) - 1, 1), Matrix(1, 1), "x").shape[1] == 1


# ---- rows in 8 bits -------------------------------------------------------------------------------------------------------------------
WIDTHS = (1, 2, 7, 8, 9, 64, 255, 256, 257, 511, 1024, 1025, 2813, 4096, 8200, 16384, 16391, 32768, 32769, 40001)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ("f32", "f16", "bf16"))
@pytest.mark.parametrize("m", WIDTHS)
def test_rows_in_8_bits(stb, m, dt):
    for rows in (1, 3) if m > 1024 else (1, 3, 160, 1500):
        x = _values(rows, m, m + rows, dt)
        if rows > 2:
            x[1] = 0
        q, s = stb.quantize_i8(x.cuda())
        assert q.shape == (rows, m) and q.dtype == torch.int8 and (rows == 1 or q.stride(0) % 16 == 0)
        _check_rows(q, s, x)
        q, s = stb.quantize_i8(_place(x, 3, 1))                     # rows on no boundary
        _check_rows(q, s, x)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ("f16", "bf16"))
@pytest.mark.parametrize("m", WIDTHS)
def test_gated_rows_in_8_bits(stb, m, dt):
    for rows in (1, 4) if m > 1024 else (2, 160, 1500):
        a, b = _values(rows, m, 3 * m + rows, dt), _values(rows, m, 5 * m + rows, dt)
        b[0] = 0
        for q, s in (stb.quantize_i8(a.cuda(), b.cuda()), stb.quantize_i8(_place(a, 8, 8), _place(b, 5, 3))):
            _check_rows(q, s, _gated64(a, b))


@pytest.mark.gpu
@pytest.mark.parametrize("m", (264, 1032, 2816, 4096, 5120, 6008, 8192, 11008, 12000, 12288, 13824, 16384, 16392, 20480, 24568, 28672, 32768))
def test_many_rows(stb, m):
    """More rows than stay on the GPU at once, of every width class: each CTA or warp takes several."""
    for k, dt in enumerate(("f16", "bf16", "f32")):
        rows = 310 + 700 * ((m + k) % 3 == 0)
        x = _values(rows, m, m + k, dt)
        x[7] = 0
        x[rows - 1, m - 1] = 300.0
        _check_rows(*stb.quantize_i8(x.cuda()), x)
        if dt != "f32":
            b = _values(rows, m, m + k + 9, dt)
            _check_rows(*stb.quantize_i8(x.cuda(), b.cuda()), _gated64(x.cuda(), b.cuda()).cpu())
    for k, kw in enumerate((dict(x="f16", r="f16", w="f16", y="bf16"), dict(x="f32", r="f32", w="f32", y="i8", kind="layer", bias=True), dict(x="bf16", r=None, post=True, w="f32", y="f32", gate=2))):
        _check_norm(stb, 310 + 200 * k, m, m + k, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ("f16", "bf16"))
def test_gated_values_next_to_their_borders(stb, dt):
    """Every pair of a grid of magnitudes from the smallest to the largest, most of all products that lie on a border of the 16-bit type."""
    t = DTYPES[dt]
    a = torch.cat([torch.arange(-120.0, 120.0, 0.75), torch.tensor([1e-30, -1e-30, 6e-8, 17.0, 37.5, 200.0, 3e4, -3e4])]).to(t)
    b = torch.cat([torch.arange(0.0, 4.0, 1 / 32), torch.tensor([6e-8, 1e-7, 1e-30, 1e30, 300.0, 6e4])]).to(t)
    b = torch.where(torch.isfinite(b), b, torch.ones_like(b))
    A, B = a[:, None].expand(-1, b.numel()).contiguous(), b[None, :].expand(a.numel(), -1).contiguous()
    q, s = stb.quantize_i8(A.cuda(), B.cuda())
    _check_rows(q, s, _gated64(A, B))


@pytest.mark.gpu
def test_rows_on_the_borders_between_whole_numbers(stb):
    """max|v| = 2^k (1 or 254/256): 127 v / max|v| is a half-odd number exactly, or one step of v beside it."""
    for top in (1.0, 254.0, 2.0 ** -20, 1.5 * 2.0 ** 60, 127.0):
        k = torch.arange(-127, 127).double()
        border = ((2 * k + 1) * top / 254.0).float()
        x = torch.stack([border, torch.nextafter(border, torch.full_like(border, 1e38)), torch.nextafter(border, torch.full_like(border, -1e38))])
        x = torch.cat([x, torch.full((3, 1), top)], 1)
        _check_rows(*stb.quantize_i8(x.cuda()), x)


@pytest.mark.gpu
@pytest.mark.parametrize("m", (40, 700, 5000, 40000))
def test_rows_without_a_scale(stb, m):
    """Zeros, magnitudes beyond the format's end, infinities and NaN."""
    x = _values(8, m, 1)
    x[0] = 0
    x[1, m // 2] = math.inf
    x[2, m - 1] = -math.inf
    x[3, 0] = math.nan
    x[4] *= 2.0 ** -130
    x[5] = torch.sign(x[5]) * 2.0 ** -118
    x[6] *= 1e37
    q, s = stb.quantize_i8(x.cuda())
    _check_rows(q, s, x)
    assert torch.isnan(s[1:4]).all() and (q[1:5] == 0).all() and s[0] == 0
    h = x.half()
    h[6] = 60000.0
    q, s = stb.quantize_i8(h.cuda(), h.cuda())                       # row 6: the product is beyond fp16
    _check_rows(q, s, _gated64(h, h))
    assert torch.isnan(s[6])


@pytest.mark.gpu
def test_quantize_i8_writes_only_its_rows(stb):
    x = _values(5, 70, 2, "f16").cuda()
    buf = torch.full((7, 96), 55, dtype=torch.int8, device="cuda")
    scale = torch.full((7,), 5.0, device="cuda")
    q, s = stb.quantize_i8(x, q=buf[1:6, :70], scale=scale[1:6])
    assert q.data_ptr() == buf[1].data_ptr() and s.data_ptr() == scale[1:].data_ptr()
    _check_rows(q, s, x.cpu())
    assert (buf[0] == 55).all() and (buf[6] == 55).all() and (buf[:, 70:] == 55).all() and scale[0] == 5 and scale[6] == 5
    q1, s1 = stb.quantize_i8(x[2])                                   # one token as a vector
    assert q1.shape == (70,) and torch.equal(q1, q[2]) and torch.equal(s1, s[2:3])


# ---- the product ----------------------------------------------------------------------------------------------------------------------
def _eight(rows, m, seed):
    q = torch.randint(-128, 128, (rows, m), generator=_gen(seed), dtype=torch.int8)
    return q, torch.rand(rows, generator=_gen(seed + 1)) * 0.01 + 1e-4


def _product(xq, xs, wq, ws, bias, dtype):
    """The definition: an exact sum, and one rounding to fp32 after each step."""
    y = torch.round(xq.double().cuda() @ wq.double().cuda().T).cpu()        # whole numbers below 2^53: exact in any order
    y = y.to(torch.float32) * xs[:, None]
    y = y * ws
    return (y if bias is None else y + bias).to(dtype)


def _i8_place(q, pad):
    rows, m = q.shape
    buf = torch.full((rows, -(-m // 16) * 16 + pad), 99, dtype=torch.int8, device="cuda")
    buf[:, :m] = q
    return buf[:, :m]


def _check_product(stb, T, n, m, seed, out="f32", with_bias=False, pad=0, **kw):
    xq, xs = _eight(T, m, seed)
    wq, ws = _eight(n, m, seed + 10)
    bias = torch.randn(n, generator=_gen(seed + 20)) if with_bias else None
    y = stb.gemm_i8(_i8_place(xq, pad), xs.cuda(), _i8_place(wq, pad), ws.cuda(), bias=bias.cuda() if with_bias else None, out_dtype=DTYPES[out], **kw)
    want = _product(xq, xs, wq, ws, bias, DTYPES[out])
    assert y.shape == (T, n) and y.dtype == DTYPES[out]
    assert torch.equal(y.cpu(), want), (T, n, m)


@pytest.mark.gpu
@pytest.mark.parametrize("T", (1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 64, 65, 96, 100, 128, 129, 200, 255, 256, 257, 300, 512, 513, 700, 1025))
def test_product_by_tokens(stb, T):
    for k, (n, m) in enumerate(((300, 1000), (1, 64), (127, 129), (512, 2048))):
        _check_product(stb, T, n, m, T + k, out=("f32", "f16", "bf16")[(T + k) % 3], with_bias=k % 2 == 0, pad=16 * (k % 2))


@pytest.mark.gpu
@pytest.mark.parametrize("m", (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1023, 1100, 4111, 20000))
def test_product_by_columns(stb, m):
    for k, (T, n) in enumerate(((1, 40), (5, 17), (16, 33), (40, 130), (150, 70), (300, 260))):
        _check_product(stb, T, n, m, m + k, out=("f32", "f16", "bf16")[(m + k) % 3], with_bias=k % 2 == 1, pad=32 * (k % 2))


@pytest.mark.gpu
@pytest.mark.parametrize("n", (1, 2, 15, 16, 17, 31, 32, 33, 64, 100, 127, 128, 129, 255, 256, 257, 400, 1001, 5003))
def test_product_by_channels(stb, n):
    for k, (T, m) in enumerate(((1, 512), (3, 300), (12, 128), (50, 640), (130, 256), (280, 384))):
        _check_product(stb, T, n, m, n + k, out=("f16", "f32", "bf16")[(n + k) % 3], with_bias=k % 2 == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("T", (1, 13, 48, 180, 400))
def test_product_at_the_ends_of_its_range(stb, T):
    """Sums of the largest magnitude that int32 takes: every product 128 * 128, as many columns as are allowed."""
    m, n = 131071, 3
    x = torch.full((T, m), -128, dtype=torch.int8, device="cuda")
    buf = torch.full((T, 131072), -128, dtype=torch.int8, device="cuda")
    w = torch.full((n, 131072), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    one = torch.ones(max(T, n), device="cuda")
    y = stb.gemm_i8(buf[:, :m], one[:T], w[:, :m], one[:n])
    want = torch.tensor([128.0 * 128 * m, -128.0 * 127 * m, 128.0 * 128 * m], dtype=torch.float64).float()
    assert torch.equal(y.cpu(), want.expand(T, n)), x.shape


@pytest.mark.gpu
@pytest.mark.parametrize("T", (1, 4, 20, 90, 300))
@pytest.mark.parametrize("out", ("f32", "f16", "bf16"))
def test_product_into_rows_of_a_larger_buffer(stb, T, out):
    """Any row stride and start of the result; nothing around it is touched."""
    n, m = 150, 260
    xq, xs = _eight(T, m, 5)
    wq, ws = _eight(n, m, 6)
    want = _product(xq, xs, wq, ws, None, DTYPES[out])
    for pad, shift in ((0, 0), (10, 0), (1, 0), (7, 3), (16, 8)):
        ld = n + pad
        buf = torch.full((T * ld + 32,), 7.0, dtype=DTYPES[out], device="cuda")
        y = buf[shift:shift + T * ld].view(T, ld)[:, :n]
        got = stb.gemm_i8(_i8_place(xq, 0), xs.cuda(), _i8_place(wq, 0), ws.cuda(), out=y)
        assert got.data_ptr() == y.data_ptr() and torch.equal(got.cpu(), want)
        y.fill_(7.0)
        assert (buf == 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", (1, 12, 100, 300))
def test_product_of_tokens_without_a_scale(stb, T):
    xq, xs = _eight(T, 320, 8)
    wq, ws = _eight(200, 320, 9)
    xs[T // 2] = math.nan
    ws[7] = 0.0
    y = stb.gemm_i8(_i8_place(xq, 0), xs.cuda(), _i8_place(wq, 0), ws.cuda())
    assert torch.isnan(y[T // 2]).all()
    keep = [t for t in range(T) if t != T // 2]
    assert torch.equal(y[keep].cpu(), _product(xq, xs, wq, ws, None, torch.float32)[keep])
    one = stb.gemm_i8(_i8_place(xq, 0)[0], xs[:1].cuda(), _i8_place(wq, 0), ws.cuda())     # one token as a vector
    assert one.shape == (200,) and _same(one, y[0])


@pytest.mark.gpu
def test_product_refuses_what_does_not_fit(stb):
    q = lambda r, m: torch.zeros(r, m, dtype=torch.int8, device="cuda")  # noqa: E731
    s = lambda r: torch.zeros(r, device="cuda")  # noqa: E731
    for call in (lambda: stb.gemm_i8(q(4, 64), s(4), q(8, 80), s(8)), lambda: stb.gemm_i8(q(4, 64), s(3), q(8, 64), s(8)), lambda: stb.gemm_i8(q(4, 64), s(4), q(8, 64), s(7)),
                 lambda: stb.gemm_i8(q(4, 64), s(4), q(8, 64), s(8), bias=s(7)), lambda: stb.gemm_i8(q(4, 64), s(4), q(8, 64), s(8), out=torch.zeros(4, 7, device="cuda")),
                 lambda: stb.gemm_i8(q(4, 64).half(), s(4), q(8, 64), s(8)), lambda: stb.gemm_i8(q(4, 64), s(4).double(), q(8, 64), s(8)),
                 lambda: stb.gemm_i8(q(64, 4).t(), s(4), q(8, 64), s(8)), lambda: stb.gemm_i8(q(4, 60), s(4), q(8, 60), s(8)),          # rows of 60 bytes
                 lambda: stb.gemm_i8(q(1, 64).expand(4, 64), s(4), q(8, 64), s(8)), lambda: stb.gemm_i8(q(4, 80)[:, 8:72], s(4), q(8, 64), s(8))):
        with pytest.raises(stb.StbError) as e:
            call()
        assert e.value.status == stb.STB_ERR_ARG
    with pytest.raises(stb.StbError) as e:
        stb.gemm_i8(q(4, 64), s(4), q(8, 64), s(8), out_dtype=torch.float64)
    assert e.value.status == stb.STB_ERR_UNSUPPORTED


# ---- norms ------------------------------------------------------------------------------------------------------------------------------
def _norm64(v, kind, eps):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    return v, 1.0 / torch.sqrt(v.square().mean(1, keepdim=True) + eps)


def _block64(x, weight, residual, bias, post, post_weight, post_bias, gate, alpha, kind, eps):
    """(y, r, bound on y's error before its rounding, bound on r's): the definition in 64 bits, and what fp32 arithmetic may be off.

    A row sum of the kernel is a chain of at most 32 additions in a thread and 10 between threads, each off by U32 of the sum of magnitudes:
    the mean square by 43 U32 relative, the reciprocal root by half that and its own 4 U32, so norm(v) by S = 32 U32 relative; a layer
    norm's mean by 43 U32 of the largest magnitude, which every centred value inherits (M = 44 U32 max|v| / sqrt(variance + eps))."""
    S, M = 32 * U32, 44 * U32
    d = lambda t: t.double()  # noqa: E731
    v, err = d(x), torch.zeros_like(d(x))
    alpha = float(torch.tensor(alpha, dtype=torch.float32))
    eps = float(torch.tensor(eps, dtype=torch.float32))

    def norm(v, err, w, b):
        c, inv = _norm64(v, kind, eps)
        # an error of the input moves its own value, and through the root mean square (and the mean) all of them
        spread = err.square().mean(1, keepdim=True).sqrt() + (err.mean(1, keepdim=True) if kind == "layer" else 0.0)
        e = inv * (err + (M * v.abs().amax(1, keepdim=True) if kind == "layer" else 0.0)) + (c * inv).abs() * (S + 2 * U32 + inv * spread) + (inv * spread if kind == "layer" else 0.0)
        y = c * inv
        if w is not None:
            y, e = y * d(w), e * d(w).abs() + 1.01 * U32 * (y * d(w)).abs()
        if b is not None:
            y = y + d(b)
            e = e + 1.01 * U32 * y.abs()
        return y, e

    if post or post_weight is not None or post_bias is not None:
        v, err = norm(v, err, post_weight, post_bias)
    if gate is not None:
        G = d(gate if gate.dim() == 2 else gate[None]).repeat_interleave(x.shape[0] // (gate.shape[0] if gate.dim() == 2 else 1), 0)
        v, err = v * G, err * G.abs() + 1.01 * U32 * (v * G).abs()
    v, err = alpha * v, abs(alpha) * err
    if residual is not None:
        v = v + d(residual)
    err = err + 1.01 * U32 * v.abs()
    y, ey = norm(v, err, weight, bias)
    return y, v, ey, err


def _half_step(dtype):
    return torch.finfo(dtype).eps / 2


def _check_norm(stb, T, h, seed, x="f16", r="f16", w="f16", y="f16", kind="rms", post=False, post_w=False, post_b=False, gate=None, bias=False, weight=True,
                alpha=1.0, eps=1e-5, place=(0, 0), inplace=False):
    ten = {"x": _values(T, h, seed, x), "residual": _values(T, h, seed + 1, r, 3.0) if r else None}
    wdt = DTYPES[w]
    vec = lambda k, on, one: (one + 0.3 * torch.randn(h, generator=_gen(seed + k))).to(wdt) if on else None  # noqa: E731
    vecs = {"weight": vec(2, weight, 1.0), "bias": vec(3, bias, 0.0), "post_weight": vec(4, post_w, 1.0), "post_bias": vec(5, post_b, 0.0)}
    if gate is not None:
        g = torch.randn(max(1, gate), h, generator=_gen(seed + 6)).to(wdt)
        vecs["gate"] = g if gate else g[0]
    want_y, want_r, ey, er = _block64(post=post, alpha=alpha, kind=kind, eps=eps, **{**{"gate": None}, **ten, **vecs})
    dev = {k: (None if v is None else _place(v, *place) if v.dim() == 2 else v.cuda()) for k, v in {**ten, **vecs}.items()}
    out_dtype = torch.int8 if y == "i8" else DTYPES[y]
    got, got_r = stb.block_norm(dev.pop("x"), dev.pop("weight"), post=post, alpha=alpha, kind=kind, eps=eps, out_dtype=out_dtype,
                                residual_out=dev["residual"] if inplace else None, **dev)
    if r:
        assert got_r.dtype == DTYPES[r]
        if inplace:
            assert got_r.data_ptr() == dev["residual"].data_ptr()
        off = (got_r.cpu().double() - want_r).abs()
        tiny = torch.finfo(DTYPES[r]).smallest_normal * torch.finfo(DTYPES[r]).eps
        assert (off <= 1.001 * (er + _half_step(DTYPES[r]) * (want_r.abs() + er)) + tiny).all(), "residual"
    else:
        assert got_r is None
    if y == "i8":
        q, s = got
        top, etop = want_y.abs().amax(1), ey.amax(1)
        s64 = s.cpu().double()
        assert ((s64 * 127 - top).abs() <= 1.001 * (etop + 2 * U32 * top)).all(), "scale"
        # half a step of 8 bits, and the value's own error
        assert ((q.cpu().double() * s64[:, None] - want_y).abs() <= 1.0001 * (0.5 * s64[:, None] + ey) + 4 * U32 * top[:, None]).all(), "values"
        assert (q.cpu().abs().amax(1)[top > 2.0 ** -100] == 127).all()
    else:
        assert got.dtype == out_dtype
        off = (got.cpu().double() - want_y).abs()
        tiny = torch.finfo(out_dtype).smallest_normal * torch.finfo(out_dtype).eps
        assert (off <= 1.001 * (ey + _half_step(out_dtype) * (want_y.abs() + ey)) + tiny).all(), "y"


NORM_WIDTHS = (1, 2, 7, 8, 31, 255, 256, 257, 512, 1000, 1024, 1025, 2048, 4096, 5111, 8192, 8200, 16384, 16385, 20000, 32768)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ("rms", "layer"))
@pytest.mark.parametrize("h", NORM_WIDTHS)
def test_norms_by_width(stb, h, kind):
    for k, T in enumerate((1, 5, 152) if h <= 4096 else (1, 3, 150)):
        types = ("f16", "bf16", "f32")
        pick = lambda j: types[(h + k + j) % 3]  # noqa: E731
        _check_norm(stb, T, h, 10 * h + k, x=pick(0), r=pick(1), w=pick(2), y=("f16", "i8", "f32", "bf16")[(h + k) % 4], kind=kind, bias=kind == "layer")
        _check_norm(stb, T, h, 10 * h + k + 5, x=pick(1), r=pick(1), w=pick(0), y=pick(2), kind=kind, post_w=True, post_b=kind == "layer", gate=0, alpha=0.3, place=(5, 3))


@pytest.mark.gpu
@pytest.mark.parametrize("h", (200, 1016, 3000, 18000))
@pytest.mark.parametrize("T", (1, 6, 300, 1200))
def test_norm_parts(stb, T, h):
    if T * h > 4_000_000:
        T = 152
    for k, kw in enumerate((dict(r=None), dict(r=None, weight=False, y="i8"), dict(post=True, weight=False), dict(gate=T), dict(gate=0, post_w=True), dict(gate=max(1, T // 3) if T % 3 == 0 else 1),
                            dict(post=True, kind="layer", bias=True, alpha=-2.0), dict(inplace=True, r="f32", y="i8"), dict(inplace=True, place=(8, 8)), dict(eps=0.0), dict(alpha=0.0),
                            dict(x="f32", w="f32", r="f32", y="f32", post_w=True, post_b=True, bias=True))):
        _check_norm(stb, T, h, 31 * h + k, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("h", (1032, 2816, 5120, 8192, 11008, 16384, 17000, 24576, 24584, 28672, 32768))
def test_norms_of_many_tokens(stb, h):
    """More tokens than CTAs stay on the GPU: the next one's values on their way, in every form that takes them."""
    T = max(310, min(1500, 5_000_000 // h))
    f32 = dict(x="f32", r="f32", w="f32", y="f32")
    for k, kw in enumerate((dict(r="f32"), dict(y="i8"), dict(x="bf16", r="bf16", w="bf16", y="bf16", post=True, post_w=True, gate=1, alpha=0.5),
                            dict(kind="layer", w="f32", bias=True, inplace=True, place=(16, 8)), f32 if h <= 28672 else dict(r=None))):
        _check_norm(stb, T, h, 17 * h + k, **kw)


@pytest.mark.gpu
def test_rows_of_fp32_off_their_pieces(stb):
    """fp32 rows on 16-byte boundaries that are on no 32-byte ones."""
    for T, h in ((3, 4096), (400, 1032)):
        buf = torch.randn(T, h + 12, generator=_gen(h), dtype=torch.float32).cuda()
        for x in (buf[:, 4:h + 4], buf.view(-1)[4:4 + T * h].view(T, h)):
            q, s = stb.quantize_i8(x)
            _check_rows(q, s, x.cpu())
            w = torch.randn(h + 4, generator=_gen(T)).cuda()[4:]
            y, _ = stb.block_norm(x, w)
            want_y, _, ey, _ = _block64(x.cpu(), w.cpu(), None, None, False, None, None, None, 1.0, "rms", 1e-5)
            assert ((y.cpu().double() - want_y).abs() <= 1.001 * (ey + U32 * want_y.abs())).all()


@pytest.mark.gpu
def test_norm_of_nothing_and_of_no_numbers(stb):
    for h in (50, 1500):
        x = _values(6, h, 3)
        x[0] = 0
        x[1, 3] = math.nan
        x[2, h - 1] = math.inf
        for kind in ("rms", "layer"):
            (q, s), _ = stb.block_norm(x.cuda(), kind=kind, out_dtype=torch.int8)
            y, _ = stb.block_norm(x.cuda(), kind=kind)
            assert (y[0] == 0).all() and (q[0] == 0).all() and s[0] == 0
            assert torch.isnan(y[1]).all() and torch.isnan(s[1]) and (q[1] == 0).all()
            assert torch.isnan(y[2, h - 1]) and torch.isnan(s[2]) and (q[2] == 0).all()
            assert torch.isfinite(y[3:]).all() and torch.isfinite(s[3:]).all()


@pytest.mark.gpu
def test_norm_in_place_and_as_vectors(stb):
    x, r = _values(4, 640, 4, "f16").cuda(), _values(4, 640, 5, "f16").cuda()
    y, rr = stb.block_norm(x, residual=r)
    x2, r2 = x.clone(), r.clone()
    y2, rr2 = stb.block_norm(x2, residual=r2, out=x2, residual_out=r2)
    assert y2 is x2 and rr2 is r2 and torch.equal(x2, y) and torch.equal(r2, rr)
    y1, r1 = stb.block_norm(x[1], residual=r[1])
    assert y1.shape == (640,) and torch.equal(y1, y[1]) and torch.equal(r1, rr[1])
    q, s = torch.full((4, 656), 3, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    (q8, s8), _ = stb.block_norm(x, residual=r, out=(q[:, :640], s))
    (w8, v8), _ = stb.block_norm(x, residual=r, out_dtype=torch.int8)
    assert torch.equal(q8, w8) and torch.equal(s8, v8) and (q[:, 640:] == 3).all()
    for bad in (dict(weight=torch.zeros(639, dtype=torch.float16, device="cuda")), dict(residual=r[:3]), dict(gate=torch.zeros(3, 640, dtype=torch.float16, device="cuda")),
                dict(weight=torch.zeros(640, dtype=torch.float16, device="cuda"), bias=torch.zeros(640, device="cuda")), dict(out=torch.zeros(4, 641, device="cuda")[:, ::1]),
                dict(residual=r, residual_out=torch.zeros(4, 640, device="cuda")), dict(residual=r.cpu())):
        with pytest.raises(stb.StbError) as e:
            stb.block_norm(x, **bad)
        assert e.value.status == stb.STB_ERR_ARG


# ---- together ---------------------------------------------------------------------------------------------------------------------------
def _mlp(stb, x, r, weight, layers):
    """The MLP of a decoder block in 8 bits, up to the norm of the next block."""
    (g, gs), (u, us), (d, ds) = layers
    (xq, xs), r = stb.block_norm(x, weight, residual=r, out_dtype=torch.int8)
    gate, up = stb.gemm_i8(xq, xs, g, gs, out_dtype=torch.float16), stb.gemm_i8(xq, xs, u, us, out_dtype=torch.float16)
    hq, hs = stb.quantize_i8(gate, up)
    return stb.block_norm(stb.gemm_i8(hq, hs, d, ds, out_dtype=torch.float16), weight, residual=r)


@pytest.mark.gpu
@pytest.mark.parametrize("T", (1, 24, 270))
def test_an_mlp_in_8_bits(stb, T):
    h, f = 512, 1376
    x, r, weight = _values(T, h, 1, "f16").cuda(), _values(T, h, 2, "f16").cuda(), (1 + 0.1 * torch.randn(h, generator=_gen(3))).half().cuda()
    dense = [(torch.randn(*s, generator=_gen(4 + k)) * 0.04).half().cuda() for k, s in enumerate(((f, h), (f, h), (h, f)))]
    layers = [stb.quantize_i8(w) for w in dense]
    y, rr = _mlp(stb, x, r, weight, layers)
    # step by step from the GPU's own operands: each is what its definition makes of them
    (xq, xs), r1 = stb.block_norm(x, weight, residual=r, out_dtype=torch.int8)
    gate = _product(xq.cpu(), xs.cpu(), layers[0][0].cpu(), layers[0][1].cpu(), None, torch.float16)
    up = _product(xq.cpu(), xs.cpu(), layers[1][0].cpu(), layers[1][1].cpu(), None, torch.float16)
    hq, hs = stb.quantize_i8(gate.cuda(), up.cuda())
    _check_rows(hq, hs, _gated64(gate, up))
    down = _product(hq.cpu(), hs.cpu(), layers[2][0].cpu(), layers[2][1].cpu(), None, torch.float16)
    y2, rr2 = stb.block_norm(down.cuda(), weight, residual=r1)
    assert torch.equal(y, y2) and torch.equal(rr, rr2)
    # and the whole is the MLP of the dense weights, to what 8 bits leave of it: three products of operands within 1/254 of their rows' largest values
    n = torch.nn.functional.rms_norm(r1.double(), (h,), weight.double(), 1e-5)
    a = torch.nn.functional.silu(n @ dense[0].double().T) * (n @ dense[1].double().T)
    want = r1.double() + a @ dense[2].double().T
    assert (rr.double() - want).norm() <= 0.1 * (want - r1.double()).norm()
    # the norm's 16-bit output is what the structured-binary layers read
    import oracle
    import stb_inputs as si
    data = si.logical_layer(96, h, 4, 77)
    layer = stb.pack_numpy(data)
    rows = y[:8].contiguous()
    got = stb.gemv(layer, rows).double().cpu().numpy()
    ref = oracle.matmul(oracle.decode(oracle.Logical(**data)), rows.double().cpu().numpy())
    assert abs(got - ref).max() <= 5e-3 * abs(ref).max()


@pytest.mark.gpu
@pytest.mark.parametrize("T", (1, 24, 270))
def test_captured_replayed_and_on_another_stream(stb, T):
    h, f = 512, 1376
    weight = torch.ones(h, dtype=torch.float16, device="cuda")
    layers = [stb.quantize_i8((torch.randn(*s, generator=_gen(14 + k)) * 0.04).half().cuda()) for k, s in enumerate(((f, h), (f, h), (h, f)))]
    x, r = torch.zeros(T, h, dtype=torch.float16, device="cuda"), torch.zeros(T, h, dtype=torch.float16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _mlp(stb, x, r, weight, layers)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = _mlp(stb, x, r, weight, layers)
        graphs.append((g, out))
    for seed in range(3):
        x.copy_(_values(T, h, 20 + seed, "f16"))
        r.copy_(_values(T, h, 30 + seed, "f16"))
        want = _mlp(stb, x, r, weight, layers)
        for g, out in graphs:
            g.replay()
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    # two streams at once, each with its own tensors
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ins = [(_values(T, h, 40 + k, "f16").cuda(), _values(T, h, 50 + k, "f16").cuda()) for k in range(2)]
    wants = [_mlp(stb, a, b, weight, layers) for a, b in ins]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(_mlp(stb, *ins[k], weight, layers))
    torch.cuda.synchronize()
    for k in range(2):
        for a, b in got[k]:
            assert torch.equal(a, wants[k][0]) and torch.equal(b, wants[k][1])
    # the stream as an argument
    q, s = stb.quantize_i8(ins[0][0], stream=side)
    y = stb.gemm_i8(q, s, *layers[0], stream=side)
    n, _ = stb.block_norm(ins[0][0], weight, stream=side)
    side.synchronize()
    q2, s2 = stb.quantize_i8(ins[0][0])
    assert torch.equal(q, q2) and torch.equal(y, stb.gemm_i8(q2, s2, *layers[0])) and torch.equal(n, stb.block_norm(ins[0][0], weight)[0])


@pytest.mark.gpu
def test_the_native_and_the_python_forms_agree(stb):
    x, x2 = _values(9, 700, 1, "f16").cuda(), _values(9, 700, 2, "f16").cuda()
    w = _eight(40, 700, 3)
    wq, ws = _i8_place(w[0], 0), w[1].cuda()
    for args in ((x, None), (x, x2)):
        a, b = stb.quantize_i8(*args), stb._quantize_i8_py(*args)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[0].stride() == b[0].stride()
    xq, xs = stb.quantize_i8(x)
    assert torch.equal(stb.gemm_i8(xq, xs, wq, ws, out_dtype=torch.bfloat16), stb._gemm_i8_py(xq, xs, wq, ws, out_dtype=torch.bfloat16))
    one = torch.ones(700, dtype=torch.float16, device="cuda")
    for kw in (dict(weight=one), dict(weight=one, residual=x2, kind="layer"), dict(residual=x2, gate=one, alpha=0.5, post=True, out_dtype=torch.float32), dict(weight=one, out_dtype=torch.int8)):
        a, b = stb.block_norm(x, **kw), stb._block_norm_py(x, **kw)
        flat = lambda o: [t for v in o for t in (v if isinstance(v, tuple) else (v,)) if t is not None]  # noqa: E731
        assert len(flat(a)) == len(flat(b)) and all(torch.equal(p, q) and p.dtype == q.dtype for p, q in zip(flat(a), flat(b)))
