"""stb_block_norm in the forms that the C interface has beside those of the Python call: the residual alone, a residual without a residual input, none written back,
rows in 16 bits and in 8 at once.  Every output lies in a larger buffer that is compared too.  Bounds as in test_i8_norm.py (derived there)."""
import ctypes as C

import pytest
import torch

from test_i8_norm import DTYPES, U32, _block64, _gen, _half_step, _place, _values, stb  # noqa: F401

FORMS = {
    "residual alone": dict(resid=True, resid_out=True, post=True),
    "residual alone, in place": dict(resid=True, resid_out="in place"),
    "residual of nothing, alone": dict(resid_out=True),
    "residual of nothing": dict(resid_out=True, y=True, weight=True, gate=True),
    "residual not written": dict(resid=True, y=True, weight=True, post=True),
    "16 and 8 bits": dict(resid=True, resid_out=True, y=True, q=True, weight=True, bias=True, gate=True),
    "16 and 8 bits, nothing else": dict(y=True, q=True),
    "8 bits, residual not written": dict(resid=True, q=True, weight=True, post=True, gate=True),
    "16 bits in place": dict(y="in place", weight=True),
}


class _Out:
    """An output of T rows in a larger buffer: `pad` values between rows, `shift` before the first."""

    def __init__(self, T, h, dtype, pad, shift):
        self.fill = 55 if dtype == torch.int8 else 7.0
        self.buf = torch.full((T * (h + pad) + shift + 16,), self.fill, dtype=dtype, device="cuda")
        self.view = self.buf[shift:shift + T * (h + pad)].view(T, h + pad)[:, :h]

    def take(self):
        got = self.view.clone()
        self.view.fill_(self.fill)
        assert bool((self.buf == self.fill).all()), "around an output"
        return got


@pytest.mark.gpu
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("T, h", ((1, 40), (3, 1000), (400, 200), (400, 1000), (2, 4096), (400, 4096), (400, 1029), (2, 17000), (330, 12000), (150, 9001)))
def test_forms(stb, T, h, form):  # noqa: F811
    f = dict(dict(resid=False, resid_out=False, y=False, q=False, weight=False, bias=False, post=False, gate=False), **FORMS[form])
    for k, (xdt, rdt, wdt, ydt, kind) in enumerate((("f16", "f16", "f16", "f16", "rms"), ("bf16", "f32", "f32", "f32", "layer"), ("f32", "bf16", "bf16", "bf16", "rms"))):
        pad, shift = ((16, 16), (0, 0), (5, 3))[(k + T + h) % 3]
        if f["y"] == "in place":
            ydt = xdt
        seed = 7 * h + T + k
        x, r = _values(T, h, seed, xdt), _values(T, h, seed + 1, rdt, 3.0)
        vec = lambda j, one: (one + 0.3 * torch.randn(h, generator=_gen(seed + j))).to(DTYPES[wdt])  # noqa: E731
        weight, bias = vec(2, 1.0) if f["weight"] else None, vec(3, 0.0) if f["bias"] else None
        post_weight = vec(4, 1.0) if f["post"] else None
        gates = T // 2 if T % 2 == 0 and T > 2 else 1
        gate = torch.randn(gates, h, generator=_gen(seed + 5)).to(DTYPES[wdt]) if f["gate"] else None
        want_y, want_r, ey, er = _block64(x, weight, r if f["resid"] else None, bias, f["post"], post_weight, None, gate, 0.5, kind, 1e-5)
        code = {"f32": stb.STB_F32, "f16": stb.STB_F16, "bf16": stb.STB_BF16}
        dx, dr = _place(x, pad, shift), _place(r, pad, shift)
        held = [t.cuda() for t in (weight, bias, post_weight, gate) if t is not None]
        names = [n for n, t in zip(("weight", "bias", "post_weight", "gate"), (weight, bias, post_weight, gate)) if t is not None]
        a = stb._Norm(tokens=T, h=h, kind=stb.STB_NORM_RMS if kind == "rms" else stb.STB_NORM_LAYER, post=int(f["post"]), eps=1e-5, alpha=0.5, x=dx.data_ptr(), xdt=code[xdt],
                      ldx=h + pad, rdt=code[rdt], wdt=code[wdt], tokens_per_gate=T // gates, ldgate=h)
        for name, t in zip(names, held):
            setattr(a, name, t.data_ptr())
        if f["resid"]:
            a.resid, a.ldr = dr.data_ptr(), h + pad
        outs = {}
        if f["resid_out"] == "in place":
            a.resid_out, a.ldro = a.resid, a.ldr
        elif f["resid_out"]:
            outs["r"] = _Out(T, h, DTYPES[rdt], pad, shift)
            a.resid_out, a.ldro = outs["r"].view.data_ptr(), h + pad
        if f["y"] == "in place":
            a.y, a.ydt, a.ldy = a.x, code[xdt], h + pad
        elif f["y"]:
            outs["y"] = _Out(T, h, DTYPES[ydt], pad, shift)
            a.y, a.ydt, a.ldy = outs["y"].view.data_ptr(), code[ydt], h + pad
        scale = torch.full((T + 1,), 5.0, device="cuda")
        if f["q"]:
            outs["q"] = _Out(T, h, torch.int8, pad, shift)
            a.q, a.ldq, a.q_scale = outs["q"].view.data_ptr(), h + pad, scale.data_ptr()
        assert stb._lib.stb_block_norm(C.byref(a), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == stb.STB_OK
        torch.cuda.synchronize()
        got = {k: o.take() for k, o in outs.items()}
        if f["resid_out"] == "in place":
            got["r"] = dr
        if f["y"] == "in place":
            got["y"] = dx
        for name, want, err, dt in (("r", want_r, er, rdt), ("y", want_y, ey, ydt)):
            if name in got:
                t = DTYPES[dt]
                tiny = torch.finfo(t).smallest_normal * torch.finfo(t).eps
                off = (got[name].cpu().double() - want).abs()
                assert (off <= 1.001 * (err + _half_step(t) * (want.abs() + err)) + tiny).all(), (form, name, k)
        if f["q"]:
            assert scale[T] == 5.0
            s64, top = scale[:T].cpu().double(), want_y.abs().amax(1)
            assert ((s64 * 127 - top).abs() <= 1.001 * (ey.amax(1) + 2 * U32 * top)).all(), (form, "scale", k)
            assert ((got["q"].cpu().double() * s64[:, None] - want_y).abs() <= 1.0001 * (0.5 * s64[:, None] + ey) + 4 * U32 * top[:, None]).all(), (form, "q", k)


@pytest.mark.gpu
def test_rows_of_a_norm_in_8_bits_repeat_themselves(stb):  # noqa: F811
    """The same call gives the same bits, whatever ran between."""
    for T, h, kw in ((333, 8192, {}), (37, 5111, dict(kind="layer")), (1200, 1000, {})):
        x, other, w = _values(T, h, 1, "bf16").cuda(), _values(T, h, 2, "bf16").cuda(), (1 + 0.1 * torch.randn(h, generator=_gen(3))).bfloat16().cuda()
        (q, s), _ = stb.block_norm(x, w, out_dtype=torch.int8, **kw)
        for k in range(40):
            if k % 3 == 1:
                stb.block_norm(other, w, out_dtype=torch.int8, **kw)
            (q2, s2), _ = stb.block_norm(x, w, out_dtype=torch.int8, **kw)
            assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.gpu
def test_a_residual_to_write_to_without_one_to_read(stb):  # noqa: F811
    """The Python call: residual_out alone takes alpha times the block."""
    for T, h in ((1, 64), (5, 1500), (400, 2048)):
        x = _values(T, h, 9, "f16").cuda()
        out = torch.full((T, h), 7.0, device="cuda")
        y, r = stb.block_norm(x, alpha=0.25, residual_out=out)
        assert r is out and torch.equal(out, 0.25 * x.float())
        assert torch.equal(y, stb.block_norm(0.25 * x.float(), out_dtype=torch.float16)[0])
