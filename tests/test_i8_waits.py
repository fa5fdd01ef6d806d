"""Bounded waits of the 8-bit product: where one runs out, the call ends, says so, and leaves NaN in place of what it could not compute."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# (n, m, T, parts of K; 0: the pair kernel)
FORMS = ((16000, 512, 64, 1), (30000, 256, 40, 1), (4000, 4096, 100, 2), (300, 1000, 40, 4), (300, 20000, 20, 8), (300, 1000, 1025, 0), (5000, 200, 705, 0))


@pytest.fixture(scope="module")
def stb():
    from paper_2408_01803_b200 import build
    build.build()
    import paper_2408_01803_b200 as stb
    return stb


def test_these_shapes_reach_every_form(tmp_path):
    exe = str(tmp_path / "host_i8_plan")
    subprocess.check_call([shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-o", exe,
                           os.path.join(ROOT, "tests", "host_i8_plan.cu")])
    out = subprocess.check_output([exe] + [str(v) for f in FORMS for v in f[:3]], text=True).split("\n")
    for (n, m, T, parts), line in zip(FORMS, out):
        gemv, pair, _, _, lks = (int(v) for v in line.split())
        assert not gemv and pair == (parts == 0) and (pair or 1 << lks == parts), (n, m, T, line)


def test_the_selftest_refuses(stb):
    one = C.c_void_p(256)
    call = lambda n, T, st: stb._lib.stb_gemm_i8_wait_selftest(one, 64, one, None, n, 64, one, 64, one, T, one, stb.STB_F32, n, st, None)  # noqa: E731
    assert call(300, 40, None) == stb.STB_ERR_ARG
    assert call(0, 40, one) == stb.STB_ERR_SHAPE
    assert call(300, 1, one) == stb.STB_ERR_UNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("dt", (torch.float32, torch.float16, torch.bfloat16))
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "%dx%d_t%d" % f[:3])
def test_a_wait_that_runs_out_leaves_no_numbers(stb, form, dt):
    n, m, T, parts = form
    g = torch.Generator(device="cuda").manual_seed(n + T)
    rows = lambda r: torch.randint(-128, 128, (r, -(-m // 16) * 16), generator=g, dtype=torch.int8, device="cuda")[:, :m]  # noqa: E731
    xq, wq = rows(T), rows(n)
    xs, ws = (torch.rand(k, generator=g, device="cuda") * 0.01 + 1e-4 for k in (T, n))
    want = torch.round(xq.double() @ wq.double().T).float().mul_(xs[:, None]).mul_(ws).to(dt)
    y, status = torch.full((T, n), 7.0, dtype=dt, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    stb.gemm_i8_wait_selftest(xq, xs, wq, ws, y, status)
    torch.cuda.synchronize()
    assert int(status.item()) == stb.STB_ERR_TIMEOUT
    if parts or n < 1000:                                    # every result lacks a part of K, or its tile
        assert bool(torch.isnan(y).all())
    else:                                                    # the first tile of every pair of CTAs has come
        assert bool((torch.isnan(y) | (y == want)).all())
        assert torch.equal(y[:64, :256], want[:64, :256]) and bool(torch.isnan(y[-1, -1])) and 0 < int(torch.isnan(y).sum()) < y.numel()
    status.zero_()
    assert torch.equal(stb.gemm_i8(xq, xs, wq, ws, out_dtype=dt, dev_status=status), want)
    assert int(status.item()) == 0
