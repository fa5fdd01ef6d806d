"""The 8-bit product of many tokens: the pair kernel (gemm_i8_prefill_kernel) through several tiles per pair of CTAs, with every width of a tile, every number of
32-token chunks behind the last token, channels on both sides of a CTA's 128, each type and both ways of storing, bit for bit against the definition in 64 bits.
Few columns keep the products short, so that one tile's stores are close behind the last one's."""
import os
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PAIRS = 74                                           # pairs of CTAs that the GPU holds at once
# (n, m, T)
SHAPES = ((1100, 128, 1500), (2100, 128, 1030), (1100, 128, 2050), (6016, 200, 777), (5000, 128, 705), (4232, 640, 2100), (2100, 200, 1537), (5003, 640, 900),
          (7040, 128, 705), (2300, 640, 2300), (8064, 128, 1300), (4992, 128, 2100), (7040, 200, 900), (4992, 128, 1800), (6016, 640, 1537), (5000, 200, 1537),
          (6016, 200, 1300), (4992, 640, 1500), (8064, 640, 777), (7040, 128, 2100), (4992, 128, 2300), (8064, 128, 1800), (8064, 128, 2300), (6016, 640, 1500),
          (6016, 640, 2100), (6016, 640, 2050))
LONGEST = (300, 131071, 710)                         # as many columns as are allowed


@pytest.fixture(scope="module")
def stb():
    from paper_2408_01803_b200 import build
    build.build()
    import paper_2408_01803_b200 as stb
    return stb


def test_these_shapes_reach_the_pair_kernel_in_every_form(tmp_path):
    """tests/host_i8_plan.cu: the library's own choice for them, so that another choice cannot take the kernel out of the tests below unseen."""
    exe = str(tmp_path / "host_i8_plan")
    subprocess.check_call([shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-o", exe,
                           os.path.join(ROOT, "tests", "host_i8_plan.cu")])
    out = subprocess.check_output([exe] + [str(v) for s in SHAPES + (LONGEST,) for v in s], text=True).split("\n")
    turns, widths, empty = set(), set(), set()
    for (n, m, T), line in zip(SHAPES + (LONGEST,), out):
        gemv, pair, bn, ttiles, _ = (int(v) for v in line.split())
        assert not gemv and pair, (n, m, T)
        if (n, m, T) == LONGEST:
            continue
        tiles = -(-n // 256) * ttiles
        assert tiles > PAIRS, (n, m, T)                      # some pair takes a second tile
        turns.add(-(-tiles // PAIRS))
        widths.add(bn)
        empty.add(bn // 32 - -(-(T - (ttiles - 1) * bn) // 32))
    assert widths == set(range(64, 257, 32)) and empty == set(range(8)) and {2, 3, 4} <= turns
    rest = {n % 256 for n, _, _ in SHAPES}
    assert 128 in rest and any(0 < r < 128 for r in rest) and any(r > 128 for r in rest)


def _eight(rows, m, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((rows, -(-m // 16) * 16), 99, dtype=torch.int8, device="cuda")
    buf[:, :m] = torch.randint(-128, 128, (rows, m), generator=g, dtype=torch.int8, device="cuda")
    return buf[:, :m], torch.rand(rows, generator=g, device="cuda") * 0.01 + 1e-4


def _same(a, b):
    return torch.equal(a, b) or (torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a, nan=0.0), torch.nan_to_num(b, nan=0.0)))


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dx%d_t%d" % s)
def test_product_of_many_tokens(stb, shape):
    n, m, T = shape
    xq, xs = _eight(T, m, n + T)
    wq, ws = _eight(n, m, n + T + 1)
    xs[T // 2] = float("nan")                                # a token without a scale
    bias = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(T), device="cuda")
    # an exact sum (whole numbers below 2^53 in any order), then one rounding to fp32 after each step
    scaled = torch.round(xq.double() @ wq.double().T).float().mul_(xs[:, None]).mul_(ws)
    for b in (None, bias):
        y32 = scaled if b is None else scaled + b
        for t in (torch.float32, torch.float16, torch.bfloat16):
            want = y32.to(t)
            calls = [stb.gemm_i8(xq, xs, wq, ws, bias=b, out_dtype=t) for _ in range(4)]
            for got in calls:
                assert _same(got, want), (shape, t, b is not None)
            # rows of a larger buffer: on 16-byte boundaries, and on none
            for pad, shift in ((32, 16), (-n % 2 + 5, 3)):
                ld = n + pad - (n % 16 if pad == 32 else 0)
                buf = torch.full((T * ld + 32,), 7.0, dtype=t, device="cuda")
                y = buf[shift:shift + T * ld].view(T, ld)[:, :n]
                stb.gemm_i8(xq, xs, wq, ws, bias=b, out=y)
                assert _same(y, want), (shape, t, b is not None, pad)
                y.fill_(7.0)
                assert bool((buf == 7.0).all()), (shape, t, "around the result")


@pytest.mark.gpu
@pytest.mark.parametrize("n", (1, 3, 7, 9, 130, 257, 263))
def test_few_channels_of_many_tokens_in_wider_rows(stb, n):
    """What lies beside the result in its rows stays as it is, wherever the last channel lies in a 16-byte piece."""
    m, T = 128, 1025
    xq, xs = _eight(T, m, n)
    wq, ws = _eight(n, m, n + 1)
    y32 = torch.round(xq.double() @ wq.double().T).float().mul_(xs[:, None]).mul_(ws)
    for t in (torch.float32, torch.float16, torch.bfloat16):
        buf = torch.full((T, 288), 7.0, dtype=t, device="cuda")
        stb.gemm_i8(xq, xs, wq, ws, out=buf[:, 16:16 + n])
        assert torch.equal(buf[:, 16:16 + n], y32.to(t))
        assert bool((buf[:, :16] == 7.0).all()) and bool((buf[:, 16 + n:] == 7.0).all()), t


@pytest.mark.gpu
def test_product_of_many_tokens_at_the_ends_of_its_range(stb):
    """Sums of the largest magnitude that int32 takes."""
    n, m, T = LONGEST
    x = torch.full((T, 131072), -128, dtype=torch.int8, device="cuda")[:, :m]
    w = torch.full((n, 131072), -128, dtype=torch.int8, device="cuda")[:, :m]
    w[1::2] = 127
    one = torch.ones(max(T, n), device="cuda")
    y = stb.gemm_i8(x, one[:T], w, one[:n])
    want = torch.tensor([128.0 * 128 * m, -128.0 * 127 * m], dtype=torch.float64).float().cuda().repeat(n // 2)
    assert torch.equal(y, want.expand(T, n))


@pytest.mark.gpu
def test_products_of_many_tokens_captured_replayed_and_side_by_side(stb):
    """Two graphs over the same weights, replayed on two streams at once with products of few tokens between them; inputs change between the replays."""
    n, m, T = 4232, 640, 2100
    wq, ws = _eight(n, m, 3)
    ins = [_eight(T, m, 10 + k) for k in range(2)]
    few = _eight(20, m, 30)
    want = lambda x, s: torch.round(x.double() @ wq.double().T).float().mul_(s[:, None]).mul_(ws)  # noqa: E731
    few_want = want(*few)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                            # (every kernel has run once before it is captured)
        stb.gemm_i8(*ins[0], wq, ws)
        stb.gemm_i8(*few, wq, ws)
    torch.cuda.synchronize()
    graphs = []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = [stb.gemm_i8(*ins[k], wq, ws) for _ in range(3)] + [stb.gemm_i8(*few, wq, ws)]
        graphs.append((g, out))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for seed in range(3):
        for k in range(2):
            x, s = _eight(T, m, 40 + 2 * seed + k)
            ins[k][0].copy_(x)
            ins[k][1].copy_(s)
        torch.cuda.synchronize()
        for _ in range(4):
            for (g, _), s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for k, (_, out) in enumerate(graphs):
            w = want(*ins[k])
            assert all(torch.equal(y, w) for y in out[:3]) and torch.equal(out[3], few_want)
