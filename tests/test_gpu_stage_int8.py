"""8-bit rows and their products.  Nothing here has a tolerance: the quantised values are exact quotients rounded once, the
sums are integers, and the two products by the scales are fp32 operations that numpy does the same way."""

import numpy as np
import pytest
import torch

from oracle import stage_oracle as so
from paper_2607_13332_b200 import binding
from paper_2607_13332_b200.stage_ops import int8_matmul, int8_quantize

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def expected(xq, xs, wq, ws, dtype):
    """The integer sums in 64 bits, then fp32 products and the rounding of the stored type."""
    total = (xq.double() @ wq.double().t()).cpu().numpy()          # whole numbers below 2^31: exact
    y = total.astype(np.float32) * xs.cpu().numpy()[:, None] * ws.cpu().numpy()[None, :]
    return torch.from_numpy(y).to(TORCH[dtype])


def same(a, b):
    a, b = a.cpu(), b.cpu()
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def operands(rng, n, inner, outer, x_pitch=None, w_pitch=None, x_at=0, w_at=0):
    """int8 operands over the whole range at given leading dimensions and byte offsets, surrounded by other values."""
    def one(rows, pitch, at):
        buf = torch.from_numpy(rng.integers(-128, 128, rows * pitch + at + 32).astype(np.int8)).cuda()
        return buf[at:at + rows * pitch].view(rows, pitch)[:, :inner]
    xq, wq = one(n, x_pitch or -(-inner // 16) * 16, x_at), one(outer, w_pitch or -(-inner // 16) * 16, w_at)
    xs = torch.from_numpy(rng.uniform(0.001, 0.1, n).astype(np.float32)).cuda()
    ws = torch.from_numpy(rng.uniform(0.001, 0.1, outer).astype(np.float32)).cuda()
    return xq, xs, wq, ws


@pytest.mark.parametrize("rows,cols,pitch,at", [(1, 4096, None, 0), (3, 1, None, 0), (5, 7, 9, 1), (33, 2000, 2000, 0), (17, 2001, 2001, 3),
                                                (700, 128, 136, 8), (2, 70001, 70001, 0), (2, 131072, None, 0), (64, 16, None, 0),
                                                (5, 5120, 5128, 4), (1200, 511, 512, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize(rows, cols, pitch, at, dtype):
    rng = np.random.default_rng(rows + cols)
    pitch = pitch or cols
    buf = torch.full((rows * pitch + at + 8,), float("nan"), dtype=TORCH[dtype], device="cuda")
    x = buf[at:at + rows * pitch].view(rows, pitch)[:, :cols]
    x.copy_(torch.from_numpy((rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-8, 8, (rows, 1)))).astype(np.float32)))
    q, scale = int8_quantize(x)
    want, want_scale = so.int8_quantize(x.double().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), want_scale) and np.array_equal(q.cpu().numpy(), want)
    # into a buffer of the caller's, at an odd place
    out = torch.full((rows * (cols + 3) + 7,), 55, dtype=torch.int8, device="cuda")
    view = out[5:5 + rows * (cols + 3)].view(rows, cols + 3)[:, :cols]
    int8_quantize(x, q=view)
    assert np.array_equal(view.cpu().numpy(), want)
    view.fill_(55)
    assert bool((out == 55).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_halves_and_neighbours(dtype):
    """Quotients at and right beside every half: scale 1 (largest value 127), and scales that are no power of two."""
    halves = np.arange(-126.5, 127, 1.0)
    rows = []
    for top in (127.0, 127.0 * 3, 100.0, 0.9990234375, 5.0e-5):
        s = float(np.float32(np.float32(top) / np.float32(127)))
        base = (halves * s).astype(np.float32)
        for step in (0, 1, -1, 2, -2):
            v = base.copy()
            for _ in range(abs(step)):
                v = np.nextafter(v, np.float32(np.inf if step > 0 else -np.inf))
            rows.append(np.concatenate((v, [np.float32(top)])))
    x = torch.from_numpy(np.stack(rows).astype(np.float32)).to(TORCH[dtype]).cuda()
    q, scale = int8_quantize(x)
    want, want_scale = so.int8_quantize(x.double().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), want_scale) and np.array_equal(q.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [40, 5000])
def test_quantize_odd_rows(dtype, cols):
    """Zeros, infinities, NaN, the largest and the smallest values."""
    rng = np.random.default_rng(cols)
    x = torch.from_numpy(rng.standard_normal((9, cols)).astype(np.float32)).to(TORCH[dtype]).cuda()
    big = torch.finfo(TORCH[dtype]).max
    x[0] = 0.0
    x[1, cols // 2] = float("inf")
    x[2, cols - 1] = float("nan")
    x[3, 3] = float("-inf")
    x[4] *= 1e-38
    x[5] *= 1e-42
    x[6, :] = 0.0
    x[6, 7] = -1e-45
    x[7, 1], x[7, 2] = big, -big
    q, scale = int8_quantize(x)
    want, want_scale = so.int8_quantize(x.double().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), want_scale, equal_nan=True) and np.array_equal(q.cpu().numpy(), want)
    assert not bool(q[0].any()) and bool(scale[1:4].isnan().all()) and float(scale[0]) == 0


SIZES = [(1, 64, 16), (1, 4096, 4096), (2, 100, 33), (7, 2048, 1000), (16, 4096, 515), (17, 129, 300), (33, 2000, 64), (64, 4096, 4099),
         (100, 48, 50), (128, 128, 256), (129, 144, 257), (200, 2048, 1030), (257, 512, 513), (777, 2000, 503), (1000, 1040, 2000), (300, 16, 16),
         (5, 1, 3), (1, 1, 1), (640, 4096, 768), (2100, 640, 530), (3, 131071, 70)]


@pytest.mark.parametrize("n,inner,outer", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_matmul(n, inner, outer, dtype):
    rng = np.random.default_rng(n + inner + outer)
    xq, xs, wq, ws = operands(rng, n, inner, outer)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = int8_matmul(xq, xs, wq, ws, dtype, dev_status=status)
    assert int(status) == 0 and same(got, expected(xq, xs, wq, ws, dtype))
    # between rows of a wider buffer
    wide = torch.full((n + 2, outer + 5), 99.0, dtype=TORCH[dtype], device="cuda")
    view = wide[1:n + 1, 2:outer + 2]
    int8_matmul(xq, xs, wq, ws, dtype, out=view)
    assert torch.equal(view, got)
    view.fill_(99.0)
    assert bool((wide == 99.0).all())
    # and in wide rows that keep 16-byte boundaries
    wide = torch.full((n, -(-outer // 8) * 8 + 16), 99.0, dtype=TORCH[dtype], device="cuda")
    int8_matmul(xq, xs, wq, ws, dtype, out=wide[:, :outer])
    assert torch.equal(wide[:, :outer], got) and bool((wide[:, outer:] == 99.0).all())


@pytest.mark.parametrize("x_pitch,w_pitch,x_at,w_at", [(2001, 2001, 0, 0), (2016, 2001, 0, 0), (2001, 2016, 0, 0), (2016, 2016, 8, 0), (2016, 2016, 0, 1),
                                                       (2008, 2012, 4, 2), (2048, 2032, 16, 32)])
@pytest.mark.parametrize("n,outer", [(1, 77), (20, 300), (150, 260), (400, 520)])
def test_matmul_alignment(x_pitch, w_pitch, x_at, w_at, n, outer):
    rng = np.random.default_rng(x_pitch + w_at + n)
    xq, xs, wq, ws = operands(rng, n, 2001 if min(x_pitch, w_pitch) > 2000 else 1990, outer, x_pitch, w_pitch, x_at, w_at)
    assert same(int8_matmul(xq, xs, wq, ws, "bf16"), expected(xq, xs, wq, ws, "bf16"))


@pytest.mark.parametrize("n", [1, 40, 300])
def test_matmul_extremes(n):
    """The largest sums there are, and scales of 0, NaN and infinity."""
    inner, outer = 131071, 260
    xq = torch.full((n, 131072), -128, dtype=torch.int8, device="cuda")[:, :inner]
    wq = torch.full((outer, 131072), -128, dtype=torch.int8, device="cuda")[:, :inner]
    wq[1::2] = 127
    xs, ws = torch.ones(n, device="cuda"), torch.ones(outer, device="cuda")
    ws[3], ws[4], ws[5] = 0.0, float("nan"), float("inf")
    xs[n - 1] = float("nan") if n > 1 else 1e-30
    got = int8_matmul(xq, xs, wq, ws, "f32")
    assert same(got, expected(xq, xs, wq, ws, "f32"))
    assert float(got[0, 0] / xs[0]) == 2.0 ** 14 * inner or n == 1


def test_matmul_far_offsets():
    """Leading dimensions past 32 bits: operands, output."""
    rng = np.random.default_rng(1)
    far = 2 ** 31 + 16
    buf = torch.empty(far + 4096, dtype=torch.int8, device="cuda")
    xq, xs, wq, ws = operands(rng, 2, 512, 2)
    want = expected(xq, xs, wq, ws, "bf16")
    xf, wf = buf.as_strided((2, 512), (far, 1)), buf.as_strided((2, 512), (far, 1), 1024)
    xf.copy_(xq)
    wf.copy_(wq)
    assert same(int8_matmul(xf, xs, wf, ws, "bf16"), want)
    out = torch.empty(far + 16, dtype=torch.bfloat16, device="cuda").as_strided((2, 2), (far, 1))
    int8_matmul(xf, xs, wf, ws, "bf16", out=out)
    assert same(out, want)


def test_many_tokens():
    """More rows than fit 16 bits of tiles, one channel block."""
    rng = np.random.default_rng(2)
    xq, xs, wq, ws = operands(rng, 70000, 64, 24)
    assert same(int8_matmul(xq, xs, wq, ws, "bf16"), expected(xq, xs, wq, ws, "bf16"))


@pytest.mark.parametrize("n", [1, 48, 400])
def test_captured_and_on_two_streams(n):
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((n, 1024)).astype(np.float32)).cuda().bfloat16()
    _, _, wq, ws = operands(rng, 1, 1024, 1500)
    want = int8_matmul(*int8_quantize(x), wq, ws)
    graphs, got = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(int8_matmul(*int8_quantize(x), wq, ws))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for t in got:
            t.fill_(-3.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, want) for t in got)


def test_queued_calls_repeat():
    """Many calls of changing sizes without a wait in between: every one gives what it gave alone."""
    rng = np.random.default_rng(4)
    sets = [operands(rng, *s) for s in ((300, 2048, 1000), (1, 2048, 1000), (64, 512, 4000), (513, 1024, 300))]
    want = [int8_matmul(*s) for s in sets]
    torch.cuda.synchronize()
    outs = [[int8_matmul(*s) for s in sets] for _ in range(200)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got in outs for a, b in zip(got, want))


def test_python_refusals():
    rng = np.random.default_rng(5)
    xq, xs, wq, ws = operands(rng, 4, 64, 32)
    assert int8_matmul(xq[:0], xs[:0], wq, ws).shape == (0, 32) and int8_matmul(xq, xs, wq[:0], ws[:0]).shape == (4, 0)
    assert int8_quantize(torch.zeros(0, 64, device="cuda"))[0].shape == (0, 64)
    for bad in ((xq[:, :32], xs, wq, ws), (xq.short(), xs, wq, ws), (xq, xs.double(), wq, ws), (xq, xs, wq, ws[:5]), (xq.t(), xs, wq, ws), (xq.cpu(), xs, wq, ws)):
        with pytest.raises(ValueError):
            int8_matmul(*bad)
    for out in (torch.empty(4, 32, device="cuda"), torch.empty(4, 31, dtype=torch.bfloat16, device="cuda")):
        with pytest.raises(ValueError):
            int8_matmul(xq, xs, wq, ws, out=out)
    for bad in (torch.zeros(4, 64, device="cuda").half(), torch.zeros(64, 4, device="cuda").t(), torch.zeros(4, 64)):
        with pytest.raises(ValueError):
            int8_quantize(bad)
    with pytest.raises(ValueError):
        int8_quantize(torch.zeros(4, 64, device="cuda"), q=torch.zeros(4, 63, dtype=torch.int8, device="cuda"))
    with pytest.raises(binding.SsnError):
        int8_quantize(torch.zeros(4, 0, device="cuda"))
