"""Layer norm and its gradients against the formula in 64 bits (tests/operators_ref.py), and against differences."""
import pytest
import torch

import operators_ref as ref
from paper_2410_20225_amd import tdf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = [(1, 1), (1, 5), (3, 8), (7, 64), (5, 63), (33, 65), (128, 512), (65, 300), (130, 128), (9, 1000), (17, 1024), (6, 2049), (5, 4096), (3, 8192), (2, 20000), (1, 70001), (1500, 40), (4099, 24), (2050, 512)]


def make(rows, cols, dtype, seed=0, gap=0, shift=0):
    """Values as a host's and the GPU's tensor; the GPU's rows are `gap` apart and begin `shift` elements after an aligned place."""
    g = torch.Generator().manual_seed(1000 * rows + cols + seed)
    x = (torch.randn(rows, cols, generator=g) * (0.5 + torch.rand(rows, 1, generator=g)) + torch.randn(rows, 1, generator=g)).to(dtype)
    wide = torch.full((rows * (cols + gap) + shift,), float("nan"), dtype=dtype, device=DEV)
    d = wide[shift:].view(rows, cols + gap)[:, :cols]
    d.copy_(x)
    return x, d


def vectors(cols, seed=1):
    g = torch.Generator().manual_seed(cols + seed)
    return 1 + 0.3 * torch.randn(cols, generator=g), 0.5 * torch.randn(cols, generator=g)


def forward(x, d, w, b, eps=1e-5, y=None):
    y = torch.empty_like(d, memory_format=torch.contiguous_format) if y is None else y
    mean, rstd = (torch.empty(d.shape[0], device=DEV) for _ in range(2))
    tdf.layer_norm(d, y, None if w is None else w.to(DEV), None if b is None else b.to(DEV), eps, mean, rstd)
    one, zero = torch.ones(d.shape[1]), torch.zeros(d.shape[1])
    want, wm, wr, e, em, er = ref.norm(x, (one if w is None else w).double(), (zero if b is None else b).double(), eps)
    ref.close(y, want, e + ref.half_step(d.dtype) * (want.abs() + e))
    ref.close(mean, wm, em)
    ref.close(rstd, wr, er)
    return y, mean, rstd


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, dtype):
    forward(*make(rows, cols, dtype), *vectors(cols))


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("gap,shift", [(8, 0), (3, 0), (0, 1), (64, 8), (5, 3)])
@pytest.mark.parametrize("cols", [48, 301, 512])
def test_rows_apart_and_places_that_are_not_aligned(cols, gap, shift, dtype):
    w, b = vectors(cols)
    x, d = make(37, cols, dtype, gap=gap, shift=shift)
    y = torch.full((37, cols + 7), -3.0, dtype=dtype, device=DEV)
    forward(x, d, w, b, y=y[:, :cols])
    assert torch.equal(y[:, cols:], torch.full_like(y[:, cols:], -3.0))
    gradient(x, d, w, gap=gap)
    off = torch.cat([torch.zeros(1), w]).to(DEV)[1:]             # vectors that begin four bytes after an aligned place
    got = torch.empty(37, cols, dtype=dtype, device=DEV)
    tdf.layer_norm(d, got, off, off)
    want = torch.empty_like(got)
    tdf.layer_norm(d.contiguous(), want, w.to(DEV), w.to(DEV))
    want, got = want.double().cpu(), got
    ref.close(got, want, 2 * ref.half_step(dtype) * want.abs() + 1e-4 * (want.abs() + 1))


@pytest.mark.parametrize("w,b", [(False, False), (True, False), (False, True)])
def test_without_weight_or_bias(w, b):
    weight, bias = vectors(300)
    forward(*make(20, 300, torch.bfloat16), weight if w else None, bias if b else None)


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("cols", [64, 300, 3001])
def test_in_place(cols, dtype):
    w, b = vectors(cols)
    x, d = make(12, cols, dtype)
    y, mean, rstd = forward(x, d, w, b)
    forward(x, d, w, b, y=d)                                     # y is x
    assert torch.equal(d, y)
    x, d = make(12, cols, dtype)
    dy = torch.randn(12, cols, device=DEV).to(dtype)
    want = grads(d, dy, mean, rstd, w.to(DEV))
    got = grads(d, dy, mean, rstd, w.to(DEV), dx=dy)             # dx is dy
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("offset", [1e3, 1e4])
def test_a_mean_far_from_zero_costs_no_variance(offset):
    # a variance from the mean of the squares would lose all its bits here
    x = (torch.randn(9, 700, generator=torch.Generator().manual_seed(3)) + offset)
    forward(x, x.to(DEV), *vectors(700))


def test_constant_rows_and_eps():
    x = torch.full((3, 100), 2.5)
    y, mean, rstd = forward(x, x.to(DEV), *vectors(100), eps=1e-3)
    x = torch.randn(3, 100, generator=torch.Generator().manual_seed(0))
    forward(x, x.to(DEV), *vectors(100), eps=0.0)


def test_values_that_are_not_finite_stay_in_their_rows():
    w, b = vectors(256)
    x, d = make(70, 256, torch.float32)
    x[3, 17], x[40, 0], x[69, 255] = float("nan"), float("inf"), float("-inf")
    d.copy_(x)
    y, mean, rstd = torch.empty_like(d), torch.empty(70, device=DEV), torch.empty(70, device=DEV)
    tdf.layer_norm(d, y, w.to(DEV), b.to(DEV), mean=mean, rstd=rstd)
    bad = torch.zeros(70, dtype=torch.bool)
    bad[[3, 40, 69]] = True
    assert torch.equal(torch.isfinite(y).all(1).cpu(), ~bad)
    good = ~bad
    want, _, _, e, _, _ = ref.norm(x[good], w.double(), b.double(), 1e-5)
    ref.close(y[good.to(DEV)], want, e)


def grads(d, dy, mean, rstd, w, dx=True, dw=True, db=True):
    rows, cols = d.shape
    dx = torch.empty(rows, cols, dtype=d.dtype, device=DEV) if dx is True else dx
    dw = torch.full((cols,), -9.0, device=DEV) if dw else None
    db = torch.full((cols,), -9.0, device=DEV) if db else None
    ws = torch.full((tdf.layer_norm_grad_workspace_size(rows, cols),), 255, dtype=torch.uint8, device=DEV)
    tdf.layer_norm_grad(d, dy, mean, rstd, dx, dw, db, ws, weight=w)
    return dx, dw, db


def gradient(x, d, w, gap=0):
    rows, cols = x.shape
    dy, ddy = make(rows, cols, x.dtype, seed=7, gap=gap)
    one = torch.ones(cols)
    _, mean, rstd, _, _, _ = ref.norm(x, one.double(), one.double(), 1e-5)
    mean, rstd = mean.float(), rstd.float()
    dx, dw, db = grads(d, ddy, mean.to(DEV), rstd.to(DEV), None if w is None else w.to(DEV))
    want = ref.norm_grad(x, dy, mean, rstd, (one if w is None else w).double())
    ref.close(dx, want[0], want[3] + ref.half_step(x.dtype) * (want[0].abs() + want[3]))
    ref.close(dw, want[1], want[4])
    ref.close(db, want[2], want[5])


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_gradient(rows, cols, dtype):
    x, d = make(rows, cols, dtype)
    gradient(x, d, vectors(cols)[0])


def test_gradient_without_weight():
    gradient(*make(40, 300, torch.float32), None)


def test_gradients_that_are_not_wanted():
    x, d = make(300, 96, torch.float32)
    w = vectors(96)[0].to(DEV)
    dy, mean, rstd = torch.randn_like(d), d.mean(1).contiguous(), torch.rand(300, device=DEV)
    dx, dw, db = grads(d, dy, mean, rstd, w)
    assert torch.equal(grads(d, dy, mean, rstd, w, dw=False, db=False)[0], dx)
    assert torch.equal(grads(d, dy, mean, rstd, w, dx=None, db=False)[1], dw)
    assert torch.equal(grads(d, dy, mean, rstd, w, dx=None, dw=False)[2], db)


def test_no_rows():
    e = torch.empty(0, 40, device=DEV)
    tdf.layer_norm(e, torch.empty_like(e))
    s = torch.empty(0, device=DEV)
    _, dw, db = grads(e, e, s, s, None)
    assert not dw.any() and not db.any()


def test_gradient_against_differences():
    g = torch.Generator().manual_seed(4)
    x, dy, way = (torch.randn(6, 50, generator=g, dtype=torch.float64).float() for _ in range(3))
    w, b = vectors(50)
    dirs = (way.double(), torch.randn(50, generator=g, dtype=torch.float64), torch.randn(50, generator=g, dtype=torch.float64))
    f = lambda k: (ref.norm(x.double() + k * dirs[0], w + k * dirs[1], b + k * dirs[2], 1e-5)[0] * dy).sum()  # noqa: E731
    slope = float(f(1e-5) - f(-1e-5)) / 2e-5
    _, mean, rstd = forward(x, x.to(DEV), w, b)
    dx, dw, db = grads(x.to(DEV), dy.to(DEV), mean, rstd, w.to(DEV))
    got = sum(float((a.cpu().double() * d).sum()) for a, d in zip((dx, dw, db), dirs))
    size = sum(float((a.cpu().double() * d).abs().sum()) for a, d in zip((dx, dw, db), dirs))
    assert abs(got - slope) <= 200 * ref.U * size + 1e-7 * size      # (gradients' roundings; the difference's third derivative)


def test_sums_over_rows_are_the_same_every_time():
    _, d = make(5000, 200, torch.bfloat16)
    dy, mean, rstd = torch.randn_like(d), torch.randn(5000, device=DEV), torch.rand(5000, device=DEV)
    first = grads(d, dy, mean, rstd, None)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(grads(d, dy, mean, rstd, None), first))


def test_rows_beyond_32_bits():
    far = 1 << 31
    buf = torch.empty(2 * far + 128, dtype=torch.bfloat16, device=DEV)       # 8.6 GB, of which three rows are touched
    d = buf.as_strided((3, 128), (far, 1))
    x, near = make(3, 128, torch.bfloat16)
    d.copy_(near)
    w, b = vectors(128)
    want, _, _ = forward(x, near, w, b)
    dy = torch.randn(3, 128, device=DEV).to(torch.bfloat16)
    mean, rstd = torch.randn(3, device=DEV), torch.rand(3, device=DEV)
    wants = grads(near, dy, mean, rstd, w.to(DEV))
    got = grads(d, dy, mean, rstd, w.to(DEV))
    assert all(torch.equal(a, b) for a, b in zip(got, wants))
    tdf.layer_norm(d, d, w.to(DEV), b.to(DEV))
    assert torch.equal(d, want)


def test_another_stream_and_a_graph():
    _, d = make(333, 300, torch.bfloat16)
    w, b = (v.to(DEV) for v in vectors(300))
    dy = torch.randn_like(d)
    y, mean, rstd = torch.empty_like(d), torch.empty(333, device=DEV), torch.empty(333, device=DEV)
    dx, dw, db = torch.empty_like(d), torch.empty(300, device=DEV), torch.empty(300, device=DEV)
    ws = torch.empty(tdf.layer_norm_grad_workspace_size(333, 300), dtype=torch.uint8, device=DEV)

    def both():
        tdf.layer_norm(d, y, w, b, mean=mean, rstd=rstd)
        tdf.layer_norm_grad(d, dy, mean, rstd, dx, dw, db, ws, weight=w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(4):
        d.copy_(torch.randn(333, 300, device=DEV, generator=torch.Generator(DEV).manual_seed(k)))
        both()
        want = [t.clone() for t in (y, mean, rstd, dx, dw, db)]
        for t in (y, mean, rstd, dx, dw, db):
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, mean, rstd, dx, dw, db), want))


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", [(65539, 24), (65537, 25), (65538, 96), (65539, 99), (16387, 300), (16385, 301), (16386, 700), (16387, 701), (4099, 1025),
                                       (4097, 1032), (4098, 1500), (4099, 1501), (4097, 2500)])
def test_rows_so_many_that_a_thread_has_several(rows, cols, dtype):
    """More than 4,096 workgroups: several rows of a thread, the last ones not there; rows at whole pieces of 16 bytes and at any element."""
    w, b = vectors(cols)
    x, d = make(rows, cols, dtype)
    y, mean, rstd = forward(x, d, w, b)
    assert torch.equal(forward(x, d, w, b, y=d)[0], y)               # in place
    if cols < 400:
        gradient(*make(rows, cols, dtype), w)


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("cols", [48, 301, 512, 3000, 9000])
def test_vectors_that_begin_four_bytes_after_an_aligned_place(cols, dtype):
    w, b = vectors(cols)
    x, d = make(37, cols, dtype)
    off_w, off_b = (torch.cat([torch.zeros(1), v]).to(DEV)[1:] for v in (w, b))
    y = torch.empty_like(d)
    tdf.layer_norm(d, y, off_w, off_b)
    want, _, _, e, _, _ = ref.norm(x, w.double(), b.double(), 1e-5)
    ref.close(y, want, e + ref.half_step(dtype) * (want.abs() + e))
    mean, rstd = torch.randn(37, device=DEV), torch.rand(37, device=DEV)
    dy = torch.randn_like(d)
    got = grads(d, dy, mean, rstd, off_w)
    want = ref.norm_grad(x, dy.cpu(), mean.cpu(), rstd.cpu(), w.double())
    ref.close(got[0], want[0], want[3] + ref.half_step(dtype) * (want[0].abs() + want[3]))
    ref.close(got[1], want[1], want[4])
    ref.close(got[2], want[2], want[5])
