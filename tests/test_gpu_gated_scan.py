"""The gated linear recurrence, its gradients and its single step against the formula in 64 bits, row after row
(tests/operators_ref.py), and against differences."""
import pytest
import torch

import operators_ref as ref
from paper_2410_20225_amd import tdf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# lengths of sequences, columns: one row, empty sequences at every place, lengths around the tiles' of 16, 64, 128 and 256 rows, long ones
CASES = [([1], 1), ([0], 5), ([0, 0, 3, 0], 7), ([5], 64), ([1, 1, 1, 1], 300), ([64, 63, 65, 1], 48), ([127, 0, 128, 129], 20), ([255, 1, 256, 0, 257], 64),
         ([700], 33), ([1000, 0, 24], 8), ([3] * 100, 16), ([0] * 70 + [9] + [0] * 70 + [200], 12), ([16, 16, 16, 15, 17], 130), ([4500], 4), ([2, 3000, 1], 72),
         ([1] * 300, 260), ([40] * 30, 516)]


def make(lengths, cols, dtype, seed=0, before=0, after=0, packed=False, shift=0, slow=0.0):
    """f, x, h0 on the host and the GPU, offsets; `before` and `after` rows belong to no sequence and hold NaN."""
    g = torch.Generator().manual_seed(cols + 7 * len(lengths) + seed)
    n = sum(lengths)
    rows = n + before + after
    f = (1 + slow + 2 * torch.randn(rows, cols, generator=g) + 2 * torch.randn(1, cols, generator=g)).to(dtype)
    x = torch.randn(rows, cols, generator=g).to(dtype)
    h0 = torch.randn(len(lengths), cols, generator=g)
    for t in (f, x):
        t[:before], t[before + n:] = float("nan"), float("nan")
    offsets = [before]
    for l in lengths:
        offsets.append(offsets[-1] + l)
    if packed:
        wide = torch.zeros(rows * 2 * cols + shift, dtype=dtype, device=DEV)[shift:].view(rows, 2 * cols)
        df, dx = wide[:, :cols], wide[:, cols:]
        df.copy_(f)
        dx.copy_(x)
    else:
        df, dx = f.to(DEV), x.to(DEV)
    return f, x, h0, offsets, df, dx


def space(rows, cols):
    return torch.full((tdf.gated_scan_workspace_size(rows, cols),), 255, dtype=torch.uint8, device=DEV)


def forward(f, x, h0, offsets, df, dx, zeros=False, none=False):
    rows, cols = f.shape
    h = torch.full((rows, cols), -7.0, dtype=f.dtype, device=DEV)
    last = torch.full((len(offsets) - 1, cols), -7.0, device=DEV)
    off = None if none else torch.tensor(offsets, dtype=torch.int64, device=DEV)
    tdf.gated_scan(df, dx, h, space(rows, cols), off, None if zeros else h0.to(DEV), last)
    want, w_last, e, e_last = ref.scan(f, x, offsets, torch.zeros_like(h0) if zeros else h0)
    a, b = offsets[0], offsets[-1]
    ref.close(h[a:b], want[a:b], (e + ref.half_step(f.dtype) * (want.abs() + e))[a:b])
    assert (h[:a] == -7).all() and (h[b:] == -7).all()
    ref.close(last, w_last, e_last)
    return h, last


def backward(f, x, h0, offsets, df, dx, zeros=False, no_dh=False, no_last=False, packed=False, none=False):
    rows, cols = f.shape
    g = torch.Generator().manual_seed(rows + cols)
    a, b = offsets[0], offsets[-1]
    h = ref.scan(f, x, offsets, torch.zeros_like(h0) if zeros else h0)[0].to(f.dtype)
    dh = torch.randn(rows, cols, generator=g).to(f.dtype)
    dh[:a], dh[b:], h[:a], h[b:] = (float("nan"),) * 4
    dlast = torch.randn(h0.shape, generator=g)
    if packed:
        wide = torch.full((rows, 2 * cols), -7.0, dtype=f.dtype, device=DEV)
        gf, gx = wide[:, :cols], wide[:, cols:]
    else:
        gf, gx = (torch.full((rows, cols), -7.0, dtype=f.dtype, device=DEV) for _ in range(2))
    dh0 = torch.full(h0.shape, -7.0, device=DEV)
    off = None if none else torch.tensor(offsets, dtype=torch.int64, device=DEV)
    tdf.gated_scan_grad(df, dx, h.to(DEV), None if no_dh else dh.to(DEV), gf, gx, space(rows, cols), off, None if zeros else h0.to(DEV),
                        None if no_last else dlast.to(DEV), dh0)
    want = ref.scan_grad(f, x, h, torch.zeros_like(dh) if no_dh else dh, offsets, torch.zeros_like(h0) if zeros else h0,
                         torch.zeros_like(dlast) if no_last else dlast)
    for got, w, e in ((gf, want[0], want[3]), (gx, want[1], want[4])):
        ref.close(got[a:b], w[a:b], (e + ref.half_step(f.dtype) * (w.abs() + e))[a:b])
        assert (got[:a] == -7).all() and (got[b:] == -7).all()
    ref.close(dh0, want[2], want[5])


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("lengths,cols", CASES, ids=lambda v: str(v)[:24])
def test_forward(lengths, cols, dtype):
    forward(*make(lengths, cols, dtype))


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("lengths,cols", CASES, ids=lambda v: str(v)[:24])
def test_gradient(lengths, cols, dtype):
    backward(*make(lengths, cols, dtype))


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("lengths,cols", [([4500], 4), ([2, 3000, 1], 72)], ids=lambda v: str(v)[:24])
def test_gates_that_keep_a_state_for_thousands_of_rows(lengths, cols, dtype):
    args = make(lengths, cols, dtype, slow=9.0)
    forward(*args)
    backward(*args)


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("cols,shift", [(64, 0), (300, 0), (37, 0), (64, 1), (128, 4)])
def test_halves_of_a_projection(cols, shift, dtype):
    args = make([5, 0, 150, 70], cols, dtype, packed=True, shift=shift)
    forward(*args)
    backward(*args, packed=True)


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("before,after", [(1, 0), (0, 3), (70, 200), (300, 300)])
def test_rows_of_no_sequence(before, after, dtype):
    args = make([9, 0, 160], 24, dtype, before=before, after=after)
    forward(*args)
    backward(*args)


@pytest.mark.parametrize("zeros,no_dh,no_last", [(True, False, False), (False, True, False), (False, False, True), (True, True, False)])
def test_arguments_left_out(zeros, no_dh, no_last):
    args = make([100, 0, 40], 40, torch.float32)
    forward(*args, zeros=zeros)
    backward(*args, zeros=zeros, no_dh=no_dh, no_last=no_last)
    one = make([140], 40, torch.float32)
    forward(*one, none=True)
    backward(*one, none=True)
    tdf.gated_scan(one[4], one[5], torch.empty_like(one[4]), space(140, 40))


def test_states_in_neighbouring_buffers():
    f, x, h0, offsets, df, dx = make([30, 0, 200], 40, torch.float32)
    off, ws, h = torch.tensor(offsets, device=DEV), space(230, 40), torch.empty_like(df)
    both = torch.empty(3, 3, 40, device=DEV)                     # h0, h_last and dh0 beside each other
    both[0].copy_(h0)
    tdf.gated_scan(df, dx, h, ws, off, both[0], both[1])
    tdf.gated_scan_grad(df, dx, h, None, torch.empty_like(df), torch.empty_like(df), ws, off, both[0], both[1], both[2])
    apart = torch.empty(3, 40, device=DEV)
    tdf.gated_scan(df, dx, h, ws, off, h0.to(DEV), apart)
    assert torch.equal(both[1], apart) and torch.equal(both[0].cpu(), h0)
    with pytest.raises(tdf.TdfError, match="h_last overlaps h0"):
        tdf.gated_scan(df, dx, h, ws, off, both[0], both[0])
    with pytest.raises(tdf.TdfError, match="dh0 overlaps dh_last"):
        tdf.gated_scan_grad(df, dx, h, None, torch.empty_like(df), torch.empty_like(df), ws, off, both[0], both[1], both[1])


@pytest.mark.parametrize("rows", [60, 140, 700])
@pytest.mark.parametrize("cols", [32, 37])
@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
def test_the_distance_of_rows_that_are_not_given_does_not_matter(dtype, cols, rows):
    f, x, h0, _, df, dx = make([rows], cols, dtype)
    h = torch.empty_like(df)
    tdf.gated_scan(df, dx, h, space(rows, cols), h0=h0.to(DEV))
    last, ws = torch.randn(1, cols, device=DEV), space(rows, cols)
    got = []
    for ld in (0, -1, 3, 1 << 20, 1 << 31, 1 << 62, -(1 << 40)):
        gf, gx, dh0 = torch.empty_like(df), torch.empty_like(df), torch.empty_like(last)
        in_ = tdf.Scan(rows, cols, 1, tdf._DTYPES[dtype], df.data_ptr(), cols, dx.data_ptr(), cols, None, None)
        grads = tdf.ScanGrads(h.data_ptr(), cols, None, ld, last.data_ptr(), gf.data_ptr(), cols, gx.data_ptr(), cols, dh0.data_ptr())
        assert tdf.lib.tdf_gated_scan_grad(in_, grads, ws.data_ptr(), ws.nbytes, tdf._stream_of(0)) == tdf.OK
        got.append((gf, gx, dh0))
    want = ref.scan_grad(f, x, h.cpu(), torch.zeros(rows, cols, dtype=dtype), [0, rows], torch.zeros_like(h0), last.cpu())
    for g, w, e in zip(got[0][:2], want[:2], want[3:5]):
        ref.close(g, w, e + ref.half_step(dtype) * (w.abs() + e))
    ref.close(got[0][2], want[2], want[5])
    assert all(torch.equal(a, b) for k in got[1:] for a, b in zip(k, got[0]))


def test_no_rows():
    e = torch.empty(0, 6, device=DEV)
    off, h0 = torch.zeros(4, dtype=torch.int64, device=DEV), torch.randn(3, 6, device=DEV)
    last, dh0 = torch.empty(3, 6, device=DEV), torch.empty(3, 6, device=DEV)
    tdf.gated_scan(e, e, torch.empty_like(e), space(0, 6), off, h0, last)
    assert torch.equal(last, h0)
    tdf.gated_scan_grad(e, e, e, None, torch.empty_like(e), torch.empty_like(e), space(0, 6), off, h0, h0, dh0)
    assert torch.equal(dh0, h0)


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
def test_values_that_are_not_finite_stay_in_their_sequences_and_columns(dtype):
    lengths = [30, 200, 30, 0, 300]
    f, x, h0, offsets, df, dx = make(lengths, 20, dtype)
    clean = forward(f, x, h0, offsets, df, dx)
    x[100, 3], x[259, 5], h0[0, 7] = float("nan"), float("inf"), float("nan")
    dx.copy_(x)
    h = torch.zeros_like(df)
    last = torch.zeros_like(h0, device=DEV)
    tdf.gated_scan(df, dx, h, space(560, 20), torch.tensor(offsets, device=DEV), h0.to(DEV), last)
    bad = torch.zeros(560, 20, dtype=torch.bool)
    bad[100:230, 3], bad[259, 5], bad[:30, 7] = True, True, True
    assert torch.equal(torch.isfinite(h).cpu(), ~bad)                       # for all rows after it, to the end of the sequence, however long
    assert torch.equal(h[~bad.to(DEV)], clean[0][~bad.to(DEV)])
    # and the gradients, towards earlier rows
    dh = torch.randn(560, 20).to(dtype)
    dh[150, 2] = float("nan")
    gf, gx, dh0 = torch.zeros_like(df), torch.zeros_like(df), torch.zeros_like(last)
    f, x, h0, offsets, df, dx = make(lengths, 20, dtype)
    tdf.gated_scan_grad(df, dx, clean[0], dh.to(DEV), gf, gx, space(560, 20), torch.tensor(offsets, device=DEV), h0.to(DEV), None, dh0)
    bad = torch.zeros(560, 20, dtype=torch.bool)
    bad[30:151, 2] = True
    assert torch.equal(torch.isfinite(gx).cpu(), ~bad) and torch.equal(torch.isfinite(gf).cpu(), ~bad)
    assert torch.equal(torch.isnan(dh0).nonzero().cpu(), torch.tensor([[1, 2]]))


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
def test_gates_at_their_ends(dtype):
    # closed (f = -inf: h = x), open (f = inf: h stays), and far out on either side
    f, x, h0, offsets, df, dx = make([40, 90], 12, dtype)
    f[::5], f[1::5], f[2::7], f[3::7] = float("inf"), float("-inf"), 90.0, -90.0
    df.copy_(f)
    h = torch.empty_like(df)
    tdf.gated_scan(df, dx, h, space(130, 12), torch.tensor(offsets, device=DEV), h0.to(DEV))
    want, _, e, _ = ref.scan(f, x, offsets, h0)
    ref.close(h, want, e + 1e-30 + ref.half_step(dtype) * (want.abs() + e))      # (gates below 1e-38 may be zero)


def test_gradient_against_differences():
    lengths, cols = [3, 0, 9], 11
    f, x, h0, offsets, df, dx = make(lengths, cols, torch.float32)
    g = torch.Generator().manual_seed(2)
    dh, dlast = torch.randn(12, cols, generator=g), torch.randn(3, cols, generator=g)
    ways = [torch.randn(t.shape, generator=g, dtype=torch.float64) for t in (f, x, h0)]

    def value(k):
        h, last, _, _ = ref.scan(f.double() + k * ways[0], x.double() + k * ways[1], offsets, h0.double() + k * ways[2])
        return (h * dh).sum() + (last * dlast).sum()
    slope = float(value(1e-5) - value(-1e-5)) / 2e-5
    h = torch.empty_like(df)
    off = torch.tensor(offsets, device=DEV)
    tdf.gated_scan(df, dx, h, space(12, cols), off, h0.to(DEV))
    gf, gx, dh0 = torch.empty_like(df), torch.empty_like(df), torch.empty(3, cols, device=DEV)
    tdf.gated_scan_grad(df, dx, h, dh.to(DEV), gf, gx, space(12, cols), off, h0.to(DEV), dlast.to(DEV), dh0)
    parts = [t.cpu().double() * w for t, w in zip((gf, gx, dh0), ways)]
    assert abs(sum(float(p.sum()) for p in parts) - slope) <= (300 * ref.U + 1e-7) * sum(float(p.abs().sum()) for p in parts)


def test_the_same_every_time():
    f, x, h0, offsets, df, dx = make([1000, 2500, 3, 800], 260, torch.bfloat16)
    off, ws = torch.tensor(offsets, device=DEV), space(4303, 260)
    dh = torch.randn_like(df)
    got = []
    for _ in range(6):
        h, last, gf, gx, dh0 = torch.empty_like(df), torch.empty(4, 260, device=DEV), torch.empty_like(df), torch.empty_like(df), torch.empty(4, 260, device=DEV)
        tdf.gated_scan(df, dx, h, ws, off, h0.to(DEV), last)
        tdf.gated_scan_grad(df, dx, h, dh, gf, gx, ws, off, h0.to(DEV), last, dh0)
        got.append((h, last, gf, gx, dh0))
    assert all(torch.equal(a, b) for k in got[1:] for a, b in zip(k, got[0]))


def test_offsets_out_of_order_touch_nothing_else():
    rows, cols = 600, 16
    f, x, h0, _, df, dx = make([rows], cols, torch.float32)
    guard = torch.full((rows + 400, cols), -7.0, device=DEV)
    h = guard[200:200 + rows]
    for offsets in ([500, 100, 600, 300], [-50, 10, 900, 700], [600, 600, 0, 0], [0, 1 << 40, -(1 << 40), 600]):
        off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
        last = torch.empty(3, cols, device=DEV)
        tdf.gated_scan(df, dx, h, space(rows, cols), off, torch.randn(3, cols, device=DEV), last)
        tdf.gated_scan_grad(df, dx, dx, df, h, torch.empty_like(df), space(rows, cols), off, last, last, torch.empty_like(last))
        torch.cuda.synchronize()
        assert (guard[:200] == -7).all() and (guard[200 + rows:] == -7).all()


def test_rows_beyond_32_bits():
    ld, rows, cols = 1 << 26, 70, 40
    buf = torch.empty(rows * ld, dtype=torch.bfloat16, device=DEV)                  # 9.4 GB, of which 70 rows are touched
    f, x, h0, offsets, df, dx = make([30, 40], cols, torch.bfloat16)
    ff, xx = buf.as_strided((rows, cols), (ld, 1)), buf.as_strided((rows, cols), (ld, 1), 1 << 20)
    hh = buf.as_strided((rows, cols), (ld, 1), 1 << 21)
    ff.copy_(df)
    xx.copy_(dx)
    h, _ = forward(f, x, h0, offsets, df, dx)
    off = torch.tensor(offsets, device=DEV)
    tdf.gated_scan(ff, xx, hh, space(rows, cols), off, h0.to(DEV))
    assert torch.equal(hh, h)
    want = [torch.empty_like(df) for _ in range(2)]
    tdf.gated_scan_grad(df, dx, h, df, *want, space(rows, cols), off, h0.to(DEV))
    gf, gx = (buf.as_strided((rows, cols), (ld, 1), k << 22) for k in (1, 2))
    tdf.gated_scan_grad(ff, xx, hh, ff, gf, gx, space(rows, cols), off, h0.to(DEV))
    assert torch.equal(gf, want[0]) and torch.equal(gx, want[1])


# ---- single rows --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("rows,cols,states,packed", [(1, 1, 1, False), (1, 512, 4, False), (5, 300, 9, True), (64, 64, 64, False), (33, 37, 100, True), (256, 512, 1024, False), (3, 4100, 3, True)])
def test_step(rows, cols, states, packed, dtype):
    f, x, _, _, df, dx = make([rows], cols, dtype, packed=packed)
    g = torch.Generator().manual_seed(rows)
    state = torch.randn(states, cols, generator=g)
    slot = torch.randperm(states, generator=g)[:rows].to(torch.int32)
    if rows > 4:
        slot[2], slot[4] = -1, states            # nobody's place, and one that is not in the table
    d_state, h = state.to(DEV), torch.full((rows, cols), -7.0, dtype=dtype, device=DEV)
    tdf.gated_scan_step(df, dx, d_state, h, slot.to(DEV))
    want, e = state.double().clone(), torch.zeros(states, cols, dtype=torch.float64)
    w_h, e_h = torch.zeros(rows, cols, dtype=torch.float64), torch.zeros(rows, cols, dtype=torch.float64)
    for r, s in enumerate(slot.tolist()):
        if 0 <= s < states:
            _, last, _, el = ref.scan(f[r:r + 1], x[r:r + 1], [0, 1], state[s:s + 1])
            want[s], e[s], w_h[r], e_h[r] = last[0], el[0], last[0], el[0]
    ref.close(d_state, want, e)
    ref.close(h, w_h, e_h + ref.half_step(dtype) * (w_h.abs() + e_h))
    again = state.to(DEV)
    tdf.gated_scan_step(df, dx, again, slot=slot.to(DEV))                 # the rows of h are not wanted
    assert torch.equal(again, d_state)


def test_steps_are_the_scan():
    f, x, h0, offsets, df, dx = make([20], 36, torch.float32)
    h, last = forward(f, x, h0, offsets, df, dx)
    state, row = h0.to(DEV).clone(), torch.empty(1, 36, device=DEV)
    for t in range(20):
        tdf.gated_scan_step(df[t:t + 1], dx[t:t + 1], state, row)
        ref.close(row, h[t:t + 1].cpu().double(), 400 * ref.U * (1 + h[t:t + 1].cpu().double().abs()))
    assert torch.equal(row, state)


def test_a_table_beyond_32_bits():
    cols, states = 4096, (1 << 31) // 4096 + 9
    state = torch.empty(states, cols, device=DEV)                         # 8.6 GB
    f, x, h0, _, df, dx = make([2], cols, torch.float32)
    slot = torch.tensor([states - 1, 3], dtype=torch.int32, device=DEV)
    state[slot.long()] = h0.to(DEV)[[0, 0]]
    tdf.gated_scan_step(df, dx, state, slot=slot)
    want = h0.to(DEV)[[0, 0]].contiguous()
    tdf.gated_scan_step(df, dx, want)
    assert torch.equal(state[slot.long()], want)


def test_another_stream_and_a_graph():
    f, x, h0, offsets, df, dx = make([700, 0, 130, 900], 96, torch.bfloat16)
    off, ws, d_h0 = torch.tensor(offsets, device=DEV), space(1730, 96), h0.to(DEV)
    outs = [torch.empty_like(df) for _ in range(4)] + [torch.empty_like(d_h0) for _ in range(3)]
    h, gf, gx, row, last, dh0, state = outs
    dh = torch.randn_like(df)

    def all_three():
        tdf.gated_scan(df, dx, h, ws, off, d_h0, last)
        tdf.gated_scan_grad(df, dx, h, dh, gf, gx, ws, off, d_h0, last, dh0)
        state.copy_(last)
        tdf.gated_scan_step(df[:4], dx[:4], state, row[:4])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_three()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_three()
    for k in range(4):
        df.copy_(torch.randn(1730, 96, device=DEV, generator=torch.Generator(DEV).manual_seed(k)))
        row.zero_()
        all_three()
        want = [t.clone() for t in outs]
        for t in outs:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
