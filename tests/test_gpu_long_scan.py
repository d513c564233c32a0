"""Sequences so long that a chain of tiles has its third level: 256 tiles and more, of 128 rows (64: gradients in float32), against the
formula in 64 bits for all rows at once."""
import pytest
import torch

import operators_ref as ref
from paper_2410_20225_amd import tdf

DEV = "cuda:0"
ROWS = 547 * 128 - 21        # two states of the third level forward, and in float32 four for the gradients; the last tile is not full


def along(a, b):
    """s_t = a_t s_(t-1) + b_t from s = 0: in step k every row takes in the 2^k rows before it."""
    k = 1
    while k < len(b):
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


def scan(f, x, offsets, h0):
    """As operators_ref.scan, of sequences that have rows and are all the rows."""
    f, x, h0 = f.double(), x.double(), h0.double()
    first, last = torch.tensor(offsets[:-1]), torch.tensor(offsets[1:]) - 1
    a, keep = torch.sigmoid(f), torch.sigmoid(-f)
    cut = a.index_fill(0, first, 0.0)
    h = along(cut, (keep * x).index_add(0, first, a[first] * h0))
    before = torch.cat([h[:1], h[:-1]]).index_copy(0, first, h0)
    e = along(cut, ref._slack(f) * ((a * before).abs() + (keep * x).abs()))
    return h, h[last], e + ref.U * h.abs(), (e + ref.U * h.abs())[last]


def scan_grad(f, x, h, dh, offsets, h0, dh_last):
    """As operators_ref.scan_grad, of the same."""
    f, x, h, dh, h0, dh_last = (t.double() for t in (f, x, h, dh, h0, dh_last))
    first, last = torch.tensor(offsets[:-1]), torch.tensor(offsets[1:]) - 1
    a, keep, k = torch.sigmoid(f), torch.sigmoid(-f), ref._slack(f)
    after = torch.cat([a[1:], a[:1]]).index_fill(0, last, 0.0)
    back = lambda c, b: along(c.flip(0), b.flip(0)).flip(0)  # noqa: E731
    ds = back(after, dh.index_add(0, last, dh_last))
    carry = ds - dh
    # of each row: U (|dh| + |carry|) of its sum, and k |ds| where it is handed on
    own, handed = ref.U * (dh.abs() + carry.abs()), k * ds.abs()
    e_ds = back(after, own + after * torch.cat([handed[1:], handed[:1]]))
    before = torch.cat([h[:1], h[:-1]]).index_copy(0, first, h0)
    d = before - x
    dx, df = ds * keep, ds * d * a * keep
    e_dx = keep * (e_ds + handed)
    e_df = a * keep * (d.abs() * (e_ds + 2 * handed) + ref.U * ds.abs() * (before.abs() + x.abs()))
    dh0, e_dh0 = (a * ds)[first], (a * (e_ds + handed))[first]
    return df, dx, dh0, e_df + ref.U * df.abs(), e_dx + ref.U * dx.abs(), e_dh0 + ref.U * dh0.abs()


def make(offsets, cols, dtype, slow):
    g = torch.Generator().manual_seed(cols + offsets[1])
    rows, seqs = offsets[-1], len(offsets) - 1
    f = (1 + slow + 2 * torch.randn(rows, cols, generator=g) + 2 * torch.randn(1, cols, generator=g)).to(dtype)
    x, dh = (torch.randn(rows, cols, generator=g).to(dtype) for _ in range(2))
    return f, x, dh, torch.randn(seqs, cols, generator=g), torch.randn(seqs, cols, generator=g)


@pytest.mark.parametrize("slow", [0.0, 9.0])
def test_the_formula_for_all_rows_at_once_is_the_one_row_after_row(slow):
    offsets = [0, 1, 60, 61, 200]
    f, x, dh, h0, dh_last = make(offsets, 5, torch.float32, slow)
    h = ref.scan(f, x, offsets, h0)[0].float()
    for got, want in ((scan(f, x, offsets, h0), ref.scan(f, x, offsets, h0)),
                      (scan_grad(f, x, h, dh, offsets, h0, dh_last), ref.scan_grad(f, x, h, dh, offsets, h0, dh_last))):
        assert len(got) == len(want)
        for a, b in zip(got, want):
            assert torch.allclose(a, b, rtol=1e-9, atol=1e-18 + 1e-11 * float(b.abs().max()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("cols", [8, 7])
@pytest.mark.parametrize("offsets,slow", [([0, ROWS], 12.0), ([0, ROWS], 3.0),
                                          # sequences that begin and end a few rows before or after tile 256: of 128 rows from the first row (32,768)
                                          # and from the last (37,248), and of 64 from the last (53,632)
                                          ([0, 32763, 37253, 53629, ROWS], 12.0), ([0, 32771, 37243, 53635, ROWS], 12.0)], ids=["keep", "forget", "before", "after"])
def test_chains_of_hundreds_of_tiles(offsets, slow, cols, dtype):
    f, x, dh, h0, dh_last = make(offsets, cols, dtype, slow)
    df, dx, ddh, d0, dl = (t.to(DEV) for t in (f, x, dh, h0, dh_last))
    off = torch.tensor(offsets, device=DEV)
    ws = torch.full((tdf.gated_scan_workspace_size(ROWS, cols),), 255, dtype=torch.uint8, device=DEV)
    h, last = torch.full_like(df, -7.0), torch.full_like(d0, -7.0)
    tdf.gated_scan(df, dx, h, ws, off, d0, last)
    want, w_last, e, e_last = scan(f, x, offsets, h0)
    ref.close(h, want, e + ref.half_step(dtype) * (want.abs() + e))
    ref.close(last, w_last, e_last)
    gf, gx, dh0 = torch.full_like(df, -7.0), torch.full_like(df, -7.0), torch.full_like(d0, -7.0)
    tdf.gated_scan_grad(df, dx, h, ddh, gf, gx, ws, off, d0, dl, dh0)
    want = scan_grad(f, x, h.cpu(), dh, offsets, h0, dh_last)
    for got, w, e in ((gf, want[0], want[3]), (gx, want[1], want[4])):
        ref.close(got, w, e + ref.half_step(dtype) * (w.abs() + e))
    ref.close(dh0, want[2], want[5])
    # and the same again
    again = torch.empty_like(h)
    tdf.gated_scan(df, dx, again, ws, off, d0, last)
    assert torch.equal(again, h)
