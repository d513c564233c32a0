"""What the operators beside the evaluations refuse, before anything is enqueued: no GPU is needed."""
import ctypes as C

import pytest
import torch

tdf = pytest.importorskip("paper_2410_20225_amd.tdf")
P = 1 << 20          # an address that no call gets as far as using


def norm(**k):
    a = dict(n_rows=4, n_cols=8, dtype=tdf.F32, eps=1e-5, x=P, ld_x=8, weight=P, bias=P)
    a.update(k)
    return tdf.Norm(*[a[n] for n, _ in tdf.Norm._fields_])


def norm_grads(**k):
    a = dict(dy=2 * P, ld_dy=8, mean=P, rstd=P, dx=3 * P, ld_dx=8, dweight=P, dbias=P)
    a.update(k)
    return tdf.NormGrads(*[a[n] for n, _ in tdf.NormGrads._fields_])


def scan(**k):
    a = dict(n_rows=4, n_cols=8, n_seqs=2, dtype=tdf.BF16, f=P, ld_f=8, x=2 * P, ld_x=16, offsets=P, h0=P)
    a.update(k)
    return tdf.Scan(*[a[n] for n, _ in tdf.Scan._fields_])


def scan_grads(**k):
    a = dict(h=3 * P, ld_h=8, dh=4 * P, ld_dh=8, dh_last=P, df=5 * P, ld_df=8, dx=6 * P, ld_dx=8, dh0=P)
    a.update(k)
    return tdf.ScanGrads(*[a[n] for n, _ in tdf.ScanGrads._fields_])


def step(**k):
    a = dict(n_rows=4, n_cols=8, n_states=9, dtype=tdf.F32, f=P, ld_f=8, x=2 * P, ld_x=8, slot=P, state=3 * P, h=4 * P, ld_h=8)
    a.update(k)
    return tdf.ScanStep(*[a[n] for n, _ in tdf.ScanStep._fields_])


def refused(status, text, code=None):
    assert status == (tdf.ERR_BAD_ARG if code is None else code)
    assert text in tdf.last_error(), tdf.last_error()


BAD_SIZES = [(dict(n_rows=-1), "out of range"), (dict(n_cols=0), "out of range"), (dict(n_cols=1 << 40), "out of range"), (dict(n_rows=1 << 50), "out of range"),
             (dict(dtype=7), "dtype")]


@pytest.mark.parametrize("change,text", BAD_SIZES + [
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(x=None), "NULL"), (dict(x=P + 2), "aligned"), (dict(ld_x=7), "distance"),
    (dict(weight=P + 1), "aligned"), (dict(bias=P + 2), "aligned"), (dict(n_rows=1 << 39, ld_x=1 << 30), "too large")])
def test_layer_norm(change, text):
    refused(tdf.lib.tdf_layer_norm(norm(**change), 2 * P, 8, None, None, None), text)
    refused(tdf.lib.tdf_layer_norm_grad(norm(**change), norm_grads(), 7 * P, 1 << 30, None), text)


def test_layer_norm_outputs():
    call = lambda y=2 * P, ld=8, mean=None, rstd=None: tdf.lib.tdf_layer_norm(norm(ld_x=16), y, ld, mean, rstd, None)  # noqa: E731
    refused(call(y=None), "NULL")
    refused(call(ld=3), "distance")
    refused(call(y=P), "overlaps")
    refused(call(mean=P + 1), "aligned")
    refused(tdf.lib.tdf_layer_norm(None, P, 8, None, None, None), "NULL")
    assert tdf.lib.tdf_layer_norm(norm(n_rows=0, x=None), None, 0, None, None, None) == tdf.OK


@pytest.mark.parametrize("change,text", [(dict(dy=None), "NULL"), (dict(ld_dy=2), "distance"), (dict(mean=None), "NULL"), (dict(rstd=P + 3), "aligned"),
                                         (dict(dx=P), "overlaps"), (dict(dx=2 * P, ld_dx=9), "overlaps"), (dict(dweight=P + 1), "aligned")])
def test_layer_norm_grad(change, text):
    refused(tdf.lib.tdf_layer_norm_grad(norm(), norm_grads(**change), 7 * P, 1 << 30, None), text)


def test_workspaces():
    need = tdf.layer_norm_grad_workspace_size(5000, 8)
    big = norm(n_rows=5000)
    for ws, n in ((None, need), (7 * P, need - 1), (7 * P + 16, need)):
        refused(tdf.lib.tdf_layer_norm_grad(big, norm_grads(), ws, n, None), "workspace", tdf.ERR_WORKSPACE)
    need = tdf.gated_scan_workspace_size(5000, 8)
    for ws, n in ((None, need), (7 * P, need - 1), (7 * P + 16, need)):
        if need:
            refused(tdf.lib.tdf_gated_scan(scan(n_rows=5000), 3 * P, 8, None, ws, n, None), "workspace", tdf.ERR_WORKSPACE)
            refused(tdf.lib.tdf_gated_scan_grad(scan(n_rows=5000), scan_grads(), ws, n, None), "workspace", tdf.ERR_WORKSPACE)
    for call in (tdf.layer_norm_grad_workspace_size, tdf.gated_scan_workspace_size):
        for size in ((-1, 8), (1, 0), (1 << 60, 8)):
            with pytest.raises(tdf.TdfError):
                call(*size)


@pytest.mark.parametrize("change,text", BAD_SIZES + [
    (dict(n_seqs=0), "n_seqs"), (dict(n_seqs=1 << 40), "n_seqs"), (dict(offsets=None), "offsets"), (dict(offsets=P + 4), "aligned"), (dict(h0=P + 2), "aligned"),
    (dict(f=None), "NULL"), (dict(x=None), "NULL"), (dict(f=P + 1), "aligned"), (dict(ld_f=7), "distance"), (dict(ld_x=1), "distance")])
def test_gated_scan(change, text):
    refused(tdf.lib.tdf_gated_scan(scan(**change), 3 * P, 8, None, 7 * P, 1 << 30, None), text)
    refused(tdf.lib.tdf_gated_scan_grad(scan(**change), scan_grads(), 7 * P, 1 << 30, None), text)


def test_gated_scan_outputs():
    call = lambda h=3 * P, ld=8, last=None: tdf.lib.tdf_gated_scan(scan(), h, ld, last, 7 * P, 1 << 30, None)  # noqa: E731
    refused(call(h=None), "NULL")
    refused(call(ld=7), "distance")
    refused(call(h=P), "overlaps")
    refused(call(last=P + 1), "aligned")
    refused(tdf.lib.tdf_gated_scan(None, P, 8, None, None, 0, None), "NULL")
    refused(tdf.lib.tdf_gated_scan_grad(scan(), None, 7 * P, 1 << 30, None), "NULL")


@pytest.mark.parametrize("change,text", [(dict(h=None), "NULL"), (dict(ld_h=3), "distance"), (dict(dh=4 * P + 1), "aligned"), (dict(df=None), "NULL"), (dict(dx=None), "NULL"),
                                         (dict(df=P), "overlaps"), (dict(dx=3 * P), "overlaps"), (dict(df=6 * P), "overlaps"), (dict(dh0=P + 1), "aligned"),
                                         (dict(dh_last=P + 2), "aligned")])
def test_gated_scan_grad(change, text):
    refused(tdf.lib.tdf_gated_scan_grad(scan(), scan_grads(**change), 7 * P, 1 << 30, None), text)


@pytest.mark.parametrize("change,text", BAD_SIZES + [
    (dict(n_states=-1), "n_states"), (dict(slot=None, n_states=3), "fewer states"), (dict(slot=P + 2), "aligned"), (dict(state=None), "NULL"), (dict(state=P + 1), "aligned"),
    (dict(f=None), "NULL"), (dict(x=None), "NULL"), (dict(ld_f=1), "distance"), (dict(h=3 * P), "overlaps"), (dict(h=P), "overlaps"), (dict(ld_h=1), "distance")])
def test_gated_scan_step(change, text):
    refused(tdf.lib.tdf_gated_scan_step(step(**change), None), text)


def adam(**k):
    a = dict(n=1000, param_dtype=tdf.F32, grad_dtype=tdf.F32, state_bits=32, weight_decay=0.0, param=P, grad=2 * P, copy=None, m=3 * P, v=4 * P, m_scale=None, v_scale=None)
    a.update(k)
    return tdf.AdamwTensor(*[a[n] for n, _ in tdf.AdamwTensor._fields_])


def build(*tensors):
    out = C.c_void_p()
    st = tdf.lib.tdf_adamw_build((tdf.AdamwTensor * max(1, len(tensors)))(*tensors), len(tensors), C.byref(out))
    return st, out


@pytest.mark.parametrize("change,text", [
    (dict(n=-1), "out of range"), (dict(param_dtype=3), "dtype"), (dict(grad_dtype=-1), "dtype"), (dict(state_bits=16), "state_bits"), (dict(weight_decay=float("nan")), "weight_decay"),
    (dict(param=None), "NULL"), (dict(grad=None), "NULL"), (dict(m=None), "NULL"), (dict(v=None), "NULL"), (dict(param=P + 2), "aligned"), (dict(m=3 * P + 1), "aligned"),
    (dict(state_bits=8), "scales"), (dict(m_scale=5 * P), "scales"), (dict(param_dtype=tdf.BF16, copy=5 * P), "copy"), (dict(copy=5 * P + 1), "aligned"),
    (dict(copy=P + 8), "overlap"), (dict(m=P + 3996), "overlap"), (dict(v=3 * P), "overlap")])
def test_adamw_tensors(change, text):
    refused(build(adam(**change))[0], text)
    refused(build(adam(n=0), adam(param=8 * P, m=9 * P, v=10 * P), adam(**change))[0], text)


def test_adamw_lists():
    refused(build()[0], "no tensors")
    refused(build(adam(), adam(param=8 * P, v=9 * P))[0], "overlap")          # the same m twice
    st, plan = build(adam(), adam(param=8 * P, m=9 * P, v=10 * P), adam(n=0, param=None, grad=None, m=None, v=None))
    assert st == tdf.OK
    n = C.c_size_t()
    assert tdf.lib.tdf_adamw_workspace_size(plan, C.byref(n)) == tdf.OK and n.value >= 3 * 64
    for ws, size in ((None, n.value), (7 * P, n.value - 1), (7 * P + 64, n.value)):
        refused(tdf.lib.tdf_adamw_prepare(plan, ws, size, None), "workspace", tdf.ERR_WORKSPACE)
    good = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, grad_scale=None, seed=0, reserved=0)
    refused(tdf.lib.tdf_adamw(plan, tdf.AdamwStep(*good.values()), None), "prepared")
    refused(tdf.lib.tdf_adamw(None, tdf.AdamwStep(*good.values()), None), "NULL")
    tdf.lib.tdf_adamw_destroy(plan)
    tdf.lib.tdf_adamw_destroy(None)


def test_the_binding_refuses_tensors_that_the_library_cannot_see_through():
    x = torch.zeros(4, 8)
    for call in (lambda: tdf.layer_norm(x, x), lambda: tdf.gated_scan(x, x, x, None), lambda: tdf.gated_scan_step(x, x, x, x),
                 lambda: tdf.adamw_build([tdf.adamw_tensor(x, x, x, x)]),
                 lambda: tdf.layer_norm_grad(x, x, x[:, 0], x[:, 0], x, None, None, None)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_more_tiles_than_a_launch_has_workgroups():
    refused(tdf.lib.tdf_gated_scan(scan(n_rows=1 << 30, n_cols=100, ld_f=100, ld_x=100), 3 * P, 100, None, 7 * P, 1 << 60, None), "out of range")
    refused(tdf.lib.tdf_gated_scan_grad(scan(n_rows=1 << 24, n_cols=1 << 14, ld_f=1 << 14, ld_x=1 << 14), scan_grads(), 7 * P, 1 << 60, None), "out of range")


@pytest.mark.parametrize("off", [0, 4, 60, -4, -60])
def test_states_that_are_carried_on_have_two_buffers(off):
    """h0 and dh_last are read while h_last and dh0 are written: 2 sequences of 8 columns, 64 bytes."""
    refused(tdf.lib.tdf_gated_scan(scan(), 3 * P, 8, P + off, 7 * P, 1 << 30, None), "h_last overlaps h0")
    refused(tdf.lib.tdf_gated_scan_grad(scan(h0=8 * P), scan_grads(dh_last=P, dh0=P + off), 7 * P, 1 << 30, None), "dh0 overlaps dh_last")
    refused(tdf.lib.tdf_gated_scan_grad(scan(h0=P), scan_grads(dh_last=8 * P, dh0=P + off), 7 * P, 1 << 30, None), "dh0 overlaps h0")
    refused(tdf.lib.tdf_gated_scan(scan(n_rows=0), None, 0, P + off, 7 * P, 1 << 30, None), "h_last overlaps h0")


def test_more_elements_than_a_launch_has_workgroups():
    huge = dict(param=1 << 45, grad=1 << 46, m=1 << 47, v=1 << 48)
    most = ((1 << 24) - 1) * 4096
    refused(build(adam(n=most + 1, **huge))[0], "too many elements")
    refused(build(adam(n=most, **huge), adam(n=1))[0], "too many elements")
    st, plan = build(adam(n=most, **huge), adam(n=0))
    assert st == tdf.OK
    tdf.lib.tdf_adamw_destroy(plan)
