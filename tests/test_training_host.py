"""Refusals of the operators around a layer's experts: bad arguments come back as an error before anything touches a GPU."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def norm(P, **kw):
    from paper_2508_02322_b200.binding import camera_norm_t
    a = dict(x=4096, ld=64, n_rows=4, dtype=1, d=64, weight=4096, bias=None, weight_dtype=1, eps=1e-6, flags=0)
    a.update(kw)
    return camera_norm_t(*[a[n] for n, _ in camera_norm_t._fields_])


BAD_NORM = [dict(n_rows=-1), dict(d=0), dict(ld=63), dict(dtype=2), dict(weight_dtype=3), dict(flags=2), dict(eps=-1.0),
            dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(x=4097), dict(weight=4097), dict(bias=4098, weight_dtype=0)]


def test_norm_refusals(P):
    lib = P.lib

    def fwd(n, r=None, r_ld=64, s=None, s_ld=64, y=4096, y_ld=64, mean=4096, rstd=4096):
        return lib.camera_norm_forward(C.byref(n), r, r_ld, s, s_ld, y, y_ld, mean, rstd, None)
    assert lib.camera_norm_forward(None, None, 0, None, 0, 4096, 64, None, None, None) == -1
    assert fwd(norm(P, n_rows=0, x=None), y=None) == 0
    for bad in BAD_NORM:
        assert fwd(norm(P, **bad)) == -1, bad
    assert fwd(norm(P, d=32769, ld=32769), y_ld=32769) == -2
    for bad in (dict(y=None), dict(y_ld=63), dict(y=4097), dict(r=4096), dict(s=4096), dict(r=4096, s=4096, r_ld=10), dict(mean=4098), dict(rstd=4097),
                dict(r=4097, s=4096), dict(r=4096, s=4096, s_ld=1)):
        assert fwd(norm(P), **bad) == -1, bad
    size = lib.camera_norm_backward_workspace_bytes(4, 64)
    assert size > 0 and lib.camera_norm_backward_workspace_bytes(0, 64) > 0
    for rows, d in ((-1, 64), (4, 0), (4, 32769)):
        assert lib.camera_norm_backward_workspace_bytes(rows, d) == 0

    def bwd(n=None, dy=4096, dy_ld=64, mean=4096, rstd=4096, ds=None, ds_ld=64, dx=4096, dx_ld=64, dw=4096, db=None, ws=4096, nbytes=size):
        return lib.camera_norm_backward(C.byref(n or norm(P)), dy, dy_ld, mean, rstd, ds, ds_ld, dx, dx_ld, dw, db, ws, nbytes, None)
    for bad in BAD_NORM:
        if "bias" not in bad:
            assert bwd(norm(P, **bad)) == -1, bad
    for bad in (dict(dy=None), dict(dy_ld=63), dict(mean=None), dict(rstd=None), dict(dx=None, dw=None), dict(dx=None, ds=4096), dict(ds=4097), dict(ds=4096, ds_ld=2),
                dict(dx=4097), dict(dx_ld=60), dict(dw=4098), dict(db=4097)):
        assert bwd(**bad) == -1, bad
    for bad in (dict(ws=None), dict(nbytes=8), dict(ws=4096 + 64)):
        assert bwd(**bad) == -3, bad


def test_moe_refusals(P):
    lib = P.lib
    big = 100000
    size = lib.camera_moe_dispatch_workspace_bytes(big, 8, 64)
    assert size > 256 and lib.camera_moe_dispatch_workspace_bytes(4, 2, 8) > 0
    for t, k, e in ((-1, 2, 8), (4, 0, 8), (4, 17, 8), (4, 2, 0), (4, 2, 1025), (1 << 30, 2, 8), (1 << 62, 4, 8)):
        assert lib.camera_moe_dispatch_workspace_bytes(t, k, e) == 0, (t, k, e)

    def dis(x=4096, dtype=1, ld=64, t=4, d=64, idx=4096, k=2, e=8, xs=4096, xs_ld=64, rows=4096, off=4096, ws=4096, n=1 << 20):
        return lib.camera_moe_dispatch(x, dtype, ld, t, d, idx, k, e, xs, xs_ld, rows, off, ws, n, None)
    for bad in (dict(dtype=2), dict(t=-1), dict(d=0), dict(k=0), dict(e=0), dict(x=None), dict(x=4097), dict(ld=63), dict(xs=None), dict(xs_ld=63), dict(idx=None),
                dict(idx=4098), dict(rows=None), dict(off=None), dict(off=4097)):
        assert dis(**bad) == -1, bad
    for bad in (dict(k=17), dict(e=1025), dict(t=1 << 31, k=1), dict(t=1 << 30, k=2), dict(d=(1 << 20) + 1, ld=1 << 21, xs_ld=1 << 21)):
        assert dis(**bad) == -2, bad
    for bad in (dict(ws=None), dict(n=100), dict(ws=4096 + 8)):
        assert dis(t=big, k=8, e=64, **bad) == -3, bad

    def com(ys=4096, dtype=1, ys_ld=64, n=8, rows=4096, w=4096, t=4, k=2, d=64, add=None, add_ld=64, y=4096, y_ld=64):
        return lib.camera_moe_combine(ys, dtype, ys_ld, n, rows, w, t, k, d, add, add_ld, y, y_ld, None)

    def dback(ys=4096, dtype=1, ys_ld=64, n=8, rows=4096, t=4, k=2, d=64, add=None, add_ld=64, y=4096, y_ld=64):
        return lib.camera_moe_dispatch_backward(ys, dtype, ys_ld, n, rows, t, k, d, add, add_ld, y, y_ld, None)
    for fn in (com, dback):
        assert fn(t=0, rows=None, y=None, ys=None, n=0) == 0
        for bad in (dict(dtype=5), dict(ys=None), dict(ys=4097), dict(ys_ld=63), dict(n=-1), dict(rows=None), dict(rows=4097), dict(t=-2), dict(k=0), dict(d=0),
                    dict(add=4097), dict(add=4096, add_ld=5), dict(y=None), dict(y_ld=9)):
            assert fn(**bad) == -1, bad
        assert fn(k=17) == -2 and fn(t=1 << 31) == -2
    assert com(w=4097) == -1

    def cback(dy=4096, dtype=1, ld=64, t=4, d=64, rows=4096, w=4096, k=2, ys=4096, ys_ld=64, n=8, dys=4096, dys_ld=64, dw=4096):
        return lib.camera_moe_combine_backward(dy, dtype, ld, t, d, rows, w, k, ys, ys_ld, n, dys, dys_ld, dw, None)
    assert cback(t=0, dy=None, rows=None) == 0
    for bad in (dict(dy=None), dict(dtype=2), dict(ld=63), dict(t=-1), dict(d=0), dict(rows=None), dict(w=4098), dict(k=0), dict(ys=None), dict(ys_ld=1), dict(n=-1),
                dict(dys=4097), dict(dys_ld=63), dict(dw=4097), dict(dys=None, dw=None)):
        assert cback(**bad) == -1, bad
    assert cback(k=17) == -2


def matrices(P, *ms):
    from paper_2508_02322_b200.binding import camera_matrix_t
    base = dict(in_=4096, out=4096, in_ld=64, out_ld=64, rows=32, cols=64)
    return (camera_matrix_t * len(ms))(*[camera_matrix_t(*[{**base, **m}[n] for n, _ in camera_matrix_t._fields_]) for m in ms])


def test_orthogonalize_refusals(P):
    lib = P.lib
    coef = (C.c_float * 3)(*P.NEWTON_SCHULZ)
    size = lib.camera_orthogonalize_workspace_bytes(matrices(P, {}), 1)
    assert size > 2 * 256 * 64 * 2
    both = lib.camera_orthogonalize_workspace_bytes(matrices(P, {}, dict(rows=300, cols=100)), 2)
    assert both > size
    assert lib.camera_orthogonalize_workspace_bytes(None, 0) > 0 and lib.camera_orthogonalize_workspace_bytes(None, 1) == 0
    for bad in (dict(rows=-1), dict(rows=131073), dict(rows=40000, cols=40000)):
        assert lib.camera_orthogonalize_workspace_bytes(matrices(P, bad), 1) == 0, bad

    def run(m={}, n=1, dtype=1, c=coef, steps=1, eps=1e-7, ws=4096, nbytes=size):
        return lib.camera_orthogonalize(matrices(P, m), n, dtype, c, steps, C.c_float(eps), ws, nbytes, None)
    for bad in (dict(in_=None), dict(out=None), dict(in_ld=63), dict(out_ld=63), dict(in_=4097), dict(out=4097), dict(rows=-1)):
        assert run(bad) == -1, bad
    assert run(dict(in_=4098), dtype=0) == -1
    assert run(dict(rows=131073)) == -2
    for bad in (dict(n=-1), dict(dtype=2), dict(c=None), dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert run(**bad) == -1, bad
    for c in ((2000.0, 0.0, 0.0), (float("nan"), 0.0, 0.0), (1.0, float("inf"), 0.0), (1.0, 0.0, 5000.0)):
        assert run(c=(C.c_float * 3)(*c)) == -1, c
    grows = (C.c_float * 9)(*[30.0, 0.0, 0.0] * 3)
    assert run(c=grows, steps=3) == -1                       # 30, 900, 27000
    for bad in (dict(ws=None), dict(nbytes=size - 1), dict(ws=4096 + 128)):
        assert run(**bad) == -3, bad


def test_tensors_are_checked_in_python(P):
    z = torch.zeros(4, 16)
    idx = torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: P.camera_norm_forward(z), lambda: P.camera_norm_backward(z, z, z[:, 0]), lambda: P.camera_moe_dispatch(z, idx, 4),
                 lambda: P.camera_moe_combine(z, idx), lambda: P.camera_moe_dispatch_backward(z, idx), lambda: P.camera_moe_combine_backward(z, z, idx),
                 lambda: P.camera_orthogonalize([z])):
        with pytest.raises(ValueError):                       # not on a GPU
            call()
    with pytest.raises(ValueError):
        P.camera_orthogonalize(z)                             # one matrix is not a list of them
    with pytest.raises(ValueError):
        P.camera_orthogonalize([z], coefficients=(1.0, 2.0))
    with pytest.raises(P.CameraError):
        P.camera_moe_dispatch_workspace_bytes(4, 99, 8)
    with pytest.raises(P.CameraError):
        P.camera_norm_backward_workspace_bytes(4, 1 << 20)
    assert P.camera_orthogonalize_workspace_bytes([z]) > 0    # shapes may be asked about anywhere


def test_coefficients_are_three_numbers_or_a_list_of_such(P):
    z = torch.zeros(4, 16)
    six = (3.0, -3.2, 1.2) * 2
    for bad in (six, six[:5], (), [six], [(3.0, -3.2, 1.2), (1.0, 2.0)], [(1.0, 2.0, 3.0), 4.0]):
        with pytest.raises(ValueError, match="coefficients must be"):
            P.camera_orthogonalize([z], coefficients=bad)
    for good in (P.NEWTON_SCHULZ, list(P.NEWTON_SCHULZ), [P.NEWTON_SCHULZ] * 5, [list(P.NEWTON_SCHULZ)]):
        with pytest.raises(ValueError, match="on the GPU"):   # past the coefficients
            P.camera_orthogonalize([z], coefficients=good)


def test_steps_and_a_list_of_coefficients_agree(P):
    z = torch.zeros(4, 16)
    three = [P.NEWTON_SCHULZ] * 3
    for bad in (1, 5, 0):
        with pytest.raises(ValueError, match="steps"):
            P.camera_orthogonalize([z], steps=bad, coefficients=three)
    for kw in (dict(coefficients=three), dict(steps=3, coefficients=three), dict(steps=7), dict()):
        with pytest.raises(ValueError, match="on the GPU"):   # past the coefficients
            P.camera_orthogonalize([z], **kw)


def test_unknown_names_of_results_are_refused(P):
    z = torch.zeros(4, 16)
    for out in ({"rstd": z[:, 0]}, {"y": z, "mean": z[:, 0]}, {"x": z}):
        with pytest.raises(ValueError, match="out"):
            P.camera_norm_forward(z, residual=z, out=out)
    with pytest.raises(ValueError, match="out"):
        P.camera_norm_forward(z, out={"sum": z})              # there is no sum without a residual
    for kw in (dict(out={"y": z}), dict(residual=z, out={"y": z, "sum": z}), dict(out={}), dict(out={"sum": None})):
        with pytest.raises(ValueError, match="on the GPU"):
            P.camera_norm_forward(z, **kw)


def test_room_for_a_result_that_is_not_asked_for_is_refused(P):
    z, idx = torch.zeros(4, 16), torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="want_x"):
        P.camera_norm_backward(z, z, z[:, 0], want_x=False, out=z)
    with pytest.raises(ValueError, match="want_y"):
        P.camera_moe_combine_backward(z, z, idx, want_y=False, out=z)
    for call in (lambda: P.camera_norm_backward(z, z, z[:, 0], want_x=False), lambda: P.camera_norm_backward(z, z, z[:, 0], out=z, d_sum=z),
                 lambda: P.camera_moe_combine_backward(z, z, idx, out=z), lambda: P.camera_moe_combine_backward(z, z, idx, want_y=False)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()
