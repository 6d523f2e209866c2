"""Layer norm, forward and backward, against the fp64 oracle on the values the
kernel was given. Tolerances count roundings: half a step of the output's type,
and the fp32 sums of a lane (up to 64 values, more in rows too long for
registers) with a tree over the lanes."""
import numpy as np
import pytest

import oracle.block as ob
from gpu_util import torch

pytestmark = pytest.mark.gpu

TYPES = ["bfloat16", "float16", "float32"]
EPS = 1e-5


def make(shape, dtype, seed, mean=0.5, sigma=1.0, layout=None):
    t = torch()
    g = t.Generator(device="cuda").manual_seed(seed)
    order = layout or list(range(len(shape)))
    x = t.randn([shape[i] for i in order], generator=g, device="cuda") * sigma + mean
    return x.to(getattr(t, dtype)).permute([order.index(i) for i in range(len(shape))])


def np64(x):
    return x.detach().double().cpu().numpy()


def half_step(dtype):
    t = torch()
    return t.finfo(getattr(t, dtype)).eps / 2


def check(x, w, b, dy, y, mean, rstd, dx, dw, db, dtype, wtype, eps=EPS):
    X, DY = np64(x), np64(dy)
    W, Bi = (None if p is None else np64(p) for p in (w, b))
    D = X.shape[-1]
    rows = X.size // D
    Y, M, R = ob.layer_norm(X, W, Bi, eps)
    DX, DW, DB = ob.layer_norm_backward(X, W, eps, DY)
    h = (X - M[..., None]) * R[..., None]
    aw = np.ones(D) if W is None else np.abs(W)
    u, f = half_step(dtype), 2.0 ** -24
    n = 96 + D // 256  # fp32 additions in a row's sum, rounded up
    r_ = R[..., None]
    # mean, then the deviation's rounding, then rstd (the variance's sum, its root)
    h_off = f * (n * r_ * np.abs(X).mean(-1, keepdims=True) + 2 * r_ * np.abs(X) + (n + 8) * np.abs(h))
    y_off = aw * h_off + 4 * f * (aw * np.abs(h) + (0 if Bi is None else np.abs(Bi)))
    tiny = 2.0 ** -24 if dtype == "float16" else 1e-37  # fp16's smallest step
    close(y, Y, y_off + u * (np.abs(Y) + y_off) + tiny, "y")
    close(mean, M, f * n * np.abs(X).mean(-1) + 1e-37, "mean")
    close(rstd, R, R * f * (n + 8) + R * f * n * np.abs(X).mean(-1) * R * 2, "rstd")
    g = DY if W is None else DY * W
    ag, ah = np.abs(g), np.abs(h)
    mean_ = lambda a: a.mean(-1, keepdims=True)  # noqa: E731
    dx_off = r_ * (f * (n + 8) * (ag + mean_(ag) + ah * mean_(ag * ah)) + h_off * np.abs(mean_(g * h)) + ah * mean_(ag * h_off))
    dx_off += f * (n + 8) * np.abs(DX)
    close(dx, DX, dx_off + u * (np.abs(DX) + dx_off) + tiny, "dx")
    lead = tuple(range(X.ndim - 1))
    sums = rows // 256 + 1100  # a lane's rows, the lanes, the partial sums
    uw = half_step(wtype)
    if dw is not None:
        off = (np.abs(DY) * (h_off + f * sums * ah)).sum(lead)
        close(dw, DW, off + uw * (np.abs(DW) + off) + 1e-7, "dw")
    if db is not None:
        off = f * sums * np.abs(DY).sum(lead)
        close(db, DB, off + uw * (np.abs(DB) + off) + 1e-7, "db")


def close(got, want, off, name):
    got = np64(got)
    assert got.shape == want.shape, name
    bad = np.abs(got - want) > off
    assert not bad.any(), (name, int(bad.sum()), float(np.max(np.abs(got - want) / off)))


def run(x, w, b, dy):
    import paper_2405_15780_amd as va

    y, mean, rstd = va.layer_norm_fwd(x, w, b, eps=EPS)
    dx, dw, db = va.layer_norm_bwd(x, w, mean, rstd, dy)
    torch().cuda.synchronize()
    return y, mean, rstd, dx, dw, db


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [1, 3, 8, 64, 72, 129, 512, 520, 1024, 2048, 2056, 4097, 5001, 8192, 16384, 16392, 40003])
def test_widths(D, dtype):
    rows = 37 if D < 4000 else 5
    print(f"case layer norm rows={rows} D={D} {dtype}", flush=True)
    x, dy = make((rows, D), dtype, D), make((rows, D), dtype, D + 1, mean=0.1)
    w, b = make((D,), dtype, D + 2, mean=1.0, sigma=0.3), make((D,), dtype, D + 3)
    check(x, w, b, dy, *run(x, w, b, dy), dtype, dtype)


@pytest.mark.parametrize("D", [4, 13, 25, 31, 33, 57, 100, 121, 125, 160, 185, 191, 193, 255, 380, 384, 500, 601, 640, 768, 1001, 1025, 1400,
                               1537, 2047])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_widths_by_lanes_and_pieces(D, dtype):
    """One to four pieces per lane, lanes of a row that divide a wave and that do not, a last piece of a few elements."""
    print(f"case layer norm D={D} {dtype} by lanes", flush=True)
    x, dy = make((301, D), dtype, D), make((301, D), dtype, D + 1)
    w, b = make((D,), "float32", D + 2, 1.0), make((D,), "float32", D + 3)
    check(x, w, b, dy, *run(x, w, b, dy), dtype, "float32")


@pytest.mark.parametrize("rows", [1, 2, 63, 64, 65, 1000, 20011])
@pytest.mark.parametrize("D", [8, 72, 768])
def test_row_counts(rows, D):
    if rows * D > 4_000_000:
        rows = 4999
    print(f"case layer norm rows={rows} D={D}", flush=True)
    x, dy = make((rows, D), "bfloat16", rows), make((rows, D), "bfloat16", rows + 1)
    w, b = make((D,), "float32", 1, mean=1.0, sigma=0.3), make((D,), "float32", 2)
    check(x, w, b, dy, *run(x, w, b, dy), "bfloat16", "float32")


LAYOUTS = {"bnhd": ((2, 3, 17, 72), [0, 2, 1, 3]), "nbhd": ((2, 3, 17, 64), [2, 0, 1, 3]), "hbnd": ((3, 2, 5, 40), [1, 0, 2, 3]),
           "3d": ((7, 11, 96), [1, 0, 2]), "5d": ((2, 3, 2, 5, 24), [0, 1, 2, 3, 4]), "5d mixed": ((2, 3, 2, 5, 24), [3, 1, 2, 0, 4])}


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_layouts(layout, dtype):
    shape, order = LAYOUTS[layout]
    print(f"case layer norm layout {layout} {dtype}", flush=True)
    x = make(shape, dtype, 5, layout=order)
    w, b = make(shape[-1:], dtype, 6, mean=1.0, sigma=0.3), make(shape[-1:], dtype, 7)
    for dy_order in (order, list(range(len(shape)))):
        dy = make(shape, dtype, 8, layout=dy_order)
        got = run(x, w, b, dy)
        assert len(shape) > 4 or got[0].stride() == x.stride()
        check(x, w, b, dy, *got, dtype, dtype)


def test_slices_odd_pitches_and_offsets():
    t = torch()
    for dtype in TYPES:
        big = make((3, 9, 131), dtype, 9)
        x, dy = big[:, 1:, 1:98], make((3, 8, 99), dtype, 10)[:, :, 2:]
        w, b = make((99,), dtype, 11)[1:98], make((97,), dtype, 12)
        assert x.shape == dy.shape == (3, 8, 97)
        check(x, w, b, dy, *run(x, w, b, dy), dtype, dtype)
        # a gradient shared by rows
        dy = make((1, 1, 97), dtype, 13).expand(3, 8, 97)
        check(x, w, b, dy, *run(x, w, b, dy), dtype, dtype)
    t.cuda.synchronize()


@pytest.mark.parametrize("w", [True, False])
@pytest.mark.parametrize("b", [True, False])
def test_without_weight_or_bias(w, b):
    x, dy = make((50, 200), "float16", 20), make((50, 200), "float16", 21)
    W = make((200,), "float32", 22) if w else None
    Bi = make((200,), "float32", 23) if b else None
    y, mean, rstd, dx, dw, db = run(x, W, Bi, dy)
    assert (dw is None) == (not w)
    check(x, W, Bi, dy, y, mean, rstd, dx, dw, db, "float16", "float32" if w else "float16")


def test_mean_far_from_zero_and_constant_rows():
    """Deviations are taken before squares, so a mean of 1,000 keeps its digits."""
    x, dy = make((64, 777), "float32", 30, mean=1000.0), make((64, 777), "float32", 31)
    w, b = make((777,), "float32", 32), make((777,), "float32", 33)
    check(x, w, b, dy, *run(x, w, b, dy), "float32", "float32")
    t = torch()
    x = t.full((4, 256), 3.0, device="cuda")
    y, mean, rstd, *_ = run(x, None, None, dy[:4, :256].contiguous())
    assert (y == 0).all() and (mean == 3).all()
    assert np.allclose(np64(rstd), 1 / np.sqrt(EPS), rtol=1e-6)


@pytest.mark.parametrize("value", [1000.0, 1000.1, -3.3e6, 1e30])
@pytest.mark.parametrize("D", [5, 100, 777, 1000, 3000, 5001, 8192, 8193, 40003, 1000003])
def test_constant_rows(D, value):
    """Deviations from the mean of equal values are zeros at any width: y is the bias and dx, dw see h = 0."""
    print(f"case layer norm constant rows D={D} value={value}", flush=True)
    t = torch()
    rows = 5 if D < 10000 else 2
    for dtype in ("float32", "bfloat16"):
        x = t.full((rows, D), value, device="cuda").to(getattr(t, dtype))
        w, b = make((D,), dtype, 34, mean=1.0), make((D,), dtype, 35)
        dy = make((rows, D), dtype, 36)
        y, mean, rstd, dx, dw, db = run(x, w, b, dy)
        assert (mean == x[:, 0].float()).all()
        assert np.allclose(np64(rstd), 1 / np.sqrt(EPS), rtol=1e-6)
        assert t.equal(y, b.expand(rows, D)) and not dw.any()


@pytest.mark.parametrize("D", [64, 100, 1000, 5001, 8193, 40003])
@pytest.mark.parametrize("sigma", [3e-4, 1e-2])
def test_rows_of_little_spread_about_a_far_mean(D, sigma):
    """The mean is the fp32 number next to the true one (2^-24 of it, and as much again for the rounding of the
    correction), the deviations x - mean are exact where x is within a factor of two of it, and the variance is
    about the true mean. So h is off by r * 2^-23 |mean| and the usual relative part (n fp32 additions)."""
    print(f"case layer norm little spread D={D} sigma={sigma}", flush=True)
    t = torch()
    g = t.Generator(device="cuda").manual_seed(D)
    x = (1000.1 + sigma * t.randn((6, D), generator=g, device="cuda", dtype=t.float64)).float()
    dy = make((6, D), "float32", 37)
    y, mean, rstd, dx, dw, db = run(x, None, None, dy)
    X = np64(x)
    Y, M, R = ob.layer_norm(X, None, None, EPS)
    f, n = 2.0 ** -24, 96 + D // 256
    close(mean, M, 2 * f * np.abs(M), "mean")
    h_off = R * 2 * f * np.abs(M)
    # r: the variance's sum, its root, and the square of the deviation of the mean that was subtracted
    r_off = R * f * (n + 8)
    close(rstd, R, r_off + 1e-30, "rstd")
    close(y, Y, h_off[:, None] * (1 + 2.0 ** -20) + (n + 12) * f * np.abs(Y), "y")


def test_other_rows_do_not_see_a_bad_one():
    t = torch()
    x, dy = make((40, 72), "float32", 40), make((40, 72), "float32", 41)
    ref = run(x, None, None, dy)
    y = x.clone()
    y[7, 3], y[21, 0] = float("nan"), float("inf")
    got = run(y, None, None, dy)
    keep = [i for i in range(40) if i not in (7, 21)]
    assert t.equal(got[0][keep], ref[0][keep]) and t.equal(got[3][keep], ref[3][keep])
    assert got[0][7].isnan().all() and got[0][21].isnan().any()


def test_in_place_and_rows_around_are_left():
    import paper_2405_15780_amd as va

    t = torch()
    for dtype in TYPES:
        big = make((20, 300), dtype, 50)
        x = big[3:9, 10:211]
        ref, *_ = va.layer_norm_fwd(x, eps=EPS)
        before = big.clone()
        va.layer_norm_fwd(x, eps=EPS, out=x)
        assert t.equal(big[3:9, 10:211], ref)
        big[3:9, 10:211] = before[3:9, 10:211]
        assert t.equal(big, before)


def test_same_bits_every_time_and_on_another_stream():
    t = torch()
    x, dy = make((3000, 768), "bfloat16", 60), make((3000, 768), "bfloat16", 61)
    w, b = make((768,), "bfloat16", 62), make((768,), "bfloat16", 63)
    ref = run(x, w, b, dy)
    s = t.cuda.Stream()
    s.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(s):
        other = run(x, w, b, dy)
    for got in (run(x, w, b, dy), other):
        for a, c in zip(got, ref):
            assert t.equal(a, c)


@pytest.mark.parametrize("need", [(1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)])
def test_autograd(need):
    import paper_2405_15780_amd as va

    t = torch()
    x, dy = make((4, 6, 96), "bfloat16", 70), make((4, 6, 96), "bfloat16", 71)
    w, b = make((96,), "bfloat16", 72), make((96,), "bfloat16", 73)
    leaves = [p.detach().requires_grad_(bool(n)) for p, n in zip((x, w, b), need)]
    y = va.layer_norm(*leaves, eps=EPS)
    y_ref, _, _, *grads = run(x, w, b, dy)
    assert t.equal(y, y_ref)
    y.backward(dy)
    for p, n, g in zip(leaves, need, grads):
        assert t.equal(p.grad, g) if n else p.grad is None
    assert t.equal(va.layer_norm(x, w, b, eps=EPS), y_ref)


@pytest.mark.parametrize("form", ["sum", "column", "transposed", "negated"])
def test_autograd_gradient_layouts(form):
    import paper_2405_15780_amd as va

    t = torch()
    x = make((12, 40), "float32", 80)
    base = make((12, 40), "float32", 81)
    dy = {"sum": t.ones((), device="cuda").expand(12, 40), "column": base[:, :1].expand(12, 40),
          "transposed": base.reshape(40, 12).t(), "negated": t._neg_view(base)}[form]
    leaf = x.detach().requires_grad_()
    va.layer_norm(leaf, eps=EPS).backward(dy)
    want = run(x, None, None, dy.resolve_neg().contiguous())[3]
    assert t.equal(leaf.grad, want)


def test_refusals():
    import paper_2405_15780_amd as va

    t = torch()
    x = make((4, 32), "bfloat16", 90)
    for bad in (x.double(), x.cpu(), x.long(), x.t(), None):
        with pytest.raises((TypeError, AttributeError)):
            va.layer_norm_fwd(bad)
    w = make((32,), "float32", 91)
    for args in ((w[:31], None), (w.half(), None), (None, w.cpu()), (w, w.bfloat16()), (make((64,), "float32", 1)[::2], None)):
        with pytest.raises(TypeError):
            va.layer_norm_fwd(x, *args)
    with pytest.raises(ValueError):
        va.layer_norm_fwd(x[:0])
    with pytest.raises(va.VitattnError):
        va.layer_norm_fwd(x, eps=-1.0)
    with pytest.raises(va.VitattnError):
        va.layer_norm_fwd(x, eps=float("nan"))
    with pytest.raises(va.VitattnError):  # the output overlaps the input, shifted
        buf = make((5, 32), "bfloat16", 92)
        va.layer_norm_fwd(buf[:4], out=buf[1:])
    y, mean, rstd = va.layer_norm_fwd(x)
    for bad in (x[:3], x.float(), x.cpu()):
        with pytest.raises(TypeError):
            va.layer_norm_bwd(x, None, mean, rstd, bad)
    with pytest.raises(TypeError):
        va.layer_norm_bwd(x, None, mean[:3], rstd, x)
    with pytest.raises(va.VitattnError):
        va.layer_norm_bwd(x, None, mean, rstd, x, workspace=t.empty(4, device="cuda"))


@pytest.mark.parametrize("windows,D,hop", [(11, 30, 1), (31, 10, 1), (9, 72, 1), (6, 30, 2), (3, 700, 1)])
def test_sliding_windows(windows, D, hop):
    """Rows that start a few elements apart: the outputs have rows of their own."""
    for dtype in TYPES:
        print(f"case layer norm windows {windows} x {D} by {hop} {dtype}", flush=True)
        long = make((2, D + hop * (windows - 1)), dtype, 93)
        x, dy = long.unfold(1, D, hop), make((2, D + hop * (windows - 1)), dtype, 94).unfold(1, D, hop)
        assert x.shape == (2, windows, D) and x.stride() == (long.shape[1], hop, 1)
        w, b = make((D,), dtype, 95, mean=1.0), make((D,), dtype, 96)
        got = run(x, w, b, dy)
        check(x, w, b, dy, *got, dtype, dtype)
        want = run(x.contiguous(), w, b, dy.contiguous())
        assert all(torch().equal(a, c) for a, c in zip(got, want))
