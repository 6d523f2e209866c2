"""The C entry points of the rms norm, dropout and the attention over chosen blocks
refuse what they cannot compute before any HIP call: a status, no output touched, no GPU
needed."""
import ctypes

import numpy as np
import pytest

va = pytest.importorskip("paper_2405_15780_amd")
from paper_2405_15780_amd.binding import DropoutSpec  # noqa: E402
from paper_2405_15780_amd.binding import Strides as S  # noqa: E402
from test_block_abi import BF16, FP16, FP32, INVAL, UNSUP, WS, Bufs, lib  # noqa: E402

ROWS = S(256, 128, 32)  # 2 x 2 x 4 rows of 32
DROP = DropoutSpec(1, 2, None, 0.5)


def rms_fwd(b, want, **o):
    a = dict(x=b[0], sx=ROWS, res=b[1], sr=ROWS, w=b[2], h=b[3], sh=ROWS, y=b[4], sy=ROWS, rstd=b[5], B=2, H=2, N=4, D=32,
             eps=1e-5, type=BF16, rtype=BF16, wtype=BF16, drop=DROP)
    a.update(o)
    b.check(lib().vitattn_rms_norm_fwd(*a.values(), None), want)


@pytest.mark.parametrize("o,want", [
    (dict(x=None), INVAL), (dict(y=None), INVAL), (dict(res=None), INVAL), (dict(h=None), INVAL), (dict(B=0), INVAL),
    (dict(H=-1), INVAL), (dict(N=0), INVAL), (dict(D=0), INVAL), (dict(D=16385), UNSUP),
    (dict(D=8193, type=FP32, rtype=FP32, wtype=FP32), UNSUP), (dict(N=2 ** 30, B=2, H=1), INVAL), (dict(type=3), UNSUP),
    (dict(type=-1), UNSUP), (dict(rtype=FP16), UNSUP), (dict(wtype=FP16), UNSUP), (dict(type=FP32), UNSUP),
    (dict(eps=-1e-9), INVAL), (dict(eps=float("nan")), INVAL), (dict(eps=float("inf")), INVAL), (dict(sx=S(-1, 128, 32)), INVAL),
    (dict(sy=S(256, 128, 31)), INVAL), (dict(sh=S(0, 128, 32)), INVAL), (dict(drop=DropoutSpec(1, 2, None, -0.1)), INVAL),
    (dict(drop=DropoutSpec(1, 2, None, 1.5)), INVAL), (dict(drop=DropoutSpec(1, 2, None, float("nan"))), INVAL),
    (dict(drop=DropoutSpec(1, 2, 12, 0.5)), INVAL),
    (dict(res=None, h=None), INVAL),  # dropout without a residual
    (dict(res=None, h=None, drop=None, rtype=FP32), INVAL)])
def test_rms_forward_refusals(o, want):
    rms_fwd(Bufs(), want, **o)


def test_rms_forward_alignment_and_overlap():
    b = Bufs()
    rms_fwd(b, INVAL, x=b[0] + 1)
    rms_fwd(b, INVAL, res=b[1] + 2, rtype=FP32)
    rms_fwd(b, INVAL, w=b[2] + 2, wtype=FP32)
    rms_fwd(b, INVAL, rstd=b[5] + 2)
    rms_fwd(b, INVAL, y=b[0] + 64)  # shifted onto the input
    rms_fwd(b, INVAL, y=b[0], sy=S(512, 256, 32))  # in place, with other strides
    rms_fwd(b, INVAL, h=b[1], sh=S(512, 256, 32))
    rms_fwd(b, INVAL, y=b[1])  # over the residual
    rms_fwd(b, INVAL, h=b[0])
    rms_fwd(b, INVAL, h=b[4])  # over the other output
    rms_fwd(b, INVAL, y=b[2])
    rms_fwd(b, INVAL, rstd=b[2])
    rms_fwd(b, INVAL, drop=DropoutSpec(1, 2, b[4], 0.5))
    # interleaved rows share nothing, but for their last bytes
    two = S(512, 256, 64)
    rms_fwd(b, INVAL, h=b[4] + 62, sh=two, sy=two)


def rms_fp8(b, want, **o):
    a = dict(x=b[0], sx=ROWS, res=b[1], sr=ROWS, w=b[2], h=b[3], sh=ROWS, y=b[4], sy=ROWS, scale=b[5], group=0, B=2, H=2, N=4,
             D=32, eps=1e-5, type=BF16, rtype=BF16, wtype=BF16)
    a.update(o)
    b.check(lib().vitattn_rms_norm_fp8(*a.values(), None), want)


@pytest.mark.parametrize("o,want", [
    (dict(group=16), UNSUP), (dict(group=-32), UNSUP), (dict(group=256), UNSUP), (dict(scale=None), INVAL), (dict(y=None), INVAL),
    (dict(x=None), INVAL), (dict(D=16385), UNSUP), (dict(sy=S(256, 128, 31)), INVAL)])
def test_rms_fp8_refusals(o, want):
    rms_fp8(Bufs(), want, **o)


def test_rms_fp8_overlap():
    b = Bufs()
    rms_fp8(b, INVAL, y=b[0])  # bytes cannot take the input's place
    rms_fp8(b, INVAL, scale=b[4] + 508)
    rms_fp8(b, INVAL, scale=b[5] + 2)
    rms_fp8(b, INVAL, scale=b[0])


def rms_bwd(b, want, **o):
    a = dict(h=b[0], sh=ROWS, w=b[1], rstd=b[2], dy=b[3], sdy=ROWS, dh=b[4], sdh=ROWS, dx=b[5], sdx=ROWS, dres=b[6], sdres=ROWS,
             dw=b[7], B=2, H=2, N=4, D=32, type=BF16, rtype=BF16, wtype=BF16, drop=DROP, ws=b[8], wsb=1 << 20)
    a.update(o)
    b.check(lib().vitattn_rms_norm_bwd(*a.values(), None), want)


@pytest.mark.parametrize("o,want", [
    (dict(h=None), INVAL), (dict(dy=None), INVAL), (dict(rstd=None), INVAL), (dict(ws=None), WS), (dict(wsb=64), WS),
    (dict(sdx=S(256, 0, 32)), INVAL), (dict(sdres=S(256, 128, 8)), INVAL), (dict(sdy=S(256, -128, 32)), INVAL), (dict(D=0), INVAL),
    (dict(D=16385), UNSUP), (dict(rtype=FP16), UNSUP), (dict(wtype=5), UNSUP), (dict(drop=DropoutSpec(1, 2, None, 2.0)), INVAL)])
def test_rms_backward_refusals(o, want):
    rms_bwd(Bufs(), want, **o)


def test_rms_backward_overlaps():
    b = Bufs()
    for i in (0, 1, 2, 4):
        rms_bwd(b, INVAL, dx=b[i])
        rms_bwd(b, INVAL, dw=b[i] + 32)
    for i in (0, 1, 2, 3, 5):
        rms_bwd(b, INVAL, dres=b[i])
    rms_bwd(b, INVAL, dx=b[3], sdx=S(512, 256, 32))
    rms_bwd(b, INVAL, dres=b[4] + 64)
    rms_bwd(b, INVAL, ws=b[0])
    rms_bwd(b, INVAL, ws=b[6])


def test_rms_workspace_bytes():
    f = lib().vitattn_rms_norm_bwd_workspace_bytes
    assert f(1, 1, 1, 64, BF16) == 64 * 4
    assert f(2, 1, 4096, 1024, BF16) % (1024 * 4) == 0 and f(2, 1, 4096, 1024, BF16) > 0
    assert f(1, 1, 1, 16385, BF16) == f(1, 1, 1, 8193, FP32) == f(0, 1, 1, 64, BF16) == f(1, 1, 1, 64, 7) == 0
    assert f(1, 1, 1, 2 ** 31, BF16) == 0


def dropout(b, want, **o):
    a = dict(x=b[0], sx=ROWS, res=b[1], sr=ROWS, y=b[2], sy=ROWS, B=2, H=2, N=4, D=32, type=BF16, rtype=BF16, drop=DROP)
    a.update(o)
    b.check(lib().vitattn_dropout(*a.values(), None), want)


@pytest.mark.parametrize("o,want", [
    (dict(x=None), INVAL), (dict(y=None), INVAL), (dict(drop=None), INVAL), (dict(B=0), INVAL), (dict(D=0), INVAL),
    (dict(type=3), UNSUP), (dict(rtype=FP16), UNSUP), (dict(res=None, rtype=FP32), INVAL), (dict(sx=S(256, 128, -32)), INVAL),
    (dict(sy=S(256, 128, 16)), INVAL), (dict(drop=DropoutSpec(1, 2, None, 1.0001)), INVAL), (dict(N=2 ** 30, B=2, H=1), INVAL),
    (dict(B=1, H=1, N=2 ** 20, D=2 ** 17 + 8, sx=S(0, 0, 0), sr=S(0, 0, 0), sy=S(0, 0, 2 ** 18), y=2 ** 44), INVAL)])
def test_dropout_refusals(o, want):
    dropout(Bufs(), want, **o)


@pytest.mark.parametrize("rtype", [BF16, FP16])
def test_dropout_to_16_bits(rtype):
    """fp32 rows without a residual may be rounded to 16 bits; what is checked of other calls is checked of these."""
    dropout(Bufs(), INVAL, res=None, type=FP32, rtype=rtype, x=None)
    dropout(Bufs(), INVAL, res=None, type=FP32, rtype=rtype, sy=S(256, 128, 16))
    dropout(Bufs(), UNSUP, type=FP32, rtype=rtype)  # beside a residual
    dropout(Bufs(), UNSUP, res=None, type=BF16, rtype=FP16)
    dropout(Bufs(), UNSUP, res=None, type=FP32, rtype=3)
    b = Bufs()
    dropout(b, INVAL, res=None, type=FP32, rtype=rtype, y=b[0])  # another type in the input's place


def test_dropout_overlap():
    b = Bufs()
    dropout(b, INVAL, y=b[0] + 64)
    dropout(b, INVAL, y=b[1] + 2)
    dropout(b, INVAL, y=b[0], sy=S(512, 256, 32))
    dropout(b, INVAL, y=b[0], rtype=FP32)  # another type in the input's place
    dropout(b, INVAL, drop=DropoutSpec(1, 2, b[2] + 8, 0.5))


HEADS = S(4 * 256 * 64, 256 * 64, 64)  # 2 x 4 x 256 rows of 64


def means(b, want, **o):
    a = dict(k=b[0], sk=HEADS, lens=b[1], means=b[2], scales=b[3], B=1, Hk=4, Nk=256, d=64, block=64)
    a.update(o)
    b.check(lib().vitattn_block_means(*a.values(), None), want)


@pytest.mark.parametrize("o,want", [
    (dict(k=None), INVAL), (dict(means=None), INVAL), (dict(scales=None), INVAL), (dict(B=0), INVAL), (dict(Hk=0), INVAL),
    (dict(Nk=0), INVAL), (dict(d=4), UNSUP), (dict(d=168), UNSUP), (dict(d=60), UNSUP), (dict(block=0), UNSUP), (dict(block=96), UNSUP),
    (dict(block=1088), UNSUP), (dict(block=-64), UNSUP), (dict(Nk=16384 * 64 + 1), UNSUP), (dict(sk=S(0, 0, 56)), INVAL),
    (dict(sk=S(0, 4, 64)), INVAL)])
def test_means_refusals(o, want):
    means(Bufs(), want, **o)


def test_means_alignment_and_overlap():
    b = Bufs()
    means(b, INVAL, k=b[0] + 8)
    means(b, INVAL, means=b[2] + 4)
    means(b, INVAL, lens=b[1] + 2)
    means(b, INVAL, means=b[0])
    means(b, INVAL, scales=b[2] + 1020)
    means(b, INVAL, scales=b[1])


def select(b, want, **o):
    a = dict(q=b[0], sq=HEADS, means=b[1], scales=b[2], blocks=b[3], B=1, H=4, Hk=2, Nq=256, d=64, nb=8, q_block=64, topk=4)
    a.update(o)
    b.check(lib().vitattn_block_select(*a.values(), None), want)


@pytest.mark.parametrize("o,want", [
    (dict(q=None), INVAL), (dict(means=None), INVAL), (dict(scales=None), INVAL), (dict(blocks=None), INVAL), (dict(Hk=3), INVAL),
    (dict(Hk=0), INVAL), (dict(nb=0), INVAL), (dict(nb=16385), UNSUP), (dict(q_block=0), INVAL), (dict(topk=0), INVAL),
    (dict(topk=257), UNSUP), (dict(d=12), UNSUP), (dict(B=65536, sq=S(0, 64, 64)), INVAL), (dict(blocks=2), INVAL)])
def test_select_refusals(o, want):
    select(Bufs(), want, **o)


def test_select_overlap():
    b = Bufs()
    for i in (0, 1, 2):
        select(b, INVAL, blocks=b[i])


def fwd(b, want, **o):
    a = dict(q=b[0], sq=HEADS, k=b[1], sk=HEADS, v=b[2], sv=HEADS, blocks=b[3], lens=b[4], o=b[5], so=HEADS, o32=b[6], lse=b[7],
             B=1, H=4, Hk=4, Nq=256, Nk=256, d=64, block=64, q_block=64, topk=8, scale=0.125, ws=b[8], wsb=1 << 20)
    a.update(o)
    b.check(lib().vitattn_block_fwd(*a.values(), None), want)


SIZES = [
    (dict(B=0), INVAL), (dict(H=6), INVAL), (dict(Hk=0), INVAL), (dict(Nq=0), INVAL), (dict(Nk=0), INVAL), (dict(d=0), UNSUP),
    (dict(d=20), UNSUP), (dict(d=168), UNSUP), (dict(block=32), UNSUP), (dict(block=100), UNSUP), (dict(block=2048), UNSUP),
    (dict(q_block=0), INVAL), (dict(topk=0), INVAL), (dict(topk=1025), UNSUP), (dict(Nk=16384 * 64 + 1), UNSUP), (dict(scale=0.0), INVAL),
    (dict(scale=float("nan")), INVAL), (dict(scale=-1.0), INVAL), (dict(H=4096, Hk=2), UNSUP), (dict(Nq=2 ** 26 + 1), INVAL),
    (dict(B=2 ** 13, H=2 ** 11, Hk=2, Nq=1024), INVAL), (dict(B=2 ** 10, H=2 ** 10, Hk=2 ** 10, Nq=300), INVAL),
    (dict(sq=S(0, 0, 60)), INVAL), (dict(sk=S(0, 12, 64)), INVAL),
    (dict(sv=S(0, 0, 2 ** 31)), INVAL), (dict(Nk=2 ** 20, sk=S(0, 0, 1024)), INVAL), (dict(q=None), INVAL), (dict(k=None), INVAL),
    (dict(v=None), INVAL), (dict(blocks=None), INVAL)]


@pytest.mark.parametrize("o,want", SIZES + [(dict(o=None), INVAL), (dict(so=S(0, 0, 64)), INVAL), (dict(ws=None), WS),
                                            (dict(wsb=64), WS)])
def test_forward_refusals(o, want):
    fwd(Bufs(), want, **o)


def test_forward_alignment_and_overlap():
    b = Bufs()
    for n in ("q", "k", "v", "o", "o32", "lse"):
        fwd(b, INVAL, **{n: b[9] + 8})
    for n in ("blocks", "lens"):
        fwd(b, INVAL, **{n: b[9] + 2})
    for n in ("o", "o32", "lse", "ws"):
        for i in (0, 1, 2, 3, 4):
            fwd(b, INVAL, **{n: b[i]})
    fwd(b, INVAL, o=b[6])
    fwd(b, INVAL, ws=b[5])


def bwd(b, want, **o):
    a = dict(q=b[0], sq=HEADS, k=b[1], sk=HEADS, v=b[2], sv=HEADS, blocks=b[3], lens=b[4], o32=b[5], lse=b[6], dout=b[7], sdo=HEADS,
             dq=b[8], sdq=HEADS, dk=b[9], sdk=HEADS, dv=b[10], sdv=HEADS, B=1, H=4, Hk=4, Nq=256, Nk=256, d=64, block=64, q_block=64,
             topk=8, scale=0.125, ws=b[11], wsb=4 << 20)
    a.update(o)
    b.check(lib().vitattn_block_bwd(*a.values(), None), want)


@pytest.mark.parametrize("o,want", SIZES + [
    (dict(dout=None), INVAL), (dict(dq=None), INVAL), (dict(dk=None), INVAL), (dict(dv=None), INVAL), (dict(o32=None), INVAL),
    (dict(lse=None), INVAL), (dict(ws=None), WS), (dict(wsb=64), WS), (dict(sdq=S(0, 0, 64)), INVAL), (dict(sdk=S(0, 64, 64)), INVAL)])
def test_backward_refusals(o, want):
    bwd(Bufs(), want, **o)


def test_backward_overlap():
    b = Bufs()
    for n in ("dq", "dk", "dv", "ws"):
        for i in range(8):
            bwd(b, INVAL, **{n: b[i]})
    bwd(b, INVAL, dk=b[8])
    bwd(b, INVAL, dv=b[9])
    bwd(b, INVAL, dq=b[7] + 64)


def test_workspace_bytes():
    f, g = lib().vitattn_block_fwd_workspace_bytes, lib().vitattn_block_bwd_workspace_bytes
    assert f(1, 8, 8, 32768, 32768, 64, 64, 64, 32) == 0  # many queries are not split
    assert f(1, 8, 8, 1, 131072, 128, 128, 1, 32) == 8 * 32 * 129 * 4
    assert f(1, 8, 8, 1, 64, 128, 64, 1, 1) == 0
    for bad in ((0, 8, 8, 1, 64, 64, 64, 1, 1), (1, 8, 3, 1, 64, 64, 64, 1, 1), (1, 8, 8, 1, 64, 60, 64, 1, 1),
                (1, 8, 8, 1, 64, 64, 65, 1, 1), (1, 8, 8, 1, 64, 64, 64, 0, 1), (1, 8, 8, 1, 64, 64, 64, 1, 1025),
                (1, 8, 8, 1, 2 ** 31, 64, 64, 1, 1)):
        assert f(*bad) == 0 and g(*bad) == 0
    # statistics, the map, counts, first items, items; no shares if no block can have two runs
    pad = lambda n: -(-n // 256) * 256  # noqa: E731
    assert g(1, 1, 1, 64, 64, 64, 64, 64, 1) == pad(2 * 64 * 4) + pad(8) + pad(4) + pad(8) + pad(16)
    # a sample's length is no reason for workspace by the square
    assert g(1, 1, 1, 1 << 20, 1 << 20, 64, 128, 128, 16) < 8 << 30


def test_host_tensors_are_refused():
    torch = pytest.importorskip("torch")
    x, q = torch.zeros(4, 64), torch.zeros(1, 1, 64, 64, dtype=torch.bfloat16)
    ids = torch.zeros(1, 1, 64, 1, dtype=torch.int32)
    for call in (lambda: va.rms_norm(x), lambda: va.rms_norm_fp8(x), lambda: va.dropout(x, 0.5, (1, 2)), lambda: va.block_means(q),
                 lambda: va.block_attention(q, q, q, ids, 64),
                 lambda: va.block_select(q, (torch.zeros(1, 1, 1, 64, dtype=torch.int8), torch.zeros(1, 1, 1)), 1)):
        with pytest.raises(TypeError):
            call()


def test_dropout_rate_is_checked_before_its_state():
    from paper_2405_15780_amd.binding import _rng

    assert _rng(0.0, None, None) is None
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(ValueError):
            _rng(p, (1, 2), None)
    with pytest.raises(ValueError):
        _rng(0.5, None, None)
    s = _rng(0.5, (-1, 2 ** 64 + 3), None)
    assert (s.seed, s.offset, s.state, s.p) == (2 ** 64 - 1, 3, None, 0.5)
    with pytest.raises(TypeError):
        _rng(0.5, (1.5, 2), None)


def test_field_layout():
    assert [getattr(DropoutSpec, n).offset for n in ("seed", "offset", "state", "p")] == [0, 8, 16, 24]
    assert ctypes.sizeof(DropoutSpec) == 32
    assert np.dtype(np.int32).itemsize == 4
