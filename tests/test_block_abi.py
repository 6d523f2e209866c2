"""The C entry points of layer norm, rotary positions and differential attention
refuse what they cannot compute before any HIP call: a status, no output touched,
no GPU needed."""
import ctypes

import numpy as np
import pytest

va = pytest.importorskip("paper_2405_15780_amd")
from paper_2405_15780_amd.binding import Strides as S  # noqa: E402

INVAL, UNSUP, WS = 1, 2, 3
BF16, FP16, FP32 = 0, 1, 2


def lib():
    try:
        return va.library()
    except ImportError as e:  # the library must be built before the tests run
        pytest.fail(str(e))


class Bufs:
    """Host buffers in the place of device memory, 1 MB apart."""

    def __init__(self, n=16):
        self.mem = np.full((n, 1 << 18), 7.0, dtype=np.float32)
        assert self.mem.ctypes.data % 16 == 0

    def __getitem__(self, i):
        return self.mem.ctypes.data + (i << 20)

    def check(self, status, want):
        assert status == want
        assert (self.mem == 7.0).all()


def norm_fwd(b, want, **o):
    a = dict(x=b[0], sx=S(256, 128, 32), w=b[1], b=b[2], y=b[3], sy=S(256, 128, 32), mean=b[4], rstd=b[5], B=2, H=2, N=4,
             D=32, eps=1e-5, type=BF16, wtype=BF16)
    a.update(o)
    b.check(lib().vitattn_layer_norm_fwd(*a.values(), None), want)


@pytest.mark.parametrize("o,want", [
    (dict(x=None), INVAL), (dict(y=None), INVAL), (dict(B=0), INVAL), (dict(H=-1), INVAL), (dict(N=0), INVAL), (dict(D=0), INVAL),
    (dict(D=(1 << 24) + 1), UNSUP), (dict(N=2 ** 30, B=2, H=1), INVAL), (dict(type=3), UNSUP), (dict(type=-1), UNSUP),
    (dict(wtype=FP16), UNSUP), (dict(eps=-1e-9), INVAL), (dict(eps=float("inf")), INVAL), (dict(eps=float("nan")), INVAL),
    (dict(mean=None), INVAL), (dict(rstd=None), INVAL), (dict(sx=S(-1, 128, 32)), INVAL), (dict(sy=S(256, 128, 31)), INVAL),
    (dict(sy=S(0, 128, 32)), INVAL), (dict(sy=S(256, 32, 32)), INVAL)])
def test_norm_forward_refusals(o, want):
    norm_fwd(Bufs(), want, **o)


def test_norm_forward_alignment_and_overlap():
    b = Bufs()
    norm_fwd(b, INVAL, x=b[0] + 1)
    norm_fwd(b, INVAL, w=b[1] + 2, wtype=FP32)
    norm_fwd(b, INVAL, mean=b[4] + 2)
    norm_fwd(b, INVAL, y=b[0] + 64)  # shifted onto the input
    norm_fwd(b, INVAL, y=b[0], sy=S(512, 256, 32))  # in place, with other strides


def norm_bwd(b, want, **o):
    a = dict(x=b[0], sx=S(256, 128, 32), w=b[1], mean=b[2], rstd=b[3], dy=b[4], sdy=S(256, 128, 32), dx=b[5],
             sdx=S(256, 128, 32), dw=b[6], db=b[7], B=2, H=2, N=4, D=32, type=BF16, wtype=BF16, ws=b[8], wsb=1 << 20)
    a.update(o)
    b.check(lib().vitattn_layer_norm_bwd(*a.values(), None), want)


@pytest.mark.parametrize("o,want", [
    (dict(x=None), INVAL), (dict(dy=None), INVAL), (dict(dx=None), INVAL), (dict(mean=None), INVAL), (dict(rstd=None), INVAL),
    (dict(ws=None), WS), (dict(wsb=64), WS), (dict(sdx=S(256, 0, 32)), INVAL), (dict(sdy=S(256, -128, 32)), INVAL),
    (dict(D=0), INVAL), (dict(wtype=5), UNSUP)])
def test_norm_backward_refusals(o, want):
    norm_bwd(Bufs(), want, **o)


def test_norm_backward_overlaps():
    b = Bufs()
    norm_bwd(b, INVAL, dx=b[0])
    norm_bwd(b, INVAL, dx=b[4] + 64)
    norm_bwd(b, INVAL, dx=b[4], sdx=S(512, 256, 32))
    rows = dict(B=1, H=1, N=2, D=16392, sx=S(0, 0, 16392), sdy=S(0, 0, 16392), sdx=S(0, 0, 16392))
    norm_bwd(b, INVAL, dx=b[4], **rows)  # dw would be summed from an overwritten dy


def test_norm_outputs_over_other_operands():
    """An output over an operand that is not its row's input: the weights, the statistics, another output."""
    b = Bufs()
    norm_fwd(b, INVAL, y=b[1])
    norm_fwd(b, INVAL, mean=b[0])
    norm_fwd(b, INVAL, rstd=b[4])  # mean's
    norm_fwd(b, INVAL, rstd=b[3] + 1016)  # y's last bytes
    norm_fwd(b, INVAL, mean=b[2] + 60)  # the bias's
    norm_bwd(b, INVAL, dx=b[1])
    norm_bwd(b, INVAL, dx=b[2])
    norm_bwd(b, INVAL, dw=b[0] + 64)
    norm_bwd(b, INVAL, dw=b[7] + 62)  # db's
    norm_bwd(b, INVAL, ws=b[0])
    norm_bwd(b, INVAL, ws=b[5])


def test_norm_most_rows():
    """A row's index and one round's rows beyond it stay below 2^31."""
    for n in (2 ** 31 - 1, 2 ** 31 - 2 ** 21, 2 ** 31 - 2 ** 22):
        one = dict(B=1, H=1, N=n, D=8, sx=S(0, 0, 0))
        norm_fwd(Bufs(), INVAL, sy=S(0, 0, 8), y=2 ** 40, mean=2 ** 41, rstd=2 ** 42, **one)
        assert lib().vitattn_layer_norm_bwd_workspace_bytes(1, 1, n, 8, BF16) == 0
    assert lib().vitattn_layer_norm_bwd_workspace_bytes(1, 1, 2 ** 31 - 2 ** 22 - 1, 8, BF16) > 0


def test_norm_workspace_bytes():
    f = lib().vitattn_layer_norm_bwd_workspace_bytes
    assert f(1, 1, 1, 64, BF16) == 2 * 64 * 4
    assert f(1, 1, 100000, 64, BF16) % (2 * 64 * 4) == 0
    assert f(2, 3, 50, 64, BF16) == f(1, 1, 300, 64, BF16)
    for bad in ((0, 1, 1, 64, BF16), (1, 1, 1, 0, BF16), (1, 1, 1, 64, 7), (1, 1, 1, (1 << 24) + 1, BF16)):
        assert f(*bad) == 0


def rotary(b, want, sections=(8, 8), **o):
    n = len(sections or ())
    a = dict(q=b[0], sq=S(640, 160, 32), q2=b[1], sq2=S(640, 160, 32), Hq=4, k=b[2], sk=S(320, 160, 32), k2=b[3],
             sk2=S(320, 160, 32), Hk=2, pos=b[4], pb=0, pr=2, pa=1, pt=1, sections=None if sections is None else (ctypes.c_int * max(n, 1))(*sections), axes=n,
             base=1e4, B=2, N=5, d=32, type=BF16, flags=0)
    a.update(o)
    b.check(lib().vitattn_rotary(*a.values(), None), want)


@pytest.mark.parametrize("o,want", [
    (dict(q=None), INVAL), (dict(q2=None), INVAL), (dict(k=None), INVAL), (dict(k2=None), INVAL), (dict(pos=None), INVAL),
    (dict(B=0), INVAL), (dict(B=65536), INVAL), (dict(N=0), INVAL), (dict(Hq=0), INVAL), (dict(Hk=-1), INVAL), (dict(d=1), INVAL),
    (dict(Hq=65536, sq=S(0, 0, 0), sq2=S(0, 160, 32), B=1), INVAL), (dict(sections=(9, 8)), INVAL), (dict(sections=(0, 0)), INVAL),
    (dict(sections=(-1, 8)), INVAL), (dict(sections=()), INVAL), (dict(sections=(1,) * 9), UNSUP), (dict(sections=None, axes=1), INVAL),
    (dict(d=65538), UNSUP), (dict(type=4), UNSUP), (dict(flags=8), INVAL), (dict(pt=3), INVAL), (dict(pt=-1), INVAL),
    (dict(base=0.0), INVAL), (dict(base=float("nan")), INVAL), (dict(pr=-1), INVAL), (dict(sq2=S(640, 0, 32)), INVAL),
    (dict(sq=S(640, -160, 32)), INVAL), (dict(N=1 << 30, d=32), INVAL)])
def test_rotary_refusals(o, want):
    rotary(Bufs(), want, **o)


def test_rotary_more_pairs_than_supported_and_overlaps():
    b = Bufs()
    rotary(b, UNSUP, sections=(129,), d=258, sq=S(0, 0, 0), sk=S(0, 0, 0), sq2=S(5160, 1290, 258), sk2=S(2580, 1290, 258))
    rotary(b, INVAL, q=b[0] + 1)
    rotary(b, INVAL, pos=b[4] + 4)  # int64
    rotary(b, INVAL, q2=b[0] + 64)
    rotary(b, INVAL, q2=b[2])  # q' over k
    rotary(b, INVAL, q2=b[0], sq2=S(640, 32, 128))  # in place, with other strides
    rotary(b, INVAL, q2=b[2], k2=b[0])
    rotary(b, INVAL, k2=b[1])  # both outputs at one address


def test_rotary_output_over_the_positions():
    b = Bufs()
    rotary(b, INVAL, q2=b[4])
    rotary(b, INVAL, k2=b[4] + 72)  # the last position's


def diff_fwd(b, want, **o):
    a = dict(q=b[0], sq=S(1280, 320, 32), k=b[1], sk=S(896, 224, 32), v=b[2], sv=S(896, 448, 64), lam=b[3], lt=FP32, lens=None,
             o=b[4], so=S(1280, 640, 64), maps=b[5], lse=b[6], B=2, H=2, Nq=10, Nk=7, d=32, e=64, scale=0.2, ws=None, wsb=0)
    a.update(o)
    b.check(lib().vitattn_diff_fwd(*a.values(), None), want)


DIFF = [(dict(q=None), INVAL), (dict(k=None), INVAL), (dict(v=None), INVAL), (dict(lam=None), INVAL), (dict(B=0), INVAL),
        (dict(H=0), INVAL), (dict(Nq=0), INVAL), (dict(Nk=-1), INVAL), (dict(d=0), UNSUP), (dict(d=12), UNSUP), (dict(d=88), UNSUP),
        (dict(e=4), UNSUP), (dict(e=168), UNSUP), (dict(scale=0.0), INVAL), (dict(scale=float("nan")), INVAL), (dict(lt=FP16), UNSUP),
        (dict(sq=S(1280, 320, 24)), INVAL), (dict(sk=S(896, 224, 33)), INVAL), (dict(sv=S(896, 444, 64)), INVAL),
        (dict(sq=S(-8, 320, 32)), INVAL), (dict(Nk=2 ** 30), INVAL), (dict(B=2 ** 15, H=2 ** 15), INVAL),
        (dict(Nk=1 << 20, sk=S(0, 0, 1024)), INVAL)]


@pytest.mark.parametrize("o,want", DIFF + [(dict(o=None), INVAL), (dict(so=S(1280, 0, 64)), INVAL), (dict(so=S(640, 640, 64)), INVAL)])
def test_diff_forward_refusals(o, want):
    diff_fwd(Bufs(), want, **o)


def test_diff_forward_alignment_and_workspace():
    b = Bufs()
    for n, i in (("q", 0), ("k", 1), ("v", 2), ("o", 4), ("maps", 5), ("lse", 6)):
        diff_fwd(b, INVAL, **{n: b[i] + 8})
    diff_fwd(b, INVAL, lam=b[3] + 2)
    diff_fwd(b, INVAL, lens=b[7] + 2)
    f = lib().vitattn_diff_fwd_workspace_bytes
    assert f(2, 2, 10, 7, 32, 64) == 0 and f(1, 1, 100000, 100000, 64, 128) == 0
    need = f(2, 2, 1, 100000, 32, 64)
    assert need > 0 and need == 4 * f(1, 1, 1, 100000, 32, 64)
    one = dict(Nq=1, Nk=100000, sq=S(128, 32, 32), sk=S(0, 0, 32), sv=S(0, 0, 64), so=S(128, 64, 64))
    diff_fwd(b, WS, **one)
    diff_fwd(b, WS, ws=b[8], wsb=need - 1, **one)
    diff_fwd(b, WS, ws=b[8] + 4, wsb=need, **one)
    for bad in ((0, 1, 1, 4096, 64, 128), (1, 1, 1, 4096, 96, 128), (1, 1, 1, 4096, 64, 20)):
        assert f(*bad) == 0


def diff_bwd(b, want, **o):
    a = dict(q=b[0], sq=S(1280, 320, 32), k=b[1], sk=S(896, 224, 32), v=b[2], sv=S(896, 448, 64), lam=b[3], lt=FP32, lens=None,
             maps=b[5], lse=b[6], dout=b[7], sdo=S(1280, 640, 64), dq=b[8], sdq=S(1280, 320, 32), dk=b[9], sdk=S(896, 224, 32),
             dv=b[10], sdv=S(896, 448, 64), dlam=b[11], B=2, H=2, Nq=10, Nk=7, d=32, e=64, scale=0.2, ws=b[12], wsb=1 << 20)
    a.update(o)
    b.check(lib().vitattn_diff_bwd(*a.values(), None), want)


@pytest.mark.parametrize("o,want", DIFF + [
    (dict(maps=None), INVAL), (dict(lse=None), INVAL), (dict(dout=None), INVAL), (dict(dq=None), INVAL), (dict(dk=None), INVAL),
    (dict(dv=None), INVAL), (dict(ws=None), WS), (dict(wsb=256), WS), (dict(sdq=S(1280, 0, 32)), INVAL),
    (dict(sdk=S(896, 224, 16)), INVAL), (dict(sdv=S(0, 448, 64)), INVAL), (dict(sdo=S(1280, 640, 0)), INVAL)])
def test_diff_backward_refusals(o, want):
    diff_bwd(Bufs(), want, **o)


def test_diff_backward_workspace():
    f = lib().vitattn_diff_bwd_workspace_bytes
    assert f(2, 2, 10, 7, 32, 64) > 0
    b = Bufs()
    diff_bwd(b, WS, wsb=f(2, 2, 10, 7, 32, 64) - 1)
    diff_bwd(b, INVAL, dlam=b[11] + 2)
    assert f(1, 1, 0, 7, 32, 64) == 0 and f(1, 1, 10, 7, 82, 64) == 0


BIG = 2 ** 32  # an int of this and a valid size has the valid size's low 32 bits


def test_sizes_past_a_c_int_are_refused_and_not_cut_off():
    """No entry may compute the part of a call that a size's low 32 bits name."""
    b = Bufs()
    for o in (dict(N=BIG + 4), dict(B=BIG + 2), dict(H=BIG + 2), dict(D=BIG + 32), dict(type=BIG), dict(wtype=BIG), dict(N=-BIG + 4)):
        norm_fwd(b, INVAL if not {"type", "wtype"} & o.keys() else UNSUP, **o)
        norm_bwd(b, INVAL if not {"type", "wtype"} & o.keys() else UNSUP, **o)
    f = lib().vitattn_layer_norm_bwd_workspace_bytes
    assert f(1, 1, BIG + 5, 8, BF16) == f(1, 1, 5, BIG + 8, BF16) == f(BIG + 1, 1, 5, 8, BF16) == 0
    for o in (dict(N=BIG + 5), dict(B=BIG + 2), dict(Hq=BIG + 4), dict(Hk=BIG + 2), dict(d=BIG + 32), dict(axes=BIG + 2), dict(pt=BIG + 1),
              dict(flags=BIG)):
        rotary(b, INVAL, **o)
    rotary(b, UNSUP, type=BIG)
    for o in (dict(B=BIG + 2), dict(H=BIG + 2), dict(Nq=BIG + 10), dict(Nk=BIG + 7)):
        diff_fwd(b, INVAL, **o)
        diff_bwd(b, INVAL, **o)
    for o in (dict(d=BIG + 32), dict(e=BIG + 64), dict(lt=BIG + FP32)):
        diff_fwd(b, UNSUP, **o)
        diff_bwd(b, UNSUP, **o)
    for f in (lib().vitattn_diff_fwd_workspace_bytes, lib().vitattn_diff_bwd_workspace_bytes):
        ok = (1, 1, 3, 5000, 64, 128)
        assert f(*ok) > 0
        for i in range(6):
            assert f(*(n + BIG * (i == j) for j, n in enumerate(ok))) == 0


def test_int_arguments():
    from paper_2405_15780_amd import binding

    conv = binding.Int.from_param
    for n in (0, 1, -1, 2 ** 31 - 1, -2 ** 31, True, np.int64(7)):
        assert conv(n) == n
    for n in (2 ** 31, -2 ** 31 - 1, BIG, BIG + 5, np.int64(BIG + 5)):
        assert conv(n) == -2 ** 31
    for bad in (1.0, "1", None):
        with pytest.raises(TypeError):
            conv(bad)
    assert list(binding._c_ints((BIG + 8, 8))) == [-2 ** 31, 8]  # a section of so many pairs
    for name, (_, args) in binding._SIGNATURES.items():
        assert ctypes.c_int not in args or name == "vitattn_status_str"


def test_rotary_outputs_that_share_elements():
    """Also where both operands are turned in place, which interleaved heads of one tensor may be."""
    b = Bufs()
    x = b[0]  # [2][N = 5][6 heads][32]: q the first four heads, k from head `h` on
    fused = dict(sq=S(960, 32, 192), sq2=S(960, 32, 192), sk=S(960, 32, 192), sk2=S(960, 32, 192), q=x, q2=x)
    for h in (0, 1, 3):
        rotary(b, INVAL, k=x + 64 * h, k2=x + 64 * h, **fused)
    rotary(b, INVAL, k=x + 64 * 4 + 2, k2=x + 64 * 4 + 2, **fused)  # its last element is the next row's first
    rotary(b, INVAL, k=x + 64 * 4 - 2, k2=x + 64 * 4 - 2, **fused)
    # one row apart: q's and k's heads one after the other, rows shared
    rotary(b, INVAL, q=x, q2=x, k=x + 64, k2=x + 64, **dict.fromkeys(("sq", "sq2"), S(640, 160, 32)), **dict.fromkeys(("sk", "sk2"), S(640, 160, 32)))
    # new outputs
    rotary(b, INVAL, k2=b[1] + 320)
    rotary(b, INVAL, k2=b[1] - 2)
    rotary(b, INVAL, q2=b[1], sq2=S(960, 32, 192), k2=b[1] + 64 * 3, sk2=S(960, 32, 192))


def test_diff_outputs_that_share_memory():
    b = Bufs()
    for n in range(8):
        if n != 4:  # on every other operand
            diff_fwd(b, INVAL, o=b[n], lens=b[7])
    diff_fwd(b, INVAL, o=b[0] + 5040)  # q's last 80 bytes
    diff_fwd(b, INVAL, maps=b[6] - 16)
    for i in (0, 1, 2, 3, 4, 6, 7):
        diff_fwd(b, INVAL, maps=b[i], lens=b[7])
    for i in (0, 1, 2, 3, 4, 5, 7):
        diff_fwd(b, INVAL, lse=b[i], lens=b[7])
    # an output among q's heads: rows of 4 * 32 + 2 * 64 columns, q's first, o one head early
    fused = dict(q=b[0], sq=S(2560, 32, 256), so=S(2560, 64, 256))
    diff_fwd(b, INVAL, o=b[0] + 2 * 96, **fused)
    diff_fwd(b, INVAL, o=b[0] + 2 * 136, **fused)
    one = dict(B=1, H=1, Nq=1, Nk=1024, sq=S(64, 32, 32), sk=S(0, 32768, 32), sv=S(0, 0, 64), so=S(64, 64, 64), wsb=1 << 20)
    for i in (0, 1, 2, 3, 4, 5, 6):
        diff_fwd(b, INVAL, ws=b[i], **one)


@pytest.mark.parametrize("out", ["dq", "dk", "dv", "dlam", "ws"])
def test_diff_gradients_that_share_memory(out):
    b = Bufs()
    base = dict(q=0, k=1, v=2, lam=3, maps=5, lse=6, dout=7, dq=8, dk=9, dv=10, dlam=11, ws=12, lens=13)
    for n, i in base.items():
        if n != out:
            diff_bwd(b, INVAL, **{"lens": b[13], out: b[i]})


@pytest.mark.parametrize("Nq,least,most", [(1, 1024, 128), (64, 1024, 128), (65, 8192, 32), (256, 8192, 32)])
def test_number_of_splits(Nq, least, most):
    """The forward's workspace holds a row of e outputs and an LSE per split, map and query."""
    def splits(Nk):
        n = lib().vitattn_diff_fwd_workspace_bytes(1, 1, Nq, Nk, 64, 128)
        assert n % (4 * 2 * Nq * 129) == 0
        return n // (4 * 2 * Nq * 129)

    assert splits(least - 1) == 0 and splits(least) > 1
    for Nk in {n + i for n in (least, 65536, 65600, 66048, 131072, 131136, 1 << 20) for i in (0, 1, 63, 64, 127, 128, 129)}:
        assert 1 < splits(Nk) <= most, Nk
    assert splits(131072) == most and splits(1 << 20) == most
