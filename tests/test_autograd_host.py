"""The autograd wrappers of layer norm, rotary positions and differential attention
on the CPU, the kernels' calls replaced by elementary torch operations: what
reaches them, and what is refused."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

import paper_2405_15780_amd as va  # noqa: E402
from paper_2405_15780_amd import binding  # noqa: E402


@pytest.fixture
def stand_ins(monkeypatch):
    """Replaces the calls that launch; returns the list of calls made."""
    calls = []

    def norm_fwd(x, weight=None, bias=None, eps=1e-5, out=None, stats=True):
        calls.append("layer_norm_fwd")
        mean, rstd = x.mean(-1), 1 / (x.var(-1, correction=0) + eps).sqrt()
        y = (x - mean[..., None]) * rstd[..., None]
        y = y if weight is None else y * weight
        y = y if bias is None else y + bias
        return y, mean, rstd

    def rotary_fwd(q, k, positions, sections, base=10000.0, interleaved=False, joint=False, inverse=False, out=None):
        calls.append(("rotary_fwd", tuple(q.shape), k is not None, inverse))
        return 2 * q if k is None else (2 * q, 2 * k)

    def diff_fwd(q, k, v, lam, scale=None, key_lens=None, out=None, save=True, workspace=None):
        calls.append("diff_fwd")
        B, H2, N, _ = q.shape
        o = torch.ones((B, H2 // 2, N, v.shape[3])) * lam.view(1, -1, 1, 1)
        return o, torch.ones((B, H2, N, v.shape[3])), torch.ones((B, H2, N))

    for f, g in (("layer_norm_fwd", norm_fwd), ("rotary_fwd", rotary_fwd), ("diff_fwd", diff_fwd)):
        monkeypatch.setattr(binding, f, g)
    return calls


X = dict(x=(3, 8), weight=(8,), bias=(8,))
QKV = dict(q=(1, 4, 5, 8), k=(1, 4, 6, 8), v=(1, 2, 6, 16), lam=(2,))
POS = torch.zeros((5, 1))


def layer_norm(ts):
    return va.layer_norm(ts["x"], ts["weight"], ts["bias"])


def rotary(ts):
    out = va.rotary(ts["q"], ts["k"][:, :, :5] if ts["k"] is not None else None, POS, (4,))
    return out[0] if isinstance(out, tuple) else out


def diff(ts):
    return va.diff_attention(ts["q"], ts["k"], ts["v"], ts["lam"])


CALLS = [(layer_norm, X, n) for n in X] + [(rotary, QKV, n) for n in ("q", "k")] + [(diff, QKV, n) for n in QKV]


@pytest.mark.parametrize("off", [False, True])
@pytest.mark.parametrize("fn,shapes,dual", CALLS)
def test_forward_mode_tangents_are_refused_and_not_dropped(stand_ins, fn, shapes, dual, off):
    """The functions have no forward-mode derivative; an output without a tangent would count as a constant. no_grad does
    not end forward mode."""
    import torch.autograd.forward_ad as fw

    with fw.dual_level(), torch.no_grad() if off else contextlib.nullcontext():
        ts = {n: torch.randn(s) for n, s in shapes.items()}
        fn(ts)  # a call without a tangent is made as ever
        assert len(stand_ins) == 1
        ts[dual] = fw.make_dual(ts[dual], torch.randn(shapes[dual]))
        with pytest.raises((NotImplementedError, RuntimeError)):
            y = fn(ts)
            assert fw.unpack_dual(y).tangent is not None


@pytest.mark.parametrize("fn,shapes", [(layer_norm, X), (rotary, QKV), (diff, QKV)])
def test_functional_derivatives_are_refused(stand_ins, fn, shapes):
    ts = {n: torch.randn(s) for n, s in shapes.items()}
    first = next(iter(shapes))
    with pytest.raises(Exception):
        torch.func.jvp(lambda x: fn({**ts, first: x}), (ts[first],), (torch.ones(shapes[first]),))


def test_the_output_of_diff_attention_is_free(stand_ins, monkeypatch):
    """The backward reads the unrounded maps' outputs, so o is neither kept alive nor held against in-place operations."""
    seen = []

    def diff_bwd(q, k, v, lam, o, o2, lse, dout, scale=None, key_lens=None, want_dlam=True, workspace=None, **wants):
        seen.append((o, dout))
        return torch.ones_like(q), torch.ones_like(k), torch.ones_like(v), torch.ones_like(lam)

    monkeypatch.setattr(binding, "diff_bwd", diff_bwd)
    ts = {n: torch.randn(s, requires_grad=True) for n, s in QKV.items()}
    saved = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: saved.append(t.shape) or t, lambda t: t):
        o = diff(ts)
    assert o.shape not in saved and ts["q"].shape in saved
    o.mul_(3.0)
    o.sum().backward()
    assert seen[0][0] is None and (seen[0][1] == 3).all()
    assert all((t.grad == 1).all() for t in ts.values())


@pytest.mark.parametrize("need", ["q", "k", "qk"])
def test_rotary_turns_back_only_what_is_asked_for(stand_ins, need):
    q, k = torch.randn((1, 4, 5, 8), requires_grad="q" in need), torch.randn((1, 2, 5, 8), requires_grad="k" in need)
    a, b = va.rotary(q, k, POS, (4,))
    (a.sum() + b.sum()).backward()
    assert stand_ins[1:] == [("rotary_fwd", tuple((k if need == "k" else q).shape), need == "qk", True)]
    for x, n in ((q, "q"), (k, "k")):
        assert x.grad is None if n not in need else (x.grad == 2).all()


def test_positions_get_no_gradient(stand_ins):
    """Also where they are all that a gradient's own backward could go to."""
    q, pos = torch.randn((1, 4, 5, 8), requires_grad=True), torch.zeros((5, 1), requires_grad=True)
    y = va.rotary(q, None, pos, (4,))
    (g,) = torch.autograd.grad(y.sum(), q, create_graph=True)
    assert (g == 2).all()
    g.sum().backward()
    assert pos.grad is None and q.grad is None
