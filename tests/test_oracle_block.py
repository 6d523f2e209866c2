"""The fp64 oracles of layer norm, rotary positions and differential attention,
pinned on the CPU: closed forms, a library's autograd in fp64 and central
differences."""
import numpy as np
import pytest

import oracle.block as ob


def rng(seed=0):
    return np.random.default_rng(seed)


def test_layer_norm_closed_form():
    y, mean, rstd = ob.layer_norm([[1.0, 3.0], [5.0, 5.0]], [2.0, 2.0], [1.0, 0.0], 0.0 + 1e-300)
    assert np.allclose(mean, [2.0, 5.0]) and np.isclose(rstd[0], 1.0)
    assert np.allclose(y[0], [-1.0, 2.0]) and np.allclose(y[1], [1.0, 0.0])


@pytest.mark.parametrize("D", [1, 2, 7, 72])
@pytest.mark.parametrize("with_w", [True, False])
def test_layer_norm_gradients(D, with_w):
    import torch

    r = rng(D)
    x, dy = r.normal(size=(3, 4, D)), r.normal(size=(3, 4, D))
    w, b = (r.normal(size=D), r.normal(size=D)) if with_w else (None, None)
    t = [None if a is None else torch.tensor(a, requires_grad=True) for a in (x, w, b)]
    y = torch.nn.functional.layer_norm(t[0], (D,), t[1], t[2], 1e-3)
    y.backward(torch.tensor(dy))
    assert np.allclose(ob.layer_norm(x, w, b, 1e-3)[0], y.detach().numpy())
    dx, dw, db = ob.layer_norm_backward(x, w, 1e-3, dy)
    assert np.allclose(dx, t[0].grad.numpy())
    if with_w:
        assert np.allclose(dw, t[1].grad.numpy()) and np.allclose(db, t[2].grad.numpy())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("joint", [False, True])
def test_rotary_turns_pairs_as_complex_numbers(interleaved, joint):
    r = rng(3)
    B, H, N, d, sections = 2, 3, 5, 14, (2, 0, 4)
    x, pos = r.normal(size=(B, H, N, d)), r.integers(0, 50, size=(B, N, 3))
    y = ob.rotary(x, pos, sections, 100.0, interleaved, joint)
    R, p = 6, 0
    for a, n in enumerate(sections):
        for i in range(n):
            lo, hi = (2 * p, 2 * p + 1) if interleaved else (p, R + p)
            f = 100.0 ** -(p / R if joint else i / n)
            z = (x[..., lo] + 1j * x[..., hi]) * np.exp(1j * pos[:, None, :, a] * f)
            assert np.allclose(y[..., lo], z.real) and np.allclose(y[..., hi], z.imag)
            p += 1
    assert np.array_equal(y[..., 12:], x[..., 12:])
    assert np.allclose(ob.rotary(y, pos, sections, 100.0, interleaved, joint, inverse=True), x)


def test_rotary_gradient_is_the_inverse_turn():
    r = rng(4)
    x, g, pos = r.normal(size=(1, 1, 4, 6)), r.normal(size=(1, 1, 4, 6)), r.integers(0, 9, size=(4, 1))
    f = lambda a: (ob.rotary(a, pos, (3,), 10.0) * g).sum()  # noqa: E731
    want = ob.rotary(g, pos, (3,), 10.0, inverse=True)
    for at in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[at] = 1e-5
        assert np.isclose((f(x + e) - f(x - e)) / 2e-5, want[at], atol=1e-8)


def test_diff_attention_is_the_difference_of_two_attentions():
    import oracle

    r = rng(5)
    B, H, N, d = 2, 2, 9, 8
    q, k, v, g = r.normal(size=(B, 2 * H, N, d)), r.normal(size=(B, 2 * H, N, d)), r.normal(size=(B, H, N, d)), \
        r.normal(size=(B, H, N, d))
    lam, scale = np.array([0.3, -1.2]), 0.25
    got = ob.diff_attention(q, k, v, lam, scale, dout=g)
    one = [oracle.forward_backward(q[:, m::2], k[:, m::2], v, g, scale) for m in (0, 1)]
    f = lam[None, :, None, None]
    assert np.allclose(got["o"], one[0]["o"] - f * one[1]["o"])
    assert np.allclose(got["o2"][:, 0::2], one[0]["o"]) and np.allclose(got["o2"][:, 1::2], one[1]["o"])
    assert np.allclose(got["dv"], one[0]["dv"] - f * one[1]["dv"])
    for n in ("dq", "dk"):
        assert np.allclose(got[n][:, 0::2], one[0][n]) and np.allclose(got[n][:, 1::2], -f * one[1][n])
    assert np.allclose(got["lse"][:, 0::2], one[0]["lse"]) and np.allclose(got["lse"][:, 1::2], one[1]["lse"])
    assert np.allclose(got["dlam"], -(g * one[1]["o"]).sum((0, 2, 3)))


def test_diff_attention_gradients_by_differences():
    r = rng(6)
    B, H, Nq, Nk, d, e = 2, 1, 3, 5, 4, 6
    x = {"q": r.normal(size=(B, 2 * H, Nq, d)), "k": r.normal(size=(B, 2 * H, Nk, d)), "v": r.normal(size=(B, H, Nk, e)),
         "lam": r.normal(size=H)}
    g, lens = r.normal(size=(B, H, Nq, e)), [5, 2]
    want = ob.diff_attention(**x, scale=0.7, key_lens=lens, dout=g)
    for n in x:
        for at in np.ndindex(x[n].shape):
            hi, lo = ({m: a.copy() for m, a in x.items()} for _ in range(2))
            hi[n][at] += 1e-5
            lo[n][at] -= 1e-5
            diff = [(ob.diff_attention(**y, scale=0.7, key_lens=lens)["o"] * g).sum() for y in (hi, lo)]
            assert np.isclose((diff[0] - diff[1]) / 2e-5, want["d" + n][at], atol=1e-7), (n, at)


def test_diff_attention_without_keys():
    r = rng(7)
    q, k, v, g = r.normal(size=(2, 2, 3, 8)), r.normal(size=(2, 2, 4, 8)), r.normal(size=(2, 1, 4, 8)), \
        r.normal(size=(2, 1, 3, 8))
    got = ob.diff_attention(q, k, v, [0.5], 0.3, key_lens=[0, 4], dout=g)
    for n in ("o", "o2", "dq", "dk", "dv"):
        assert not got[n][0].any() and got[n][1].any()
    assert np.isneginf(got["lse"][0]).all()
