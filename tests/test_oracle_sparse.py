"""The fp64 oracle of the rms norm, dropout's counter and the attention over chosen
blocks against published vectors, library routines and finite differences."""
import numpy as np
import pytest

import oracle.sparse as os_

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("counter,key,want", [
    # the known answers published with the generator
    ([0, 0, 0, 0], [0, 0], [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
    ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
    ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
     [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1])])
def test_philox(counter, key, want):
    assert os_.philox(np.array(counter, dtype=np.uint64), np.array(key, dtype=np.uint64)).tolist() == want


def test_kept():
    keep, up = os_.kept((3, 5, 1001), 0.3, 12345, 2 ** 40 + 7)
    t = round(0.3 * 65536)
    assert up == 65536 / (65536 - t)
    n = keep.size
    assert abs(keep.mean() - (1 - t / 65536)) < 5 * np.sqrt(0.21 / n)
    # rows, offsets and seeds are apart; a row's head is that of a longer row
    assert not np.array_equal(keep[0, 0], keep[0, 1])
    assert not np.array_equal(keep, os_.kept((3, 5, 1001), 0.3, 12345, 2 ** 40 + 8)[0])
    assert not np.array_equal(keep, os_.kept((3, 5, 1001), 0.3, 12346, 2 ** 40 + 7)[0])
    assert np.array_equal(keep[..., :17], os_.kept((3, 5, 17), 0.3, 12345, 2 ** 40 + 7)[0])
    assert os_.kept((4, 9), 0.0, 1, 1)[0].all() and not os_.kept((4, 9), 1.0, 1, 1)[0].any()
    assert np.array_equal(os_.kept((4, 9), 0.5, -1, 3)[0], os_.kept((4, 9), 0.5, 2 ** 64 - 1, 3)[0])


def test_rms_norm_gradients():
    rng = np.random.default_rng(1)
    h, w, dy = rng.standard_normal((4, 3, 13)), rng.standard_normal(13), rng.standard_normal((4, 3, 13))
    dh, dw = os_.rms_norm_backward(h, w, 1e-3, dy)
    f = lambda h, w: (os_.rms_norm(h, w, 1e-3)[0] * dy).sum()  # noqa: E731
    for i in ((0, 0, 0), (2, 1, 7), (3, 2, 12)):
        e = np.zeros_like(h)
        e[i] = 1e-5
        assert abs((f(h + e, w) - f(h - e, w)) / 2e-5 - dh[i]) < 1e-8
    e = np.zeros(13)
    e[4] = 1e-5
    assert abs((f(h, w + e) - f(h, w - e)) / 2e-5 - dw[4]) < 1e-8


def test_select_by_hand():
    k = np.zeros((1, 1, 256, 8))
    k[0, 0, :64, 0], k[0, 0, 64:128, 0], k[0, 0, 128:192, 1], k[0, 0, 192:, 0] = 1, 3, 5, 3
    m, scale = os_.block_means(k, 64)
    assert m[0, 0, :, 0].tolist() == [127, 127, 0, 127] and m[0, 0, 2, 1] == 127
    assert np.array_equal(scale[0, 0], np.float32(np.array([1, 3, 5, 3]) * (1 / 127)))
    q = np.zeros((1, 1, 2, 8))
    q[0, 0, 0, 0], q[0, 0, 1, 1] = 2, 1
    assert os_.block_select(q, (m, scale), 1, 1)[0, 0].tolist() == [[1], [2]]  # (of equal ones the lowest)
    assert os_.block_select(q, (m, scale), 3, 1)[0, 0].tolist() == [[0, 1, 3], [0, 1, 2]]
    assert os_.block_select(q, os_.block_means(k, 64, [100]), 3, 2)[0, 0].tolist() == [[0, 1, -1]]


@pytest.mark.parametrize("q_block,lens", [(1, None), (3, [50, 0]), (64, [96, 70])])
def test_attention(q_block, lens):
    rng = np.random.default_rng(q_block)
    B, H, Hk, Nq, Nk, d, block = 2, 4, 2, 37, 96, 8, 32
    q, k, v, g = (rng.standard_normal(s) for s in ((B, H, Nq, d), (B, Hk, Nk, d), (B, Hk, Nk, d), (B, H, Nq, d)))
    blocks = rng.integers(-1, 4, (B, H, -(-Nq // q_block), 2)).astype(np.int32)
    mask = os_.allowed(blocks, Nq, Nk, block, q_block, lens)
    r = os_.block_attention(q, k, v, mask, 0.3, g)
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    s = 0.3 * tq @ tk.repeat_interleave(2, 1).transpose(-1, -2)
    m = torch.tensor(mask)
    p = torch.softmax(s.masked_fill(~m, -1e300), -1) * m.any(-1, keepdim=True)
    o = p @ tv.repeat_interleave(2, 1)
    o.backward(torch.tensor(g))
    for got, want in ((r["o"], o.detach()), (r["dq"], tq.grad), (r["dk"], tk.grad), (r["dv"], tv.grad)):
        assert np.abs(got - want.numpy()).max() < 1e-12
    lse = torch.logsumexp(s.masked_fill(~m, -np.inf), -1).detach().numpy()
    some = mask.any(-1)
    assert np.abs(r["lse"] - lse)[some].max() < 1e-12 and (r["lse"][~some] == -np.inf).all()
