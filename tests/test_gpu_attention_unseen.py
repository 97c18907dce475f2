"""Pairs that do not see each other contribute exactly nothing to attention and its gradient, however large the finite values on
either side are: 0 x 3e38 is 0, and an overflow in a product that the formula does not contain stays out of the sums."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2510_03515_b200 import binding as rb  # noqa: E402

BF = torch.bfloat16
HUGE = 3e38


def _rows(n, length, heads, kv, hd, seed):
    g = torch.Generator().manual_seed(seed)
    mk = lambda h: torch.randn(n * length, h, hd, generator=g).to(BF).cuda()  # noqa: E731
    return mk(heads), mk(kv), mk(kv), mk(heads)


def _signs(x, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randint(0, 2, x.shape, generator=g) * 2 - 1).to(BF).to(x.device) * HUGE


# n_seq = 1: length, head_dim, window, first position with other values
SEEN = [(100, 64, 0, 40), (300, 64, 0, 131), (300, 128, 0, 131), (700, 128, 0, 390), (700, 64, 0, 512), (130, 80, 0, 3)]
WINDOWED = [(300, 64, 20, 131), (700, 128, 130, 257), (700, 64, 256, 300), (90, 128, 7, 40)]


@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("length,hd,window,s", SEEN)
def test_later_keys(length, hd, window, s, what):
    q, k, v, dout = _rows(1, length, 4, 2, hd, 1)
    out, lse = rb.attention(q, k, v, 1, length, None, window)
    grads = rb.attention_grad(q, k, v, out, lse, dout, 1, length, None, window)
    k2, v2 = k.clone(), v.clone()
    (k2 if what == "k" else v2)[s:] = _signs(v[s:], 2)
    out2, lse2 = rb.attention(q, k2, v2, 1, length, None, window)
    assert torch.equal(out2[:s], out[:s]) and torch.equal(lse2[:, :, :s], lse[:, :, :s])
    got = rb.attention_grad(q, k2, v2, out, lse, dout, 1, length, None, window)
    assert torch.equal(got.dq[:s], grads.dq[:s])


@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("length,hd,window,s", WINDOWED)
def test_keys_before_the_window(length, hd, window, s, what):
    q, k, v, dout = _rows(1, length, 4, 2, hd, 3)
    out, lse = rb.attention(q, k, v, 1, length, None, window)
    grads = rb.attention_grad(q, k, v, out, lse, dout, 1, length, None, window)
    k2, v2 = k.clone(), v.clone()
    (k2 if what == "k" else v2)[:s] = _signs(v[:s], 4)
    out2, lse2 = rb.attention(q, k2, v2, 1, length, None, window)
    first = s + window - 1  # sees nothing before s
    assert torch.equal(out2[first:], out[first:]) and torch.equal(lse2[:, :, first:], lse[:, :, first:])
    got = rb.attention_grad(q, k2, v2, out, lse, dout, 1, length, None, window)
    assert torch.equal(got.dq[first:], grads.dq[first:])


@pytest.mark.parametrize("length,hd,window,s", SEEN)
def test_gradients_of_earlier_rows(length, hd, window, s):
    """Keys from s on are not seen by the rows before."""
    q, k, v, dout = _rows(1, length, 4, 2, hd, 5)
    out, lse = rb.attention(q, k, v, 1, length, None, window)
    grads = rb.attention_grad(q, k, v, out, lse, dout, 1, length, None, window)
    d2 = dout.clone()
    d2[:s] = _signs(dout[:s], 6)
    got = rb.attention_grad(q, k, v, out, lse, d2, 1, length, None, window)
    assert torch.equal(got.dk[s:], grads.dk[s:]) and torch.equal(got.dv[s:], grads.dv[s:]) and torch.equal(got.dq[s:], grads.dq[s:])


@pytest.mark.parametrize("length,hd,window,s", WINDOWED)
def test_gradients_of_rows_beyond_the_window(length, hd, window, s):
    q, k, v, dout = _rows(1, length, 4, 2, hd, 7)
    out, lse = rb.attention(q, k, v, 1, length, None, window)
    grads = rb.attention_grad(q, k, v, out, lse, dout, 1, length, None, window)
    d2 = dout.clone()
    d2[s + window - 1:] = _signs(dout[s + window - 1:], 8)
    got = rb.attention_grad(q, k, v, out, lse, d2, 1, length, None, window)
    assert torch.equal(got.dk[:s], grads.dk[:s]) and torch.equal(got.dv[:s], grads.dv[:s])


@pytest.mark.parametrize("n,length,hd", [(11, 21, 64), (40, 8, 128), (6, 64, 64), (130, 1, 128)])
def test_live_neighbours_in_a_tile(n, length, hd):
    """Short generations share tiles: what a live neighbour holds does not reach the others."""
    q, k, v, dout = _rows(n, length, 4, 2, hd, 9)
    out, lse = rb.attention(q, k, v, n, length)
    grads = rb.attention_grad(q, k, v, out, lse, dout, n, length)
    grid = lambda x: x.view(n, length, -1, hd)  # noqa: E731
    for which in range(4):
        x = [t.clone() for t in (q, k, v, dout)]
        grid(x[which])[1::2] = _signs(grid(x[which])[1::2], 10)
        out2, lse2 = rb.attention(*x[:3], n, length)
        assert torch.equal(grid(out2)[::2], grid(out)[::2]) and torch.equal(lse2[::2], lse[::2]), which
        got = rb.attention_grad(*x[:3], out, lse, x[3], n, length)
        for name in ("dq", "dk", "dv"):
            assert torch.equal(grid(getattr(got, name))[::2], grid(getattr(grads, name))[::2]), (which, name)
