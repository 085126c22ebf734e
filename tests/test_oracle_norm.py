"""The head norm's oracle: its gradients against fp64 autograd of the formula written
out, and against central differences."""
import pytest
import torch

from oracle import norm as N
from oracle import rope as R

F64 = torch.float64


def _formula(x, weight, pos, w, inter, amp, eps, offset, centred):
    """y, element by element of the definition."""
    rows = []
    for t in range(x.shape[0]):
        heads = []
        for h in range(x.shape[1]):
            v = x[t, h]
            if centred:
                v = v - v.sum() / v.numel()
            n = v / ((v * v).sum() / v.numel() + eps) ** 0.5
            k = weight if weight.dim() == 1 else weight[h]
            heads.append(n * (k + offset))
        rows.append(torch.stack(heads))
    y = torch.stack(rows)
    m = 2 * len(w)
    ia, ib = (range(0, m, 2), range(1, m, 2)) if inter else (range(0, m // 2), range(m // 2, m))
    c = torch.cos(pos.to(F64)[:, None] * torch.tensor(w, dtype=F64)) * amp
    s = torch.sin(pos.to(F64)[:, None] * torch.tensor(w, dtype=F64)) * amp
    cols = list(y.unbind(-1))
    for i, (a, b) in enumerate(zip(ia, ib)):
        ya, yb = cols[a], cols[b]
        cols[a], cols[b] = c[:, i:i + 1] * ya - s[:, i:i + 1] * yb, c[:, i:i + 1] * yb + s[:, i:i + 1] * ya
    return torch.stack(cols, -1)


@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("inter,m", [(False, 8), (True, 8), (False, 6), (True, 4), (False, 0)])
def test_gradients(inter, m, per_head, centred):
    g = torch.Generator().manual_seed(m + 2 * per_head + 4 * centred)
    T, H, d = 5, 3, 8
    x = torch.randn(T, H, d, generator=g, dtype=F64).requires_grad_()
    wt = torch.randn(*((H, d) if per_head else (d,)), generator=g, dtype=F64).requires_grad_()
    pos, w = torch.tensor([0, 1, 7, 100, 3]), [0.7 / (i + 1) for i in range(m // 2)]
    dy = torch.randn(T, H, d, generator=g, dtype=F64)
    kw = dict(w=w, inter=inter, amp=1.3, eps=0.05, offset=0.5, centred=centred)
    y = _formula(x, wt, pos, w, inter, 1.3, 0.05, 0.5, centred)
    got, _ = N.forward(x.detach(), wt.detach(), pos, **kw)
    torch.testing.assert_close(got, y.detach(), rtol=1e-12, atol=1e-12)
    y.backward(dy)
    dx, _, dw, _ = N.backward(dy, x.detach(), wt.detach(), pos, **kw)
    torch.testing.assert_close(dx, x.grad, rtol=1e-11, atol=1e-12)
    torch.testing.assert_close(dw if per_head else dw.sum(0), wt.grad, rtol=1e-11, atol=1e-12)
    # central differences of <dy, y>
    f = lambda a, b: float((N.forward(a, b, pos, **kw)[0] * dy).sum())  # noqa: E731
    h = 1e-5
    for i in range(0, x.numel(), 7):
        e = torch.zeros(x.numel(), dtype=F64)
        e[i] = h
        e = e.view_as(x)
        fd = (f(x.detach() + e, wt.detach()) - f(x.detach() - e, wt.detach())) / (2 * h)
        assert abs(fd - float(dx.flatten()[i])) < 1e-7 * max(1, abs(fd))
    for i in range(0, wt.numel(), 5):
        e = torch.zeros(wt.numel(), dtype=F64)
        e[i] = h
        e = e.view_as(wt)
        fd = (f(x.detach(), wt.detach() + e) - f(x.detach(), wt.detach() - e)) / (2 * h)
        want = (dw if per_head else dw.sum(0)).flatten()[i]
        assert abs(fd - float(want)) < 1e-7 * max(1, abs(fd))


def test_without_weights_or_rotation():
    x = torch.randn(4, 2, 16, dtype=F64)
    y, _ = N.forward(x, None, torch.arange(4), eps=1e-9)
    torch.testing.assert_close(y.square().mean(-1), torch.ones(4, 2, dtype=F64), rtol=1e-6, atol=0)
    # R's angle 0 is the identity, times the amplitude
    z, _ = N.forward(x, None, torch.zeros(4), w=[1.0] * 8, amp=2.0, eps=1e-9)
    torch.testing.assert_close(z, 2 * y, rtol=1e-12, atol=0)
    torch.testing.assert_close(R.rotate(y, torch.zeros(4), [1.0]), y)
