"""Gradients through Rotary.apply: those of the formula in 64 bits, with every way in which they come."""
import pytest
import torch

from paper_2603_06274_amd.decode import Rotary
from paper_2603_06274_amd.prefill import StemPrefill

import decode_util as du

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


def make(dtype, layout="half", T=33, Hq=4, Hkv=2, d=64, rot=48):
    g = torch.Generator().manual_seed(5)
    rows = lambda h: torch.randn(T, h, d, generator=g).to(dtype).to(DEV)
    r = Rotary(d, rot, theta=10000.0, layout=layout, scaling="yarn", factor=4.0, trained_length=2048.0)
    pos = torch.randint(0, 100000, (T,), generator=g).to(torch.int32)
    return r, pos, rows


def wanted(r, pos, grad):
    """The gradient of the formula: what autograd finds in 64 bits, and the bound of the transposed map's roundings."""
    x = torch.zeros(grad.shape, dtype=torch.float64, requires_grad=True)
    du.rotary_reference(x, pos, r.turns.cpu(), r.attention_factor, r.rotary_dim, r.layout)[0].backward(grad.cpu().double())
    return x.grad, du.rotary_reference(grad.cpu(), pos, r.turns.cpu(), r.attention_factor, r.rotary_dim, r.layout, True)[1]


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_gradients_of_the_formula(dtype, layout):
    r, pos, rows = make(dtype, layout)
    q, k, gq, gk = rows(4).requires_grad_(), rows(2).requires_grad_(), rows(4), rows(2)
    yq, yk = r.apply(q, k, pos.to(DEV))
    with torch.no_grad():
        zq, zk = r.apply(q, k, pos.to(DEV))
        back = r.backward(gq, gk, pos.to(DEV))
    assert torch.equal(yq, zq) and torch.equal(yk, zk) and zq.grad_fn is None
    torch.autograd.backward((yq, yk), (gq, gk))
    for x, g, b in ((q, gq, back[0]), (k, gk, back[1])):
        want, bound = wanted(r, pos, g)
        assert ((x.grad.cpu().double() - want).abs() <= bound).all() and torch.equal(x.grad, b)


def test_gradients_of_any_strides():
    r, pos, rows = make(FP)
    q = rows(4).requires_grad_()
    one = torch.ones((), device=DEV)
    wide = torch.zeros(33, 4, 66, device=DEV)
    for g in (one.expand(33, 4, 64), rows(4)[:1].expand(33, 4, 64), rows(1).expand(33, 4, 64), wide[..., 1:65].copy_(rows(4)),
              torch.zeros(1 + 33 * 4 * 64, device=DEV)[1:].view(33, 4, 64).copy_(rows(4)),
              rows(4).transpose(1, 2).contiguous().transpose(1, 2), rows(4).transpose(0, 1).contiguous().transpose(0, 1)):
        y, none = r.apply(q, None, pos.to(DEV))
        assert none is None
        got, = torch.autograd.grad(y, q, g)
        want, bound = wanted(r, pos, g.contiguous())
        assert ((got.cpu().double() - want).abs() <= bound).all()


def test_one_of_the_two():
    r, pos, rows = make(BF)
    q, k = rows(4), rows(2).requires_grad_()
    yq, yk = r.apply(q, k, pos.to(DEV))
    assert not yq.requires_grad and yk.requires_grad
    g = rows(2)
    got, = torch.autograd.grad(yk, k, g)
    assert torch.equal(got, r.backward(None, g, pos.to(DEV))[1])
    q.requires_grad_()
    yq, yk = r.apply(q, k, pos.to(DEV))                # a loss of one output alone
    yq.float().sum().backward()
    assert k.grad is None and q.grad is not None


def test_gradients_of_gradients():
    """The map is linear in its rows, so the gradient's gradient is the map of what comes."""
    r, pos, rows = make(FP)
    q, g, u = rows(4).requires_grad_(), rows(4).requires_grad_(), rows(4)
    y, _ = r.apply(q, None, pos.to(DEV))
    x, = torch.autograd.grad(y, q, g, create_graph=True)
    again, = torch.autograd.grad(x, g, u)
    assert torch.equal(again, r.apply(u, None, pos.to(DEV))[0])


def test_given_outputs_and_changed_positions():
    r, pos, rows = make(BF)
    q, p = rows(4).requires_grad_(), pos.to(DEV)
    for out in (torch.empty_like(q), q):
        with pytest.raises(ValueError):
            r.apply(q, None, p, out)
    with torch.no_grad():
        r.apply(q, None, p, torch.empty_like(q))
    y, _ = r.apply(q, None, p)
    p += 1
    with pytest.raises(RuntimeError):                  # positions that the backward pass would need
        y.float().sum().backward()


def test_a_prompt_that_requires_gradients_is_pre_filled():
    g = torch.Generator().manual_seed(6)
    q, k, v = (torch.randn(130, 1, 64, generator=g).to(BF).to(DEV) for _ in range(3))
    make = lambda q: StemPrefill(q, k, v, [0, 130], 64, [3], 1.0, n_sink=1, n_local=1, rotary=Rotary(64))
    want = make(q).run()
    assert torch.equal(make(q.clone().requires_grad_()).run(), want)


def test_captured_forward_and_backward():
    r, pos, rows = make(BF)
    q, g, p = rows(4).requires_grad_(), rows(4), pos.to(DEV)

    def both():
        y, _ = r.apply(q, None, p)
        return y.detach(), torch.autograd.grad(y, q, g)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, x = both()
    for step in range(4):
        with torch.no_grad():
            q.copy_(rows(4)), g.copy_(rows(4)), p.copy_((pos + 100 * step).to(torch.int32))
        graph.replay()
        if step % 2:
            torch.cuda.synchronize()
        with torch.no_grad():
            eager = r.apply(q, None, p)[0], r.backward(g, None, p)[0]
        torch.cuda.synchronize()
        assert torch.equal(y, eager[0]) and torch.equal(x, eager[1])
