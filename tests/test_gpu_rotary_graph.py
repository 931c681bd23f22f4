"""Turned rows whose inputs require gradients, and tables to the last bits that they can have.  References: oracle/blocks_oracle.py."""
import numpy as np
import pytest
import torch

import paper_2406_09041_amd as mes
from oracle import blocks_oracle as BO

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("interleaved,dims", [(False, 64), (True, 48)])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_gradients_reach_the_rows(kind, interleaved, dims, transpose):
    """Bit by bit those of the call turned back; rows without a position get none."""
    g = torch.Generator().manual_seed(dims)
    angles = mes.Angles(mes.mes_rotary_table(40, dims, magnitude=1.25), interleaved=interleaved)
    at = _ints([3, -1, 39, 0, 40])
    q, k, wq, wk = (torch.randn(5, h, 64, generator=g).to(kind).to(DEV) for h in (4, 2, 4, 2))
    q.requires_grad_(), k.requires_grad_()
    out = mes.mes_rotary(angles, at, q, k, transpose=transpose)
    with torch.no_grad():
        plain = mes.mes_rotary(angles, at, q, k, transpose=transpose)
        back = mes.mes_rotary(angles, at, wq, wk, transpose=not transpose)
    assert all(torch.equal(a, b) and a.requires_grad and not b.requires_grad for a, b in zip(out, plain))
    got = torch.autograd.grad(out, (q, k), (wq, wk))
    assert all(torch.equal(a, b) for a, b in zip(got, back)) and not got[0][1].any() and not got[1][4].any()
    # one of the two, gradients whose rows are no rows, through views of one buffer, and twice
    out = mes.mes_rotary(angles, at, q, k, transpose=transpose)
    assert torch.equal(torch.autograd.grad(out[1], k, wk)[0], back[1])
    out = mes.mes_rotary(angles, at, q, transpose=transpose)
    ones = torch.autograd.grad(out.sum(), q)[0]
    assert torch.equal(ones, mes.mes_rotary(angles, at, torch.ones_like(wq), transpose=not transpose))
    wide = torch.randn(5, 7, 64, generator=g).to(kind).to(DEV).requires_grad_()
    out = mes.mes_rotary(angles, at, wide[:, :4], wide[:, 4:6], transpose=transpose)
    grad = torch.autograd.grad(out, wide, (wq, wk))[0]
    assert torch.equal(grad[:, :4], back[0]) and torch.equal(grad[:, 4:6], back[1]) and not grad[:, 6].any()
    w = wq.clone().requires_grad_()
    first = torch.autograd.grad(mes.mes_rotary(angles, at, q, transpose=transpose), q, w, create_graph=True)[0]
    assert torch.equal(torch.autograd.grad(first, w, wq)[0], mes.mes_rotary(angles, at, wq, transpose=transpose))


def test_gradients_by_differences():
    """<w, turned(x)> is linear in x: a step of 1 in one number moves it by that number's gradient, but for rounding: each of two turned
    values moves by up to 4 roundings of fp32 of values up to about 8, as do their products with w (up to about 4)."""
    g = torch.Generator().manual_seed(7)
    angles, at = mes.Angles(mes.mes_rotary_table(30, 32), interleaved=True), _ints([1, 29])
    x, w = (torch.randn(2, 1, 48, generator=g).to(DEV) for _ in range(2))
    x.requires_grad_()
    (mes.mes_rotary(angles, at, x) * w).sum().backward()
    f = lambda y: (mes.mes_rotary(angles, at, y).double() * w.double()).sum().item()  # noqa: E731
    with torch.no_grad():
        here = f(x)
        for t in range(2):
            for d in range(48):
                y = x.clone()
                y[t, 0, d] += 1.0
                assert abs(f(y) - here - x.grad[t, 0, d].item()) < 2 * 4 * 2.0 ** -24 * 8 * 4 * 2


def test_what_would_lose_gradients_is_refused():
    angles, at = mes.Angles(mes.mes_rotary_table(8, 16)), _ints([1, 2, 3])
    q = torch.randn(3, 2, 16, device=DEV, requires_grad=True)
    y = q * 1.0
    with pytest.raises(AssertionError, match="require gradients"):
        mes.mes_rotary(angles, at, y, q_out=y)
    with pytest.raises(AssertionError, match="require gradients"):
        mes.mes_rotary(angles, at, q, q_out=torch.empty(3, 2, 16, device=DEV))
    with torch.no_grad():
        mes.mes_rotary(angles, at, y, q_out=y)
    out = mes.mes_rotary(angles, at, q)
    at.fill_(0)                                                  # the gradient would be that of other positions
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_gradients_in_a_captured_graph():
    g = torch.Generator().manual_seed(9)
    angles, at = mes.Angles(mes.mes_rotary_table(512, 128)), torch.arange(300, dtype=torch.int32, device=DEV)
    q, k, wq, wk = (torch.randn(300, h, 128, generator=g).to(torch.bfloat16).to(DEV) for h in (8, 2, 8, 2))
    q.requires_grad_(), k.requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(mes.mes_rotary(angles, at, q, k), (q, k), (wq, wk))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(mes.mes_rotary(angles, at, q, k), (q, k), (wq, wk))
    for step in range(3):
        at.copy_(torch.arange(300, dtype=torch.int32) + 70 * step)
        for x in got:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        with torch.no_grad():
            want = mes.mes_rotary(angles, at, wq, wk, transpose=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n,dims,magnitude", [(1, 16, 1.0), (40, 64, 1.0), (5000, 128, -1.5), (131072, 96, 1.0)])
def test_tables_to_the_last_bits(n, dims, magnitude):
    """Rounded once: half a step of fp32.  Angles in fp64: a frequency is off by a few units of 2^-53 (a power, a product), times the position; the
    first cosine and sine of a run of 16 positions and their product with the magnitude by 2^-52 each, and each of the 15 products by three
    roundings of 2^-53 and the step's own error, sqrt 2 times 2^-52: below 2 + 15 * 3 < 48 times 2^-52, each time the magnitude."""
    got = mes.mes_rotary_table(n, dims, magnitude=magnitude)
    f = BO.frequencies(dims, 10000.0)
    rows = np.unique(np.concatenate([np.arange(min(n, 300)), np.linspace(0, n - 1, 300).astype(int), [n - 1]]))
    angle = rows[:, None] * f
    want = np.stack([np.cos(angle), np.sin(angle)], 1) * magnitude
    tol = 2.0 ** -24 * np.abs(want) + abs(magnitude) * (32 * 2.0 ** -53 * angle[:, None] + 48 * 2.0 ** -52) + 2.0 ** -149
    assert (np.abs(got[torch.from_numpy(rows).to(DEV)].double().cpu().numpy() - want) <= tol).all()
