"""Rows turned by their positions, against the definition in 64 bits; the inverse as the gradient, against differences."""
import numpy as np
import pytest
import torch

import paper_2608_03537_b200 as cf
from oracle import kv_oracle as orc
from tests import kv, parity as P

pytestmark = pytest.mark.gpu


def _freqs(pairs, device, base=10000.0):
    return base ** (-torch.arange(pairs, dtype=torch.float64, device=device) / pairs)


def _check(x, positions, freqs, out, sections, adjacent, inverse=False):
    pairs = len(freqs)
    parts = sections or (pairs,)
    xs, pos, fr = kv.f64(x), positions.cpu().numpy(), freqs.cpu().numpy()
    want = orc.rotary(xs, pos, fr, parts, adjacent, inverse)
    bound = kv.turned_bound(want, xs, pairs, adjacent, kv.raw_angle(pos, fr, parts), x.dtype)
    assert np.all(np.abs(kv.f64(out) - want) <= bound)
    assert torch.equal(out[..., 2 * pairs:], x[..., 2 * pairs:])


SHAPES = [(1, 1, 8, 1, 4), (1, 32, 128, 1, 64), (3, 5, 80, 2, 40), (17, 12, 64, 3, 32), (777, 3, 128, 3, 64), (40, 7, 256, 1, 64), (9, 2, 512, 4, 256), (5, 3, 96, 1, 20), (2100, 2, 72, 2, 9),
          (6, 1, 24, 1, 1), (5000, 1, 64, 1, 32)]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,heads,D,axes,pairs", SHAPES)
def test_rotary(tokens, heads, D, axes, pairs, name, adjacent, cuda_device):
    g = torch.Generator(device=cuda_device).manual_seed(tokens + D)
    x = torch.randn(tokens, heads, D, device=cuda_device, generator=g).to(kv.TYPES[name])
    positions = torch.randint(-100, 200000, (axes, tokens), dtype=torch.int32, device=cuda_device, generator=g)
    cut = sorted(np.random.RandomState(D).randint(0, pairs + 1, axes - 1))
    sections = tuple(int(b - a) for a, b in zip([0, *cut], [*cut, pairs]))
    if axes == 1:
        positions, sections = positions[0], None
    freqs = _freqs(pairs, cuda_device)
    out = P.guarded(x.shape, x.dtype, -77.0, cuda_device)
    assert cf.rotary(x, positions, freqs, out, sections=sections, adjacent=adjacent) is out
    torch.cuda.synchronize()
    P.check_canaries({"out": out})
    _check(x, positions, freqs, out, sections, adjacent)
    again = x.clone()
    cf.rotary(again, positions, freqs, again, sections=sections, adjacent=adjacent)   # in place
    assert torch.equal(again, out)
    cf.rotary(x, positions, freqs, out, sections=sections, adjacent=adjacent, inverse=True)
    _check(x, positions, freqs, out, sections, adjacent, True)


@pytest.mark.parametrize("adjacent", [False, True])
def test_far_positions(adjacent, cuda_device):
    positions = torch.tensor([0, 1, 2 ** 20 + 1, 2 ** 31 - 1, -2 ** 31, -1, 123456789], dtype=torch.int32, device=cuda_device)
    x = torch.randn(7, 2, 32, device=cuda_device)
    freqs = torch.tensor([1.0, 0.5, 1 / 3, 3.0, 1e-3, 1e-9, 0.0, -0.7, 1, 1, 1, 1, 1, 1, 1, 1], dtype=torch.float64, device=cuda_device)
    out = torch.empty_like(x)
    cf.rotary(x, positions, freqs, out, adjacent=adjacent)
    _check(x, positions, freqs, out, None, adjacent)


def test_strides_and_rows_that_are_not_finite(cuda_device):
    """Heads of one projection's output, turned where they stand; what lies around them stays."""
    base = torch.randn(11, 9, 64, device=cuda_device).bfloat16()
    base[4, 2, 5] = float("inf")
    base[7, 3, 9] = float("nan")
    before = base.clone()
    x = base[:, 2:6, :]
    positions, freqs = torch.arange(11, dtype=torch.int32, device=cuda_device), _freqs(32, cuda_device)
    cf.rotary(x, positions, freqs, x)
    torch.cuda.synchronize()
    assert torch.equal(base[:, 6:], before[:, 6:]) and torch.equal(base[:, :2], before[:, :2])
    bad = torch.zeros(11, 4, 64, dtype=torch.bool, device=cuda_device)
    bad[4, 0, 5] = bad[4, 0, 37] = bad[7, 1, 9] = bad[7, 1, 41] = True
    assert torch.equal(torch.isfinite(x), ~bad)
    # heads and tokens exchanged: any order of strides
    y, out = before.transpose(0, 1)[:, :4], torch.empty(9, 4, 64, dtype=torch.bfloat16, device=cuda_device)
    cf.rotary(y, positions[:9], freqs, out)
    dense = torch.empty_like(out)
    cf.rotary(y.contiguous(), positions[:9], freqs, dense)
    assert torch.equal(out, dense)


@pytest.mark.parametrize("adjacent", [False, True])
def test_inverse_is_the_gradient(adjacent, cuda_device):
    """d/dx of sum(dy * rotary(x)) is rotary(dy, inverse); rotary is linear, so a difference is exact but for rounding.  In fp32: each side is a sum of 48 products off by 2^-20 of
    their magnitudes."""
    g = torch.Generator(device=cuda_device).manual_seed(5)
    x, dy, dx = (torch.randn(6, 2, 24, device=cuda_device, generator=g) for _ in range(3))
    positions = torch.randint(0, 5000, (2, 6), dtype=torch.int32, device=cuda_device, generator=g)
    freqs, kw = _freqs(10, cuda_device), dict(sections=(4, 6), adjacent=adjacent)
    turn = lambda t, **more: cf.rotary(t, positions, freqs, torch.empty_like(t), **kw, **more)  # noqa: E731
    grad = turn(dy, inverse=True)
    left = (dy.double() * (turn(x + dx).double() - turn(x).double())).sum((1, 2))
    right = (grad.double() * ((x + dx).double() - x.double())).sum((1, 2))
    size = (dy.double().abs().sum((1, 2)) * (x.abs() + dx.abs()).double().amax((1, 2))) * 4
    assert torch.all((left - right).abs() <= size * 2.0 ** -20)
    back = turn(turn(x), inverse=True)
    assert torch.all((back - x).abs() <= 2.0 ** -19 * x.abs().amax() * 2)


def test_trains_through_autograd_and_graphs(cuda_device):
    """As a training program has it: a function whose backward pass is the inverse, captured while an eager graph of the same leaves lives."""
    positions, freqs = torch.arange(40, dtype=torch.int32, device=cuda_device), _freqs(16, cuda_device)

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return cf.rotary(x, positions, freqs, torch.empty_like(x))

        @staticmethod
        def backward(ctx, dy):
            dy = dy.contiguous()
            return cf.rotary(dy, positions, freqs, torch.empty_like(dy), inverse=True)

    x = torch.randn(40, 4, 32, device=cuda_device, requires_grad=True)
    w = torch.randn(40, 4, 32, device=cuda_device)
    want = cf.rotary(w, positions, freqs, torch.empty_like(w), inverse=True)
    eager = (Turn.apply(x) * w).sum()
    eager.backward()
    assert torch.equal(x.grad, want)
    x.grad = None
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = x.detach().clone().requires_grad_(True)
        (Turn.apply(y) * w).sum().backward()
        y.grad = None
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        (Turn.apply(y) * w).sum().backward()
    w.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y.grad, 2 * want)


def test_refusals(cuda_device):
    x, positions, freqs = torch.zeros(4, 2, 32, device=cuda_device), torch.zeros(4, dtype=torch.int32, device=cuda_device), _freqs(16, cuda_device)
    out = torch.full_like(x, 3.0)
    for args, kw, error in (((x, positions, _freqs(17, cuda_device), out), {}, cf.ComfuseError), ((x, positions.long(), freqs, out), {}, AssertionError), ((x, positions, freqs.float(), out), {}, AssertionError),
                            ((x, positions, freqs, out.bfloat16()), {}, AssertionError), ((x, positions[:3], freqs, out), {}, AssertionError), ((x, positions.cpu(), freqs, out), {}, AssertionError),
                            ((x, positions[None].repeat(2, 1), freqs, out), {}, AssertionError), ((x, positions[None].repeat(2, 1), freqs, out), {"sections": (8, 7)}, AssertionError),
                            ((x, positions, freqs, out[:, :, ::2]), {}, AssertionError), ((x[:0], positions[:0], freqs, out[:0]), {}, cf.ComfuseError)):
        with pytest.raises(error):
            cf.rotary(*args, **kw)
    torch.cuda.synchronize()
    assert torch.all(out == 3.0)
