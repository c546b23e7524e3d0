"""Rotated heads where a number is none or a row is left out, against the definition in 64 bits.

Tolerances are those of test_gpu_rotary.py: half a unit in the last place of an output, and what its terms may be off by in 32 bits.
"""
import math

import pytest
import torch

from .test_gpu_rotary import BF16, DEV, F16, F32, angles, inputs, normal, normed, ops, to, turn  # noqa: F401
from .test_gpu_rotary import near as near_finite

pytestmark = pytest.mark.gpu

INF, NAN = math.inf, math.nan


def near(got, want, terms):
    """near_finite where `want` is finite; what is infinite or NaN there is the same here."""
    g, fine = got.cpu(), torch.isfinite(want)
    assert torch.equal(torch.isnan(g), torch.isnan(want))
    assert torch.equal(g[torch.isinf(want)].double(), want[torch.isinf(want)])
    near_finite(g[fine], want[fine], terms[fine])


def same(got, want):
    """Bit for bit, a NaN's own bits apart."""
    kind = {2: torch.int16, 4: torch.int32}[got.element_size()]
    nan = torch.isnan(want)
    return torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan].view(kind), want[~nan].view(kind))


def spoil(x, tail):
    """Writes infinities, NaN and a -0 into both halves of what is not turned, x [1, 4, 3, dim], from element `tail` on."""
    rest = (x.shape[-1] - tail) // 2
    x[0, 0, 0, tail] = INF                       # (its partner keeps its number)
    x[0, 0, 1, tail + rest] = -INF
    x[0, 1, 2, tail + 1] = NAN
    x[0, 2, 0, tail + rest + 1] = NAN
    x[0, 3, 1, tail:] = -0.0
    x[0, 3, 2, tail + rest:] = INF


# (By how many of a lane's elements lie together: 8, 4 or 1.)
TAILS = [(64, 16, False), (64, 20, True), (128, 40, False), (40, 12, False), (40, 7, True), (88, 32, False), (34, 5, False), (34, 6, True), (250, 99, False)]


@pytest.mark.parametrize("dim,pairs,interleaved", TAILS)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_what_is_not_turned_stays(ops, dim, pairs, interleaved, dtype):  # noqa: F811
    q, k, positions, f, qw, kw, _ = inputs(dim + pairs, 1, 4, 3, 3, dim, pairs, 0, True, dtype, 100)
    dq, dk = normal(9, *q.shape).to(dtype), normal(10, *k.shape).to(dtype)
    for x in (q, k, dq, dk):
        spoil(x, 2 * pairs)
    a = angles(positions, f, None)
    at, fr = to(DEV, positions, f)
    args = to(DEV, q, k)
    for got, x in zip(ops.rotary_norm(*args, at, fr, interleaved=interleaved), (q, k)):
        assert same(got[..., 2 * pairs:].cpu(), x[..., 2 * pairs:])
        want, both = turn(x.double(), a, interleaved)
        near(got, want, both * 2.0 ** -19)
    grads = ops.rotary_norm_backward(*to(DEV, dq, dk), *args, at, fr, interleaved=interleaved)
    for got, x in zip(grads, (dq, dk)):
        assert same(got[..., 2 * pairs:].cpu(), x[..., 2 * pairs:])
        want, both = turn(x.double(), a, interleaved, back=True)
        near(got, want, both * 2.0 ** -19)
    # With a norm an infinite element is NaN and leaves 0 of the others.
    w = to(DEV, qw, kw)
    for got, x, weight in zip(ops.rotary_norm(*args, at, fr, *w, interleaved=interleaved, eps=1e-5), (q, k), (qw, kw)):
        want, both = turn(normed(x.double(), weight.double(), 1e-5), a, interleaved)
        near(got, want, both * 2.0 ** -19)


@pytest.mark.parametrize("dim,pairs,interleaved", TAILS)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_gradient_behind_a_norm_of_what_is_not_turned(ops, dim, pairs, interleaved, dtype):  # noqa: F811
    q, k, positions, f, qw, kw, _ = inputs(dim + pairs + 1, 1, 4, 3, 3, dim, pairs, 0, True, dtype, 100)
    dq, dk = normal(9, *q.shape).to(dtype), normal(10, *k.shape).to(dtype)
    for x in (dq, dk):
        spoil(x, 2 * pairs)
    a = angles(positions, f, None)
    got = ops.rotary_norm_backward(*to(DEV, dq, dk, q, k, positions, f, qw, kw), interleaved=interleaved, eps=1e-5)
    for i, (d, x, w) in enumerate(zip((dq, dk), (q, k), (qw, kw))):
        g, both = turn(d.double(), a, interleaved, back=True)
        x, w = x.double(), w.double()
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
        n, e = x * r, g * w
        inner, magnitude = (e * n).mean(-1, keepdim=True), (e * n).abs().mean(-1, keepdim=True)
        slack = both * 2.0 ** -21
        near(got[i], r * (e - n * inner),
             r * (slack * w.abs() + n.abs() * ((slack * w.abs() * n.abs()).mean(-1, keepdim=True) + magnitude * 2.0 ** -18) + e.abs() * 2.0 ** -19))
        near(got[2 + i], (g * n).sum((0, 1, 2)), (both * n.abs()).sum((0, 1, 2)) * 2.0 ** -18)


@pytest.mark.parametrize("dim,heads,kv", [(32, 5, 16), (64, 17, 3), (80, 9, 8), (128, 3, 9), (250, 5, 2)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradient_without_eps(ops, dim, heads, kv, dtype):  # noqa: F811
    """eps = 0 over numbers of heads that leave lanes without one."""
    q, k, positions, f, qw, kw, _ = inputs(dim, 2, 3, heads, kv, dim, dim // 2, 0, True, dtype, 100)
    dy = [normal(90 + i, *x.shape).to(dtype) for i, x in enumerate((q, k))]
    got = ops.rotary_norm_backward(*to(DEV, *dy, q, k, positions, f, qw, kw), eps=0.0)
    a = angles(positions, f, None)
    for i, (d, x, w) in enumerate(zip(dy, (q, k), (qw, kw))):
        g, both = turn(d.double(), a, False, back=True)
        x, w = x.double(), w.double()
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True))
        n, e = x * r, g * w
        inner, magnitude = (e * n).mean(-1, keepdim=True), (e * n).abs().mean(-1, keepdim=True)
        slack = both * 2.0 ** -21
        near_finite(got[i], r * (e - n * inner),
                    r * (slack * w.abs() + n.abs() * ((slack * w.abs() * n.abs()).mean(-1, keepdim=True) + magnitude * 2.0 ** -18) + e.abs() * 2.0 ** -19))
        near_finite(got[2 + i], (g * n).sum((0, 1, 2)), (both * n.abs()).sum((0, 1, 2)) * 2.0 ** -18)


# Tokens and heads of which a wave takes 2, 3, 4, 2 and 2 groups of heads, more than one chunk of them but in the fourth, the last one ragged.
SEVERAL = [(1, 1700, 37, 9, 128, 64, 0, False), (3, 700, 19, 5, 256, 100, 0, False), (2, 1024, 70, 33, 64, 32, 0, False), (2, 1221, 16, 16, 80, 40, 3, True),
           (1, 2100, 33, 17, 32, 16, 2, True)]


@pytest.mark.parametrize("shape", SEVERAL)
def test_several_groups_of_heads_a_wave(ops, shape):  # noqa: F811
    *size, interleaved = shape
    q, k, positions, f, qw, kw, sections = inputs(sum(size), *size, True, F32, 5000)
    args = to(DEV, q, k, positions, f, qw, kw)
    a = angles(positions, f, sections)
    got = ops.rotary_norm(*args, sections=sections, interleaved=interleaved, eps=1e-5)
    for g, x, w in zip(got, (q, k), (qw, kw)):
        want, both = turn(normed(x.double(), w.double(), 1e-5), a, interleaved)
        near_finite(g, want, both * 2.0 ** -19)
    plain = ops.rotary_norm(*args[:4], sections=sections, interleaved=interleaved)
    for g, x in zip(plain, (q, k)):
        want, both = turn(x.double(), a, interleaved)
        near_finite(g, want, both * 2.0 ** -19)


@pytest.mark.parametrize("shape", SEVERAL)
def test_gradient_of_several_groups_of_heads_a_wave(ops, shape):  # noqa: F811
    """A weight's sum has at most 51 roundings (8 in a lane, 4 between lanes, 2 between waves, 37 over the blocks) and its terms are off by 24 * 2^-24
    of |a| + |b|: less than 2^-17."""
    *size, interleaved = shape
    q, k, positions, f, qw, kw, sections = inputs(sum(size) + 5, *size, True, F32, 5000)
    dy = [normal(90 + i, *x.shape) for i, x in enumerate((q, k))]
    got = ops.rotary_norm_backward(*to(DEV, *dy, q, k, positions, f, qw, kw), sections=sections, interleaved=interleaved, eps=1e-5)
    a = angles(positions, f, sections)
    for i, (d, x, w) in enumerate(zip(dy, (q, k), (qw, kw))):
        g, both = turn(d.double(), a, interleaved, back=True)
        x, w = x.double(), w.double()
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
        n, e = x * r, g * w
        inner, magnitude = (e * n).mean(-1, keepdim=True), (e * n).abs().mean(-1, keepdim=True)
        near_finite(got[i], r * (e - n * inner), r * (both * w.abs() + n.abs() * ((both * w.abs() * n.abs()).mean(-1, keepdim=True) + magnitude)) * 2.0 ** -18)
        near_finite(got[2 + i], (g * n).sum((0, 1, 2)), (both * n.abs()).sum((0, 1, 2)) * 2.0 ** -17)
