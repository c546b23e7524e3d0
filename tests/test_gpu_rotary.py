"""Normed and rotated heads and their gradients on the GPU against their definitions in 64 bits.

Tolerances: half a unit in the last place of an output (bfloat16 2^-8, float16 2^-11, float32 2^-24, relative), and in front of
it, in 32 bits: a vector's sum of squares is off by up to 22 roundings of 2^-24 (16 + 2 in a lane, 4 between lanes), its root by
half of that, quotient and products by 5 more: 2^-20. A cosine or sine is off by 2^-22 (the angle's rounding to 32 bits and its
factor, pi / 4 * 2^-23, and the polynomial's last steps), so that a turned element is off by (|a| + |b|) (2^-20 + 2^-22 + 2^-23),
less than (|a| + |b|) 2^-19. Sums for the weights add up to 2^-18 of their terms' magnitudes (at most 60 roundings each).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64
HALF_ULP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF16: 2.0 ** -133, F16: 2.0 ** -25, F32: 2.0 ** -149}


@pytest.fixture(scope="module")
def ops():
    from paper_1905_13298_amd import ops as o
    return o


def normal(seed, *shape, std=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std


def near(got, want, terms=0.0):
    t = got.dtype
    assert torch.isfinite(got).all()
    off = (got.cpu().double() - want).abs()
    tol = want.abs() * HALF_ULP[t] * 1.01 + TINY[t] + terms * (1 + HALF_ULP[t])
    assert torch.all(off <= tol), float((off / tol.clamp(min=1e-300)).max())


def angles(positions, frequencies, sections):
    """[batch, tokens, 1, pairs]."""
    f = frequencies.double()
    if positions.dim() == 2:
        a = positions.double()[..., None] * f
    else:
        axis = torch.tensor([i for i, n in enumerate(sections or (f.numel(),)) for _ in range(n)])
        a = positions.double()[axis].permute(1, 2, 0) * f
    return a[:, :, None]


def turn(x, a, interleaved, back=False):
    """(x turned, |a| + |b| of each element's pair)."""
    n = a.shape[-1]
    i = torch.arange(n)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    c, s = torch.cos(a), torch.sin(a) * (-1 if back else 1)
    y, size = x.clone(), x.abs()
    p, q = x[..., first], x[..., second]
    y[..., first], y[..., second] = p * c - q * s, q * c + p * s
    size[..., first] = size[..., second] = p.abs() + q.abs()
    return y, size


def normed(x, w, eps):
    if w is None:
        return x
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w


def inputs(seed, batch, tokens, heads, kv, dim, pairs, axes, norm, dtype, far, wtype=None):
    q, k = normal(seed, batch, tokens, heads, dim).to(dtype), normal(seed + 1, batch, tokens, kv, dim).to(dtype)
    gen = torch.Generator().manual_seed(seed + 2)
    shape = (batch, tokens) if axes == 0 else (axes, batch, tokens)
    positions = torch.randint(-far, far + 1, shape, generator=gen, dtype=torch.int64).to(torch.int32)
    f = torch.pow(torch.tensor(1e4, dtype=F64), -torch.arange(pairs, dtype=F64) / pairs)
    w = [(1 + normal(seed + 3 + i, dim, std=0.2)).to(wtype or dtype) if norm else None for i in range(2)]
    sections = None
    if axes > 1:
        cut = sorted(torch.randint(0, pairs + 1, (axes - 1,), generator=gen).tolist())
        sections = tuple(b - a for a, b in zip([0, *cut], [*cut, pairs]))
    return q, k, positions, f, *w, sections


def to(dev, *ts):
    return [None if t is None else t.to(dev) for t in ts]


SHAPES = [  # batch, tokens, heads, kv heads, dim, pairs, axes, norm, interleaved, far
    (1, 1, 1, 1, 2, 1, 0, True, False, 10), (2, 3, 5, 2, 16, 8, 0, True, False, 1000), (1, 7, 9, 3, 64, 32, 0, True, False, 100000),
    (3, 5, 32, 8, 128, 64, 0, True, False, 1 << 30), (2, 9, 4, 4, 80, 40, 3, False, True, 64), (2, 9, 4, 1, 80, 40, 0, True, False, 64),
    (1, 6, 3, 3, 96, 36, 2, True, False, 5000), (2, 4, 17, 2, 256, 128, 4, True, True, 300), (1, 33, 2, 1, 130, 27, 1, True, False, 100),
    (1, 4, 20, 9, 34, 17, 2, False, False, 9), (2, 5, 6, 6, 192, 48, 0, True, True, 70), (1, 3, 2, 2, 128, 32, 3, True, False, 9999),
    (5, 130, 3, 1, 64, 24, 0, True, False, 1 << 20), (1, 2, 70, 70, 32, 16, 0, True, False, 50), (1, 5, 3, 2, 250, 125, 0, True, True, 1000),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_rotary(ops, shape, dtype):
    *size, interleaved, far = shape
    q, k, positions, f, qw, kw, sections = inputs(sum(size[:6]), *size, dtype, far)
    args = to(DEV, q, k, positions, f, qw, kw)
    got = ops.rotary_norm(*args, sections=sections, interleaved=interleaved, eps=1e-5)
    a = angles(positions, f, sections)
    for g, x, w in zip(got, (q, k), (qw, kw)):
        want, both = turn(normed(x.double(), None if w is None else w.double(), 1e-5), a, interleaved)
        assert g.dtype == dtype and g.shape == x.shape
        near(g, want, both * (2.0 ** -19 + 2.0 ** -52 * a.abs().max()))
    alone, none = ops.rotary_norm(args[0], None, *args[2:5], sections=sections, interleaved=interleaved, eps=1e-5)
    assert none is None and torch.equal(alone, got[0])


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_rotary_gradient(ops, shape, dtype):
    *size, interleaved, far = shape
    q, k, positions, f, qw, kw, sections = inputs(sum(size[:6]) + 7, *size, dtype, far)
    dy = [normal(90 + i, *x.shape).to(dtype) for i, x in enumerate((q, k))]
    args = to(DEV, *dy, q, k, positions, f, qw, kw)
    got = ops.rotary_norm_backward(*args, sections=sections, interleaved=interleaved, eps=1e-5)
    a = angles(positions, f, sections)
    for i, (d, x, w) in enumerate(zip(dy, (q, k), (qw, kw))):
        g, both = turn(d.double(), a, interleaved, back=True)
        slack = both * (2.0 ** -21 + 2.0 ** -52 * a.abs().max())
        if w is None:
            assert got[2 + i] is None
            near(got[i], g, slack)
            continue
        x, w = x.double(), w.double()
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
        n, e = x * r, g * w
        inner, magnitude = (e * n).mean(-1, keepdim=True), (e * n).abs().mean(-1, keepdim=True)
        near(got[i], r * (e - n * inner),
             r * (slack * w.abs() + n.abs() * ((slack * w.abs() * n.abs()).mean(-1, keepdim=True) + magnitude * 2.0 ** -18) + e.abs() * 2.0 ** -19))
        near(got[2 + i], (g * n).sum((0, 1, 2)), (both * n.abs()).sum((0, 1, 2)) * 2.0 ** -18)
    again = ops.rotary_norm_backward(*args, sections=sections, interleaved=interleaved, eps=1e-5)
    assert all(x is None and y is None or torch.equal(x, y) for x, y in zip(got, again))


def test_gradient_of_many_tokens(ops):
    """More tokens than the launch has waves: every wave's sums are of several."""
    q, k, positions, f, qw, kw, _ = inputs(1, 3, 1999, 5, 2, 64, 32, 0, True, F32, 5000)
    dy = [normal(90 + i, *x.shape) for i, x in enumerate((q, k))]
    got = ops.rotary_norm_backward(*to(DEV, *dy, q, k, positions, f, qw, kw))
    a = angles(positions, f, None)
    for i, (d, x, w) in enumerate(zip(dy, (q, k), (qw, kw))):
        g, both = turn(d.double(), a, False, back=True)
        x, w = x.double(), w.double()
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        n, e = x * r, g * w
        inner, magnitude = (e * n).mean(-1, keepdim=True), (e * n).abs().mean(-1, keepdim=True)
        near(got[i], r * (e - n * inner), r * (both * w.abs() + n.abs() * ((both * w.abs() * n.abs()).mean(-1, keepdim=True) + magnitude)) * 2.0 ** -18)
        near(got[2 + i], (g * n).sum((0, 1, 2)), (both * n.abs()).sum((0, 1, 2)) * 2.0 ** -18)


def test_gradient_against_differences(ops):
    """Central differences of the definition in 64 bits, sum(y * c), along random directions."""
    q, k, positions, f, qw, kw, sections = inputs(3, 2, 3, 3, 2, 40, 13, 2, True, F32, 50)
    c = [normal(50 + i, *x.shape) for i, x in enumerate((q, k))]
    a = angles(positions, f, sections)
    loss = lambda *v: sum(float((turn(normed(x, w, 1e-6), a, True)[0] * y.double()).sum()) for x, w, y in zip(v[:2], v[2:], c))  # noqa: E731
    grads = ops.rotary_norm_backward(*to(DEV, *c, q, k, positions, f, qw, kw), sections=sections, interleaved=True)
    at = [t.double() for t in (q, k, qw, kw)]
    for seed in range(5):
        u = [normal(seed * 7 + i, *t.shape).double() for i, t in enumerate(at)]
        t = 1e-4
        num = (loss(*(x + t * d for x, d in zip(at, u))) - loss(*(x - t * d for x, d in zip(at, u)))) / (2 * t)
        parts = [(g.cpu().double() * d) for g, d in zip(grads, u)]
        # t^2 times third derivatives of the terms' order for the differences, 2^-18 a term for the gradients.
        assert abs(num - float(sum(p.sum() for p in parts))) <= 1e-5 * float(sum(p.abs().sum() for p in parts))


@pytest.mark.parametrize("far", [0, 1, 12345, 2 ** 24 + 1, 2 ** 31 - 1])
def test_far_positions(ops, far):
    """Angles of far positions: as near as those of near ones, and a rotation's length stays."""
    for position in (far, -far):
        q = normal(1, 1, 1, 1, 128)
        positions = torch.full((1, 1), position, dtype=torch.int32)
        for theta in (1e4, 5e5):
            f = ops.rotary_frequencies(64, theta)
            got, _ = ops.rotary_norm(q.to(DEV), None, positions.to(DEV), f)
            want, both = turn(q.double(), angles(positions, f.cpu(), None), False)
            near(got, want, both * (2.0 ** -21 + abs(far) * 2.0 ** -52))


def test_quarter_turns_are_exact(ops):
    q = normal(1, 1, 8, 1, 16)
    f = torch.full((8,), math.pi / 2, dtype=F64)
    got, _ = ops.rotary_norm(q.to(DEV), None, torch.arange(8, dtype=torch.int32, device=DEV)[None], f.to(DEV))
    a, b = q[..., :8], q[..., 8:]
    for t in range(8):
        c, s = ((1, 0), (0, 1), (-1, 0), (0, -1))[t % 4]
        want = torch.cat([a[0, t] * c - b[0, t] * s, b[0, t] * c + a[0, t] * s], -1)
        assert torch.allclose(got[0, t].cpu(), want, rtol=0, atol=2.0 ** -48)     # (pi / 2 itself is off by 2^-54)


def test_types_strides_and_broadcasts(ops):
    batch, tokens, heads, kv, dim = 2, 6, 4, 2, 64
    qkv = normal(1, batch, tokens, heads + 2 * kv, dim).to(BF16).to(DEV)
    q, k, _ = qkv.split([heads, kv, kv], dim=2)
    positions = torch.arange(tokens, dtype=torch.int32, device=DEV)[None].expand(batch, tokens)
    f = ops.rotary_frequencies(32)
    w = (1 + normal(2, dim, std=0.2)).to(DEV)
    got = ops.rotary_norm(q, k, positions, f, w, w)
    want = ops.rotary_norm(q.contiguous(), k.contiguous(), positions.contiguous(), f, w, w)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    # Rows that begin anywhere, and a token's vector that every token shares.
    wide = normal(3, tokens, batch, heads, dim + 3).to(F16).to(DEV)
    view = wide.transpose(0, 1)[..., 1:1 + dim]
    one = view[:, :1].expand(batch, tokens, heads, dim)
    assert torch.equal(ops.rotary_norm(view, None, positions, f)[0], ops.rotary_norm(view.contiguous(), None, positions, f)[0])
    assert torch.equal(ops.rotary_norm(one, None, positions, f)[0], ops.rotary_norm(one.contiguous(), None, positions, f)[0])
    # Frequencies in 32 bits are taken as they are.
    assert torch.equal(ops.rotary_norm(q, k, positions, f.float())[0], ops.rotary_norm(q, k, positions, f.float().double())[0])
    # A weight for one of the two alone; weights in 32 bits get gradients in 32 bits.
    only, plain = ops.rotary_norm(q, k, positions, f, w), ops.rotary_norm(q, k, positions, f)
    assert torch.equal(only[0], got[0]) and torch.equal(only[1], plain[1])
    grads = ops.rotary_norm_backward(q, k, q, k, positions, f, None, w)
    both = ops.rotary_norm_backward(q, k, q, k, positions, f, w, w)
    assert grads[2] is None and grads[3].dtype == F32 and torch.equal(grads[1], both[1]) and torch.equal(grads[3], both[3])
    assert torch.equal(grads[0], ops.rotary_norm_backward(q, None, q, None, positions, f)[0])


def test_nothing_and_what_is_no_number(ops):
    f = ops.rotary_frequencies(16)
    w = torch.ones(32, device=DEV)
    none = torch.empty(2, 0, 3, 32, device=DEV)
    positions = torch.zeros(2, 4, dtype=torch.int32, device=DEV)
    assert ops.rotary_norm(none, none[:, :, :1], positions[:, :0], f, w, w)[1].shape == (2, 0, 1, 32)
    _, _, dq, dk = ops.rotary_norm_backward(none, none, none, none, positions[:, :0], f, w, w)
    assert torch.all(dq == 0) and torch.all(dk == 0)
    x = normal(1, 2, 4, 3, 32)
    want, _ = ops.rotary_norm(x.to(DEV), None, positions, f, w)
    x[1, 2, 1, 5] = float("nan")
    x[0, 0, 0] = 0
    got, _ = ops.rotary_norm(x.to(DEV), None, positions, f, w)
    keep = torch.ones(2, 4, 3, dtype=torch.bool)
    keep[1, 2, 1] = keep[0, 0, 0] = False
    assert torch.isnan(got[1, 2, 1]).all() and torch.all(got[0, 0, 0] == 0) and torch.equal(got.cpu()[keep], want.cpu()[keep])


def test_other_streams_and_graphs(ops):
    """Forward and backward on a stream of the caller's, and replayed from a graph, between the caller's own work: the eager results."""
    q, k, positions, f, qw, kw, _ = inputs(4, 2, 40, 4, 2, 64, 32, 0, True, BF16, 100)
    q, k, positions, f, qw, kw = to(DEV, q, k, positions, f, qw, kw)

    def step():
        y = ops.rotary_norm(q, k, positions, f, qw, kw)
        return (*y, *ops.rotary_norm_backward(*y, q, k, positions, f, qw, kw))

    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step()
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        q.copy_(normal(10 + i, *q.shape).to(BF16))
        positions += 17
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(x, y) for x, y in zip(got, step()))


def test_refusals(ops):
    x = torch.zeros(2, 3, 4, 64, device=DEV)
    at = torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    f, w = ops.rotary_frequencies(32), torch.ones(64, device=DEV)
    both = torch.stack([at, at])
    bad = [
        lambda: ops.rotary_norm(x[0], x, at, f),
        lambda: ops.rotary_norm(x.int(), None, at, f),
        lambda: ops.rotary_norm(x, x[:1], at, f),
        lambda: ops.rotary_norm(x, x[0], at, f),
        lambda: ops.rotary_norm(x, x.to(BF16), at, f),
        lambda: ops.rotary_norm(x, x[..., :32], at, f),
        lambda: ops.rotary_norm(x.transpose(2, 3), None, at, f),
        lambda: ops.rotary_norm(x, x, at.long(), f),
        lambda: ops.rotary_norm(x, x, at[:, :2], f),
        lambda: ops.rotary_norm(x, x, at.cpu(), f),
        lambda: ops.rotary_norm(x, x, at, f.to(F16)),
        lambda: ops.rotary_norm(x, x, at, ops.rotary_frequencies(33)),
        lambda: ops.rotary_norm(x, x, at, f[::2]),
        lambda: ops.rotary_norm(x, x, at, f[None]),
        lambda: ops.rotary_norm(x, x, both, f),
        lambda: ops.rotary_norm(x, x, both, f, sections=(16, 15)),
        lambda: ops.rotary_norm(x, x, both, f, sections=(33, -1)),
        lambda: ops.rotary_norm(x, x, both, f, sections=(2 ** 32, 32)),
        lambda: ops.rotary_norm(x, x, at, f, sections=(16, 16)),
        lambda: ops.rotary_norm(x, x, at, f, w[:32]),
        lambda: ops.rotary_norm(x, x, at, f, w.to(BF16)),
        lambda: ops.rotary_norm(x.to(BF16), x.to(BF16), at, f, w, w.to(BF16)),
        lambda: ops.rotary_norm(x, None, at, f, w, w),
        lambda: ops.rotary_norm(x, x, at, f, w, w, eps=-1.0),
        lambda: ops.rotary_norm(x[..., :63], None, at, ops.rotary_frequencies(8)),
        lambda: ops.rotary_norm(torch.zeros(2, 3, 4, 258, device=DEV), None, at, f),
        lambda: ops.rotary_norm_backward(x, None, x, x, at, f),
        lambda: ops.rotary_norm_backward(x, x, x[:, :2], x, at, f),
        lambda: ops.rotary_norm_backward(x, x[:, :, :2], x, x, at, f),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((TypeError, ValueError, ops.DeepShiftError)):
            call()
            pytest.fail(f"case {i} was accepted")
