"""Rotary positions on the GPU against the formula in 64 bits.

Tolerance.  An output u = m (a cos - b sin) is formed in fp32 from sines and cosines that are off by at
most 2^-23 (the angle's conversion to fp32, at most pi/4 2^-24, two half steps of the polynomial and one of
the magnitude's product), in one product and one fused multiply and add: with B = |m| (|a| + |b|) it is off by at most
2^-23 B + 2 2^-24 B, then rounded to the output's type (bf16 2^-8, fp32 2^-24 of the value)."""
import math

import pytest
import torch

from gpu_common import DEV
from paper_2609_37988_amd import kvk

pytestmark = pytest.mark.gpu
F64 = torch.float64


def _reference(x, pos, freq, layout, first, magnitude, inverse):
    """x [B, heads, n, d], pos [B, n]: the turned rows in 64 bits and their tolerance."""
    f = torch.tensor(freq, dtype=F64, device=x.device)
    angle = pos.to(F64)[:, None, :, None] * f
    c, s = angle.cos() * magnitude, angle.sin() * magnitude * (-1 if inverse else 1)
    half = len(freq)
    i = torch.arange(half, device=x.device)
    i, j = (first + i, first + half + i) if layout == kvk.HALVES else (first + 2 * i, first + 2 * i + 1)
    y = x.to(F64).clone()
    bound = torch.zeros_like(y)
    a, b = y[..., i].clone(), y[..., j].clone()
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    bound[..., i] = bound[..., j] = abs(magnitude) * (a.abs() + b.abs())
    own = 2.0**-8 if x.dtype == torch.bfloat16 else 2.0**-24
    return y, 1.01 * (2.0**-22 * bound + torch.where(bound > 0, own * y.abs(), 0 * y)) + 1e-37


def _check(got, x, pos, freq, layout, first, magnitude=1.0, inverse=False):
    want, tol = _reference(x, pos, freq, layout, first, magnitude, inverse)
    err = (got.to(F64) - want).abs()
    assert (err <= tol).all(), f"worst {float((err / tol).max()):.2f} of the tolerance"


def _inputs(seed, b, heads, n, d, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(b, heads, n, d, generator=g, device=DEV).to(dtype), g


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", [kvk.HALVES, kvk.PAIRS])
@pytest.mark.parametrize("b,n,hq,hk,d,width,first", [
    (1, 1, 1, 1, 64, 64, 0), (1, 1, 40, 8, 128, 128, 0), (3, 7, 5, 1, 128, 64, 64), (2, 33, 4, 2, 192, 64, 128),
    (2, 5, 3, 1, 80, 32, 0), (1, 130, 9, 2, 72, 8, 40), (2, 65, 2, 1, 104, 24, 16), (1, 3, 2, 1, 576, 512, 8), (4, 257, 28, 4, 128, 128, 0)])
def test_rotate(b, n, hq, hk, d, width, first, layout, dtype, inverse):
    q, g = _inputs(1, b, hq, n, d, dtype)
    k, _ = _inputs(2, b, hk, n, d, dtype)
    pos = torch.randint(0, 200000, (b, n), generator=g, device=DEV, dtype=torch.int32)
    freq = kvk.rotary_frequencies(width, 1e6, factor=4.0, original_tokens=8192)
    r = kvk.rotary(width, freq, layout, 1.139)
    outs = [torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))]
    kvk.rotate(r, pos, [q, k], outs, first, inverse=inverse)
    for x, y in zip((q, k), outs):
        _check(y, x, pos, freq, layout, first, 1.139, inverse)
    # in place: the same bits
    x, y = q.clone(), k.clone()
    kvk.rotate(r, pos, [x, y], first=first, inverse=inverse)
    assert torch.equal(x, outs[0]) and torch.equal(y, outs[1])


@pytest.mark.parametrize("pos", [0, 1, 2**24 + 1, 2**31 - 1, -1, -2**31])
def test_far_positions(pos):
    """Every 32-bit position keeps its angle: the frequency's 64 bits of a turn times the position.  (The
    reference's own angle in 64 bits is off by 2^31 2^-53 radians, far below the tolerance.)"""
    x, _ = _inputs(3, 1, 3, 4, 64, torch.float32)
    freq = [1.0, 3.0, -0.7, math.pi, 2 * math.pi, 0.25, 1e-9, 0.0, 1e5, -2e4] + [10000.0 ** (-i / 22) for i in range(22)]
    r = kvk.rotary(64, freq, kvk.PAIRS)
    p = torch.full((4,), pos, dtype=torch.int32, device=DEV)
    out = torch.empty_like(x)
    kvk.rotate(r, p, [x], [out])
    _, tol = _reference(x, p[None], freq, kvk.PAIRS, 0, 1.0, False)
    # a product position * frequency of up to 2^31 1e5 rounds to 2^-6 radians in 64 bits: in exact arithmetic instead
    from fractions import Fraction
    two_pi = Fraction("6.28318530717958647692528676655900576839433879875021164194988918461563281257")
    angle = [float((Fraction(f) * pos) % two_pi) for f in freq]
    c = torch.tensor([math.cos(a) for a in angle], dtype=F64, device=DEV)
    s = torch.tensor([math.sin(a) for a in angle], dtype=F64, device=DEV)
    y = x.to(F64)
    want = torch.stack((y[..., 0::2] * c - y[..., 1::2] * s, y[..., 1::2] * c + y[..., 0::2] * s), -1).flatten(-2)
    # a frequency of F turns is held to 2^-63 F turns (F <= 2^14) and 2^-65: at 2^31 positions 2^-18 turns for the largest one
    held = torch.tensor([abs(pos) * 2 * math.pi * (2.0**-63 * abs(f) + 2.0**-64) for f in freq], dtype=F64, device=DEV)
    big = (y[..., 0::2].abs() + y[..., 1::2].abs()) * held
    assert ((out.to(F64) - want).abs() <= tol + torch.stack((big, big), -1).flatten(-2) + 2.0**-24 * want.abs()).all()


def test_back_is_the_gradient():
    """<y, R x> = <R^T y, x>, and with magnitude 1 back and forth gives the row again."""
    x, g = _inputs(4, 2, 6, 19, 128, torch.float32)
    y, _ = _inputs(5, 2, 6, 19, 128, torch.float32)
    pos = torch.randint(0, 5000, (2, 19), generator=g, device=DEV, dtype=torch.int32)
    for layout in (kvk.HALVES, kvk.PAIRS):
        r = kvk.rotary(64, kvk.rotary_frequencies(64), layout, 1.25)
        fwd, back = torch.empty_like(x), torch.empty_like(y)
        kvk.rotate(r, pos, [x], [fwd], 32)
        kvk.rotate(r, pos, [y], [back], 32, inverse=True)
        lhs, rhs = (y.to(F64) * fwd.to(F64)).sum(), (back.to(F64) * x.to(F64)).sum()
        bound = 2.0**-21 * 2.5 * (x.to(F64).abs().sum() * y.abs().max() + y.to(F64).abs().sum() * x.abs().max())
        assert abs(lhs - rhs) <= bound
        # differences: the map is linear
        step = torch.zeros_like(x)
        step[0, 0, 3, 40] = 1.0
        moved = torch.empty_like(x)
        kvk.rotate(r, pos, [step], [moved], 32)
        assert abs((moved.to(F64) * y.to(F64)).sum() - back[0, 0, 3, 40].to(F64)) <= 2.0**-20 * 2.5 * y.abs().max()
        one = kvk.rotary(64, kvk.rotary_frequencies(64), layout)
        z = x.clone()
        kvk.rotate(one, pos, [z], first=32)
        kvk.rotate(one, pos, [z], first=32, inverse=True)
        assert (z - x).abs().max() <= 2.0**-20 * x.abs().max()


def test_layouts_and_positions():
    """Views of one fused projection, packed and padded, head-major and token-major, shared and repeated positions;
    the channels between and the rows around stay as they were."""
    freq = kvk.rotary_frequencies(128)
    r = kvk.rotary(128, freq)
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    x = torch.randn(50, 7, 128, generator=g, device=DEV).bfloat16()
    pos = torch.randint(0, 999, (50,), generator=g, device=DEV, dtype=torch.int32)
    was = x.clone()
    kvk.rotate(r, pos, [x[:, :4], x[:, 5:6]])  # in place in the projection; heads 4 and 6 are no keys
    for lo, hi in ((0, 4), (5, 6)):
        _check(x[:, lo:hi].transpose(0, 1)[None], was[:, lo:hi].transpose(0, 1)[None], pos[None], freq, kvk.HALVES, 0)
    assert torch.equal(x[:, 4], was[:, 4]) and torch.equal(x[:, 6], was[:, 6])
    # token-major in, head-major out; positions by sequence, shared, and repeated by layer
    y = torch.randn(6, 11, 3, 128, generator=g, device=DEV).transpose(1, 2)
    for p in (torch.randint(0, 999, (6, 11), generator=g, device=DEV, dtype=torch.int32),
              torch.randint(0, 999, (11,), generator=g, device=DEV, dtype=torch.int32),
              torch.randint(0, 999, (3, 11), generator=g, device=DEV, dtype=torch.int32)):
        out = torch.empty(6, 3, 11, 128, device=DEV)
        kvk.rotate(r, p, [y], [out])
        rows = p[None].expand(6, 11) if p.dim() == 1 else p.repeat(6 // p.shape[0], 1)
        _check(out, y, rows, freq, kvk.HALVES, 0)
    # one head read for several (a broadcast input)
    one = torch.randn(2, 1, 9, 128, generator=g, device=DEV).expand(2, 5, 9, 128)
    out, p = torch.empty(2, 5, 9, 128, device=DEV), torch.arange(9, dtype=torch.int32, device=DEV)
    kvk.rotate(r, p, [one], [out])
    _check(out, one, p[None].expand(2, 9), freq, kvk.HALVES, 0)


def test_four_tensors_of_their_own_widths():
    freq = kvk.rotary_frequencies(64)
    r = kvk.rotary(64, freq, kvk.PAIRS)
    xs = [_inputs(10 + i, 2, h, 21, d, torch.bfloat16)[0] for i, (h, d) in enumerate(((32, 192), (1, 64), (3, 96), (17, 128)))]
    firsts = [128, 0, 32, 8]
    pos = torch.arange(42, dtype=torch.int32, device=DEV).view(2, 21)
    outs = [torch.empty_like(x) for x in xs]
    kvk.rotate(r, pos, xs, outs, firsts)
    for x, y, f in zip(xs, outs, firsts):
        _check(y, x, pos, freq, kvk.PAIRS, f)
        keep = torch.ones(x.shape[-1], dtype=torch.bool, device=DEV)
        keep[f:f + 64] = False
        assert torch.equal(y[..., keep], x[..., keep])


def test_long_and_wide():
    """Runs of heads per thread, and a buffer past 2^31 elements."""
    freq = kvk.rotary_frequencies(128)
    r = kvk.rotary(128, freq)
    x, _ = _inputs(7, 1, 48, 20000, 128, torch.bfloat16)
    pos = torch.arange(20000, dtype=torch.int32, device=DEV)
    out = torch.empty_like(x)
    kvk.rotate(r, pos, [x], [out])
    at = torch.tensor([0, 1, 4095, 9999, 19998, 19999], device=DEV)
    _check(out[:, :, at], x[:, :, at], pos[at][None], freq, kvk.HALVES, 0)
    del x, out
    big = torch.zeros((2**31 + 2**20) // (33 * 128), 33, 128, dtype=torch.bfloat16, device=DEV)
    n = big.shape[0]
    big[-3:] = torch.randn(3, 33, 128, device=DEV).bfloat16()
    was = big[-3:].clone()
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    kvk.rotate(r, pos, [big])
    _check(big[-3:].transpose(0, 1)[None], was.transpose(0, 1)[None], pos[-3:][None], freq, kvk.HALVES, 0)


def test_infinite_values_stay_in_their_pair():
    freq = kvk.rotary_frequencies(64)
    r = kvk.rotary(64, freq)
    x, _ = _inputs(8, 1, 2, 6, 64, torch.float32)
    x[0, 0, 2, 5], x[0, 1, 4, 40] = float("inf"), float("nan")
    out = torch.empty_like(x)
    kvk.rotate(r, torch.arange(6, dtype=torch.int32, device=DEV), [x], [out])
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[0, 0, 2, [5, 37]] = True
    want[0, 1, 4, [8, 40]] = True
    assert torch.equal(bad, want)


def test_another_stream_and_a_captured_call():
    freq = kvk.rotary_frequencies(128)
    r = kvk.rotary(128, freq)
    x, g = _inputs(9, 2, 5, 31, 128, torch.bfloat16)
    pos = torch.arange(62, dtype=torch.int32, device=DEV).view(2, 31)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(x)
    kvk.rotate(r, pos, [x], [out], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    _check(out, x, pos, freq, kvk.HALVES, 0)
    with torch.cuda.stream(side):
        kvk.rotate(r, pos, [x], [out])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvk.rotate(r, pos, [x], [out])
    del r  # (the captured launch holds what it needs)
    for i in range(3):
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        pos.add_(1000)
        graph.replay()
        torch.cuda.synchronize()
        _check(out, x, pos, freq, kvk.HALVES, 0)
