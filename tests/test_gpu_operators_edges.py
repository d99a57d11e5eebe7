"""The multi-token operators at the edges of what they accept: infinite values at visible
tokens, with and without mass, small values and queries, and group scales halfway between two
fp16 values.
"""
import math

import pytest
import torch

from paper_2609_37988_amd import kvk
from gpu_common import DEV
from test_gpu_operators import Streams, _check_chunk, _prompt_inputs, _run_chunk, _run_prompt

pytestmark = pytest.mark.gpu
NAN = float("nan")


# --------------------------------------------------------------------------------------
# Infinite values at visible tokens
# --------------------------------------------------------------------------------------

# Score of the token that holds the infinities, relative to the others' (of order 1), and what an
# infinite value there gives: probability 0 times infinity is NaN, a positive one leaves infinity.
SCALE = 0.1
SCORES = [(-math.inf, NAN), (-30000.0, NAN), (-50.0, math.inf), (400.0, math.inf)]


def _spoil(q, k, v, t, score):
    """Channel 0 of the keys decides the score of token t; channels 5 to 7 of its values are not finite."""
    q[..., 0], k[..., 0] = 1.0, 0.0
    k[..., t, :] = 0.0
    k[..., t, 0] = score / SCALE
    v[..., t, 5], v[..., t, 6], v[..., t, 7] = math.inf, -math.inf, NAN


def _check_spoilt(out, ref, t, want):
    """out, ref [rows, heads, d], row i that of token i; ref without the infinities."""
    d = out.shape[-1]
    clean = [c for c in range(d) if c not in (5, 6, 7)]
    assert torch.equal(out[:, :, clean], ref[:, :, clean]) and torch.equal(out[:t], ref[:t])
    for ch, x in ((5, want), (6, -want), (7, NAN)):
        got = out[t:, :, ch].float()
        wrong = ~(torch.isnan(got) if math.isnan(x) else got == x).all(-1)
        assert not wrong.any(), f"channel {ch}: rows {(wrong.nonzero().flatten() + t).tolist()} are not {x}"


@pytest.mark.parametrize("score,want", SCORES)
@pytest.mark.parametrize("d", [64, 128])
def test_prompt_infinite_values_agree(d, score, want):
    """Rows that see the token in the tile of the diagonal, and rows that see it in a tile which
    the whole workgroup sees."""
    n, t = 500, 150
    q, k, v = _prompt_inputs(30, [n], 2, 1, d, "padded")
    _spoil(q, k, v, t, score)
    out, _ = _run_prompt(q, k, v, [n], SCALE)
    v[..., t, 5:8] = 0.0
    ref, _ = _run_prompt(q, k, v, [n], SCALE)
    _check_spoilt(out[0, :, :n].transpose(0, 1), ref[0, :, :n].transpose(0, 1), t, want)


@pytest.mark.parametrize("score,want", SCORES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq", [3, 20, 64])
def test_chunk_infinite_values_agree(hq, d, score, want):
    """The same for chunks of a 16-bit layer, in narrow and wide workgroups, and in the window."""
    n, t = 430, 150
    for start, m, at in ((0, n, t), (n - 5, 5, t), (n - 12, 12, 425)):
        c = Streams([(0, 16)], hq, 1, d, 1, n, kvk.KIVI32, seed=31)
        q = torch.randn(1, 1, hq, m, d, device=DEV).bfloat16()
        _spoil(q, c.k, c.v, at, score)
        c.append([0], [n])
        _, out = _run_chunk(c, 0, 1, [n], [m], SCALE, q=q)
        c.v[..., at, 5:8] = 0.0
        c.append([0], [n])
        _, ref = _run_chunk(c, 0, 1, [n], [m], SCALE, q=q)
        _check_spoilt(out[0, 0].transpose(0, 1), ref[0, 0].transpose(0, 1), max(at - start, 0), want)


@pytest.mark.parametrize("score,want", SCORES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq", [3, 20, 64])
def test_chunk_infinite_values_in_the_window_of_a_quantised_layer(hq, d, score, want):
    n, m, at = 430, 12, 425
    c = Streams([(0, 4)], hq, 1, d, 1, n, kvk.KIVI32, seed=36)
    q = torch.randn(1, 1, hq, m, d, device=DEV).bfloat16()
    _spoil(q, c.k, c.v, at, score)
    c.append([0], [n])
    _, out = _run_chunk(c, 0, 1, [n], [m], SCALE, q=q)
    c.v[..., at, 5:8] = 0.0
    c.append([0], [n])
    _, ref = _run_chunk(c, 0, 1, [n], [m], SCALE, q=q)
    _check_spoilt(out[0, 0].transpose(0, 1), ref[0, 0].transpose(0, 1), at - (n - m), want)


# --------------------------------------------------------------------------------------
# Small values
# --------------------------------------------------------------------------------------

STORED = [1, 20, 33, 64, 129, 200, 517, 97]
NEW = [[1] * 8, [1, 20, 33, 4, 6, 7, 3, 1], [1, 11, 20, 33, 60, 100, 0, 40]]


def _small(scheme, d, bits, hq, kv, qf):
    """Keys and values scaled by kv, queries by qf, the softmax scale to match."""
    c = Streams([(0, bits)], hq, 1, d, 8, 520, scheme, seed=32)
    c.k, c.v = c.k * kv, c.v * kv
    c.append([0] * 8, STORED)
    scale = 0.8 / math.sqrt(d) / (kv * qf)
    for new in NEW:
        q = (torch.randn(1, 8, hq, max(new), d, device=DEV) * qf).bfloat16()
        _, out = _run_chunk(c, 0, 1, STORED, new, scale, q=q)
        _check_chunk(c, 0, 1, STORED, new, scale, q, out)


@pytest.mark.parametrize("scheme", [kvk.KIVI32, kvk.GROUP64])
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
@pytest.mark.parametrize("d,hq", [(64, 64), (128, 5)])
@pytest.mark.parametrize("kv,qf", [(2.0**-12, 1.0), (2.0**-18, 1.0), (1.0, 2.0**-12), (1.0, 2.0**-30), (2.0**-18, 2.0**12)])
def test_chunk_small_values(kv, qf, d, hq, bits, scheme):
    """Values and queries below fp16's normal range, in full blocks and in the window."""
    _small(scheme, d, bits, hq, kv, qf)


# --------------------------------------------------------------------------------------
# Group scales halfway between two fp16 values
# --------------------------------------------------------------------------------------


def _tied_ranges(levels):
    """(lowest, highest) bf16 values whose difference is `levels` times a 12-bit odd number (times
    2^-10): the scale lies halfway between two fp16 values."""
    out = []
    for odd in range(2049, 4096, 2):
        d = levels * odd
        for k in range(4, 13):
            hi, lo = d >> k << k, d & ((1 << k) - 1)
            if hi >> k < 256 and lo < 256 and hi >> k:
                out.append((-lo / 1024, hi / 1024))
                break
    assert len(out) >= 64
    return out[::len(out) // 64][:64]


@pytest.mark.parametrize("bits", [8, 4, 2])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scheme", [kvk.KIVI32, kvk.GROUP64])
def test_group_scales_round_twice_as_documented(scheme, d, bits):
    """The scale is the fp32 quotient rounded to fp16 (the oracle's chain), in ties too: by the
    chunk append and by the prefill write."""
    n = 64
    ranges = _tied_ranges((1 << bits) - 1)
    c = Streams([(0, bits)], 1, 1, d, 1, n, scheme, seed=35)
    for x, per_channel in ((c.k, scheme == kvk.KIVI32), (c.v, False)):
        u = x.float().sigmoid()
        for i in range(n if not per_channel else d):
            lo, hi = ranges[i % len(ranges)]
            g = u[0, 0, 0, :, i] if per_channel else u[0, 0, 0, i]
            g.mul_(hi - lo).add_(lo)
            g[0::32], g[1::32] = lo, hi
        x.copy_(u)
    c.append([0], [n])
    want = c.values(0, 0, 0, n)
    for write in ("append", "prefill"):
        if write == "prefill":
            c.arena.fill_(0xFF)
            kvk.compress_layer(c.t, 0, c.k[0], c.v[0], n, None, c.arena)
        got = [torch.empty((1, 1, n, d), dtype=torch.float32, device=DEV) for _ in range(2)]
        kvk.debug_dequantize(c.t, 0, n, c.arena, *got)
        for g, w, name in zip(got, want, "kv"):
            wrong = (g[0, 0] != w.float()).sum()
            assert wrong == 0, f"{write}: {int(wrong)} of {n * d} {name} values differ"
