"""The multi-token operators at the edges of what they accept: infinite values at visible
tokens, with and without mass, small values and queries, drafts that are taken back or complete
a group, group scales halfway between two fp16 values, launches of many sequences, repeated inputs
and captured calls of the long forms.  Tolerances as in test_gpu_operators.py.
"""
import math

import numpy as np
import pytest
import torch

from paper_2609_37988_amd import kvk
from gpu_common import DEV
import test_gpu_operators as base
from test_gpu_operators import Streams, _attend, _check, _gen, _prompt_inputs, _randn, _run_chunk, _run_prompt, _same

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
        q = _randn(_gen(40), 1, 1, hq, m, d).bfloat16()
        _spoil(q, c.k, c.v, at, score)
        c.append([0], [n])
        _, out = _run_chunk(c, 0, 1, [n], [m], SCALE, q=q)
        c.v[..., at, 5:8] = 0.0
        c.append([0], [n])
        _, ref = _run_chunk(c, 0, 1, [n], [m], SCALE, q=q)
        _check_spoilt(out[0, 0].transpose(0, 1), ref[0, 0].transpose(0, 1), max(at - start, 0), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq", [3, 20])
@pytest.mark.parametrize("first", [0.0, 20.0, 60.0])
def test_chunk_infinite_values_after_two_jumps(first, hq, d):
    """A partly seen tile whose first half raises the rows' logits a little and whose second one by
    more than fp32's range, for some rows of a wave."""
    n, low, t = 430, 200, 240  # (the second tile of its split)
    c = Streams([(0, 16)], hq, 1, d, 1, n, kvk.KIVI32, seed=48)
    q = _randn(_gen(49), 1, 1, hq, n, d).bfloat16()
    _spoil(q, c.k, c.v, t, 400.0)
    c.k[..., low, :] = 0.0
    c.k[..., low, 0] = first / SCALE
    c.append([0], [n])
    _, out = _run_chunk(c, 0, 1, [n], [n], SCALE, q=q)
    c.v[..., t, 5:8] = 0.0
    c.append([0], [n])
    _, ref = _run_chunk(c, 0, 1, [n], [n], SCALE, q=q)
    # the reference maximum moves earlier for the wave's other rows: rounding, not bits (each side
    # is off by its own rounding and the probabilities', 2^-8 of the largest value each)
    _check_rows(c, [n], [n], SCALE, q, ref)
    clean = [x for x in range(d) if x not in (5, 6, 7)]
    assert ((out - ref).abs()[..., clean] <= 2.0**-6 * c.v.abs().max()).all()
    assert (out[0, 0, :, t:, 5] == math.inf).all() and (out[0, 0, :, t:, 6] == -math.inf).all()
    assert torch.isnan(out[0, 0, :, t:, 7]).all() and torch.isfinite(out[0, 0, :, :t]).all()


@pytest.mark.parametrize("score,want", SCORES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq", [3, 20, 64])
def test_chunk_infinite_values_in_the_window_of_a_quantised_layer(hq, d, score, want):
    n, m, at = 430, 12, 425
    c = Streams([(0, 4)], hq, 1, d, 1, n, kvk.KIVI32, seed=36)
    q = _randn(_gen(40), 1, 1, hq, m, d).bfloat16()
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


def _check_rows(c, stored, new, scale, q, out, held=None):
    """The outputs of layer 0 with the tolerance of test_gpu_operators.py and what it leaves out:
    probabilities beneath fp16's normal range (quantised layers).  A row's largest probability
    enters the product as 2^7 or more and fp16 rounds small ones by at most 2^-25, so each
    probability is off by at most 2^-32 of the largest.  SYMROW scales the values of 32 tokens by
    the power of two of their largest scale, and the probabilities against it: there 2^-32 of the
    largest product of a probability and its group's scale, here 2^-31 of that with the
    group's largest value (a scale is between it and half of it, times a constant).  held: tokens
    in the cache, where they are more than the rows' (which groups are complete goes by them)."""
    grp = c.hq // c.hkv
    for b, (n, m) in enumerate(zip(stored, new)):
        assert (out[:, b, :, m:] == 7.0).all(), "rows past the new tokens"
        last = torch.arange(n - m, n, device=DEV)
        for h in range(c.hkv if m else 0):
            K, V, bits = c.values(0, b, h, held or n)
            K, V = K[:n], V[:n]
            rows = q[0, b, h * grp:(h + 1) * grp, :m]
            err = (0.0, 2.0**-8, 0.0) if bits == 16 else (2.0**-11, 2.0**-11, 2.0**-11)
            o, lse, tol, _ = _attend(rows, K, V, scale, last, *err)
            if bits != 16:
                top = V.abs().amax(-1)
                top = torch.cat([x.amax().clamp(min=1e-30).expand(x.numel()) for x in top.split(32)])
                if c.dims.qscheme != kvk.SYMROW:
                    top = torch.ones_like(top)
                p = torch.exp((rows.double() @ K.double().t()) * scale - lse[..., None])
                seen = torch.arange(n, device=DEV) <= last[:, None]
                p = torch.where(seen, p, torch.zeros_like(p))
                off = seen.double() @ (V.abs().double() / top[:, None])  # [rows, channels]
                tol = tol + 2.0**-31 * (p * top).amax(-1, keepdim=True) * off
            _check(out[0, b, h * grp:(h + 1) * grp, :m], o, tol, f"sequence {b} head {h}")


def _small(scheme, d, bits, hq, kv, qf):
    """Keys and values scaled by kv, queries by qf, the softmax scale to match."""
    c = Streams([(0, bits)], hq, 1, d, 8, 520, scheme, seed=32)
    c.k, c.v = c.k * kv, c.v * kv
    c.append([0] * 8, STORED)
    scale = 0.8 / math.sqrt(d) / (kv * qf)
    for new in NEW:
        q = (_randn(_gen(41), 1, 8, hq, max(new), d) * qf).bfloat16()
        _, out = _run_chunk(c, 0, 1, STORED, new, scale, q=q)
        _check_rows(c, STORED, new, scale, q, out)


@pytest.mark.parametrize("scheme", [kvk.KIVI32, kvk.GROUP64])
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
@pytest.mark.parametrize("d,hq", [(64, 64), (128, 5)])
@pytest.mark.parametrize("kv,qf", [(2.0**-12, 1.0), (2.0**-18, 1.0), (1.0, 2.0**-12), (1.0, 2.0**-30), (2.0**-18, 2.0**12)])
def test_chunk_small_values(kv, qf, d, hq, bits, scheme):
    """Values and queries below fp16's normal range, in full blocks and in the window."""
    _small(scheme, d, bits, hq, kv, qf)


@pytest.mark.parametrize("bits", [8, 4, 2])
@pytest.mark.parametrize("d,hq", [(64, 64), (128, 5)])
@pytest.mark.parametrize("kv,qf", [(2.0**-12, 1.0), (2.0**-18, 1.0), (2.0**-40, 2.0**-10), (2.0**12, 1.0)])
def test_chunk_small_symrow_values(kv, qf, d, hq, bits):
    """The same where a row's scale is bf16, which reaches further than fp16."""
    _small(kvk.SYMROW, d, bits, hq, kv, qf)


@pytest.mark.parametrize("bits", [8, 4, 2])
@pytest.mark.parametrize("d,hq", [(64, 64), (128, 5), (128, 30)])
def test_chunk_symrow_values_of_many_sizes(d, hq, bits):
    """Tokens whose values, and whose keys, differ by up to 2^16 from one to the next and by 2^20
    from one group to the next; contexts in one piece and split."""
    cap = 3000
    c = Streams([(0, bits)], hq, 1, d, 2, cap, kvk.SYMROW, seed=33)
    g = _gen(34)
    for x, top in ((c.k, 1.0), (c.v, 1.0)):
        per_token = torch.exp2(-16 * torch.rand(1, 2, 1, cap, 1, generator=g, device=DEV))
        per_group = torch.exp2(-20 * torch.rand(1, 2, 1, cap // 30, 1, generator=g, device=DEV)).repeat_interleave(32, 3)[:, :, :, :cap]
        x.copy_(x.float() * per_token * per_group)
    c.k[:, :, :, ::7] = (c.k[:, :, :, ::7].float() * 2.0**10).bfloat16()
    stored = [2990, 96]
    c.append([0, 0], stored)
    for new in ([1, 96], [7, 40], [33, 1]):
        q, out = _run_chunk(c, 0, 1, stored, new, 0.1)
        _check_rows(c, stored, new, 0.1, q, out)


@pytest.mark.parametrize("d,hq", [(64, 64), (128, 5), (128, 20)])
@pytest.mark.parametrize("scale", [0.25, -0.25, 1e30, 1e-38])
def test_chunk_symrow_values_2_to_80_apart(scale, d, hq):
    """One token with values of 2^40 among many of 2^-40 that together weigh a fifth of it: they count
    in the sum.  Softmax scales to both ends, the queries to match."""
    n, t = 2047, 1000
    c = Streams([(0, 8)], hq, 1, d, 1, n, kvk.SYMROW, seed=50)
    c.v.copy_(c.v.float() * 2.0**-40)
    c.v[..., t, :] = (c.v[..., t, :].float() * 2.0**80).bfloat16()
    c.k[..., :] = 0.0
    c.k[..., 0] = 1.0
    c.k[..., t, 0] = 10.0  # ln of 2^13: 9 more than the others
    c.append([0], [n])
    q = (_randn(_gen(51), 1, 1, hq, 3, d) * abs(0.01 / scale)).bfloat16()
    q[..., 0] = 1.0 / scale
    _, out = _run_chunk(c, 0, 1, [n], [3], scale, q=q)
    _check_rows(c, [n], [3], scale, q, out)


@pytest.mark.parametrize("bits", [8, 4, 2])
@pytest.mark.parametrize("d,hq", [(64, 64), (128, 5), (128, 20)])
def test_chunk_symrow_infinite_token(d, hq, bits):
    """A token with infinities has an infinite scale: its group's earlier tokens, and their rows, do
    not notice; the rows that see it are NaN."""
    n, t = 70, 40
    c = Streams([(0, bits)], hq, 1, d, 1, n, kvk.SYMROW, seed=37)
    c.k[..., t, 3], c.v[..., t, 4] = math.inf, -math.inf
    c.append([0], [n])
    q, out = _run_chunk(c, 0, 1, [n], [n], 0.1)
    assert torch.isnan(out[..., t:, :]).all()
    c.k[..., t, 3], c.v[..., t, 4] = 0.0, 0.0  # (hidden from the rows before it)
    _check_rows(c, [t], [t], 0.1, q[..., :t, :].contiguous(), out[..., :t, :].contiguous(), held=n)


@pytest.mark.parametrize("scheme", [kvk.SYMROW, kvk.GROUP64])
@pytest.mark.parametrize("bits", [8, 4, 2])
def test_chunk_one_token_matches_decode_element_by_element(bits, scheme):
    """The decode step rounds less than what the tolerance of a chunk's row counts (codes are exact
    in its products), but GROUP64's codes and zeros enter apart: each of the two is at most twice
    the group's largest value."""
    hq, d, n = 10, 128, 333
    c = Streams([(0, bits)], hq, 2, d, 2, 400, scheme, seed=17)
    c.append([0, 0], [n, n])
    q, out = _run_chunk(c, 0, 1, [n, n], [1, 1], 0.09)
    ws = torch.empty(kvk.workspace_bytes(c.t, 0, 1), dtype=torch.uint8, device=DEV)
    dec = torch.empty((1, 2, hq, d), dtype=torch.float32, device=DEV)
    kvk.decode_attention(c.t, 0, 1, q[:, :, :, 0].contiguous(), n, 0.09, c.arena, dec, ws)
    last = torch.tensor([n - 1], device=DEV)
    for b in range(2):
        for h in range(2):
            rows = slice(5 * h, 5 * h + 5)
            K, V, _ = c.values(0, b, h, n)
            o, _, tol, _ = _attend(q[0, b, rows], K, V, 0.09, last, 2.0**-11, 2.0**-11, 2.0**-11)
            wide = V.abs().reshape(n, d // 64, 64).amax(-1, keepdim=True).expand(n, d // 64, 64).reshape(n, d)
            _, _, more, _ = _attend(q[0, b, rows], K, 4 * wide, 0.09, last, 2.0**-11, 2.0**-11, 2.0**-11)
            _check(out[0, b, rows], o, tol, "chunk")
            _check(dec[0, b, rows][:, None], o, tol + (more if scheme == kvk.GROUP64 else 0), "decode")


# --------------------------------------------------------------------------------------
# Drafts: taken back, and in a group that they complete
# --------------------------------------------------------------------------------------


@pytest.mark.parametrize("scheme", [kvk.KIVI32, kvk.SYMROW, kvk.GROUP64])
@pytest.mark.parametrize("d", [64, 128])
def test_chunk_drafts_taken_back(d, scheme):
    """Sequences whose drafts are rejected in part, inside a group and after completing one (or
    two): the streams go on as those that never held the drafts."""
    L, B, hkv = 3, 5, 2
    plan = [(0, 16), (0, 8), (0, 2)]
    c = Streams(plan, 4, hkv, d, B, 200, scheme, seed=38)
    never = c.new_arena()
    start, drafts, kept = [60, 62, 30, 64, 5], [3, 6, 70, 4, 20], [1, 1, 1, 0, 20]
    c.append([0] * B, start)
    c.append([0] * B, start, arena=never)
    other = Streams(plan, 4, hkv, d, B, 200, scheme, seed=39)  # rejected tokens: other values after the kept ones
    for b in range(B):
        at = start[b] + kept[b]
        other.k[:, b, :, :at], other.v[:, b, :, :at] = c.k[:, b, :, :at], c.v[:, b, :, :at]
    other.append(start, drafts, arena=c.arena)
    now = [s + n for s, n in zip(start, kept)]
    again = [n % 32 if n // 32 < (s + m) // 32 else 0 for n, s, m in zip(now, start, drafts)]
    assert again == [0, 31, 31, 0, 0]
    c.append([n // 32 * 32 if a else n for n, a in zip(now, again)], again)
    c.append(start, kept, arena=never)
    _same(c.streams(c.arena, now), c.streams(never, now))
    for l in (0, 2):
        q, out = _run_chunk(c, l, l + 1, now, [5, 3, 1, 2, 7], 0.1)
        c.arena, never = never, c.arena
        _, ref = _run_chunk(c, l, l + 1, now, [5, 3, 1, 2, 7], 0.1, q=q)
        c.arena, never = never, c.arena
        assert torch.equal(out, ref)
    more = [40, 1, 5, 33, 64]
    c.append(now, more)
    c.append(now, more, arena=never)
    now = [n + m for n, m in zip(now, more)]
    _same(c.streams(c.arena, now), c.streams(never, now))


@pytest.mark.parametrize("scheme", [kvk.KIVI32, kvk.SYMROW, kvk.GROUP64])
@pytest.mark.parametrize("bits", [8, 4, 2])
@pytest.mark.parametrize("d,hq", [(64, 64), (128, 5)])
def test_chunk_rows_of_a_completed_group_with_a_late_outlier(d, hq, bits, scheme):
    """Rows of a group that the chunk completes attend to its quantised form, whose scales a later
    token of it may have set."""
    c = Streams([(0, bits)], hq, 1, d, 2, 100, scheme, seed=42)
    for x in (c.k, c.v):
        x[:, 0, :, 60] *= 50.0
        x[:, 1, :, 31] *= 50.0
    stored, new = [64, 40], [20, 40]
    c.append([0, 0], [44, 0])
    c.append([44, 0], new)
    q, out = _run_chunk(c, 0, 1, stored, new, 0.02)
    _check_rows(c, stored, new, 0.02, q, out)


@pytest.mark.parametrize("scheme,keys", [(kvk.KIVI32, False), (kvk.GROUP64, True)])
@pytest.mark.parametrize("bits", [8, 4, 2])
@pytest.mark.parametrize("d,hq", [(64, 64), (128, 5), (128, 20)])
def test_chunk_infinite_token_of_a_group(d, hq, bits, scheme, keys):
    """As for SYMROW, where the scales are each token's own: GROUP64, and the values of KIVI32."""
    n, t = 70, 40
    c = Streams([(0, bits)], hq, 1, d, 1, n, scheme, seed=43)
    c.v[..., t, 4] = math.inf
    if keys:
        c.k[..., t, 3] = math.inf
    c.append([0], [n])
    q, out = _run_chunk(c, 0, 1, [n], [n], 0.1)
    group = slice(0, 32 if scheme == kvk.KIVI32 else 64)  # the channels that share the infinite scale
    assert not torch.isfinite(out[..., t:, group]).any()
    c.v[..., t, 4] = 0.0
    if keys:
        c.k[..., t, 3] = 0.0
    _check_rows(c, [t], [t], 0.1, q[..., :t, :].contiguous(), out[..., :t, :].contiguous(), held=n)


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


# --------------------------------------------------------------------------------------
# Launches of many sequences, long prompts, repeated inputs, unlike row counts
# --------------------------------------------------------------------------------------


@pytest.mark.parametrize("d,hq,hkv", [(64, 2, 1), (128, 3, 3)])
@pytest.mark.parametrize("count", [65, 128, 256])
def test_prompt_and_weight_many_sequences(count, d, hq, hkv):
    """More sequences than a wave has lanes, up to the limit, of lengths that repeat and end
    inside blocks of either kernel, empty ones among them."""
    rng = np.random.default_rng(count)
    lens = [int(x) for x in rng.choice([0, 1, 17, 64, 127, 128, 129, 256, 257, 300], count)]
    base.test_prompt_attention(lens, hq, hkv, d, "packed")
    base.test_attention_weight(lens, hq, hkv, d, "packed")


@pytest.mark.parametrize("lens,hq,hkv,d", [([5003], 2, 1, 64), ([2049, 4100], 3, 1, 128)])
def test_prompt_and_weight_long(lens, hq, hkv, d):
    base.test_prompt_attention(lens, hq, hkv, d, "fused")
    base.test_attention_weight(lens, hq, hkv, d, "padded")


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_repeated_inputs(d):
    """Heads, and tokens, that share one place (strides of 0), without the log-sum-exps."""
    lens, scale = [150, 33], 0.2
    q, k, v = _prompt_inputs(44, lens, 4, 2, d, "packed")
    k, v = k[:, :1].expand(-1, 2, -1), v[:, 1:].expand(-1, 2, -1)
    q = q[5:6].expand(183, -1, -1)
    out, lse = _run_prompt(q, k, v, lens, scale)
    base._check_prompt(q, k, v, lens, scale, out, lse)
    again = torch.full_like(out, NAN)
    kvk.prompt_attention(q, k, v, lens, scale, again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("scheme", [kvk.KIVI32, kvk.SYMROW])
def test_chunk_of_a_prompt_beside_single_tokens(scheme):
    """One long chunk sets the launch's row blocks; the other sequences have one row per head, or
    a few, or none."""
    stored = [1500] + [1, 700, 32, 64, 95, 1024, 5, 333, 64, 31]
    new = [600] + [1, 1, 1, 4, 2, 1, 5, 1, 0, 31]
    c = Streams([(0, 8)], 5, 1, 128, len(stored), 1500, scheme, seed=45)
    c.append([0] * len(stored), stored)
    q, out = _run_chunk(c, 0, 1, stored, new, 0.08)
    _check_rows(c, stored, new, 0.08, q, out)


def test_keep_heaviest_long_and_all_recent():
    n, keep = 40000, 333
    t = kvk.layer_table(kvk.make_dims(kvk.GQA, 1, 2, 2, 64, batch=1, max_tokens=n, keep_tokens=keep), kvk.make_plan([(0, 8)]))
    out = torch.full((1, 2, keep), -1, dtype=torch.int32, device=DEV)
    kvk.keep_heaviest(t, torch.rand(1, 2, n, device=DEV), n, keep, out)
    assert torch.equal(out, torch.arange(n - keep, n, dtype=torch.int32, device=DEV).expand(1, 2, keep))


def test_long_forms_captured():
    """The keep list of a long prompt and a chunk whose context is split, captured into one graph
    with workspaces of their own and replayed on new inputs, eager calls in between."""
    B, hq, hkv, d, n, keep = 2, 4, 2, 128, 20000, 5000
    c = Streams([(0, 4), (1, 4)], hq, hkv, d, B, n, kvk.KIVI32, seed=46)
    stored, new = [19990, 7001], [3, 2]
    c.append([0, 0], stored)
    dims = kvk.make_dims(kvk.GQA, 1, hq, hkv, d, batch=B, max_tokens=n, keep_tokens=keep)
    te = kvk.layer_table(dims, kvk.make_plan([(0, 8)]))
    g = _gen(47)
    w, q = _randn(g, B, hkv, n).exp(), _randn(g, 2, B, hq, 3, d).bfloat16()
    idx = torch.full((B, hkv, keep), -1, dtype=torch.int32, device=DEV)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((kvk.chunk_workspace_bytes(c.t, 0, 2, 3),), 0xFF, dtype=torch.uint8, device=DEV)
    kws = torch.full((kvk.keep_workspace_bytes(te, n),), 0xFF, dtype=torch.uint8, device=DEV)
    assert kws.numel() > 0 and ws.numel() > 256

    def path():
        kvk.keep_heaviest(te, w, n, 32, idx, kws)
        kvk.chunk_attention(c.t, 0, 2, q, stored, new, 0.09, c.arena, out, ws)

    path()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        path()
    for _ in range(3):
        w.copy_(_randn(g, *w.shape).exp()), q.copy_(_randn(g, *q.shape))
        path()
        eager = idx.clone(), out.clone()
        idx.fill_(-1), out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(idx, eager[0]) and torch.equal(out, eager[1])
        assert np.array_equal(idx.cpu().numpy().reshape(-1, keep), base._keep_ref(w.cpu().numpy(), keep, 32))
        assert (out[:, 1, :, 2:] == 7.0).all()
    base._check_chunk(c, 0, 2, stored, new, 0.09, q, out)
