"""The block index, the choice of blocks and the attention over chosen blocks, on the GPU, against 64-bit
references made from the stored values (the test dequantiser's, which the oracle pins bit for bit).

The index and the choice are exact: codes, scales and lists have to be equal.

Tolerance of the attention, roundings counted as in test_gpu_operators: with A = sum_t p_t |v_t| (p the softmax)
an output o is off by at most
  2^-8 |o|          its own rounding,
  e_p A             probabilities rounded to bf16 (16-bit layers: 2^-8) or fp16 (2^-11; SYMROW's twice: with the scale),
  e_v A             values rounded to fp16 (KIVI32, GROUP64: 2^-11),
  2 d (A + |o|)     scores off by at most d: fp32 sums of products whose absolute sum is S, (d_h + 16) 2^-24 S, keys
                    rounded to fp16 (KIVI32: 2^-11 S), GROUP64's scale and zero parts, each at most 3 S',
  2^-31 sum_t max|v| probabilities below fp16's steps (2^-25, against a sum of at least 2^6),
and 2 % more for products of these terms."""
import math

import pytest
import torch

from gpu_common import DEV
from paper_2609_37988_amd import kvk

pytestmark = pytest.mark.gpu
F64 = torch.float64
NAN, INF = float("nan"), float("inf")
SCHEMES = {"kivi": kvk.KIVI32, "sym": kvk.SYMROW, "g64": kvk.GROUP64}


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


class Cache:
    """A GQA table (one plan, or one per sequence) with caches of the stored lengths."""

    def __init__(self, hq, hkv, d, stored, plan, scheme="kivi", cap=None, seed=1, plans=None, values=None):
        self.hq, self.hkv, self.d, self.stored = hq, hkv, d, list(stored)
        self.B, self.nl = len(stored), len(plans[0] if plans else plan)
        cap = cap or max(32, max(stored))
        self.cap = cap
        dims = kvk.make_dims(kvk.GQA, self.nl, hq, hkv, d, qscheme=SCHEMES[scheme], batch=self.B, max_tokens=cap)
        if plans:
            self.table = kvk.layer_table_batched(dims, [kvk.make_plan(p) for p in plans])
        else:
            self.table = kvk.layer_table(dims, kvk.make_plan(plan))
        self.plans = plans or [plan] * self.B
        self.scheme = scheme
        g = _gen(seed)
        n = max(stored)
        self.arena = torch.zeros(self.table.arena_bytes, dtype=torch.uint8, device=DEV)
        if values is None:
            k = _randn(g, self.nl, self.B, hkv, max(n, 1), d) * torch.exp(_randn(g, self.nl, 1, hkv, 1, d))
            v = _randn(g, self.nl, self.B, hkv, max(n, 1), d)
            values = k.bfloat16(), v.bfloat16()
        self.k, self.v = values
        kvk.append_chunk(self.table, 0, self.nl, self.k, self.v, 0, self.stored, self.arena)

    def anchor(self, l, b):
        return max(a for a in range(l + 1) if not self.plans[b][a][0])

    def bits(self, l, b):
        return self.plans[b][self.anchor(l, b)][1]

    def values(self, l):
        """What layer l reads, [B, Hkv, n, d] fp32 each, n the longest sequence's."""
        n = max(self.stored)
        k = torch.empty((self.B, self.hkv, max(n, 1), self.d), dtype=torch.float32, device=DEV)
        v = torch.empty_like(k)
        kvk.debug_dequantize(self.table, l, n, self.arena, k, v)
        return k, v

    def token_values(self, l, b, h, k, v):
        """K, V [n, d] of a stream as sequence b stores it: the dequantiser took the longest sequence's length, so
        the window of a shorter one comes from the inputs."""
        n, full = self.stored[b], self.stored[b] // 32 * 32
        a = self.anchor(l, b)
        return (torch.cat((k[b, h, :full], self.k[a, b, h, full:n].float())),
                torch.cat((v[b, h, :full], self.v[a, b, h, full:n].float())))


# --------------------------------------------------------------------------------------
# Index
# --------------------------------------------------------------------------------------


def _summary(keys):
    """Codes and scales of blocks keys [..., 32, d] by the definition."""
    x = keys.to(F64)
    lo, hi = x.amin(-2), x.amax(-2)
    y = torch.stack(((hi + lo) / 2, (hi - lo) / 2), -2)
    bad = ~torch.isfinite(x).all(-1).all(-1)
    y = torch.where(bad[..., None, None], torch.zeros_like(y), y)
    scale = (y.abs().amax(-1) / 127).float()
    s = scale.to(F64)[..., None]
    code = torch.where(s > 0, (y / torch.where(s > 0, s, torch.ones_like(s))).round().clamp(-127, 127), torch.zeros_like(y))
    scale[..., 1] = torch.where(bad, torch.full_like(scale[..., 1], INF), scale[..., 1])
    return code.to(torch.int8), scale


def _index_of(c, n_indexed=None, fill=0x55):
    index = torch.full((kvk.index_bytes(c.table),), fill, dtype=torch.uint8, device=DEV)
    kvk.index_blocks(c.table, 0, c.nl, c.stored, c.arena, index, n_indexed)
    return index


def _check_index(c, index, n_indexed=None, fill=0x55):
    for l in range(c.nl):
        k, _ = c.values(l)
        for b in range(c.B):
            codes, scales = kvk.index_views(c.table, index, l, b if c.table.plans else 0)
            codes, scales = (x[0] if c.table.plans else x[b] for x in (codes, scales))
            full, first = c.stored[b] // 32, (n_indexed[b] // 32 if n_indexed else 0)
            want, ws = _summary(k[b, :, :full * 32].reshape(c.hkv, full, 32, c.d))
            at = f"layer {l} sequence {b}"
            assert torch.equal(codes[:, first:full], want[:, first:]), at
            assert torch.equal(scales[:, first:full], ws[:, first:]), at
            # blocks that the index has already, and places past the stored ones, stay
            for rest in (codes[:, :first], codes[:, full:], scales[:, :first], scales[:, full:]):
                assert (rest.contiguous().view(torch.uint8) == fill).all(), at


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scheme", ["kivi", "sym", "g64"])
@pytest.mark.parametrize("hkv", [1, 3])
def test_index(d, scheme, hkv):
    plan = [(0, 16), (0, 8), (1, 8), (0, 4), (0, 2)]
    c = Cache(hkv, hkv, d, [0, 1, 31, 32, 33, 64, 500, 1023], plan, scheme)
    _check_index(c, _index_of(c))
    done = [0, 0, 31, 32, 5, 33, 480, 40]
    _check_index(c, _index_of(c, done), done)


def test_index_follows_appends():
    """A token at a time and chunks: after each append only the blocks it completed are written."""
    c = Cache(2, 1, 64, [40, 63, 7], [(0, 4), (0, 16)], cap=200)
    index = _index_of(c)
    g = _gen(5)
    for m in (1, 24, 30, 64):
        k, v = (_randn(g, 2, 3, 1, m, 64).bfloat16() for _ in range(2))
        before = list(c.stored)
        kvk.append_chunk(c.table, 0, 2, k, v, before, None, c.arena)
        c.stored = [n + m for n in before]
        kvk.index_blocks(c.table, 0, 2, c.stored, c.arena, index, before)
        _check_index(c, index)


@pytest.mark.parametrize("bits,scheme", [(16, "kivi"), (8, "sym"), (4, "kivi"), (2, "g64")])
def test_index_values(bits, scheme):
    """Blocks of zeros and of one value, tiny and huge keys, one key far from the others."""
    g = _gen(3)
    n, d = 32 * 9, 64
    k = _randn(g, 1, 1, 1, n, d)
    k[0, 0, 0, :32] = 0
    k[0, 0, 0, 32:64] = 0.75
    k[0, 0, 0, 64:96] *= 2.0**-13
    k[0, 0, 0, 96:128] *= 60000 / k[0, 0, 0, 96:128].abs().max()
    k[0, 0, 0, 130, 7] = -5000
    if scheme == "sym" or bits == 16:
        k[0, 0, 0, 160:192] *= 1e36
        k[0, 0, 0, 192:224] *= 1e-30
    k = k.bfloat16()
    c = Cache(1, 1, d, [n], [(0, bits)], scheme, values=(k, k))
    _check_index(c, _index_of(c))


def test_index_of_infinite_and_nan_keys():
    g = _gen(4)
    k = _randn(g, 1, 2, 2, 160, 128).bfloat16()
    k[0, 0, 0, 3, 5], k[0, 0, 1, 40, 127], k[0, 1, 0, 70, 64], k[0, 1, 1, 159, 0] = INF, -INF, NAN, INF
    c = Cache(2, 2, 128, [160, 160], [(0, 16)], values=(k, k))
    index = _index_of(c)
    _check_index(c, index)
    codes, scales = kvk.index_views(c.table, index, 0)
    bad = torch.isinf(scales[..., 1])
    assert bad.nonzero().tolist() == [[0, 0, 0], [0, 1, 1], [1, 0, 2], [1, 1, 4]]


def test_index_per_sequence_plans_and_many_sequences():
    plans = [[(0, (16, 8, 4, 2)[b % 4]), (1, 16) if b % 3 == 0 else (0, 4), (0, 2)] for b in range(7)]
    c = Cache(2, 1, 64, [100, 32, 31, 64, 200, 0, 96], None, plans=plans)
    _check_index(c, _index_of(c))
    stored = [32 + 3 * i for i in range(150)]
    c = Cache(1, 1, 64, stored, [(0, 4), (0, 8)])
    _check_index(c, _index_of(c))


# --------------------------------------------------------------------------------------
# Choice
# --------------------------------------------------------------------------------------


def _chosen(q, codes, scales, nb, n_select, first, recent):
    """The list of one (layer, sequence, KV head): q [G, d] bf16, codes [nb, 2, d], scales [nb, 2]."""
    if nb <= n_select:
        return list(range(nb)) + [-1] * (n_select - nb)
    x = q.float()
    top = x.abs().amax(-1, keepdim=True)
    s = top * torch.tensor(1 / 127, dtype=torch.float32, device=q.device)
    s = torch.where(torch.isfinite(x).all(-1, keepdim=True), s, torch.zeros_like(s))
    q8 = torch.where(s > 0, torch.round(x / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(x)).to(F64)
    m = codes[:nb].to(F64)
    dm, dh = q8 @ m[:, 0].t(), q8.abs() @ m[:, 1].t()
    t = (dh * scales[:nb, 1].to(F64)).float()
    u = (dm * scales[:nb, 0].to(F64) + t.to(F64)).float()
    u = (u.to(F64) * s.to(F64)).float()
    u = torch.where(torch.isnan(u), torch.full_like(u, INF), u).amax(0)
    mid = u[first:nb - recent]
    order = torch.sort(mid, descending=True, stable=True)[1][:n_select - first - recent] + first
    return sorted(list(range(first)) + order.tolist() + list(range(nb - recent, nb)))


def _fake_index(c, seed, ties=False):
    """An index of made-up summaries (codes over their whole range), so that long contexts need no caches."""
    index = torch.zeros(kvk.index_bytes(c.table), dtype=torch.uint8, device=DEV)
    g = _gen(seed)
    for l in range(c.nl):
        for b in range(c.B if c.table.plans else 1):
            if l and c.anchor(l, b) != l:
                continue
            codes, scales = kvk.index_views(c.table, index, l, b)
            codes.copy_(torch.randint(-127, 128, codes.shape, generator=g, device=DEV))
            codes[..., 1, :].abs_()
            scales.copy_(torch.rand(scales.shape, generator=g, device=DEV) * 0.02)
            if ties:  # few different blocks
                i = torch.randint(0, 3, (codes.shape[2],), generator=g, device=DEV)
                codes.copy_(codes[:, :, i])
                scales.copy_(scales[:, :, i])
    return index


class Shape(Cache):
    """A table without caches, for choices from a made-up index."""

    def __init__(self, hq, hkv, d, stored, plan, cap=None, plans=None):
        self.hq, self.hkv, self.d, self.stored, self.B, self.nl = hq, hkv, d, list(stored), len(stored), len(plans[0] if plans else plan)
        dims = kvk.make_dims(kvk.GQA, self.nl, hq, hkv, d, batch=self.B, max_tokens=cap or max(32, max(stored)))
        self.table = kvk.layer_table_batched(dims, [kvk.make_plan(p) for p in plans]) if plans else kvk.layer_table(dims, kvk.make_plan(plan))
        self.plans = plans or [plan] * self.B


def _workspace(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) if n else None


def _select(c, q, index, n_select, first=0, recent=0, stream=None):
    blocks = torch.full((c.nl, c.B, c.hkv, n_select), -77, dtype=torch.int32, device=DEV)
    kvk.select_blocks(c.table, 0, c.nl, q, c.stored, index, blocks, first, recent,
                      _workspace(kvk.select_workspace_bytes(c.table, 0, c.nl)), stream)
    return blocks


def _check_select(c, q, index, blocks, first, recent):
    G, got = c.hq // c.hkv, blocks.cpu()
    for l in range(c.nl):
        for b in range(c.B):
            codes, scales = kvk.index_views(c.table, index, l, b if c.table.plans else 0)
            codes, scales = (x[0] if c.table.plans else x[b] for x in (codes, scales))
            for h in range(c.hkv):
                want = _chosen(q[l, b, h * G:(h + 1) * G], codes[h], scales[h], c.stored[b] // 32, blocks.shape[3], first, recent)
                assert got[l, b, h].tolist() == want, f"layer {l} sequence {b} head {h}"


@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 64), (4, 1, 64), (28, 4, 128), (40, 8, 128), (16, 1, 128), (17, 1, 64), (33, 1, 128),
                                      (64, 1, 64), (64, 1, 128)])
@pytest.mark.parametrize("n_select,first,recent", [(1, 0, 0), (5, 0, 0), (7, 1, 2), (3, 1, 2), (64, 0, 0)])
def test_select(hq, hkv, d, n_select, first, recent):
    c = Shape(hq, hkv, d, [0, 31, 32, 100, 5000, 32 * 64, 32 * 65 + 3, 1337], [(0, 4)] + ([(1, 4)] if hq < 32 else []))
    index, g = _fake_index(c, 1), _gen(2)
    q = _randn(g, c.nl, c.B, hq, d).bfloat16()
    blocks = _select(c, q, index, n_select, first, recent)
    _check_select(c, q, index, blocks, first, recent)
    assert torch.equal(blocks, _select(c, q, index, n_select, first, recent))


@pytest.mark.parametrize("stored", [[131072], [32 * 8192], [32 * 8193 + 5, 40], [400000, 131071, 1]])
@pytest.mark.parametrize("n_select,first,recent", [(1, 0, 0), (256, 1, 4), (4096, 0, 0)])
def test_select_long(stored, n_select, first, recent):
    """Rows whose scores go through the workspace, and those at the edge of LDS."""
    c = Shape(10, 2, 128, stored, [(0, 4)])
    index, g = _fake_index(c, 3), _gen(4)
    q = _randn(g, 1, c.B, 10, 128).bfloat16()
    _check_select(c, q, index, _select(c, q, index, n_select, first, recent), first, recent)


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("n_select", [4, 130, 255])
def test_select_about_256_and_512_competing_blocks(n_select, ties):
    c = Shape(4, 2, 64, [32 * (n + 3) + 1 for n in (255, 256, 257, 511, 512, 513, 700)], [(0, 4), (0, 2)])
    index, g = _fake_index(c, 65, ties), _gen(66)
    q = _randn(g, c.nl, c.B, 4, 64).bfloat16()
    _check_select(c, q, index, _select(c, q, index, n_select, 1, 2), 1, 2)


@pytest.mark.parametrize("hq,hkv", [(65, 1), (96, 1), (256, 2)])
@pytest.mark.parametrize("stored", [[3200, 700], [64000]])
def test_select_groups_of_many_heads(hq, hkv, stored):
    """More than 64 heads of a KV head, any of which may hold the largest score."""
    c = Shape(hq, hkv, 64, stored, [(0, 4), (1, 4)])
    index, g = _fake_index(c, 61), _gen(62)
    q = _randn(g, c.nl, c.B, hq, 64)
    q = (q * (1 + 3 * torch.rand(q.shape[:-1] + (1,), generator=g, device=DEV))).bfloat16()
    _check_select(c, q, index, _select(c, q, index, 20, 1, 2), 1, 2)


@pytest.mark.parametrize("hq,hkv,readers", [(40, 1, 3), (14, 2, 9), (4, 1, 40), (7, 1, 10)])
def test_select_anchors_of_many_readers(hq, hkv, readers):
    """More than 64 rows read one anchor's index."""
    c = Shape(hq, hkv, 64, [64000, 40000], [(0, 4)] + [(1, 4)] * (readers - 1) + [(0, 2), (1, 2)])
    assert kvk.select_workspace_bytes(c.table, 0, c.nl) > 0
    index, g = _fake_index(c, 63), _gen(64)
    q = _randn(g, c.nl, c.B, hq, 64).bfloat16()
    _check_select(c, q, index, _select(c, q, index, 9, 1, 2), 1, 2)


def test_select_many_rows():
    """Launches of more rows than go through the workspace, at the longest that LDS holds, and of many sequences."""
    c = Shape(4, 4, 64, [32 * 8192] + [32 * 70] * 129, [(0, 4)])
    index, g = _fake_index(c, 5), _gen(6)
    q = _randn(g, 1, c.B, 4, 64).bfloat16()
    assert kvk.select_workspace_bytes(c.table, 0, 1) == 0
    _check_select(c, q, index, _select(c, q, index, 33, 1, 1), 1, 1)


@pytest.mark.parametrize("stored", [[3200], [64000]])
def test_select_ties_go_to_the_lower_block(stored):
    c = Shape(4, 2, 64, stored, [(0, 4)])
    index, g = _fake_index(c, 7, ties=True), _gen(8)
    q = _randn(g, 1, 1, 4, 64).bfloat16()
    for n in (1, 10, 50, 99):
        _check_select(c, q, index, _select(c, q, index, n), 0, 0)
    q.zero_()  # every score is 0
    assert _select(c, q, index, 6, 1, 2)[0, 0].tolist() == [[0, 1, 2, 3, stored[0] // 32 - 2, stored[0] // 32 - 1]] * 2


def test_select_odd_queries_and_blocks():
    """Queries of zeros, with infinities and NaN, tiny and huge; blocks with infinite keys come first."""
    c = Shape(6, 1, 128, [3200] * 6, [(0, 4)])
    index, g = _fake_index(c, 9), _gen(10)
    codes, scales = kvk.index_views(c.table, index, 0)
    for blk in (17, 60):
        codes[:, :, blk] = 0
        scales[:, :, blk, 0], scales[:, :, blk, 1] = 0, INF
    q = _randn(g, 1, 6, 6, 128).bfloat16()
    q[0, 0] = 0
    q[0, 1, 2, 5], q[0, 1, 3, 7] = INF, NAN
    q[0, 2] *= 2.0**-100
    q[0, 3] = (q[0, 3].float() * 1e37).bfloat16()
    q[0, 4, 1:] = 0
    blocks = _select(c, q, index, 4)
    _check_select(c, q, index, blocks, 0, 0)
    # (sequence 3: s_q = 3e37 / 127 times products of about 4e4 overflows too, and equal scores go to the lower block)
    assert all({17, 60} <= set(x) for b, x in enumerate(blocks[0, :, 0].tolist()) if b != 3)


def test_select_finds_planted_keys():
    """Through a real cache: a block that holds the query itself, much larger than the rest, is chosen."""
    g = _gen(11)
    k = _randn(g, 1, 1, 2, 6400, 128)
    q = _randn(g, 1, 1, 4, 128).bfloat16()
    for h, t in ((0, 1000), (1, 5555)):
        k[0, 0, h, t] = 6 * q[0, 0, 2 * h].float()
    k = k.bfloat16()
    for bits in (16, 8, 4, 2):
        c = Cache(4, 2, 128, [6400], [(0, bits)], values=(k, k))
        blocks = _select(c, q, _index_of(c), 3)
        assert 1000 // 32 in blocks[0, 0, 0].tolist() and 5555 // 32 in blocks[0, 0, 1].tolist()


def test_select_per_sequence_plans():
    plans = [[(0, 8), (1, 8), (0, 4)], [(0, 4), (0, 4), (1, 2)], [(0, 16), (1, 16), (1, 16)]]
    c = Shape(6, 2, 64, [3000, 640, 35000], None, plans=plans)
    index, g = _fake_index(c, 12), _gen(13)
    for l in range(3):  # layers that own a cache in some sequence only are filled above where any() does
        for b in range(3):
            if c.anchor(l, b) == l and l:
                codes, scales = kvk.index_views(c.table, index, l, b)
                codes.copy_(torch.randint(-127, 128, codes.shape, generator=g, device=DEV))
                scales.copy_(torch.rand(scales.shape, generator=g, device=DEV))
    q = _randn(g, 3, 3, 6, 64).bfloat16()
    _check_select(c, q, index, _select(c, q, index, 20, 1, 1), 1, 1)


# --------------------------------------------------------------------------------------
# Attention
# --------------------------------------------------------------------------------------


def _attend(c, q, blocks, scale, stream=None):
    out = torch.full(q.shape, NAN, dtype=torch.bfloat16, device=DEV)
    ws = _workspace(kvk.block_workspace_bytes(c.table, 0, c.nl, blocks.shape[3]))
    kvk.block_attention(c.table, 0, c.nl, q, c.stored, blocks, scale, c.arena, out, ws, stream)
    return out


def _check_attend(c, q, blocks, scale, out):
    G, lists = c.hq // c.hkv, blocks.cpu()
    for l in range(c.nl):
        k, v = c.values(l)
        for b in range(c.B):
            bits, full = c.bits(l, b), c.stored[b] // 32
            for h in range(c.hkv):
                blk = lists[l, b, h]
                blk = blk[(blk >= 0) & (blk < full)].long()
                at = (blk[:, None] * 32 + torch.arange(32)).reshape(-1)
                at = torch.cat((at, torch.arange(full * 32, c.stored[b]))).to(DEV)
                K, V = c.token_values(l, b, h, k, v)
                rows = slice(h * G, (h + 1) * G)
                got = out[l, b, rows].to(F64)
                what = f"layer {l} sequence {b} head {h}"
                if at.numel() == 0:
                    assert (got == 0).all(), what
                    continue
                K, V, x = K[at].to(F64), V[at].to(F64), q[l, b, rows].to(F64)
                p = torch.softmax(x @ K.t() * scale, -1)
                o, A = p @ V, p @ V.abs()
                S = (x.abs() @ K.abs().t()).amax(-1, keepdim=True) * abs(scale)
                if bits == 16:
                    e_p, e_v, e_k = 2.0**-8, 0.0, 0.0
                else:
                    e_p = 2.0**-10 if c.scheme == "sym" else 2.0**-11
                    e_v, e_k = (0.0 if c.scheme == "sym" else 2.0**-11), (2.0**-11 if c.scheme == "kivi" else 0.0)
                if c.scheme == "g64":
                    far = (x.abs().sum(-1, keepdim=True) * K.abs().amax()) * abs(scale) * 3
                else:
                    far = 0.0
                ds = ((c.d + 16) * 2.0**-24 + e_k) * S + (c.d + 16) * 2.0**-24 * far + 2.0**-22 * (1 + S)
                small = 2.0**-31 * V.abs().amax(-1).sum() if bits != 16 else 0.0
                tol = 1.02 * (2.0**-8 * o.abs() + (e_p + e_v) * A + 2 * ds * (A + o.abs())) + small + 1e-30
                err = (got - o).abs()
                assert (err <= tol).all(), f"{what}: worst {float((err / tol).nan_to_num(nan=INF).max()):.2f} of the tolerance"


def _lists(g, c, n, kind="rising"):
    """Lists [layers, B, Hkv, n]: rising distinct blocks, then -1; or any."""
    nb = max(1, max(c.stored) // 32)
    full = torch.tensor([s // 32 for s in c.stored], device=DEV)[None, :, None, None]
    if kind == "any":  # in any order, repeated, and some that name no block
        x = torch.randint(-2, nb + 3, (c.nl, c.B, c.hkv, n), generator=g, device=DEV)
        return torch.where(torch.rand(x.shape, generator=g, device=DEV) < 0.1, 2**31 - 1 - x.abs(), x).int()
    r = torch.rand(c.nl, c.B, c.hkv, nb, generator=g, device=DEV)
    r = r.masked_fill(torch.arange(nb, device=DEV) >= full, 2.0).argsort(-1)[..., :n]
    r = torch.where(r < full, r, torch.full_like(r, 1 << 20)).sort(-1)[0]
    r = torch.nn.functional.pad(r, (0, n - r.shape[-1]), value=1 << 20)
    return torch.where(r < 1 << 20, r, torch.full_like(r, -1)).int()


@pytest.mark.parametrize("bits,scheme", [(16, "kivi")] + [(b, s) for b in (8, 4, 2) for s in ("kivi", "sym", "g64")])
@pytest.mark.parametrize("hq,hkv,d,n", [(4, 1, 64, 1), (28, 4, 128, 16), (40, 8, 128, 7), (17, 1, 64, 9), (64, 1, 128, 33), (3, 3, 64, 70)])
def test_block_attention(hq, hkv, d, n, bits, scheme):
    readers = 1 if hq // hkv > 16 else 2
    c = Cache(hq, hkv, d, [0, 1, 31, 32, 33, 1000, 2047, 2048], [(0, bits)] + [(1, 16)] * (readers - 1), scheme)
    g = _gen(21)
    q = _randn(g, c.nl, c.B, hq, d).bfloat16()
    for kind in ("rising", "any"):
        blocks = _lists(g, c, n, kind)
        out = _attend(c, q, blocks, 1.2 / math.sqrt(d))
        _check_attend(c, q, blocks, 1.2 / math.sqrt(d), out)
        assert torch.equal(out, _attend(c, q, blocks, 1.2 / math.sqrt(d)))


@pytest.mark.parametrize("bits,scheme", [(16, "kivi"), (8, "sym"), (4, "kivi"), (2, "g64")])
@pytest.mark.parametrize("hq,hkv,d", [(65, 1, 64), (194, 2, 128)])
def test_block_attention_groups_of_many_heads(hq, hkv, d, bits, scheme):
    c = Cache(hq, hkv, d, [33, 1000], [(0, bits), (1, 16)], scheme)
    g = _gen(23)
    q = _randn(g, c.nl, c.B, hq, d).bfloat16()
    blocks = _lists(g, c, 20, "any")
    _check_attend(c, q, blocks, 1.0 / math.sqrt(d), _attend(c, q, blocks, 1.0 / math.sqrt(d)))


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
@pytest.mark.parametrize("bits,scheme", [(16, "kivi"), (8, "sym"), (4, "kivi"), (2, "g64")])
def test_block_attention_scales(scale, bits, scheme):
    c = Cache(5, 1, 128, [700, 41], [(0, bits)], scheme)
    g = _gen(22)
    q, blocks = _randn(g, 1, 2, 5, 128).bfloat16(), _lists(g, c, 12)
    _check_attend(c, q, blocks, scale, _attend(c, q, blocks, scale))


def test_block_attention_many_entries():
    """Lists longer than a wave looks at in one go, split over workgroups, and with gaps."""
    c = Cache(4, 1, 64, [32 * 700 + 9], [(0, 4)])
    g = _gen(23)
    q = _randn(g, 1, 1, 4, 64).bfloat16()
    for n in (255, 256, 257, 700, 3000):
        blocks = _lists(g, c, n)
        _check_attend(c, q, blocks, 0.1, _attend(c, q, blocks, 0.1))
        gaps = torch.full((1, 1, 1, 4 * n), -1, dtype=torch.int32, device=DEV)
        gaps[..., 3::4] = blocks
        _check_attend(c, q, gaps, 0.1, _attend(c, q, gaps, 0.1))
    c = Cache(4, 4, 64, [32 * 300] * 70, [(0, 2)])  # rows enough: no split, waves look several times
    q, blocks = _randn(g, 1, 70, 4, 64).bfloat16(), _lists(g, c, 300)
    _check_attend(c, q, blocks, 0.1, _attend(c, q, blocks, 0.1))


@pytest.mark.parametrize("bits,scheme", [(16, "kivi"), (8, "kivi"), (4, "sym"), (8, "g64"), (2, "kivi")])
@pytest.mark.parametrize("d,hq,hkv,B", [(128, 5, 1, 256), (128, 34, 2, 70), (64, 6, 2, 150)])
def test_block_attention_eight_waves(bits, scheme, d, hq, hkv, B):
    """Launches of a workgroup per CU and more, whose rows eight waves share."""
    c = Cache(hq, hkv, d, [(37 * b) % 1500 for b in range(B)], [(0, bits)], scheme)
    g = _gen(31)
    q = _randn(g, 1, B, hq, d).bfloat16()
    for n in (17, 40):
        blocks = _lists(g, c, n)
        _check_attend(c, q, blocks, 0.1, _attend(c, q, blocks, 0.1))


@pytest.mark.parametrize("bits,scheme", [(16, "kivi"), (8, "kivi"), (4, "sym")])
def test_every_block_is_the_chunk_attention(bits, scheme):
    c = Cache(10, 2, 128, [1003, 320, 5], [(0, bits), (1, 2)], scheme)
    g = _gen(24)
    q = _randn(g, 2, 3, 10, 128).bfloat16()
    blocks = torch.arange(31, device=DEV, dtype=torch.int32).expand(2, 3, 2, 31).contiguous()
    out = _attend(c, q, blocks, 0.09)
    want = torch.empty(2, 3, 10, 1, 128, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(kvk.chunk_workspace_bytes(c.table, 0, 2, 1), dtype=torch.uint8, device=DEV)
    kvk.chunk_attention(c.table, 0, 2, q.unsqueeze(3).contiguous(), c.stored, None, 0.09, c.arena, want, ws)
    a, b = out.to(F64), want[:, :, :, 0].to(F64)
    assert ((a - b).abs() <= 2.0**-6 * b.abs() + 2.0**-7 * b.abs().amax()).all()
    _check_attend(c, q, blocks, 0.09, out)


def test_block_attention_small_and_large_values():
    """Values and keys far from 1, and scales that differ from block to block (SYMROW)."""
    g = _gen(25)
    n = 32 * 12 + 7
    q = _randn(g, 1, 1, 4, 64).bfloat16()
    for scheme, bits, size in (("kivi", 8, 2.0**-9), ("kivi", 4, 2.0**-12), ("g64", 8, 2.0**-9), ("kivi", 8, 3000.0),
                               ("sym", 8, 2.0**-35), ("sym", 4, 2.0**35), ("sym", 8, 2.0**-12), (None, 16, 2.0**-60), (None, 16, 2.0**60)):
        k, v = _randn(g, 1, 1, 1, n, 64).bfloat16(), (_randn(g, 1, 1, 1, n, 64) * size).bfloat16()
        c = Cache(4, 1, 64, [n], [(0, bits)], scheme or "kivi", values=(k, v))
        blocks = _lists(g, c, 9)
        _check_attend(c, q, blocks, 0.125, _attend(c, q, blocks, 0.125))
    k = _randn(g, 1, 1, 1, n, 64).bfloat16()
    grow = torch.exp2(torch.linspace(-30, 30, n // 32 + 1, device=DEV).round()).repeat_interleave(32)[:n]
    v = (_randn(g, 1, 1, 1, n, 64) * grow[:, None]).bfloat16()
    c = Cache(4, 1, 64, [n], [(0, 8)], "sym", values=(k, v))
    blocks = torch.arange(12, dtype=torch.int32, device=DEV).view(1, 1, 1, 12)
    _check_attend(c, q, blocks, 0.125, _attend(c, q, blocks, 0.125))
    # large keys with small queries, and small keys with large queries
    for up in (40, 100, -40, -100):
        k2, q2 = (k.float() * 2.0**up).bfloat16(), (q.float() * 2.0**-up).bfloat16()
        for scheme, bits in (("sym", 8), ("sym", 2), ("kivi", 16)):
            c = Cache(4, 1, 64, [n], [(0, bits)], scheme, values=(k2, k))
            _check_attend(c, q2, blocks, 0.125, _attend(c, q2, blocks, 0.125))


def test_block_attention_rising_scores():
    """Blocks whose maximum keeps rising, and far apart from the window's."""
    g = _gen(26)
    n = 32 * 40 + 3
    k = _randn(g, 1, 1, 1, n, 64) * torch.linspace(0.01, 9.0, n, device=DEV)[:, None]
    for bits in (16, 8, 2):
        c = Cache(2, 1, 64, [n], [(0, bits)], values=(k.bfloat16(), _randn(g, 1, 1, 1, n, 64).bfloat16()))
        q = (_randn(g, 1, 1, 2, 64) * 2).bfloat16()
        for order in (range(40), range(39, -1, -1)):
            blocks = torch.tensor(list(order), dtype=torch.int32, device=DEV).view(1, 1, 1, 40)
            _check_attend(c, q, blocks, 0.125, _attend(c, q, blocks, 0.125))


def test_block_attention_infinite_values():
    """At seen tokens infinite and NaN values count by channel; in blocks left out and in stale slots of the window
    they reach no row; infinite scores."""
    g = _gen(27)
    n = 32 * 6 + 5
    k, v = _randn(g, 1, 1, 1, n + 20, 64).bfloat16(), _randn(g, 1, 1, 1, n + 20, 64).bfloat16()
    v[0, 0, 0, 40, 3], v[0, 0, 0, 70, 5], v[0, 0, 0, n - 1, 9] = INF, NAN, -INF
    v[0, 0, 0, 100, 7] = k[0, 0, 0, 101, 7] = NAN  # block 3 is left out
    v[0, 0, 0, n + 2, :] = NAN                     # slots past the stored tokens
    k[0, 0, 0, n + 3, :] = INF
    for bits in (16, 8):
        kb, vb = k.clone(), v.clone()
        if bits == 8:  # the window alone holds such values
            kb[0, 0, 0, :192], vb[0, 0, 0, :192] = 0.5, 0.25
        c = Cache(4, 1, 64, [n + 20], [(0, bits)], values=(kb, vb))
        c.stored = [n]
        q = _randn(g, 1, 1, 4, 64).bfloat16()
        blocks = torch.tensor([0, 1, 2, 4, 5], dtype=torch.int32, device=DEV).view(1, 1, 1, 5)
        out = _attend(c, q, blocks, 0.125).float()
        want = torch.ones(64, dtype=torch.bool, device=DEV)
        want[9] = False
        assert (out[0, 0, :, 9] == -INF).all()
        if bits == 16:
            want[[3, 5]] = False
            assert (out[0, 0, :, 3] == INF).all() and torch.isnan(out[0, 0, :, 5]).all()
        assert torch.isfinite(out[0, 0][:, want]).all()
    # rows whose seen scores are all -inf, or NaN in one
    q = torch.ones(1, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    k = torch.zeros(1, 1, 1, 64, 64, dtype=torch.bfloat16, device=DEV)
    k[0, 0, 0, :32, 0], k[0, 0, 0, 40, 1] = -INF, NAN
    c = Cache(2, 1, 64, [64], [(0, 16)], values=(k, torch.ones_like(k)))
    for blk in (0, 1):
        assert torch.isnan(_attend(c, q, torch.tensor([[[[blk]]]], dtype=torch.int32, device=DEV), 1.0)).all()
    k[0, 0, 0, 40, 1] = 0
    c = Cache(2, 1, 64, [64], [(0, 16)], values=(k, torch.ones_like(k)))
    assert (_attend(c, q, torch.tensor([[[[0, 1]]]], dtype=torch.int32, device=DEV), 1.0) == 1).all()


def test_block_attention_per_sequence_plans_and_many_sequences():
    plans = [[(0, (16, 8, 4, 2)[b % 4]), (1, 16) if b % 3 == 0 else (0, 4), (0, 2)] for b in range(7)]
    c = Cache(6, 2, 64, [100, 32, 31, 64, 200, 0, 96], None, plans=plans)
    g = _gen(28)
    q, blocks = _randn(g, 3, 7, 6, 64).bfloat16(), _lists(g, c, 4)
    _check_attend(c, q, blocks, 0.15, _attend(c, q, blocks, 0.15))
    c = Cache(2, 1, 64, [20 + 3 * i for i in range(150)], [(0, 4), (0, 8)])
    q, blocks = _randn(g, 2, 150, 2, 64).bfloat16(), _lists(g, c, 5)
    _check_attend(c, q, blocks, 0.15, _attend(c, q, blocks, 0.15))


def test_block_attention_past_4_gib():
    """Streams past 2^32 bytes of the arena, blocks late in a long stream."""
    B, n = 9, 131072
    c = Shape(4, 4, 128, [n] * B, [(0, 16), (0, 16)], cap=n + 40)
    assert c.table.arena_bytes > 2**32 + 2**27
    c.arena, c.scheme = torch.zeros(c.table.arena_bytes, dtype=torch.uint8, device=DEV), "kivi"
    g = _gen(29)
    k, v = (_randn(g, 2, B, 4, 40, 128).bfloat16() for _ in range(2))
    kvk.append_chunk(c.table, 0, 2, k, v, n, None, c.arena)  # the last block and a window of 8 tokens
    c.stored = [n + 40] * B
    q = _randn(g, 2, B, 4, 128).bfloat16()
    blocks = torch.full((2, B, 4, 1), n // 32, dtype=torch.int32, device=DEV)
    out = _attend(c, q, blocks, 0.1)
    index = _index_of(c, [n] * B)  # the last block's summaries, of every stream
    for l in range(2):
        codes, scales = kvk.index_views(c.table, index, l)
        want, ws = _summary(k[l, :, :, :32].float())
        assert torch.equal(codes[:, :, n // 32], want) and torch.equal(scales[:, :, n // 32], ws)
    p = torch.softmax((q.to(F64).unsqueeze(3) * k.to(F64)).sum(-1) * 0.1, -1)
    want = (p[..., None] * v.to(F64)).sum(3)
    assert ((out.to(F64) - want).abs() <= 2.0**-6 * (p[..., None] * v.to(F64).abs()).sum(3) + 1e-3).all()


def test_select_past_4_gib():
    """The last sequence's part of the last anchor of an index of 4.4 GB."""
    n = 524288
    c = Shape(8, 8, 128, [0] * 63 + [n], [(0, 4), (0, 4)], cap=n)
    assert kvk.index_bytes(c.table) > 2**32 + 2**26
    index, g = torch.zeros(kvk.index_bytes(c.table), dtype=torch.uint8, device=DEV), _gen(32)
    codes, scales = kvk.index_views(c.table, index, 1)
    codes[63] = torch.randint(-127, 128, codes[63].shape, generator=g, device=DEV)
    scales[63] = torch.rand(scales[63].shape, generator=g, device=DEV)
    q = _randn(g, 2, 64, 8, 128).bfloat16()
    blocks = _select(c, q, index, 100, 1, 2)
    for h in range(8):
        assert blocks[1, 63, h].tolist() == _chosen(q[1, 63, h:h + 1], codes[63, h], scales[63, h], n // 32, 100, 1, 2)
    assert (blocks[:, :63] == -1).all()


def test_captured_index_and_long_choice():
    """The index's launch and the choice in two launches, captured and replayed on other contents."""
    c = Cache(4, 2, 64, [300, 64], [(0, 8), (0, 4)])
    long = Shape(8, 2, 64, [64000, 40000], [(0, 4), (1, 4)])
    index, g = torch.zeros(kvk.index_bytes(c.table), dtype=torch.uint8, device=DEV), _gen(33)
    far, q = _fake_index(long, 34), _randn(g, 2, 2, 8, 64).bfloat16()
    blocks = torch.zeros(2, 2, 2, 50, dtype=torch.int32, device=DEV)
    ws = _workspace(kvk.select_workspace_bytes(long.table, 0, 2))
    assert ws is not None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvk.index_blocks(c.table, 0, 2, c.stored, c.arena, index)
        kvk.select_blocks(long.table, 0, 2, q, long.stored, far, blocks, 1, 1, ws)
    for i in range(3):
        k, v = (_randn(g, 2, 2, 2, 300, 64).bfloat16() for _ in range(2))
        kvk.append_chunk(c.table, 0, 2, k, v, 0, c.stored, c.arena)
        q.copy_(_randn(g, *q.shape))
        c.k, c.v = k, v
        index.fill_(0x55)
        graph.replay()
        torch.cuda.synchronize()
        _check_index(c, index)
        _check_select(long, q, far, blocks, 1, 1)


def test_streams_graphs_and_shared_workspaces():
    """Choice and attention on another stream, captured into graphs that share workspaces, replayed with new
    queries between eager calls."""
    c = Cache(10, 2, 128, [2000, 1500], [(0, 4)])
    index, g = _index_of(c), _gen(30)
    q = _randn(g, 1, 2, 10, 128).bfloat16()
    blocks, out = torch.zeros(1, 2, 2, 8, dtype=torch.int32, device=DEV), torch.zeros_like(q)
    ws = _workspace(max(kvk.block_workspace_bytes(c.table, 0, 1, 8), 256))
    ws2 = _workspace(kvk.select_workspace_bytes(c.table, 0, 1))

    def step(stream=None):
        kvk.select_blocks(c.table, 0, 1, q, c.stored, index, blocks, 1, 1, ws2, stream)
        kvk.block_attention(c.table, 0, 1, q, c.stored, blocks, 0.09, c.arena, out, ws, stream)

    def check():
        torch.cuda.synchronize()
        _check_select(c, q, index, blocks, 1, 1)
        _check_attend(c, q, blocks, 0.09, out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    check()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        graphs.append(graph)
    for i in range(4):
        q.copy_(_randn(g, *q.shape))
        graphs[i % 2].replay()
        check()
        q.copy_(_randn(g, *q.shape))
        step()
        check()
