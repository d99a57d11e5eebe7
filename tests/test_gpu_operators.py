"""The multi-token operators on the GPU against 64-bit references: prompt attention, the weight
positions collect, the keep list of the heaviest, the chunk append and the chunk attention.

Tolerances count roundings.  A value rounded to bf16 is off by at most 2^-8 of it, to fp16 by
2^-11, to fp32 by 2^-24.  With A = sum_t p_t |v_t| (p the softmax), an output o = sum_t p_t v_t
is off by at most
  2^-8 |o|        its own rounding,
  e_p A           probabilities rounded to bf16 (e_p = 2^-8) or fp16 (2^-11),
  e_v A           values rounded to fp16 (e_v = 2^-11, quantised layers only),
  2 d (A + |o|)   scores off by at most d: fp32 sums, d_h + 16 additions of products whose
                  absolute sum is S, d = (d_h + 16) 2^-24 S, and keys rounded to fp16, 2^-11 S,
and 2 % more for products of these terms.
"""
import math

import numpy as np
import pytest
import torch

from oracle import cache as OC
from oracle import plan as OP
from paper_2609_37988_amd import kvk
from gpu_common import DEV

pytestmark = pytest.mark.gpu
F64 = torch.float64
NAN = float("nan")


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _attend(q, k, v, scale, last, k_err=0.0, p_err=2.0**-8, v_err=0.0):
    """64-bit attention of rows q [H, m, d] over k, v [n, d] where row i sees tokens 0..last[i];
    the outputs, log-sum-exps, their tolerances, and the largest absolute score sum per row."""
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    hidden = torch.arange(k.shape[0], device=k.device) > last[:, None]
    s = (q @ k.t()) * scale
    s = torch.where(hidden, torch.full_like(s, -math.inf), s)
    lse = torch.logsumexp(s, -1)
    p = torch.where(hidden, torch.zeros_like(s), torch.exp(s - lse[..., None]))
    o, a = p @ v, p @ v.abs()
    big = torch.where(hidden, torch.zeros_like(s), q.abs() @ k.abs().t() * abs(scale)).amax(-1)
    d_s = ((q.shape[-1] + 16) * 2.0**-24 + k_err) * big
    tol = 1.02 * (2.0**-8 * o.abs() + (p_err + v_err) * a + 2 * d_s[..., None] * (a + o.abs())) + 1e-30
    return o, lse, tol, d_s + 2.0**-21 * (1 + lse.abs())


def _check(got, want, tol, what):
    err = (got.to(F64) - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / tol).nan_to_num(nan=math.inf).max()):.2f} of the tolerance"


# --------------------------------------------------------------------------------------
# Prompt attention and the collected weights
# --------------------------------------------------------------------------------------


def _prompt_inputs(seed, lens, hq, hkv, d, layout):
    g = _gen(seed)
    if layout == "padded":
        n = max(lens) + 3
        return [_randn(g, len(lens), h, n, d).bfloat16() for h in (hq, hkv, hkv)]
    t = sum(lens)
    if layout == "fused":  # views of one projection, with a gap between its rows
        x = _randn(g, t, hq + 2 * hkv + 1, d).bfloat16()
        return [x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:hq + 2 * hkv]]
    return [_randn(g, t, h, d).bfloat16() for h in (hq, hkv, hkv)]


def _seq(x, lens, s):
    """[heads, length, d] of sequence s."""
    if x.dim() == 4:
        return x[s, :, :lens[s]]
    first = sum(lens[:s])
    return x[first:first + lens[s]].transpose(0, 1)


def _run_prompt(q, k, v, lens, scale):
    out = torch.full(q.shape, NAN, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((q.shape[1] * sum(lens),), NAN, dtype=torch.float32, device=DEV)
    kvk.prompt_attention(q, k, v, lens, scale, out, lse)
    return out, lse


def _check_prompt(q, k, v, lens, scale, out, lse):
    hq, grp, at = q.shape[1], q.shape[1] // k.shape[1], 0
    for s, n in enumerate(lens):
        qs, ks, vs, os = (_seq(x, lens, s) for x in (q, k, v, out))
        last = torch.arange(n, device=DEV)
        for j in range(ks.shape[0] if n else 0):
            rows = slice(j * grp, (j + 1) * grp)
            o, l, tol, ltol = _attend(qs[rows], ks[j], vs[j], scale, last)
            _check(os[rows], o, tol, f"sequence {s} KV head {j}")
            _check(lse[at + j * grp * n:at + (j + 1) * grp * n].view(grp, n), l, ltol, f"lse of sequence {s}")
        at += hq * n


PROMPTS = [
    ([1], 1, 1, 64), ([1], 4, 2, 128), ([2, 1, 3], 5, 1, 128), ([31, 32, 33], 4, 4, 64), ([63, 64, 65, 0, 127], 2, 1, 128),
    ([128, 129, 255], 6, 2, 64), ([300, 1, 17], 7, 1, 128), ([513], 3, 3, 128), ([700, 257], 8, 2, 64), ([1500], 10, 2, 128),
]


@pytest.mark.parametrize("layout", ["packed", "fused", "padded"])
@pytest.mark.parametrize("lens,hq,hkv,d", PROMPTS)
def test_prompt_attention(lens, hq, hkv, d, layout):
    q, k, v = _prompt_inputs(1, lens, hq, hkv, d, layout)
    scale = 1.3 / math.sqrt(d)
    out, lse = _run_prompt(q, k, v, lens, scale)
    _check_prompt(q, k, v, lens, scale, out, lse)
    if layout == "padded":  # the padding rows stay as they were
        for s, n in enumerate(lens):
            assert torch.isnan(out[s, :, n:]).all()


@pytest.mark.parametrize("scale", [-0.2, 0.0, 2.0])
def test_prompt_attention_scales(scale):
    lens = [70, 200]
    q, k, v = _prompt_inputs(2, lens, 4, 2, 128, "packed")
    out, lse = _run_prompt(q, k, v, lens, scale)
    _check_prompt(q, k, v, lens, scale, out, lse)


def test_prompt_attention_growing_scores():
    """Rows whose maximum keeps rising, and large negative starts."""
    lens = [400]
    q, k, v = _prompt_inputs(3, lens, 2, 1, 64, "packed")
    k = (k.float() * torch.linspace(0.01, 12.0, 400, device=DEV)[:, None, None]).bfloat16()
    out, lse = _run_prompt(q, k, v, lens, 0.125)
    _check_prompt(q, k, v, lens, 0.125, out, lse)


def test_prompt_attention_hides_later_infinities():
    """Infinities and NaN in later tokens' keys and values do not reach a row; the rows that see
    them get them."""
    lens = [200, 90]
    for d in (64, 128):
        q, k, v = _prompt_inputs(4, lens, 2, 1, d, "packed")
        ref, _ = _run_prompt(q, k, v, lens, 0.1)
        v2, k2 = v.clone(), k.clone()
        v2[150, 0, 5], v2[151, 0, 6], v2[152, 0, 7] = math.inf, -math.inf, NAN
        v2[160, 0, 5] = -math.inf
        k2[190] = NAN
        v2[200 + 89, 0, :] = NAN  # the last token of the second sequence
        out, lse = _run_prompt(q, k2, v2, lens, 0.1)
        assert torch.equal(out[:150], ref[:150])
        assert torch.equal(out[200:200 + 89], ref[200:200 + 89])
        clean = [c for c in range(d) if c not in (5, 6, 7)]
        assert torch.equal(out[150:190][:, :, clean], ref[150:190][:, :, clean])
        assert (out[150:160, :, 5] == math.inf).all() and torch.isnan(out[160:190, :, 5]).all()
        assert (out[151:190, :, 6] == -math.inf).all() and torch.isnan(out[152:190, :, 7]).all()
        assert torch.isnan(out[190:200]).all() and torch.isnan(out[200 + 89]).all()
        assert torch.isfinite(lse.view(-1)[:2 * 200].view(2, 200)[:, :190]).all()


def test_prompt_attention_rows_of_minus_infinity():
    """Keys that give -inf scores carry no mass; a row that sees nothing else is NaN."""
    lens = [100]
    q, k, v = _prompt_inputs(5, lens, 1, 1, 64, "packed")
    q[:, :, 0] = 1.0
    k[:70, :, 0] = -math.inf
    out, lse = _run_prompt(q, k, v, lens, 0.1)
    assert torch.isnan(out[:70]).all() and (lse[:70] == -math.inf).all()
    o, l, tol, ltol = _attend(q[70:, 0][None], k[70:, 0], v[70:, 0], 0.1, torch.arange(30, device=DEV))
    _check(out[70:, 0][None], o, tol, "rows after the first finite score")
    _check(lse[70:][None], l, ltol, "lse")


def test_prompt_attention_beyond_32_bits():
    """Rows whose byte offsets pass 2^32."""
    d, n = 64, 70
    wide = torch.zeros(n * (1 << 25) + 4096, dtype=torch.bfloat16, device=DEV)  # 4.7 GB
    st = (1 << 25, d, 1)
    g = _gen(6)
    q = _randn(g, n, 2, d).bfloat16()
    k, v = torch.as_strided(wide, (n, 1, d), st, 0), torch.as_strided(wide, (n, 1, d), st, 1024)
    k.copy_(_randn(g, n, 1, d)), v.copy_(_randn(g, n, 1, d))
    out, lse = _run_prompt(q, k, v, [n], 0.2)
    _check_prompt(q, k.contiguous(), v.contiguous(), [n], 0.2, out, lse)


@pytest.mark.parametrize("layout", ["packed", "padded"])
@pytest.mark.parametrize("lens,hq,hkv,d", PROMPTS)
def test_attention_weight(lens, hq, hkv, d, layout):
    q, k, v = _prompt_inputs(7, lens, hq, hkv, d, layout)
    scale, grp = 0.9 / math.sqrt(d), hq // hkv
    _, lse = _run_prompt(q, k, v, lens, scale)
    need = kvk.attention_weight_workspace_bytes(hq, hkv, d, lens)
    ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device=DEV)
    w = torch.full((hkv * sum(lens),), NAN, dtype=torch.float32, device=DEV)
    kvk.attention_weight(q, k, lse, lens, scale, w, ws)
    again = torch.full_like(w, NAN)
    kvk.attention_weight(q, k, lse, lens, scale, again, ws)
    assert torch.equal(w, again)
    at = 0
    for s, n in enumerate(lens):
        qs, ks = _seq(q, lens, s).to(F64), _seq(k, lens, s).to(F64)
        for j in range(hkv if n else 0):
            l = lse[at * hq + j * grp * n:at * hq + (j + 1) * grp * n].view(grp, n).to(F64)
            x = qs[j * grp:(j + 1) * grp] @ ks[j].t() * scale
            big = (qs[j * grp:(j + 1) * grp].abs() @ ks[j].abs().t() * scale).max()
            p = torch.tril(torch.exp(x - l[..., None]))
            want = p.sum((0, 1))
            # a probability is off by its exponent's rounding: the score's sum, two products and the
            # difference; their sum by one rounding for each addition a lane makes (n / 32) and the joins
            rel = (d + 16) * 2.0**-24 * big + 2.0**-21 * (1 + l.abs().max()) + (n / 32 + 8 + grp) * 2.0**-24
            _check(w[at * hkv + j * n:at * hkv + (j + 1) * n], want, rel * want + 1e-30, f"sequence {s} head {j}")
        at += n


def test_attention_weight_rows_without_mass_and_nan():
    """A row with the log-sum-exp -inf adds nothing; a NaN row spoils the tokens it sees only."""
    lens, d = [150, 60], 64
    q, k, v = _prompt_inputs(20, lens, 2, 1, d, "packed")
    q[:, :, 0] = 1.0
    k[:40, :, 0] = -math.inf  # rows 0..39 have no finite score
    q[100, 0] = NAN           # one row of one head
    _, lse = _run_prompt(q, k, v, lens, 0.1)
    assert (lse[:40] == -math.inf).all() and torch.isnan(lse[100])
    ws = torch.empty(kvk.attention_weight_workspace_bytes(2, 1, d, lens), dtype=torch.uint8, device=DEV)
    w = torch.full((210,), 7.0, dtype=torch.float32, device=DEV)
    kvk.attention_weight(q, k, lse, lens, 0.1, w, ws)
    assert torch.isnan(w[:101]).all()  # tokens that row 100 sees
    assert torch.isfinite(w[101:]).all()
    q[100, 0] = q[99, 0]
    _, lse = _run_prompt(q, k, v, lens, 0.1)
    kvk.attention_weight(q, k, lse, lens, 0.1, w, ws)
    assert (w[:40] == 0).all() and torch.isfinite(w).all()
    assert abs(float(w[:150].sum()) / (2 * 110) - 1) < 1e-5  # 110 rows of each head carry mass


# --------------------------------------------------------------------------------------
# The keep list
# --------------------------------------------------------------------------------------


def _keep_ref(w, keep, recent):
    """Per row: the heaviest, by a stable sort (NaN last), then the recent window; sorted."""
    n = w.shape[-1]
    rows = []
    for r in w.reshape(-1, n).astype(np.float64):
        key = np.where(np.isnan(r), -math.inf, r)[:n - recent]
        order = np.lexsort((np.arange(n - recent), np.isnan(r[:n - recent]), -key))[:keep - recent]
        rows.append(np.sort(np.concatenate([order, np.arange(n - recent, n)])))
    return np.stack(rows).astype(np.int32)


@pytest.mark.parametrize("n,keep,recent", [(1, 1, 0), (1, 1, 1), (5, 3, 3), (64, 64, 0), (65, 1, 0), (1000, 250, 64), (1024, 1000, 0),
                                           (4097, 33, 32), (16384, 8192, 1), (16400, 8200, 16), (16385, 1, 0), (16385, 16385, 0),
                                           (33000, 32999, 5), (40001, 20000, 333), (131072, 65536, 4096)])
@pytest.mark.parametrize("kind", ["spread", "equal", "ties", "signs"])
def test_keep_heaviest(n, keep, recent, kind):
    rng = np.random.default_rng(n + keep)
    shape = (2, 3, n)
    w = {"spread": np.exp(3 * rng.standard_normal(shape)), "equal": np.full(shape, 0.25),
         "ties": rng.integers(0, 5, shape) / 4.0, "signs": rng.standard_normal(shape) * 10.0 ** rng.integers(-40, 30, shape)}[kind]
    w = w.astype(np.float32)
    if kind == "signs":
        w[rng.random(shape) < 0.1] = np.nan
        w[rng.random(shape) < 0.1] = -0.0
        w[rng.random(shape) < 0.1] = 0.0
        w[rng.random(shape) < 0.02] = np.inf
        w[rng.random(shape) < 0.02] = -np.inf
    dims = kvk.make_dims(kvk.GQA, 1, 3, 3, 64, batch=2, max_tokens=n, keep_tokens=keep)
    t = kvk.layer_table(dims, kvk.make_plan([(0, 8)]))
    out = torch.full((2, 3, keep), -1, dtype=torch.int32, device=DEV)
    kvk.keep_heaviest(t, torch.from_numpy(w).to(DEV), n, recent, out)
    assert np.array_equal(out.cpu().numpy().reshape(6, keep), _keep_ref(w, keep, recent))


def test_keep_heaviest_on_a_stream():
    """A long list on a side stream, whose workspace the call brings itself, and in one of exactly
    the size asked for."""
    n, keep, recent = 50000, 700, 32
    dims = kvk.make_dims(kvk.GQA, 1, 2, 2, 64, batch=2, max_tokens=n, keep_tokens=keep)
    t = kvk.layer_table(dims, kvk.make_plan([(0, 8)]))
    w = torch.rand(2, 2, n, device=DEV)
    want = _keep_ref(w.cpu().numpy(), keep, recent)
    outs = [torch.full((2, 2, keep), -1, dtype=torch.int32, device=DEV) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kvk.keep_heaviest(t, w, n, recent, outs[0], stream=side)
    side.synchronize()
    ws = torch.full((kvk.keep_workspace_bytes(t, n),), 0xFF, dtype=torch.uint8, device=DEV)
    kvk.keep_heaviest(t, w, n, recent, outs[1], ws)
    for out in outs:
        assert np.array_equal(out.cpu().numpy().reshape(4, keep), want)


def test_keep_heaviest_mla():
    dims = kvk.make_dims(kvk.MLA, 1, 8, 1, 128, latent_dim=256, rope_dim=64, nope_dim=128, v_dim=128, batch=3,
                         max_tokens=500, keep_tokens=100)
    t = kvk.layer_table(dims, kvk.make_plan([(0, 8, 256)]))
    w = torch.rand(3, 500, device=DEV)
    out = torch.empty((3, 100), dtype=torch.int32, device=DEV)
    kvk.keep_heaviest(t, w, 500, 10, out)
    assert np.array_equal(out.cpu().numpy(), _keep_ref(w.cpu().numpy(), 100, 10))


# --------------------------------------------------------------------------------------
# The chunk append
# --------------------------------------------------------------------------------------

SCHEMES = [kvk.KIVI32, kvk.SYMROW, kvk.GROUP64]


class Streams:
    """A table with its arena, and its inputs: K, V [layers, B, Hkv, cap, d]."""

    def __init__(self, plan, hq, hkv, d, B, cap, scheme, seed=0, dtype=torch.bfloat16, plans=None):
        L = len(plans[0] if plans else plan)
        self.dims = kvk.make_dims(kvk.GQA, L, hq, hkv, d, qscheme=scheme, batch=B, max_tokens=cap)
        self.t = (kvk.layer_table_batched(self.dims, [kvk.make_plan(p) for p in plans]) if plans
                  else kvk.layer_table(self.dims, kvk.make_plan(plan)))
        self.L, self.hq, self.hkv, self.d, self.B, self.cap = L, hq, hkv, d, B, cap
        self.arena = self.new_arena()
        g = _gen(seed)
        self.k = (_randn(g, L, B, hkv, cap, d) * torch.exp(_randn(g, hkv, 1, d))).to(dtype)
        self.v = _randn(g, L, B, hkv, cap, d).to(dtype)
        self.od = OP.Dims(OP.GQA, L, hq, hkv, d, qscheme=scheme, batch=B, max_tokens=cap)
        self.plans = plans or [plan] * B

    def new_arena(self):
        return torch.full((kvk.table_query(self.t).arena_bytes,), 0xFF, dtype=torch.uint8, device=DEV)

    def append(self, start, new, l0=0, l1=None, arena=None):
        """Tokens start[b] .. start[b] + new[b] of every sequence, in one call."""
        l1 = self.L if l1 is None else l1
        m = max(max(new), 1)
        shape = (l1 - l0, self.B, self.hkv, m, self.d)
        k, v = (torch.full(shape, NAN, dtype=self.k.dtype, device=DEV) for _ in range(2))
        for b in range(self.B):
            for to, x in ((k, self.k), (v, self.v)):
                to[:, b, :, :new[b]] = x[l0:l1, b, :, start[b]:start[b] + new[b]]
        kvk.append_chunk(self.t, l0, l1, k, v, start, new, self.arena if arena is None else arena)

    def streams(self, arena, stored):
        """The meaningful bytes of every stream with stored[b] tokens."""
        out = []
        host = arena.cpu().numpy()
        for b in range(self.B):
            info = kvk.table_sequence_query(self.t, b) if self.t.plans else kvk.table_query(self.t)
            for l in range(self.L):
                inherit, bits = self.plans[b][l][:2]
                if inherit:
                    continue
                for h in range(self.hkv):
                    at = info.layer_offset[l] + ((0 if self.t.plans else b * self.hkv) + h) * info.stream_bytes[l]
                    blocks, tail = OC.layout.split_stream(self.od, bits, host[at:at + info.stream_bytes[l]], stored[b])
                    # of the tail block the filled slots: zero the others
                    out.append((blocks.reshape(-1).copy(), _tail_tokens(tail, self.d, stored[b] % 32)))
        return out

    def values(self, l, b, h, n):
        """K, V of a stream as stored, in 64 bits, from the oracle's quantiser."""
        a = max(x for x in range(l + 1) if not self.plans[b][x][0])
        bits = self.plans[b][a][1]
        k, v = (x[a, b, h, :n].bfloat16().float().cpu().numpy() for x in (self.k, self.v))
        K, V = OC.dequant_stream(self.od, bits, OC.compress_stream(self.od, bits, k, v), n)
        return torch.from_numpy(np.asarray(K)).to(DEV), torch.from_numpy(np.asarray(V)).to(DEV), bits


def _tail_tokens(tail, d, n):
    """The bf16 values of the first n tokens of a tail block, K then V, by the layout's slot maps."""
    x = tail[:128 * d].view(np.uint16)
    t = np.arange(n)
    c = np.arange(d)
    T, C = np.meshgrid(t, c, indexing="ij")

    def share(P, lam, o):
        return np.where(P > 16, 1024 * (o // 16) + 16 * lam + o % 16, lam * P + o)

    kb = 32 * d * (T // 16) + share(d // 2, 16 * (C % 32 // 8) + T % 16, 16 * (C // 32) + 2 * (C % 8))
    vb = 64 * d + share(d, 16 * (T % 16 // 4) + C % 16, 16 * (C // 16) + 2 * (4 * (T // 16) + T % 4))
    return np.concatenate([x[kb.reshape(-1) // 2], x[vb.reshape(-1) // 2]])


def _same(a, b):
    assert len(a) == len(b)
    for i, (x, y) in enumerate(zip(a, b)):
        assert np.array_equal(x[0], y[0]), f"stream {i}: full blocks differ"
        assert np.array_equal(x[1], y[1]), f"stream {i}: tail differs"


PLAN = [(0, 16), (0, 8), (1, 8), (0, 4), (0, 2)]


@pytest.mark.parametrize("scheme", SCHEMES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_chunk_equals_append_token(scheme, d, dtype):
    """Chunks of ragged lengths leave the streams as single appends do."""
    c = Streams(PLAN, 4, 2, d, 4, 160, scheme, seed=8, dtype=dtype)
    one = c.new_arena()
    # token by token; every sequence gets the same tokens, the chunks stop at its own length
    steps = [[0, 5, 31, 32], [3, 1, 33, 0], [64, 60, 0, 95], [29, 0, 1, 1], [1, 2, 95, 31]]
    stored = [0] * 4
    for new in steps:
        c.append(stored, new)
        stored = [s + n for s, n in zip(stored, new)]
    seen = {}
    for n in range(max(stored)):
        kvk.append_token(c.t, 0, c.L, c.k[:, :, :, n].contiguous(), c.v[:, :, :, n].contiguous(), n, one)
        for b in range(4):
            if stored[b] == n + 1:
                seen[b] = c.streams(one, [n + 1] * 4)
    got = c.streams(c.arena, stored)
    per = len(got) // 4
    for b in range(4):
        _same(got[per * b:per * (b + 1)], seen[b][per * b:per * (b + 1)])


def test_append_chunk_per_sequence_plans_and_ranges():
    """Per-sequence plans, a sub-range of layers, and sequences with nothing new."""
    plans = [[(0, 4), (1, 4), (0, 8)], [(0, 16), (0, 2), (1, 2)], [(0, 2), (0, 2), (0, 2)]]
    c = Streams(None, 4, 2, 128, 3, 100, kvk.KIVI32, seed=9, plans=plans)
    one = c.new_arena()
    stored = [0, 0, 0]
    for new in ([40, 0, 7], [33, 64, 25], [0, 1, 0]):
        for l in range(3):
            c.append(stored, new, l, l + 1)
        stored = [s + n for s, n in zip(stored, new)]
    snap = {}
    for n in range(max(stored)):
        kvk.append_token(c.t, 0, 3, c.k[:, :, :, n].contiguous(), c.v[:, :, :, n].contiguous(), n, one)
        for b in range(3):
            if stored[b] == n + 1:
                snap[b] = c.streams(one, [n + 1] * 3)
    got = c.streams(c.arena, stored)
    counts = [sum(not a[0] for a in p) * 2 for p in plans]
    at = 0
    for b in range(3):
        _same(got[at:at + counts[b]], snap[b][at:at + counts[b]])
        at += counts[b]


def test_append_chunk_writes_nothing_else():
    """Bytes of sequences without new tokens, of later blocks and of other layers stay."""
    c = Streams([(0, 4), (0, 4)], 2, 1, 128, 2, 128, kvk.KIVI32, seed=10)
    c.append([0, 0], [40, 70])
    before = c.arena.clone()
    c.append([40, 70], [30, 0], 0, 1)
    info = kvk.table_query(c.t)
    sb, bb = info.stream_bytes[0], 8 * 128 * 5
    changed = (c.arena != before).nonzero().flatten().cpu().numpy()
    assert changed.size and changed.min() >= bb and changed.max() < sb  # sequence 0, from its second block on
    assert not ((changed >= 2 * bb) & (changed < 4 * bb)).any()          # its blocks past the full ones


# --------------------------------------------------------------------------------------
# The chunk attention
# --------------------------------------------------------------------------------------


def _run_chunk(c, l0, l1, stored, new, scale, seed=0, q=None):
    m = max(new)
    g = _gen(100 + seed)
    if q is None:
        q = _randn(g, l1 - l0, c.B, c.hq, m, c.d).bfloat16()
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((kvk.chunk_workspace_bytes(c.t, l0, l1, m),), 0xFF, dtype=torch.uint8, device=DEV)
    kvk.chunk_attention(c.t, l0, l1, q, stored, new, scale, c.arena, out, ws)
    return q, out


def _check_chunk(c, l0, l1, stored, new, scale, q, out):
    grp = c.hq // c.hkv
    for b in range(c.B):
        n, m = stored[b], new[b]
        assert (out[:, b, :, m:] == 7.0).all(), "rows past the new tokens"
        last = torch.arange(n - m, n, device=DEV)
        for l in range(l0, l1) if m else []:
            for h in range(c.hkv):
                K, V, bits = c.values(l, b, h, n)
                err = (0.0, 2.0**-8, 0.0) if bits == 16 else (2.0**-11, 2.0**-11, 2.0**-11)
                o, _, tol, _ = _attend(q[l - l0, b, h * grp:(h + 1) * grp, :m], K, V, scale, last, *err)
                _check(out[l - l0, b, h * grp:(h + 1) * grp, :m], o, tol, f"layer {l} sequence {b} head {h}")


@pytest.mark.parametrize("scheme", SCHEMES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
def test_chunk_attention(bits, scheme, d):
    """Ragged lengths around the blocks' and tiles' edges; one, two and three row groups."""
    stored = [1, 31, 32, 33, 128, 129, 300, 517]
    c = Streams([(0, bits)], 5, 1, d, 8, 520, scheme, seed=11)
    c.append([0] * 8, stored)
    for new in ([1] * 8, [1, 3, 2, 1, 6, 4, 5, 2], [1, 10, 11, 0, 9, 12, 7, 8], [1, 31, 20, 33, 60, 100, 0, 40]):
        q, out = _run_chunk(c, 0, 1, stored, new, 0.8 / math.sqrt(d))
        _check_chunk(c, 0, 1, stored, new, 0.8 / math.sqrt(d), q, out)


@pytest.mark.parametrize("bits", [16, 4])
def test_chunk_attention_long(bits):
    """Contexts split over workgroups, next to short ones; a prompt's chunks of many rows."""
    c = Streams([(0, bits)], 4, 1, 128, 3, 6000, kvk.KIVI32, seed=12)
    stored = [5999, 40, 3333]
    c.append([0] * 3, stored)
    for new in ([1, 1, 1], [4, 2, 13], [200, 40, 33], [1000, 0, 5]):
        q, out = _run_chunk(c, 0, 1, stored, new, 0.09)
        _check_chunk(c, 0, 1, stored, new, 0.09, q, out)


@pytest.mark.parametrize("scheme", SCHEMES)
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
@pytest.mark.parametrize("d", [64, 128])
def test_chunk_attention_splits(bits, scheme, d):
    """Split contexts in every row shape, ten query heads to a KV head."""
    c = Streams([(0, bits)], 20, 2, d, 2, 2900, scheme, seed=20)
    stored = [2881, 1600]
    c.append([0] * 2, stored)
    for new in ([1, 2], [4, 6], [9, 33]):
        q, out = _run_chunk(c, 0, 1, stored, new, 0.7 / math.sqrt(d))
        _check_chunk(c, 0, 1, stored, new, 0.7 / math.sqrt(d), q, out)


def test_chunk_many_sequences_and_layers():
    """More sequences than one attention launch takes, more anchors than one append launch."""
    B, L = 203, 60
    rng = np.random.default_rng(21)
    plan = [(0, (4, 8, 2, 16)[l % 4]) for l in range(L)]
    c = Streams(plan, 2, 1, 64, B, 80, kvk.KIVI32, seed=21)
    first = [int(x) for x in rng.integers(0, 41, B)]
    new = [int(x) for x in rng.integers(0, 40, B)]
    stored = [a + b for a, b in zip(first, new)]
    c.append([0] * B, first)
    c.append(first, new)
    q, out = _run_chunk(c, 56, 58, stored, new, 0.1)
    some = [0, 1, 95, 96, 97, 150, 191, 192, 202]
    for b in some:
        n, m = stored[b], new[b]
        assert (out[:, b, :, m:] == 7.0).all()
        for l in (56, 57) if m else ():
            K, V, _ = c.values(l, b, 0, n)
            o, _, tol, _ = _attend(q[l - 56, b, :, :m], K, V, 0.1, torch.arange(n - m, n, device=DEV), 2.0**-11, 2.0**-11, 2.0**-11)
            _check(out[l - 56, b, :, :m], o, tol, f"layer {l} sequence {b}")


def test_append_chunk_many_equal_sequences():
    """Sequences of one length beyond the limit of ragged ones."""
    B = 300
    c = Streams([(0, 4)], 1, 1, 64, B, 40, kvk.KIVI32, seed=22)
    c.append([0] * B, [33] * B)
    one = c.new_arena()
    for n in range(33):
        kvk.append_token(c.t, 0, 1, c.k[:, :, :, n].contiguous(), c.v[:, :, :, n].contiguous(), n, one)
    _same(c.streams(c.arena, [33] * B), c.streams(one, [33] * B))


def test_chunk_few_rows_in_a_large_workspace():
    """A call whose rows are few beside n_chunk fits the workspace asked for n_chunk; rows that
    are not new, and a call without new rows, leave the output alone."""
    c = Streams([(0, 8), (1, 8)], 4, 1, 128, 3, 9000, kvk.KIVI32, seed=23)
    stored = [8999, 5000, 64]
    c.append([0] * 3, stored)
    m = 300
    g = _gen(24)
    q = _randn(g, 2, 3, 4, m, 128).bfloat16()
    ws = torch.empty(kvk.chunk_workspace_bytes(c.t, 0, 2, m), dtype=torch.uint8, device=DEV)
    for new in ([1, 0, 1], [3, 5, 8], [20, 1, 30], [0, 0, 0]):
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        kvk.chunk_attention(c.t, 0, 2, q, stored, new, 0.09, c.arena, out, ws)
        _check_chunk(c, 0, 2, stored, new, 0.09, q, out)


def test_chunk_beyond_32_bits():
    """Caches, inputs and arena offsets past 4 GiB (16-bit layers hold the bf16 inputs)."""
    B, hkv, n, d = 17, 8, 131000, 128
    dims = kvk.make_dims(kvk.GQA, 1, 16, hkv, d, batch=B, max_tokens=131072)
    t = kvk.layer_table(dims, kvk.make_plan([(0, 16)]))
    arena = torch.empty(kvk.table_query(t).arena_bytes, dtype=torch.uint8, device=DEV)
    assert arena.numel() > 2**32 and B * hkv * n * d > 2**31
    k, v = (torch.zeros((1, B, hkv, n, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    g = _gen(25)
    for x in (k, v):
        x[0, -1, -1] = _randn(g, n, d).bfloat16()
        x[0, 0, 0] = _randn(g, n, d).bfloat16()
    kvk.append_chunk(t, 0, 1, k, v, 0, None, arena)
    q = _randn(g, 1, B, 16, 3, d).bfloat16()
    out = torch.empty_like(q)
    ws = torch.empty(kvk.chunk_workspace_bytes(t, 0, 1, 3), dtype=torch.uint8, device=DEV)
    kvk.chunk_attention(t, 0, 1, q, n, None, 0.1, arena, out, ws)
    last = torch.arange(n - 3, n, device=DEV)
    for b, h in ((0, 0), (B - 1, hkv - 1)):
        o, _, tol, _ = _attend(q[0, b, 2 * h:2 * h + 2], k[0, b, h], v[0, b, h], 0.1, last, 0.0, 2.0**-8, 0.0)
        _check(out[0, b, 2 * h:2 * h + 2], o, tol, f"sequence {b}")
    assert (out[0, 1:-1] == 0).all()


@pytest.mark.parametrize("scale", [-0.1, 0.0])
def test_chunk_attention_scales(scale):
    c = Streams([(0, 8)], 2, 1, 64, 1, 100, kvk.KIVI32, seed=13)
    c.append([0], [77])
    q, out = _run_chunk(c, 0, 1, [77], [9], scale)
    _check_chunk(c, 0, 1, [77], [9], scale, q, out)


def test_chunk_attention_shared_anchors_and_ranges():
    """Layers sharing an anchor, ranges that begin at an inheriting layer, plans per sequence."""
    plan = [(0, 8), (1, 8), (1, 8), (0, 2), (1, 2)]
    c = Streams(plan, 6, 2, 64, 2, 200, kvk.SYMROW, seed=14)
    c.append([0, 0], [150, 99])
    for l0, l1 in ((0, 5), (1, 2), (1, 4), (4, 5)):
        q, out = _run_chunk(c, l0, l1, [150, 99], [5, 7], 0.1)
        _check_chunk(c, l0, l1, [150, 99], [5, 7], 0.1, q, out)
    plans = [[(0, 4), (1, 4), (0, 8)], [(0, 16), (0, 2), (1, 2)], [(0, 4), (1, 4), (1, 8)], [(0, 4), (1, 4), (0, 8)]]
    c = Streams(None, 4, 2, 128, 4, 130, kvk.KIVI32, seed=15, plans=plans)
    stored, new = [130, 64, 33, 70], [3, 40, 0, 6]
    c.append([0] * 4, stored)
    for l0, l1 in ((0, 3), (1, 3), (2, 3)):
        q, out = _run_chunk(c, l0, l1, stored, new, 0.1)
        _check_chunk(c, l0, l1, stored, new, 0.1, q, out)


def test_chunk_attention_hides_later_infinities():
    """16-bit layers hold infinities and NaN as they are: later tokens' do not reach a row."""
    for d in (64, 128):
        c = Streams([(0, 16)], 3, 1, d, 1, 200, kvk.KIVI32, seed=16)
        c.append([0], [170])
        q, ref = _run_chunk(c, 0, 1, [170], [40], 0.1)
        c.v[0, 0, 0, 150, 3], c.v[0, 0, 0, 165, 4] = math.inf, NAN
        c.k[0, 0, 0, 168] = NAN
        c.append([0], [170])
        _, out = _run_chunk(c, 0, 1, [170], [40], 0.1, q=q)
        out, ref = out[0, 0], ref[0, 0]  # row i is token 130 + i
        keep = [x for x in range(d) if x not in (3, 4)]
        assert torch.equal(out[:, :38][:, :, keep], ref[:, :38][:, :, keep])
        assert torch.equal(out[:, :20, 3], ref[:, :20, 3]) and (out[:, 20:38, 3] == math.inf).all()
        assert torch.equal(out[:, :35, 4], ref[:, :35, 4]) and torch.isnan(out[:, 35:38, 4]).all()
        assert torch.isnan(out[:, 38:]).all()


@pytest.mark.parametrize("scheme", SCHEMES)
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
@pytest.mark.parametrize("d", [64, 128])
def test_chunk_attention_wide(bits, scheme, d):
    """Many rows (sixty-four query heads to a KV head), the widest workgroups."""
    c = Streams([(0, bits)], 64, 1, d, 3, 400, scheme, seed=26)
    stored = [390, 33, 96]
    c.append([0] * 3, stored)
    new = [41, 33, 7]
    q, out = _run_chunk(c, 0, 1, stored, new, 0.9 / math.sqrt(d))
    _check_chunk(c, 0, 1, stored, new, 0.9 / math.sqrt(d), q, out)


@pytest.mark.parametrize("d", [64, 128])
def test_chunk_attention_wide_hides_later_infinities(d):
    """As above in the widest workgroups: in full blocks, in the window, and past its tokens."""
    hq, n, m = 64, 170, 40
    c = Streams([(0, 16)], hq, 1, d, 1, 200, kvk.KIVI32, seed=27)
    c.append([0], [n])
    q, ref = _run_chunk(c, 0, 1, [n], [m], 0.1)
    c.v[0, 0, 0, 150, 3], c.v[0, 0, 0, 165, 4] = math.inf, NAN
    c.v[0, 0, 0, n:] = NAN
    c.append([0], [192])  # (the slots past token 170 of the window hold NaN, then block 5 is full)
    c.append([0], [n])
    _, out = _run_chunk(c, 0, 1, [n], [m], 0.1, q=q)
    out, ref = out[0, 0], ref[0, 0]  # row i is token 130 + i
    keep = [x for x in range(d) if x not in (3, 4)]
    assert torch.equal(out[:, :, keep], ref[:, :, keep])
    assert torch.equal(out[:, :20, 3], ref[:, :20, 3]) and (out[:, 20:, 3] == math.inf).all()
    assert torch.equal(out[:, :35, 4], ref[:, :35, 4]) and torch.isnan(out[:, 35:, 4]).all()


def test_chunk_attention_one_token_matches_decode():
    """With one new token the chunk attention is the decode step."""
    c = Streams([(0, 4), (1, 4), (0, 16)], 10, 2, 128, 2, 400, kvk.KIVI32, seed=17)
    c.append([0, 0], [333, 333])
    q, out = _run_chunk(c, 0, 3, [333, 333], [1, 1], 0.09)
    ws = torch.empty(kvk.workspace_bytes(c.t, 0, 3), dtype=torch.uint8, device=DEV)
    dec = torch.empty((3, 2, 10, 128), dtype=torch.float32, device=DEV)
    kvk.decode_attention(c.t, 0, 3, q[:, :, :, 0].contiguous(), 333, 0.09, c.arena, dec, ws)
    # the decode's own 2e-3 of the largest output, and the bf16 rounding of this one's
    tol = 2e-3 * dec.abs().amax() + (2.0**-8 + 2.0**-8) * dec.abs()
    assert ((out[:, :, :, 0].float() - dec).abs() <= tol).all()


# --------------------------------------------------------------------------------------
# Together, on other streams, and captured
# --------------------------------------------------------------------------------------


def test_prefill_with_eviction_by_collected_weight():
    """A prompt's attention, the weights it gives, the keep list, the compressed write, and a
    draft on top: the path of one layer."""
    B, hq, hkv, d, n, keep = 2, 4, 2, 64, 300, 150
    g = _gen(18)
    q, k, v = (_randn(g, B, h, n, d).bfloat16() for h in (hq, hkv, hkv))
    lens, scale = [n] * B, 0.2
    out, lse = _run_prompt(q, k, v, lens, scale)
    _check_prompt(q, k, v, lens, scale, out, lse)
    w = torch.empty((B, hkv, n), dtype=torch.float32, device=DEV)
    ws = torch.empty(kvk.attention_weight_workspace_bytes(hq, hkv, d, lens), dtype=torch.uint8, device=DEV)
    kvk.attention_weight(q, k, lse, lens, scale, w, ws)
    # every row's probabilities sum to one
    assert abs(float(w.sum()) / (B * hq * n) - 1) < 1e-5
    dims = kvk.make_dims(kvk.GQA, 1, hq, hkv, d, batch=B, max_tokens=n, keep_tokens=keep)
    t = kvk.layer_table(dims, kvk.make_plan([(0, 8)]))
    idx = torch.empty((B, hkv, keep), dtype=torch.int32, device=DEV)
    kvk.keep_heaviest(t, w, n, 32, idx)
    assert np.array_equal(idx.cpu().numpy().reshape(-1, keep), _keep_ref(w.cpu().numpy(), keep, 32))
    arena = torch.zeros(kvk.table_query(t).arena_bytes, dtype=torch.uint8, device=DEV)
    kvk.compress_layer(t, 0, k, v, n, idx, arena)
    K, V = (torch.empty((B, hkv, keep, d), dtype=torch.float32, device=DEV) for _ in range(2))
    kvk.debug_dequantize(t, 0, keep, arena, K, V)
    q2 = _randn(g, 1, B, hq, 1, d).bfloat16()
    o2 = torch.empty_like(q2)
    ws2 = torch.empty(kvk.chunk_workspace_bytes(t, 0, 1, 1), dtype=torch.uint8, device=DEV)
    kvk.chunk_attention(t, 0, 1, q2, keep, None, scale, arena, o2, ws2)
    for b in range(B):
        for h in range(hkv):
            o, _, tol, _ = _attend(q2[0, b, 2 * h:2 * h + 2], K[b, h], V[b, h], scale, torch.tensor([keep - 1], device=DEV),
                                   2.0**-11, 2.0**-11, 2.0**-11)
            _check(o2[0, b, 2 * h:2 * h + 2], o, tol, "draft after eviction")


def test_operators_on_a_stream_and_captured():
    """The whole path on a side stream, then captured into a graph and replayed with new inputs,
    with eager work between the replays."""
    B, hq, hkv, d, n = 2, 4, 2, 128, 200
    lens, scale = [n, n], 0.1
    g = _gen(19)
    c = Streams([(0, 4)], hq, hkv, d, B, n + 8, kvk.KIVI32, seed=19)
    q, k, v = (_randn(g, B, h, n, d).bfloat16() for h in (hq, hkv, hkv))
    dims = kvk.make_dims(kvk.GQA, 1, hq, hkv, d, batch=B, max_tokens=n, keep_tokens=64)
    te = kvk.layer_table(dims, kvk.make_plan([(0, 8)]))
    bufs = dict(out=torch.empty_like(q), lse=torch.empty(B * hq * n, device=DEV), w=torch.empty((B, hkv, n), device=DEV),
                ws=torch.empty(kvk.attention_weight_workspace_bytes(hq, hkv, d, lens), dtype=torch.uint8, device=DEV),
                idx=torch.empty((B, hkv, 64), dtype=torch.int32, device=DEV),
                cq=torch.empty((1, B, hq, n, d), dtype=torch.bfloat16, device=DEV),
                co=torch.empty((1, B, hq, n, d), dtype=torch.bfloat16, device=DEV),
                cws=torch.empty(kvk.chunk_workspace_bytes(c.t, 0, 1, n), dtype=torch.uint8, device=DEV))

    def path(stream):
        kvk.prompt_attention(q, k, v, lens, scale, bufs["out"], bufs["lse"], stream=stream)
        kvk.attention_weight(q, k, bufs["lse"], lens, scale, bufs["w"], bufs["ws"], stream=stream)
        kvk.keep_heaviest(te, bufs["w"], n, 16, bufs["idx"], stream=stream)
        kvk.append_chunk(c.t, 0, 1, k[None], v[None], 0, None, c.arena, stream=stream)
        kvk.chunk_attention(c.t, 0, 1, q[None], n, None, scale, c.arena, bufs["co"], bufs["cws"], stream=stream)

    names = ("out", "lse", "w", "idx", "co")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    path(side)
    side.synchronize()
    first = {x: bufs[x].clone() for x in names}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        path(torch.cuda.current_stream())
    for r in range(3):
        q.copy_(_randn(g, *q.shape)), k.copy_(_randn(g, *k.shape)), v.copy_(_randn(g, *v.shape))
        path(None)
        torch.cuda.synchronize()
        eager = {x: bufs[x].clone() for x in names}
        for x in names:
            bufs[x].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x in names:
            assert torch.equal(bufs[x], eager[x]), (r, x)
            assert not torch.equal(bufs[x], first[x]), (r, x)
