"""The long-context operators together, as a serving loop runs them: rotary positions, the chunk append, the block
index, the choice, the attention over chosen blocks, and eviction by block into another slot."""
import math

import pytest
import torch

from gpu_common import DEV
from paper_2609_37988_amd import kvk

pytestmark = pytest.mark.gpu
F64 = torch.float64


@pytest.mark.parametrize("bits,scheme", [(16, kvk.KIVI32), (8, kvk.SYMROW), (4, kvk.KIVI32), (2, kvk.GROUP64)])
def test_a_serving_loop(bits, scheme):
    B, hq, hkv, d, cap, nl = 3, 10, 2, 128, 1200, 2
    scale, n_select = 1 / math.sqrt(d), 6
    plan = [(0, bits), (1, 16)]
    t = kvk.layer_table(kvk.make_dims(kvk.GQA, nl, hq, hkv, d, qscheme=scheme, batch=B, max_tokens=cap), kvk.make_plan(plan))
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    arena = torch.zeros(t.arena_bytes, dtype=torch.uint8, device=DEV)
    index = torch.zeros(kvk.index_bytes(t), dtype=torch.uint8, device=DEV)
    rot = kvk.rotary(d, kvk.rotary_frequencies(d, 1e6))
    freq = torch.tensor(kvk.rotary_frequencies(d, 1e6), dtype=F64, device=DEV)
    blocks = torch.zeros(nl, B, hkv, n_select, dtype=torch.int32, device=DEV)
    ws = torch.empty(max(kvk.block_workspace_bytes(t, 0, nl, n_select), 256), dtype=torch.uint8, device=DEV)
    lens = [1000, 700, 33]
    x = torch.randn(B, hkv, max(lens), d, generator=g, device=DEV).bfloat16()
    v = torch.randn(B, hkv, max(lens), d, generator=g, device=DEV).bfloat16()

    # prefill of ragged prompts
    pos = torch.arange(max(lens), dtype=torch.int32, device=DEV)
    k = torch.empty_like(x)
    kvk.rotate(rot, pos, [x], [k])
    angle = pos.to(F64)[:, None] * freq
    a, b = x[..., :64].to(F64), x[..., 64:].to(F64)
    want = torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1)
    assert ((k.to(F64) - want).abs() <= 2.0**-8 * want.abs() + 2.0**-20 * (a.abs() + b.abs()).repeat(1, 1, 1, 2)).all()
    kvk.append_chunk(t, 0, 1, k[None], v[None], 0, lens, arena)
    kvk.index_blocks(t, 0, nl, lens, arena, index)

    # decode steps: a token each
    stored = list(lens)
    for step in range(40):
        q = torch.randn(nl, B, hq, 1, d, generator=g, device=DEV).bfloat16()
        kn = torch.randn(1, B, hkv, 1, d, generator=g, device=DEV).bfloat16()
        vn = torch.randn(1, B, hkv, 1, d, generator=g, device=DEV).bfloat16()
        at = torch.tensor(stored, dtype=torch.int32, device=DEV).view(B, 1)
        kvk.rotate(rot, at, [q.view(nl * B, hq, 1, d), kn.view(B, hkv, 1, d).repeat(nl, 1, 1, 1)])
        kvk.rotate(rot, at, [kn.view(B, hkv, 1, d)])
        before = list(stored)
        kvk.append_chunk(t, 0, 1, kn, vn, before, None, arena)
        stored = [n + 1 for n in stored]
        kvk.index_blocks(t, 0, nl, stored, arena, index, before)
    q1 = q.view(nl, B, hq, d)
    kvk.select_blocks(t, 0, nl, q1, stored, index, blocks, 1, 1)
    out = torch.empty_like(q1)
    kvk.block_attention(t, 0, nl, q1, stored, blocks, scale, arena, out, ws)

    # against the stored values, from the lists
    n = max(stored)
    K, V = (torch.empty(B, hkv, n, d, device=DEV) for _ in range(2))
    kvk.debug_dequantize(t, 0, n, arena, K, V)
    for bq in range(B):
        full = stored[bq] // 32
        for h in range(hkv):
            for l in range(nl):
                lst = [i for i in blocks[l, bq, h].tolist() if i >= 0]
                assert len(lst) == min(n_select, full) and lst == sorted(set(lst)) and lst[-1] == full - 1 and lst[0] == 0
    # the longest sequence, whose window the dequantiser returned
    for l in range(nl):
        for h in range(hkv):
            lst = blocks[l, 0, h].tolist()
            at = torch.cat([torch.arange(32 * i, 32 * i + 32) for i in lst] + [torch.arange(stored[0] // 32 * 32, stored[0])]).to(DEV)
            rows = slice(h * 5, h * 5 + 5)
            p = torch.softmax(q1[l, 0, rows].to(F64) @ K[0, h, at].to(F64).t() * scale, -1)
            o, size = p @ V[0, h, at].to(F64), p @ V[0, h, at].to(F64).abs()
            assert ((out[l, 0, rows].to(F64) - o).abs() <= 2.0**-8 * o.abs() + 2.0**-6 * size).all()

    # eviction by block: layer 0's choice goes to a slot of another arena, and attention over all of it there is the
    # attention over the chosen blocks here
    t2 = kvk.layer_table(kvk.make_dims(kvk.GQA, nl, hq, hkv, d, qscheme=scheme, batch=2, max_tokens=320), kvk.make_plan(plan))
    arena2 = torch.zeros(t2.arena_bytes, dtype=torch.uint8, device=DEV)
    kvk.copy_sequences(t, arena, t2, arena2, [0], [1], [stored[0]], blocks)
    kept = 32 * n_select + stored[0] % 32
    ws2 = torch.empty(kvk.chunk_workspace_bytes(t2, 0, 1, 1), dtype=torch.uint8, device=DEV)
    q2 = q1[:1, :1].expand(1, 2, hq, d).reshape(1, 2, hq, 1, d).contiguous()
    out2 = torch.zeros_like(q2)
    kvk.chunk_attention(t2, 0, 1, q2, [0, kept], [0, 1], scale, arena2, out2, ws2)
    x, y = out[0, 0].to(F64), out2[0, 1, :, 0].to(F64)
    assert ((x - y).abs() <= 2.0**-6 * y.abs() + 2.0**-7 * y.abs().amax()).all()
    index2 = torch.zeros(kvk.index_bytes(t2), dtype=torch.uint8, device=DEV)
    kvk.index_blocks(t2, 0, nl, [0, kept], arena2, index2)
    c1, c2 = kvk.index_views(t, index, 0)[0], kvk.index_views(t2, index2, 0)[0]
    for h in range(hkv):
        assert torch.equal(c2[1, h, :n_select], c1[0, h, blocks[0, 0, h].long()])
