// What the kernels over stored 32-token blocks share: the layers and sequences of a launch.
#pragma once

#include <algorithm>
#include <type_traits>

#include "kvk_internal.h"

namespace kvk {

constexpr int kGroupSeqs = 64;  // sequences of a launch
constexpr int kReaderRows = 64; // query rows of layers that are read for together

// Layers of one launch: each an entry of its own, or (of Layers::readers) the layers that read one anchor together.
struct GroupLayer {
  int64_t region, index;  // byte offsets in the arena and in the index of the anchor's part
  int32_t stream_bytes;
  uint8_t layer, count;   // the first layer (of the call's) and how many
  uint8_t row0;           // layers in the entries before
  uint8_t bits;
};
// Sequences of one launch: where the region of a sequence starts is the layer's plus its own, plus
// `mult` sequences' streams (one plan: a layer's sequences follow each other; per-sequence plans:
// the sequence's own table lies at `region`, its index at `index`, and a launch has one layer and bit-width).
struct GroupSeq {
  int64_t region, index;
  int32_t mult;
  int32_t seq;           // of the batch
  int32_t first, stored; // blocks to leave out at the front, tokens stored
};
struct Group {
  int32_t n_layers, n_seqs, Hkv;
  int32_t n_rows;  // layers in all entries
  GroupLayer layers[KVK_MAX_LAYERS];
  GroupSeq seqs[kGroupSeqs];
#ifdef __HIPCC__
  __host__ __device__
#endif
  int64_t stream_at(const GroupLayer& l, const GroupSeq& s, int kvh) const {
    return l.region + s.region + ((int64_t)s.mult * Hkv + kvh) * l.stream_bytes;
  }
};
static_assert(sizeof(Group) <= 3600, "leaves room for a kernel's own arguments");

// The index of a one-plan table's anchor, `blocks` = streams * nb_cap summaries: [blocks][2 D] 8-bit
// codes, then [blocks][2] fp32 scales, each part 256-byte aligned; the anchors in layer order.
inline int64_t index_codes_bytes(const kvk_table* t) {
  return round256((int64_t)t->d.batch * t->d.n_kv_heads * t->nb_cap * 2 * t->d.head_dim);
}
inline int64_t index_anchor_bytes(const kvk_table* t) {
  return index_codes_bytes(t) + round256((int64_t)t->d.batch * t->d.n_kv_heads * t->nb_cap * 8);
}
inline int64_t index_offset(const kvk_table* t, int anchor) {
  return t->anchors_before[anchor] * index_anchor_bytes(t);
}
inline int64_t index_total(const kvk_table* t) { return t->info.n_anchors * index_anchor_bytes(t); }

enum class Layers {
  anchors,  // of the range
  each,     // of the range, with its anchor's part
  readers,  // of the range that read one anchor: one entry for at most kReaderRows rows (per-sequence plans: each)
};

// Calls f(bits, group) for the layers of [l0, l1) of a GQA table, all bit-widths of a one-plan table in one group
// (f's bits is then 0) unless by_bits.  of(b, seq) fills first and stored of sequence b and says whether it
// takes part.
template <class Of, class F>
kvk_status for_groups(const kvk_table* t, int l0, int l1, Layers which, bool by_bits, Group& g, Of of, F f) {
  g.Hkv = t->d.n_kv_heads;
  const int together = std::max(1, kReaderRows / (t->d.n_q_heads / t->d.n_kv_heads));
  constexpr int kBits[4] = {16, 8, 4, 2};
  if (t->seq.empty()) {
    for (int k = 0; k < (by_bits ? 4 : 1); ++k) {
      const int bits = by_bits ? kBits[k] : 0;
      g.n_layers = 0;
      int rows = 0;
      for (int l = l0; l < l1;) {
        const int anc = t->info.anchor_of[l];
        const int n = which == Layers::readers ? std::min(together, std::min<int>(t->next_anchor[anc], l1) - l) : 1;
        if ((!by_bits || t->bits[anc] == bits) && (which != Layers::anchors || anc == l)) {
          g.layers[g.n_layers++] = GroupLayer{t->info.layer_offset[anc], index_offset(t, anc), (int32_t)t->info.stream_bytes[anc],
                                              (uint8_t)(l - l0), (uint8_t)n, (uint8_t)rows, (uint8_t)t->bits[anc]};
          rows += n;
        }
        l += n;
      }
      if (g.n_layers == 0) continue;
      g.n_rows = rows;
      g.n_seqs = 0;
      for (int b = 0; b < t->d.batch; ++b) {
        GroupSeq& s = g.seqs[g.n_seqs];
        s = GroupSeq{0, 0, b, b, 0, 0};
        if (of(b, s)) ++g.n_seqs;
        if (g.n_seqs == kGroupSeqs || (b == t->d.batch - 1 && g.n_seqs)) {
          if (kvk_status st = f(bits, g)) return st;
          g.n_seqs = 0;
        }
      }
    }
    return KVK_OK;
  }
  for (int l = l0; l < l1; ++l)
    for (const int bits : kBits) {
      g.n_layers = g.n_rows = 1;
      g.n_seqs = 0;
      int64_t index = 0;
      for (int b = 0; b < t->d.batch; ++b) {
        const kvk_table* x = t->seq[b];
        const int anc = x->info.anchor_of[l];
        const int64_t at = index;
        index += round256(index_total(x));
        if (x->bits[anc] == bits && (which != Layers::anchors || anc == l)) {
          GroupSeq& s = g.seqs[g.n_seqs];
          s = GroupSeq{t->seq_base[b] + x->info.layer_offset[anc], at + index_offset(x, anc), 0, b, 0, 0};
          if (of(b, s)) {
            // (streams of one bit-width have one size)
            g.layers[0] = GroupLayer{0, 0, (int32_t)x->info.stream_bytes[anc], (uint8_t)(l - l0), 1, 0, (uint8_t)bits};
            ++g.n_seqs;
          }
        }
        if (g.n_seqs == kGroupSeqs || (b == t->d.batch - 1 && g.n_seqs)) {
          if (kvk_status st = f(bits, g)) return st;
          g.n_seqs = 0;
        }
      }
    }
  return KVK_OK;
}

}  // namespace kvk
