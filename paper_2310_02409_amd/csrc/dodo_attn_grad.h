// What the kernels of dodo_nugget_attention_grad share: arguments, the ranges of an entry, tiles of keys.
#pragma once
#include "dodo_common.h"

namespace dodo {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kGradWaves = 4;
constexpr int kGradThreads = kGradWaves * kWave;

struct GradParams {
  const void *Q, *Kn, *Vn, *Kl, *Vl, *dO, *O;
  const float* lse;
  float *lse2, *neg_d;  // workspace [H][Sq]: log-sum-exp in base 2, -D = -dO . O
  const int32_t *cu_q, *cu_nuggets, *cu_local;
  const int32_t *nug_len, *loc_len;  // null: ranges end where the next begins
  int shared;                        // != 0: entries may share rows, so that key tiles run over all rows instead of a sequence's
  int32_t B, H, H_kv, max_q, max_k, max_local;
  int64_t Sq, Kt, Sm;
  int64_t nug_tok_stride, nug_head_stride, loc_tok_stride, loc_head_stride;  // elements
  float scale, scale_log2e;
  void *dQ, *dKn, *dVn, *dKl, *dVl;
  hipStream_t stream;
};

// Rows of entry e: queries, nuggets, local rows.
struct Entry {
  int q0, q_b, k0, k_b, l0, m_b;
};
__device__ __forceinline__ Entry entry_of(const GradParams& p, int e) {
  const int32_t *k_end_p = p.nug_len != nullptr ? p.nug_len + e : p.cu_nuggets + e + 1, *l_end_p = p.loc_len != nullptr ? p.loc_len + e : p.cu_local + e + 1;
  Entry s;  // (six loads at once)
  s.q0 = p.cu_q[e];
  const int q_end = p.cu_q[e + 1];
  s.k0 = p.cu_nuggets[e];
  const int k_end = *k_end_p;
  s.l0 = p.cu_local[e];
  const int l_end = *l_end_p;
  s.q_b = q_end - s.q0;
  s.k_b = p.nug_len != nullptr ? k_end : k_end - s.k0;
  s.m_b = p.loc_len != nullptr ? l_end : l_end - s.l0;
  return s;
}

// `rows` consecutive key rows of a K/V head from `first` on, in the nugget cache or among the local rows, and the entries
// that may see them.
struct KeyTile {
  const void *K, *V;
  void *dK, *dV;
  int64_t first, tok_stride, head_stride;
  int rows, kvh, entry0, entry1;
  bool local;
};
// Tile `item` of a grid of (n_nug_tiles + n_loc_tiles) tiles of `size` rows per K/V head (and sequence, unless rows are shared);
// rows <= 0: nothing there.
__device__ __forceinline__ KeyTile key_tile(const GradParams& p, unsigned item, int n_nug_tiles, int n_loc_tiles, int size) {
  KeyTile t;
  const unsigned tiles = n_nug_tiles + n_loc_tiles;
  int tile = item % tiles;
  const unsigned rest = item / tiles;
  t.kvh = rest % p.H_kv;
  const int b = rest / p.H_kv;
  t.local = tile >= n_nug_tiles;
  if (t.local) tile -= n_nug_tiles;
  int64_t begin = 0, end = t.local ? p.Sm : p.Kt;
  if (!p.shared) {
    const Entry s = entry_of(p, b);
    begin = t.local ? s.l0 : s.k0;
    end = begin + (t.local ? s.m_b : s.k_b);
  }
  t.first = begin + static_cast<int64_t>(tile) * size;
  t.rows = static_cast<int>(min(static_cast<int64_t>(size), end - t.first));
  t.entry0 = p.shared ? 0 : b;
  t.entry1 = p.shared ? p.B : b + 1;
  t.K = t.local ? p.Kl : p.Kn;
  t.V = t.local ? p.Vl : p.Vn;
  t.dK = t.local ? p.dKl : p.dKn;
  t.dV = t.local ? p.dVl : p.dVn;
  t.tok_stride = t.local ? p.loc_tok_stride : p.nug_tok_stride;
  t.head_stride = t.local ? p.loc_head_stride : p.nug_head_stride;
  return t;
}

// Which query rows of an entry see a tile's keys: key j of the entry (of len from row key0 on) is seen by the query rows from
// max(0, j - lag) on, up to q_b.
struct SeenBy {
  int q0, q_b, key0, len, lag, first_row;
  bool any;
  __device__ __forceinline__ int least(int j, bool ok) const { return ok && j >= 0 && j < len ? max(0, j - lag) : 0x7fffffff; }
};
__device__ __forceinline__ SeenBy seen_by(const GradParams& p, const KeyTile& t, int e, int size) {
  const Entry s = entry_of(p, e);
  SeenBy r;
  r.q0 = s.q0;
  r.q_b = s.q_b;
  r.key0 = t.local ? s.l0 : s.k0;
  r.len = t.local ? s.m_b : s.k_b;
  r.lag = t.local ? s.m_b - s.q_b : 0x7fffffff;  // (a nugget: all rows)
  const int64_t j = t.first - r.key0;           // of the tile's first row
  r.any = s.q_b > 0 && j < r.len && j + min(t.rows, size) > 0;
  r.first_row = t.local ? static_cast<int>(max(static_cast<int64_t>(0), max(j, static_cast<int64_t>(0)) - r.lag)) : 0;
  return r;
}

// bf16, on the bf16 matrix instructions.
int launch_grad_mfma(const GradParams& p, int32_t d_h);

// Four fp32 numbers to elements i to i + 3 (16 or 8 bytes, aligned to as much).
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
template <int DTYPE>
__device__ __forceinline__ void store4(void* p, int64_t i, float a, float b, float c, float d) {
  if (DTYPE == DODO_DTYPE_F32)
    *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = make_float4(a, b, c, d);
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = __builtin_bit_cast(uint2, __builtin_convertvector((floatx4){a, b, c, d}, bf16x4));
}

}  // namespace dodo
