// dodo_gather_nuggets_grad: the gradient of the sub-selection (Eq. 5 of the Dodo paper).  The gather copies token idx[p] to
// row p of the cache, so the gradient of a token's row is the sum of the cache rows whose index it is: one row for a nugget, none
// for the other tokens (nine in ten at the usual compression), more where a list holds an index twice.
//
// A pass over memory that mostly writes zeros.  Without accumulation a workgroup writes the rows of kTokens consecutive tokens, of
// K and of V: one search in the sequence's ascending list for the first of them, then the list is read on from
// there, one entry per lane, and a ballot tells each token how many rows are its own.  So no row is written twice and
// there are no atomics, and a list with repeated indices gives the same sum every time.  8 sequences of 4096 tokens at 10x, 32 heads of
// 128, bf16: 114 us, 5.2 TB/s of the bytes that have to move (a fill reaches 6.9, a copy 4.9); a workgroup per token and tensor took 155.  With accumulation only
// the nuggets' tokens are touched: one workgroup per cache row and tensor, of which the first of a run of equal indices adds the run; 4 sequences
// of 3500 to 4096 tokens at 10x, 32 heads of 128, bf16: 22 us, 3.3 TB/s (each row waits for a round of lookups and then for two reads).
#include "dodo_lists.h"

namespace dodo {
namespace {

constexpr int kTokens = 2;      // consecutive tokens per workgroup
constexpr int kMaxThreads = 256;

template <int DTYPE>
__device__ __forceinline__ uint4 add16(const uint4& a, const uint4& b) {
  if (DTYPE == DODO_DTYPE_F32)
    return make_uint4(__float_as_uint(__uint_as_float(a.x) + __uint_as_float(b.x)), __float_as_uint(__uint_as_float(a.y) + __uint_as_float(b.y)),
                      __float_as_uint(__uint_as_float(a.z) + __uint_as_float(b.z)), __float_as_uint(__uint_as_float(a.w) + __uint_as_float(b.w)));
  return make_uint4(pack_bf16(bf16_lo(a.x) + bf16_lo(b.x), bf16_hi(a.x) + bf16_hi(b.x)),
                    pack_bf16(bf16_lo(a.y) + bf16_lo(b.y), bf16_hi(a.y) + bf16_hi(b.y)),
                    pack_bf16(bf16_lo(a.z) + bf16_lo(b.z), bf16_hi(a.z) + bf16_hi(b.z)),
                    pack_bf16(bf16_lo(a.w) + bf16_lo(b.w), bf16_hi(a.w) + bf16_hi(b.w)));
}

// 16 bytes of a gradient row of the cache: piece c (of vec_per_head per head) of row p.
template <bool HEAD_MAJOR>
__device__ __forceinline__ const uint4* cache_piece(const uint4* base, int64_t p, int c, int64_t Kt, int vec_per_head, int vec_per_row) {
  if (!HEAD_MAJOR) return base + p * vec_per_row + c;
  const int h = c / vec_per_head;
  return base + (static_cast<int64_t>(h) * Kt + p) * vec_per_head + (c - h * vec_per_head);
}

// to[c] = (base[c] +) sum of rows p0 .. p0 + cnt of the cache, in fp32, rounded once.
template <int DTYPE, bool HEAD_MAJOR, bool ADD>
__device__ __forceinline__ void write_row(const uint4* __restrict__ src, int64_t p0, int cnt, int64_t Kt, int vec_per_head,
                                          int vec_per_row, uint4* __restrict__ to) {
  for (int c = threadIdx.x; c < vec_per_row; c += blockDim.x) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (cnt == 1) {
      v = load16_stream(cache_piece<HEAD_MAJOR>(src, p0, c, Kt, vec_per_head, vec_per_row));
      if (ADD) v = add16<DTYPE>(to[c], v);
    } else if (cnt > 1) {
      constexpr int kElems = DTYPE == DODO_DTYPE_F32 ? 4 : 8;
      float acc[kElems] = {};
      const auto add = [&](const uint4& x) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (DTYPE == DODO_DTYPE_F32) {
            acc[i] += __uint_as_float(w[i]);
          } else {
            acc[2 * i % kElems] += bf16_lo(w[i]);
            acc[(2 * i + 1) % kElems] += bf16_hi(w[i]);
          }
        }
      };
      if (ADD) add(to[c]);
      for (int r = 0; r < cnt; ++r) add(*cache_piece<HEAD_MAJOR>(src, p0 + r, c, Kt, vec_per_head, vec_per_row));
      if (DTYPE == DODO_DTYPE_F32)
        v = make_uint4(__float_as_uint(acc[0]), __float_as_uint(acc[1]), __float_as_uint(acc[2]), __float_as_uint(acc[3]));
      else
        v = make_uint4(pack_bf16(acc[0], acc[1 % kElems]), pack_bf16(acc[2 % kElems], acc[3 % kElems]),
                       pack_bf16(acc[4 % kElems], acc[5 % kElems]), pack_bf16(acc[6 % kElems], acc[7 % kElems]));
    }
    to[c] = v;
  }
}

struct GradRows {
  const uint4 *dKn, *dVn;
  uint4 *dK, *dV;
  const int32_t *nugget_idx, *cu_seqlens, *cu_nuggets;
  int B, vec_per_head, vec_per_row;
  int64_t Kt, token_vec, src_layer_vec, dst_layer_vec;
};

// Grid: (chunk of kTokens tokens; layer).
template <int DTYPE, bool HEAD_MAJOR>
__global__ __launch_bounds__(kMaxThreads) void scatter_rows_kernel(GradRows a) {
  const uint4 *dKn = a.dKn + blockIdx.y * a.src_layer_vec, *dVn = a.dVn + blockIdx.y * a.src_layer_vec;
  uint4 *dK = a.dK + blockIdx.y * a.dst_layer_vec, *dV = a.dV + blockIdx.y * a.dst_layer_vec;
  int64_t tok = static_cast<int64_t>(blockIdx.x) * kTokens;
  const int64_t end = tok + kTokens;
  const SequenceLookup sequences(a.cu_seqlens, a.cu_nuggets, a.B);
  while (tok < end) {
    int s0, s1, p0, p1;
    if (!sequences.find(tok, s0, s1, p0, p1)) return;  // behind the last sequence
    const int k_b = p1 - p0;
    const int32_t* list = a.nugget_idx + p0;
    const int stop = static_cast<int>(min(end, static_cast<int64_t>(s1)) - s0);
    const auto write = [&](int token, int first, int cnt) {
      const int64_t to = (s0 + static_cast<int64_t>(token)) * a.token_vec;
      write_row<DTYPE, HEAD_MAJOR, false>(dKn, p0 + first, cnt, a.Kt, a.vec_per_head, a.vec_per_row, dK + to);
      write_row<DTYPE, HEAD_MAJOR, false>(dVn, p0 + first, cnt, a.Kt, a.vec_per_head, a.vec_per_row, dV + to);
    };
    int t = static_cast<int>(tok - s0);
    int seen = before_lower_bound(list, k_b, t);  // lane l holds list[seen + l]
    int entry = seen + lane_id() < k_b ? list[seen + lane_id()] : 0x7fffffff;
    if (~__ballot(entry < stop) != 0) {  // the 64 entries reach past these tokens (but for long runs of one index, always)
      // the rows of zeros first: they wait for nothing
      for (int z = t; z < stop; ++z)
        if (__ballot(entry == z) == 0) write(z, 0, 0);
      for (; t < stop; ++t) {
        const uint64_t mine = __ballot(entry == t);
        if (mine != 0) write(t, seen + __ffsll(static_cast<long long>(mine)) - 1, __popcll(mine));
      }
    }
    int p = seen + __popcll(__ballot(entry < t));
    for (; t < stop; ++t) {
      const int first = p;
      while (true) {
        if (p >= seen + kWave) {
          seen = p;
          entry = seen + lane_id() < k_b ? list[seen + lane_id()] : 0x7fffffff;
        }
        const int mine = __popcll(__ballot(entry == t && seen + lane_id() >= p));
        p += mine;
        if (p < seen + kWave) break;  // (a run of equal indices may go on in the next 64)
      }
      write(t, first, p - first);
    }
    tok = s0 + static_cast<int64_t>(stop);
  }
}

// Grid: (row of the cache, tensor; layer).
template <int DTYPE, bool HEAD_MAJOR>
__global__ __launch_bounds__(kMaxThreads) void add_rows_kernel(GradRows a) {
  const bool is_v = blockIdx.x & 1;
  const int64_t row = blockIdx.x >> 1;
  const uint4* src = (is_v ? a.dVn : a.dKn) + blockIdx.y * a.src_layer_vec;
  uint4* dst = (is_v ? a.dV : a.dK) + blockIdx.y * a.dst_layer_vec;
  const int b = sequence_of(a.cu_nuggets, a.B, row);
  if (b < 0) return;  // Kt may be an upper bound of the nugget count
  const int p0 = a.cu_nuggets[b], p1 = a.cu_nuggets[b + 1];
  const int idx = a.nugget_idx[row];
  const int s0 = a.cu_seqlens[b], n_b = a.cu_seqlens[b + 1] - s0;
  if (idx < 0 || idx >= n_b) return;
  if (row > p0 && a.nugget_idx[row - 1] == idx) return;  // not the first of its run
  int cnt = 1;
  while (row + cnt < p1 && a.nugget_idx[row + cnt] == idx) ++cnt;
  write_row<DTYPE, HEAD_MAJOR, true>(src, row, cnt, a.Kt, a.vec_per_head, a.vec_per_row, dst + (s0 + static_cast<int64_t>(idx)) * a.token_vec);
}

int gather_grad_entry(const void* dKn, const void* dVn, int dtype, const int32_t* nugget_idx, const int32_t* cu_seqlens,
                      const int32_t* cu_nuggets, int32_t B, int64_t Kt, int64_t N, int32_t L, int32_t H_kv, int32_t d_h,
                      int64_t token_stride, int64_t src_layer_stride, int64_t dst_layer_stride, int accumulate, void* dK,
                      void* dV, int layout, void* stream) {
  if (B < 0 || Kt < 0 || N < 0 || L < 0 || H_kv <= 0 || d_h <= 0) return DODO_ERR_INVALID_ARG;
  const int64_t row = static_cast<int64_t>(H_kv) * d_h;
  if (token_stride < row) return DODO_ERR_INVALID_ARG;
  if (layout != DODO_LAYOUT_TOKEN_MAJOR && layout != DODO_LAYOUT_HEAD_MAJOR) return DODO_ERR_INVALID_ARG;
  if (L > 1 && ((src_layer_stride != 0 && src_layer_stride < Kt * row) || (N > 0 && dst_layer_stride < (N - 1) * token_stride + row)))
    return DODO_ERR_INVALID_ARG;
  if (B == 0 || L == 0 || N == 0 || (accumulate && Kt == 0)) return DODO_OK;
  if (!dK || !dV || !cu_seqlens || !cu_nuggets || (Kt > 0 && (!dKn || !dVn || !nugget_idx))) return DODO_ERR_INVALID_ARG;
  if (!dtype_ok(dtype)) return DODO_ERR_UNSUPPORTED;
  if (Kt > 0x3fffffffLL || N > 0x3fffffffLL || L > 65535) return DODO_ERR_UNSUPPORTED;
  const int es = elem_bytes(dtype);
  if ((static_cast<int64_t>(d_h) * es) % 16 != 0 || (token_stride * es) % 16 != 0) return DODO_ERR_UNSUPPORTED;
  if ((src_layer_stride * es) % 16 != 0 || (dst_layer_stride * es) % 16 != 0) return DODO_ERR_UNSUPPORTED;
  if (!aligned16(dKn) || !aligned16(dVn) || !aligned16(dK) || !aligned16(dV)) return DODO_ERR_UNSUPPORTED;
  GradRows a;
  a.dKn = static_cast<const uint4*>(dKn); a.dVn = static_cast<const uint4*>(dVn);
  a.dK = static_cast<uint4*>(dK); a.dV = static_cast<uint4*>(dV);
  a.nugget_idx = nugget_idx; a.cu_seqlens = cu_seqlens; a.cu_nuggets = cu_nuggets; a.B = B;
  a.vec_per_head = d_h * es / 16; a.vec_per_row = a.vec_per_head * H_kv;
  a.Kt = Kt; a.token_vec = token_stride * es / 16;
  a.src_layer_vec = src_layer_stride * es / 16; a.dst_layer_vec = dst_layer_stride * es / 16;
  const int threads = min(kMaxThreads, (a.vec_per_row + kWave - 1) / kWave * kWave);
  const int64_t items = accumulate ? Kt : (N + kTokens - 1) / kTokens;
  const dim3 grid(static_cast<unsigned>(accumulate ? 2 * items : items), static_cast<unsigned>(L)), block(static_cast<unsigned>(threads));
  const bool hm = layout == DODO_LAYOUT_HEAD_MAJOR, f32 = dtype == DODO_DTYPE_F32;
  const auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, grid, block, 0, static_cast<hipStream_t>(stream), a); };
  if (accumulate) {
    if (f32) { if (hm) launch(add_rows_kernel<DODO_DTYPE_F32, true>); else launch(add_rows_kernel<DODO_DTYPE_F32, false>); }
    else { if (hm) launch(add_rows_kernel<DODO_DTYPE_BF16, true>); else launch(add_rows_kernel<DODO_DTYPE_BF16, false>); }
  } else {
    if (f32) { if (hm) launch(scatter_rows_kernel<DODO_DTYPE_F32, true>); else launch(scatter_rows_kernel<DODO_DTYPE_F32, false>); }
    else { if (hm) launch(scatter_rows_kernel<DODO_DTYPE_BF16, true>); else launch(scatter_rows_kernel<DODO_DTYPE_BF16, false>); }
  }
  return launch_status();
}

}  // namespace
}  // namespace dodo

extern "C" int dodo_gather_nuggets_grad(const void* dKn, const void* dVn, int dtype, const int32_t* nugget_idx,
                                        const int32_t* cu_seqlens, const int32_t* cu_nuggets, int32_t B, int64_t Kt, int64_t N,
                                        int32_t H_kv, int32_t d_h, int64_t token_stride, int accumulate, void* dK, void* dV,
                                        int layout, void* stream) {
  return dodo::gather_grad_entry(dKn, dVn, dtype, nugget_idx, cu_seqlens, cu_nuggets, B, Kt, N, 1, H_kv, d_h, token_stride, 0, 0,
                                 accumulate, dK, dV, layout, stream);
}

extern "C" int dodo_gather_nuggets_grad_layers(const void* dKn, const void* dVn, int dtype, const int32_t* nugget_idx,
                                               const int32_t* cu_seqlens, const int32_t* cu_nuggets, int32_t B, int64_t Kt,
                                               int64_t N, int32_t L, int32_t H_kv, int32_t d_h, int64_t token_stride,
                                               int64_t src_layer_stride, int64_t dst_layer_stride, int accumulate, void* dK,
                                               void* dV, int layout, void* stream) {
  return dodo::gather_grad_entry(dKn, dVn, dtype, nugget_idx, cu_seqlens, cu_nuggets, B, Kt, N, L, H_kv, d_h, token_stride,
                                 src_layer_stride, dst_layer_stride, accumulate, dK, dV, layout, stream);
}
