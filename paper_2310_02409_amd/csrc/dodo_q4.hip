// Nugget caches in 4 bits (the format is described in dodo.h): dodo_gather_nuggets_q4 packs the chosen tokens' K and V rows
// (Eq. 5 of the Dodo paper) into one, dodo_unpack_nuggets_q4 reads one back.
//
// Both are passes over memory.  A thread takes 8 consecutive channels, so the four lanes of a quad hold a block of 32: the block's
// largest magnitude takes two lane exchanges within the quad, its exponent follows from that number's bits (the mantissa
// tells whether it is above 1.75, that is 7 / 4), and the conversion instructions divide by the scale and round to nearest,
// ties to the even index.  8 sequences of 4096 tokens at 10x, 32 heads of 128, bf16: packing 18.7 us (3.6 TB/s: single rows
// of 8 KiB behind a round of lookups; 20.7 with two rounds and 8 channels a thread; both tensors by one workgroup is no faster), unpacking
// 10 us (6.9 TB/s).
#include <type_traits>

#include "dodo_lists.h"
#include "dodo_q4.h"

namespace dodo {
namespace {

constexpr int kPackThreads = 256;

// Largest of an unsigned number over the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0xB1, 0xf, 0xf, false)));  // quad_perm [1,0,3,2]
  return max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x4E, 0xf, 0xf, false)));  // quad_perm [2,3,0,1]
}

template <int DTYPE>
__device__ __forceinline__ void load8(const void* p, float (&x)[8]) {
  if (DTYPE == DODO_DTYPE_F32) {
    const uint4 a = load16_stream(p), b = load16_stream(static_cast<const char*>(p) + 16);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
  } else {
    const uint4 a = load16_stream(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  }
}

// Codes of this lane's 8 channels, and the scale byte of the block that the quad holds.
__device__ __forceinline__ uint32_t pack8(const float (&x)[8], uint32_t& scale_byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = quad_max(top);
  const bool bad = top >= 0x7f800000u;  // a NaN or an infinity
  const int e = min(kMostExpQ4, max(kLeastExpQ4, static_cast<int>(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0)));
  scale_byte = bad ? kScaleBadQ4 : static_cast<uint32_t>(e + 127);
  const float scale = scale_q4(static_cast<uint32_t>(bad ? 127 : e + 127));
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
  return bad ? 0u : codes;
}

// One workgroup per destination row, tensor (the lowest bit of blockIdx.x) and layer (blockIdx.y).  A thread requests two units of 8
// channels before it packs the first.
template <int DTYPE, bool HEAD_MAJOR>
__global__ __launch_bounds__(kPackThreads) void gather_q4_kernel(
    const char* __restrict__ K, const char* __restrict__ V, const int32_t* __restrict__ nugget_idx,
    const int32_t* __restrict__ cu_seqlens, const int32_t* __restrict__ cu_nuggets, int B, int64_t Kt, int units_per_head,
    int units, int64_t token_bytes, int64_t layer_bytes, uint8_t* __restrict__ Kc, uint8_t* __restrict__ Ks,
    uint8_t* __restrict__ Vc, uint8_t* __restrict__ Vs) {
  const int64_t row = blockIdx.x >> 1, layer = blockIdx.y;
  const bool is_v = blockIdx.x & 1;
  const int64_t tok = token_of(cu_seqlens, cu_nuggets, nugget_idx, B, row);
  if (tok < 0) return;  // Kt may be an upper bound of the nugget count
  const char* src = (is_v ? V : K) + layer * layer_bytes + tok * token_bytes;
  uint32_t* codes = reinterpret_cast<uint32_t*>(is_v ? Vc : Kc) + layer * Kt * units;
  uint8_t* scales = (is_v ? Vs : Ks) + layer * Kt * (units / 4);
  constexpr int kUnitBytes = DTYPE == DODO_DTYPE_F32 ? 32 : 16;
  for (int u0 = threadIdx.x; u0 < units; u0 += 2 * blockDim.x) {  // (units is a multiple of 4: quads stay together)
    const int u1 = u0 + static_cast<int>(blockDim.x);
    float x[2][8];
    load8<DTYPE>(src + static_cast<int64_t>(u0) * kUnitBytes, x[0]);
    if (u1 < units) load8<DTYPE>(src + static_cast<int64_t>(u1) * kUnitBytes, x[1]);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int u = c == 0 ? u0 : u1;
      if (u >= units) break;
      uint32_t byte;
      const uint32_t w = pack8(x[c], byte);
      int64_t at = row * units + u;
      if (HEAD_MAJOR) {
        const int h = u / units_per_head;
        at = (static_cast<int64_t>(h) * Kt + row) * units_per_head + (u - h * units_per_head);
      }
      codes[at] = w;
      if ((u & 3) == 0) scales[at >> 2] = static_cast<uint8_t>(byte);
    }
  }
}

// A thread reads the codes of 8 channels of K (blockIdx.y = 0) or V.  BLOCKS = 0: what they stand for.  BLOCKS (2 or 4) scale bytes a row
// and head: for the attention kernels, which answer a NaN among their logits each in its own way, but all hand on one in V.  So a
// bad block of K becomes zeros, and that row and head of V NaN in all channels.  Without / with: 8 sequences of 410 nuggets, 32 heads of 128, bf16
// 8.9 / 8.9 us; 32 of 3277, 8 heads of 128, fp32 345 / 392.
template <int DTYPE, int BLOCKS>
__global__ __launch_bounds__(256) void unpack_q4_kernel(const uint32_t* __restrict__ Kc, const uint8_t* __restrict__ Ks,
                                                        const uint32_t* __restrict__ Vc, const uint8_t* __restrict__ Vs,
                                                        int64_t units, void* __restrict__ Kn, void* __restrict__ Vn) {
  const int64_t u = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (u >= units) return;
  uint32_t codes = (blockIdx.y ? Vc : Kc)[u];
  uint32_t byte = (blockIdx.y ? Vs : Ks)[u >> 2];
  if constexpr (BLOCKS > 0) {
    if (blockIdx.y) {
      if (any_bad_q4(row_scales_q4<BLOCKS>(Ks, u / (4 * BLOCKS)))) byte = kScaleBadQ4;
    } else if (byte == kScaleBadQ4) {
      codes = 0;
      byte = 127;
    }
  }
  const uint4 v = unpack8_bf16(codes, scale_q4(byte));
  void* out = blockIdx.y ? Vn : Kn;
  if (DTYPE == DODO_DTYPE_BF16) {
    store16_stream(static_cast<uint4*>(out) + u, v);
  } else {
    uint4* to = static_cast<uint4*>(out) + 2 * u;
    store16_stream(to, make_uint4(v.x << 16, v.x & 0xffff0000u, v.y << 16, v.y & 0xffff0000u));
    store16_stream(to + 1, make_uint4(v.z << 16, v.z & 0xffff0000u, v.w << 16, v.w & 0xffff0000u));
  }
}

int gather_q4_entry(const void* K, const void* V, int dtype, const int32_t* nugget_idx, const int32_t* cu_seqlens,
                    const int32_t* cu_nuggets, int32_t B, int64_t Kt, int32_t L, int32_t H_kv, int32_t d_h,
                    int64_t token_stride, int64_t src_layer_stride, uint8_t* Kc, uint8_t* Ks, uint8_t* Vc, uint8_t* Vs,
                    int layout, void* stream) {
  if (B < 0 || Kt < 0 || L < 0 || H_kv <= 0 || d_h <= 0) return DODO_ERR_INVALID_ARG;
  if (token_stride < static_cast<int64_t>(H_kv) * d_h) return DODO_ERR_INVALID_ARG;
  if (layout != DODO_LAYOUT_TOKEN_MAJOR && layout != DODO_LAYOUT_HEAD_MAJOR) return DODO_ERR_INVALID_ARG;
  if (L > 1 && src_layer_stride < 0) return DODO_ERR_INVALID_ARG;
  if (Kt == 0 || B == 0 || L == 0) return DODO_OK;
  if (!K || !V || !nugget_idx || !cu_seqlens || !cu_nuggets || !Kc || !Ks || !Vc || !Vs) return DODO_ERR_INVALID_ARG;
  if (!dtype_ok(dtype) || d_h % kBlockQ4 != 0) return DODO_ERR_UNSUPPORTED;
  if (Kt > 0x3fffffffLL || L > 65535 || static_cast<int64_t>(H_kv) * d_h > 0x3fffffffLL) return DODO_ERR_UNSUPPORTED;
  const int es = elem_bytes(dtype);
  if ((token_stride * es) % 16 != 0 || (src_layer_stride * es) % 16 != 0) return DODO_ERR_UNSUPPORTED;
  if (!aligned16(K) || !aligned16(V) || !aligned16(Kc) || !aligned16(Vc)) return DODO_ERR_UNSUPPORTED;
  if (((reinterpret_cast<uintptr_t>(Ks) | reinterpret_cast<uintptr_t>(Vs)) & 3u) != 0) return DODO_ERR_UNSUPPORTED;
  const int units_per_head = d_h / 8, units = units_per_head * H_kv;
  // as many threads as units, up to four wavefronts
  const int threads = units >= kPackThreads ? kPackThreads : (units + kWave - 1) / kWave * kWave;
  const dim3 grid(static_cast<unsigned>(2 * Kt), static_cast<unsigned>(L)), block(static_cast<unsigned>(threads));
  const auto launch = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, block, 0, static_cast<hipStream_t>(stream), static_cast<const char*>(K),
                       static_cast<const char*>(V), nugget_idx, cu_seqlens, cu_nuggets, B, Kt, units_per_head, units,
                       token_stride * es, src_layer_stride * es, Kc, Ks, Vc, Vs);
  };
  const bool hm = layout == DODO_LAYOUT_HEAD_MAJOR;
  if (dtype == DODO_DTYPE_F32) {
    if (hm) launch(gather_q4_kernel<DODO_DTYPE_F32, true>); else launch(gather_q4_kernel<DODO_DTYPE_F32, false>);
  } else {
    if (hm) launch(gather_q4_kernel<DODO_DTYPE_BF16, true>); else launch(gather_q4_kernel<DODO_DTYPE_BF16, false>);
  }
  return launch_status();
}

}  // namespace
}  // namespace dodo

extern "C" int dodo_gather_nuggets_q4(const void* K, const void* V, int dtype, const int32_t* nugget_idx,
                                      const int32_t* cu_seqlens, const int32_t* cu_nuggets, int32_t B, int64_t Kt,
                                      int32_t H_kv, int32_t d_h, int64_t token_stride, uint8_t* Kc, uint8_t* Ks, uint8_t* Vc,
                                      uint8_t* Vs, int layout, void* stream) {
  return dodo::gather_q4_entry(K, V, dtype, nugget_idx, cu_seqlens, cu_nuggets, B, Kt, 1, H_kv, d_h, token_stride, 0, Kc, Ks, Vc,
                               Vs, layout, stream);
}

extern "C" int dodo_gather_nuggets_q4_layers(const void* K, const void* V, int dtype, const int32_t* nugget_idx,
                                             const int32_t* cu_seqlens, const int32_t* cu_nuggets, int32_t B, int64_t Kt,
                                             int32_t L, int32_t H_kv, int32_t d_h, int64_t token_stride,
                                             int64_t src_layer_stride, uint8_t* Kc, uint8_t* Ks, uint8_t* Vc, uint8_t* Vs,
                                             int layout, void* stream) {
  return dodo::gather_q4_entry(K, V, dtype, nugget_idx, cu_seqlens, cu_nuggets, B, Kt, L, H_kv, d_h, token_stride,
                               src_layer_stride, Kc, Ks, Vc, Vs, layout, stream);
}

namespace dodo {

int unpack_q4(const uint8_t* Kc, const uint8_t* Ks, const uint8_t* Vc, const uint8_t* Vs, int64_t rows, int32_t d_h, int dtype,
              bool for_attention, void* Kn, void* Vn, void* stream) {
  if (rows < 0 || d_h <= 0) return DODO_ERR_INVALID_ARG;
  if (rows == 0) return DODO_OK;
  if (!Kc || !Ks || !Vc || !Vs || !Kn || !Vn) return DODO_ERR_INVALID_ARG;
  if (!dtype_ok(dtype) || d_h % kBlockQ4 != 0) return DODO_ERR_UNSUPPORTED;
  if (!aligned16(Kc) || !aligned16(Vc) || !aligned16(Kn) || !aligned16(Vn)) return DODO_ERR_UNSUPPORTED;
  if (rows > 0x7fffffffLL * 32 / (d_h / 8)) return DODO_ERR_UNSUPPORTED;
  if (for_attention && d_h != 64 && d_h != 128) return DODO_ERR_UNSUPPORTED;
  const int64_t units = rows * (d_h / 8);
  const dim3 grid(static_cast<unsigned>((units + 255) / 256), 2), block(256);
  const auto launch = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, block, 0, static_cast<hipStream_t>(stream), reinterpret_cast<const uint32_t*>(Kc), Ks,
                       reinterpret_cast<const uint32_t*>(Vc), Vs, units, Kn, Vn);
  };
  const auto launch_as = [&](auto blocks) {
    constexpr int kBlocks = decltype(blocks)::value;
    if (dtype == DODO_DTYPE_F32) launch(unpack_q4_kernel<DODO_DTYPE_F32, kBlocks>); else launch(unpack_q4_kernel<DODO_DTYPE_BF16, kBlocks>);
  };
  if (!for_attention) launch_as(std::integral_constant<int, 0>{});
  else if (d_h == 64) launch_as(std::integral_constant<int, 2>{});
  else launch_as(std::integral_constant<int, 4>{});
  return launch_status();
}

}  // namespace dodo

extern "C" int dodo_unpack_nuggets_q4(const uint8_t* Kc, const uint8_t* Ks, const uint8_t* Vc, const uint8_t* Vs, int64_t rows,
                                      int32_t d_h, int dtype, void* Kn, void* Vn, void* stream) {
  return dodo::unpack_q4(Kc, Ks, Vc, Vs, rows, d_h, dtype, false, Kn, Vn, stream);
}
