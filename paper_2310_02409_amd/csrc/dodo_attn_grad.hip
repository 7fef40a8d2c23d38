// dodo_nugget_attention_grad: gradients of nugget attention (Eq. 13 / Eq. 9 of the Dodo paper) in Q, K and V.  With s = scale q.k the
// logit of a visible pair and lse, O the forward pass's results, the probabilities are made again, never stored:
//     P[j,i] = exp(s[j,i] - lse[j]),   dS[j,i] = P[j,i] (dO[j].v_i - D[j]),   D[j] = dO[j].O[j],
//     dV_i = sum_j P dO_j,   dK_i = scale sum_j dS q_j,   dQ_j = scale sum_i dS k_i.
//
// Two kernels, so that every sum has one owner and a fixed order, without
// atomics: one walks over the query rows and owns key rows (dK, dV; with grouped-query heads all heads that read the row),
// the other walks over the keys and owns query rows (dQ).  S and dP are formed in both: 7 products instead of 5.  bf16 inputs
// have kernels of their own (dodo_attn_grad_mfma.hip); those here take fp32 inputs.
#include "dodo_attn_grad.h"

namespace dodo {
namespace {

typedef __attribute__((ext_vector_type(16))) float floatx16;

// lse2[h][row] = lse[row,h] * log2(e) and neg_d[h][row] = -dO[row,h] . O[row,h], by heads, so that the rows of a head lie side by side.
// A row that sees nothing (lse = -inf) gets +inf: its weights are 0.  16 lanes per (row, head).
__global__ __launch_bounds__(256) void grad_rows_kernel(const float* __restrict__ dO, const float* __restrict__ O,
                                                        const float* __restrict__ lse, int64_t Sq, int H, int d_h,
                                                        float* __restrict__ lse2, float* __restrict__ neg_d) {
  const int64_t t = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / 16;
  if (t >= Sq * H) return;
  const int sub = threadIdx.x % 16;
  float acc = 0.f;
  for (int c = sub * 4; c < d_h; c += 64) {
    const float4 a = *reinterpret_cast<const float4*>(dO + t * d_h + c), o = *reinterpret_cast<const float4*>(O + t * d_h + c);
    acc = fmaf(a.w, o.w, fmaf(a.z, o.z, fmaf(a.y, o.y, fmaf(a.x, o.x, acc))));
  }
  acc = lanes_sum<16>(acc);
  if (sub == 0) {
    const float l = lse[t];
    lse2[(t % H) * Sq + t / H] = l == -__builtin_inff() ? __builtin_inff() : l * kLog2e;
    neg_d[(t % H) * Sq + t / H] = -acc;
  }
}

// ---- fp32 inputs, on the fp32 matrix instructions -------------------------------------------------------------------------
// 32 x 32 blocks of S and dP from v_mfma_f32_32x32x2_f32; every wavefront fetches its fragments from memory itself.  A block's
// accumulator v holds row 8 (v / 4) + 4 g + v % 4 (g = lane / 32) and the lane's column, which is just what the next product wants
// as its right operand in step v, so P and dS stay where they are; the left operand's rows follow the same order.  The four
// wavefronts of a workgroup take the walked tiles in turn and meet in LDS at the end, added in wavefront order.

template <int DH>
using OutBlocks = floatx16[DH / 32];

template <int DH>
__device__ __forceinline__ void clear(OutBlocks<DH>& acc) {
#pragma unroll
  for (int cb = 0; cb < DH / 32; ++cb)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[cb][v] = 0.f;
}

// A row's channels as fragments: step 4 s + e of a product takes channel 8 s + 4 g + e.
template <int DH>
__device__ __forceinline__ void load_row(const void* base, int64_t off, float (&f)[DH / 2]) {
#pragma unroll
  for (int s = 0; s < DH / 8; ++s) {
    float x[4];
    load4<DODO_DTYPE_F32>(base, off + 8 * s, x);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[4 * s + e] = x[e];
  }
}
// acc = (rows at base + off, one per lane) x (fragments of the columns)
template <int DH>
__device__ __forceinline__ floatx16 dot_rows(const void* base, int64_t off, const float (&f)[DH / 2]) {
  floatx16 acc;
#pragma unroll
  for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
  for (int s = 0; s < DH / 8; ++s) {
    float x[4];
    load4<DODO_DTYPE_F32>(base, off + 8 * s, x);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], f[4 * s + e], acc, 0, 0, 0);
  }
  return acc;
}

// Sums of the workgroup's wavefronts, in wavefront order, in wavefront 0.
template <int DH>
__device__ __forceinline__ void sum_wavefronts(OutBlocks<DH>& acc, int wave, int lane, float* lds) {
  for (int w = 1; w < kGradWaves; ++w) {
    __syncthreads();
    if (wave == w)
#pragma unroll
      for (int cb = 0; cb < DH / 32; ++cb)
#pragma unroll
        for (int v = 0; v < 16; ++v) lds[(cb * 16 + v) * kWave + lane] = acc[cb][v];
    __syncthreads();
    if (wave == 0)
#pragma unroll
      for (int cb = 0; cb < DH / 32; ++cb)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[cb][v] += lds[(cb * 16 + v) * kWave + lane];
  }
}

// Row `off` of a gradient from the transposed blocks: lane (row, g) holds channels 32 cb + 8 v4 + 4 g .. + 4.
template <int DH>
__device__ __forceinline__ void store_row(void* base, int64_t off, int g, const OutBlocks<DH>& acc, float scale) {
#pragma unroll
  for (int cb = 0; cb < DH / 32; ++cb)
#pragma unroll
    for (int v4 = 0; v4 < 4; ++v4)
      store4<DODO_DTYPE_F32>(base, off + 32 * cb + 8 * v4 + 4 * g, acc[cb][4 * v4] * scale, acc[cb][4 * v4 + 1] * scale,
                    acc[cb][4 * v4 + 2] * scale, acc[cb][4 * v4 + 3] * scale);
}

template <int DH>
__global__ __launch_bounds__(kGradThreads, 1) void grad_kv_plain_kernel(GradParams p, int n_nug_tiles, int n_loc_tiles) {
  __shared__ float lds[DH / 32 * 16 * kWave];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id(), n = lane & 31, g = lane >> 5;
  const KeyTile t = key_tile(p, blockIdx.x, n_nug_tiles, n_loc_tiles, 32);
  if (t.rows <= 0) return;
  const int64_t row = t.first + min(n, t.rows - 1);
  const int64_t off = row * t.tok_stride + t.kvh * t.head_stride;
  float kf[DH / 2], vf[DH / 2];
  load_row<DH>(t.K, off + 4 * g, kf);
  load_row<DH>(t.V, off + 4 * g, vf);
  OutBlocks<DH> dk, dv;
  clear<DH>(dk);
  clear<DH>(dv);
  const int G = p.H / p.H_kv;
  for (int e = t.entry0; e < t.entry1; ++e) {
    const SeenBy s = seen_by(p, t, e, 32);
    if (!s.any) continue;
    const int least = s.least(static_cast<int>(t.first - s.key0) + n, n < t.rows);  // first query row that sees this lane's key
    for (int hg = 0; hg < G; ++hg) {
      const int h = t.kvh * G + hg;
      const int64_t stat = static_cast<int64_t>(h) * p.Sq + s.q0;
      for (int i0 = s.first_row / 32 * 32 + 32 * wave; i0 < s.q_b; i0 += 32 * kGradWaves) {
        const int64_t a_off = (static_cast<int64_t>(s.q0 + min(i0 + n, s.q_b - 1)) * p.H + h) * DH + 4 * g;
        floatx16 ds = dot_rows<DH>(p.Q, a_off, kf), dp = dot_rows<DH>(p.dO, a_off, vf);
        floatx16 pr;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int i = i0 + 8 * (v >> 2) + 4 * g + (v & 3), ic = min(i, s.q_b - 1);
          const bool vis = i >= least && i < s.q_b;
          const float w = __builtin_amdgcn_exp2f(ds[v] * p.scale_log2e - p.lse2[stat + ic]);
          pr[v] = vis ? w : 0.f;
          ds[v] = vis ? w * (dp[v] + p.neg_d[stat + ic]) : 0.f;
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int ic = min(i0 + 8 * (v >> 2) + 4 * g + (v & 3), s.q_b - 1);
          const int64_t r_off = (static_cast<int64_t>(s.q0 + ic) * p.H + h) * DH + n;
#pragma unroll
          for (int cb = 0; cb < DH / 32; ++cb) {
            dv[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(load_elem<DODO_DTYPE_F32>(p.dO, r_off + 32 * cb), pr[v], dv[cb], 0, 0, 0);
            dk[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(load_elem<DODO_DTYPE_F32>(p.Q, r_off + 32 * cb), ds[v], dk[cb], 0, 0, 0);
          }
        }
      }
    }
  }
  sum_wavefronts<DH>(dk, wave, lane, lds);
  sum_wavefronts<DH>(dv, wave, lane, lds);
  if (wave == 0 && n < t.rows) {
    store_row<DH>(t.dK, off, g, dk, p.scale);
    store_row<DH>(t.dV, off, g, dv, 1.f);
  }
}

template <int DH>
__global__ __launch_bounds__(kGradThreads, 1) void grad_q_plain_kernel(GradParams p, int n_blocks) {
  __shared__ float lds[DH / 32 * 16 * kWave];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id(), n = lane & 31, g = lane >> 5;
  const int blk = blockIdx.x % n_blocks, h = blockIdx.x / n_blocks % p.H, e = blockIdx.x / n_blocks / p.H;
  const Entry s = entry_of(p, e);
  const int i0 = blk * 32;
  if (i0 >= s.q_b) return;
  const int i = min(i0 + n, s.q_b - 1);
  const int64_t off = (static_cast<int64_t>(s.q0 + i) * p.H + h) * DH;
  float qf[DH / 2], df[DH / 2];
  load_row<DH>(p.Q, off + 4 * g, qf);
  load_row<DH>(p.dO, off + 4 * g, df);
  const float lse2 = p.lse2[static_cast<int64_t>(h) * p.Sq + s.q0 + i], neg_d = p.neg_d[static_cast<int64_t>(h) * p.Sq + s.q0 + i];
  const int kvh = h / (p.H / p.H_kv);
  const int vis = max(0, min(s.m_b, s.m_b - s.q_b + i + 1));  // local rows that this lane's row sees
  const int most = max(0, min(s.m_b, s.m_b - s.q_b + min(i0 + 32, s.q_b)));
  const int n_nug = (s.k_b + 31) / 32, n_tiles = n_nug + (most + 31) / 32;
  OutBlocks<DH> dq;
  clear<DH>(dq);
  for (int tile = wave; tile < n_tiles; tile += kGradWaves) {
    const bool nug = tile < n_nug;
    const int j0 = 32 * (nug ? tile : tile - n_nug), len = nug ? s.k_b : most, seen = nug ? s.k_b : vis;
    const void *K = nug ? p.Kn : p.Kl, *V = nug ? p.Vn : p.Vl;
    const int64_t tok = nug ? p.nug_tok_stride : p.loc_tok_stride;
    const int64_t first = (nug ? s.k0 : s.l0) * tok + kvh * (nug ? p.nug_head_stride : DH);
    const int64_t a_off = first + min(j0 + n, len - 1) * tok + 4 * g;
    floatx16 ds = dot_rows<DH>(K, a_off, qf), dp = dot_rows<DH>(V, a_off, df);
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int j = j0 + 8 * (v >> 2) + 4 * g + (v & 3);
      const float w = __builtin_amdgcn_exp2f(ds[v] * p.scale_log2e - lse2);
      ds[v] = j < seen ? w * (dp[v] + neg_d) : 0.f;
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int64_t r_off = first + min(j0 + 8 * (v >> 2) + 4 * g + (v & 3), len - 1) * tok + n;
#pragma unroll
      for (int cb = 0; cb < DH / 32; ++cb)
        dq[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(load_elem<DODO_DTYPE_F32>(K, r_off + 32 * cb), ds[v], dq[cb], 0, 0, 0);
    }
  }
  sum_wavefronts<DH>(dq, wave, lane, lds);
  if (wave == 0 && i0 + n < s.q_b) store_row<DH>(p.dQ, off, g, dq, p.scale);
}

template <int DH>
int launch_plain(const GradParams& p) {
  // one workgroup per 32 keys: of every sequence, or of all rows where entries share them
  const int64_t nug_rows = p.shared ? p.Kt : p.max_k, loc_rows = p.shared ? p.Sm : p.max_local;
  const int64_t nug = (nug_rows + 31) / 32, loc = (loc_rows + 31) / 32;
  const int64_t owners = (nug + loc) * p.H_kv * (p.shared ? 1 : p.B);
  const int64_t blocks = (static_cast<int64_t>(p.max_q) + 31) / 32, rows = blocks * p.H * p.B;
  if (owners > 0x7fffffffLL || rows > 0x7fffffffLL) return DODO_ERR_UNSUPPORTED;
  if (owners > 0) {
    hipLaunchKernelGGL(HIP_KERNEL_NAME(grad_kv_plain_kernel<DH>), dim3(static_cast<unsigned>(owners)), dim3(kGradThreads), 0,
                       p.stream, p, static_cast<int>(nug), static_cast<int>(loc));
    const int rc = launch_status();
    if (rc != DODO_OK) return rc;
  }
  if (rows == 0) return DODO_OK;
  hipLaunchKernelGGL(HIP_KERNEL_NAME(grad_q_plain_kernel<DH>), dim3(static_cast<unsigned>(rows)), dim3(kGradThreads), 0, p.stream,
                     p, static_cast<int>(blocks));
  return launch_status();
}

size_t workspace_bytes(int64_t Sq, int32_t H) { return static_cast<size_t>(2) * Sq * H * sizeof(float); }

int grad_entry(GradParams& p, int32_t d_h, int dtype, int layout, void* ws, size_t ws_bytes) {
  if (p.B < 0 || p.H <= 0 || p.H_kv <= 0 || d_h <= 0 || p.max_q < 0 || p.max_k < 0 || p.max_local < 0 || p.Sq < 0 || p.Kt < 0 || p.Sm < 0)
    return DODO_ERR_INVALID_ARG;
  if (p.H % p.H_kv != 0) return DODO_ERR_INVALID_ARG;
  if (layout != DODO_LAYOUT_TOKEN_MAJOR && layout != DODO_LAYOUT_HEAD_MAJOR) return DODO_ERR_INVALID_ARG;
  if (!(p.scale == p.scale)) return DODO_ERR_INVALID_ARG;
  if (p.B == 0 && !p.shared) return DODO_OK;
  if (p.B > 0 && (!p.cu_q || !p.cu_nuggets || !p.cu_local || (p.shared && (!p.nug_len || !p.loc_len)))) return DODO_ERR_INVALID_ARG;
  if (p.B == 0 || p.Sq == 0) p.max_q = 0;
  if (p.Kt == 0) p.max_k = 0;
  if (p.Sm == 0) p.max_local = 0;
  const bool nuggets = p.shared ? p.Kt > 0 : p.max_k > 0, locals = p.shared ? p.Sm > 0 : p.max_local > 0;
  if (p.max_q > 0 && (!p.Q || !p.dO || !p.O || !p.lse || !p.dQ)) return DODO_ERR_INVALID_ARG;
  if (nuggets && (!p.Kn || !p.Vn || !p.dKn || !p.dVn)) return DODO_ERR_INVALID_ARG;
  if (locals && (!p.Kl || !p.Vl || !p.dKl || !p.dVl)) return DODO_ERR_INVALID_ARG;
  if (!dtype_ok(dtype)) return DODO_ERR_UNSUPPORTED;
  if (d_h != 64 && d_h != 128) return DODO_ERR_UNSUPPORTED;
  if (!aligned16(p.Q) || !aligned16(p.Kn) || !aligned16(p.Vn) || !aligned16(p.Kl) || !aligned16(p.Vl) || !aligned16(p.dO) || !aligned16(p.O) ||
      !aligned16(p.dQ) || !aligned16(p.dKn) || !aligned16(p.dVn) || !aligned16(p.dKl) || !aligned16(p.dVl) || !aligned16(ws))
    return DODO_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(p.H) * d_h >= 1 << 24) return DODO_ERR_UNSUPPORTED;  // (offsets between 128 rows in 32 bits)
  if (p.Sq * p.H > 0x7fffffffLL || p.Kt > 0x7fffffffLL || p.Sm > 0x7fffffffLL) return DODO_ERR_UNSUPPORTED;
  if (!nuggets && !locals && p.max_q == 0) return DODO_OK;
  if (p.max_q > 0 && (!ws || ws_bytes < workspace_bytes(p.Sq, p.H))) return DODO_ERR_WORKSPACE_TOO_SMALL;
  p.nug_tok_stride = layout == DODO_LAYOUT_TOKEN_MAJOR ? static_cast<int64_t>(p.H_kv) * d_h : d_h;
  p.nug_head_stride = layout == DODO_LAYOUT_TOKEN_MAJOR ? d_h : p.Kt * d_h;
  p.loc_tok_stride = static_cast<int64_t>(p.H_kv) * d_h;
  p.loc_head_stride = d_h;
  p.scale_log2e = p.scale * kLog2e;
  p.lse2 = static_cast<float*>(ws);
  p.neg_d = p.lse2 + p.Sq * p.H;
  if (dtype == DODO_DTYPE_BF16) return launch_grad_mfma(p, d_h);
  if (p.max_q > 0) {
    hipLaunchKernelGGL(grad_rows_kernel, dim3(static_cast<unsigned>((p.Sq * p.H * 16 + 255) / 256)), dim3(256), 0, p.stream,
                       static_cast<const float*>(p.dO), static_cast<const float*>(p.O), p.lse, p.Sq, p.H, d_h, p.lse2, p.neg_d);
    const int rc = launch_status();
    if (rc != DODO_OK) return rc;
  }
  return d_h == 128 ? launch_plain<128>(p) : launch_plain<64>(p);
}

}  // namespace
}  // namespace dodo

extern "C" size_t dodo_nugget_attention_grad_workspace_bytes(int32_t B, int32_t H, int32_t H_kv, int32_t d_h, int32_t max_q,
                                                             int32_t max_k, int32_t max_local, int64_t Sq, int64_t Kt, int64_t Sm,
                                                             int dtype) {
  if (B <= 0 || H <= 0 || H_kv <= 0 || d_h <= 0 || max_q <= 0 || max_k < 0 || max_local < 0 || Sq <= 0 || Kt < 0 || Sm < 0) return 0;
  return dodo::workspace_bytes(Sq, H);
}

extern "C" int dodo_nugget_attention_grad(const void* Q, const void* Kn, const void* Vn, const void* Kl, const void* Vl,
                                          const void* dO, const void* O, const float* lse, const int32_t* cu_q,
                                          const int32_t* cu_nuggets, const int32_t* cu_local, int32_t B, int32_t H, int32_t H_kv,
                                          int32_t d_h, int32_t max_q, int32_t max_k, int32_t max_local, int64_t Sq, int64_t Kt,
                                          int64_t Sm, float softmax_scale, int dtype, int layout, void* dQ, void* dKn, void* dVn,
                                          void* dKl, void* dVl, void* ws, size_t ws_bytes, void* stream) {
  dodo::GradParams p = {};
  p.Q = Q; p.Kn = Kn; p.Vn = Vn; p.Kl = Kl; p.Vl = Vl; p.dO = dO; p.O = O; p.lse = lse;
  p.cu_q = cu_q; p.cu_nuggets = cu_nuggets; p.cu_local = cu_local;
  p.B = B; p.H = H; p.H_kv = H_kv; p.max_q = max_q; p.max_k = max_k; p.max_local = max_local;
  p.Sq = Sq; p.Kt = Kt; p.Sm = Sm; p.scale = softmax_scale;
  p.dQ = dQ; p.dKn = dKn; p.dVn = dVn; p.dKl = dKl; p.dVl = dVl;
  p.stream = static_cast<hipStream_t>(stream);
  return dodo::grad_entry(p, d_h, dtype, layout, ws, ws_bytes);
}

extern "C" int dodo_nugget_attention_segments_grad(const void* Q, const void* Kn, const void* Vn, const void* K, const void* V,
                                                   const void* dO, const void* O, const float* lse, const int32_t* seg_cu_q,
                                                   const int32_t* seg_nug_start, const int32_t* seg_nug_len,
                                                   const int32_t* seg_loc_start, const int32_t* seg_loc_len, int32_t n_segments,
                                                   int32_t H, int32_t H_kv, int32_t d_h, int32_t max_q, int32_t max_k,
                                                   int32_t max_local, int64_t Sq, int64_t Kt, int64_t N, float softmax_scale,
                                                   int dtype, int layout, void* dQ, void* dKn, void* dVn, void* dK, void* dV,
                                                   void* ws, size_t ws_bytes, void* stream) {
  dodo::GradParams p = {};
  p.Q = Q; p.Kn = Kn; p.Vn = Vn; p.Kl = K; p.Vl = V; p.dO = dO; p.O = O; p.lse = lse;
  p.cu_q = seg_cu_q; p.cu_nuggets = seg_nug_start; p.nug_len = seg_nug_len; p.cu_local = seg_loc_start; p.loc_len = seg_loc_len;
  p.shared = 1;
  p.B = n_segments; p.H = H; p.H_kv = H_kv; p.max_q = max_q; p.max_k = max_k; p.max_local = max_local;
  p.Sq = Sq; p.Kt = Kt; p.Sm = N; p.scale = softmax_scale;
  p.dQ = dQ; p.dKn = dKn; p.dVn = dVn; p.dKl = dK; p.dVl = dV;
  p.stream = static_cast<hipStream_t>(stream);
  return dodo::grad_entry(p, d_h, dtype, layout, ws, ws_bytes);
}
