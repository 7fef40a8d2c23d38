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

// ---- fp32 inputs, on the fp32 matrix instructions -------------------------------------------------------------------------
// 16 x 16 blocks of S and dP from v_mfma_f32_16x16x4_f32; every wavefront fetches its fragments from memory itself, 16 bytes a load.
// Lane (n, g) = (lane % 16, lane / 16) owns row n of what the kernel sums.  A block's accumulator v holds walked row 4 g + v and the
// lane's own one, which is just what the next product wants as its right operand in step v, so P and dS stay where they are; its
// left operand, block 4 hi + e of the sums, takes channels 64 hi + 4 n + e, so that one load brings four blocks' and the sums are
// stored four channels at a time.
// A workgroup owns 16 rows; its wavefronts take the walked blocks in turn and their sums meet in LDS, added in wavefront order.  (64
// rows, 16 a wavefront, walked together, is slower where it leaves compute units idle and little faster elsewhere.  This / that, dQ
// and dK with dV, us: 1 sequence, 4 heads of 64, 32 rows, 51 nuggets, 48 local rows 6.7 + 6.7 / 10.5 + 9.2; 8 sequences, 32 heads of 128,
// 512 rows, 410 nuggets, 640 local rows 1256 + 1422 / 1169 + 1379; 2, 2048 rows, 410, 2048 1871 + 2291 / 2490 + 2508; 8, 128 rows, 100, 256
// 140 + 187 / 110 + 168.)  The large ones run at half of the fp32 matrix rate, 70 TFLOP/s: the fragments come through the vector memory path,
// whose data return is busy in 86% (dQ) and 95% (dK, dV) of the cycles, the matrix pipes in 43 and 51.  The smallest are a chain of
// loads: the ranges, the owned rows, the walked rows, some 2 us each with the launch.

constexpr int kPlainRows = 16;  // owned by a workgroup
template <int DH>
using OutBlocks = floatx4[DH / 16];

template <int DH>
__device__ __forceinline__ void clear(OutBlocks<DH>& acc) {
#pragma unroll
  for (int cb = 0; cb < DH / 16; ++cb) acc[cb] = floatx4{0.f, 0.f, 0.f, 0.f};
}

// A row's channels as fragments: step 4 s + e of a product takes channel 16 s + 4 g + e.
template <int DH>
__device__ __forceinline__ void load_row(const void* base, int64_t off, float (&f)[DH / 4]) {
#pragma unroll
  for (int s = 0; s < DH / 16; ++s) {
    const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(base) + off + 16 * s);
    f[4 * s] = x.x; f[4 * s + 1] = x.y; f[4 * s + 2] = x.z; f[4 * s + 3] = x.w;
  }
}
__device__ __forceinline__ floatx4 mfma(float a, float b, const floatx4& c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
// s += (a's rows) x (k's columns), dp += (b's) x (v's)
template <int DH>
__device__ __forceinline__ void dot_rows(const float (&a)[DH / 4], const float (&b)[DH / 4], const float (&k)[DH / 4], const float (&v)[DH / 4],
                                         floatx4& s, floatx4& dp) {
#pragma unroll
  for (int c = 0; c < DH / 4; ++c) {
    s = mfma(a[c], k[c], s);
    dp = mfma(b[c], v[c], dp);
  }
}
// acc += (walked row `base + off`, one per lane group g, as a column) x (w of the owned rows)
template <int DH>
__device__ __forceinline__ void add_column(OutBlocks<DH>& acc, const void* base, int64_t off, float w) {
#pragma unroll
  for (int hi = 0; hi < DH / 64; ++hi) {
    const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(base) + off + 64 * hi);
    acc[4 * hi] = mfma(x.x, w, acc[4 * hi]);
    acc[4 * hi + 1] = mfma(x.y, w, acc[4 * hi + 1]);
    acc[4 * hi + 2] = mfma(x.z, w, acc[4 * hi + 2]);
    acc[4 * hi + 3] = mfma(x.w, w, acc[4 * hi + 3]);
  }
}

// A row of a gradient: every wavefront puts its sums into LDS and then stores a quarter of all.
template <int DH>
constexpr int kMeetWords = kGradWaves * DH / 16 * kWave;  // of 16 bytes, for one tensor
template <int DH>
__device__ __forceinline__ void put_sums(float4* lds, int wave, int lane, const OutBlocks<DH>& acc) {
#pragma unroll
  for (int hi = 0; hi < DH / 64; ++hi)
#pragma unroll
    for (int v = 0; v < 4; ++v)
      lds[((wave * (DH / 64) + hi) * 4 + v) * kWave + lane] = make_float4(acc[4 * hi][v], acc[4 * hi + 1][v], acc[4 * hi + 2][v], acc[4 * hi + 3][v]);
}
template <int DH>
__device__ __forceinline__ void store_sums(const float4* lds, int wave, int lane, void* base, int64_t off, bool row_ok, float scale) {
#pragma unroll
  for (int hi = 0; hi < DH / 64; ++hi) {
    float4 sum = lds[(hi * 4 + wave) * kWave + lane];
#pragma unroll
    for (int w = 1; w < kGradWaves; ++w) {
      const float4 x = lds[((w * (DH / 64) + hi) * 4 + wave) * kWave + lane];
      sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
    }
    if (row_ok) store4<DODO_DTYPE_F32>(base, off + 64 * hi + 16 * (lane >> 4) + 4 * wave, sum.x * scale, sum.y * scale, sum.z * scale, sum.w * scale);
  }
}

template <int DH>
__global__ __launch_bounds__(kGradThreads, 2) void grad_kv_plain_kernel(GradParams p, int n_nug_tiles, int n_loc_tiles) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id(), n = lane & 15, g = lane >> 4;
  const KeyTile t = key_tile(p, blockIdx.x, n_nug_tiles, n_loc_tiles, kPlainRows);
  if (t.rows <= 0) return;
  const int64_t off = (t.first + min(n, t.rows - 1)) * t.tok_stride + t.kvh * t.head_stride;
  float kf[DH / 4], vf[DH / 4];
  load_row<DH>(t.K, off + 4 * g, kf);
  load_row<DH>(t.V, off + 4 * g, vf);
  OutBlocks<DH> dk, dv;
  clear<DH>(dk);
  clear<DH>(dv);
  const int G = p.H / p.H_kv;
  for (int e0 = t.entry0; e0 < t.entry1; e0 += kWave) {  // entries that see any of the keys are looked for 64 at a time
    SeenBy of_lane = {};
    if (e0 + lane < t.entry1) of_lane = seen_by(p, t, e0 + lane, kPlainRows);
    for (uint64_t todo = __ballot(of_lane.any && of_lane.first_row < of_lane.q_b); todo != 0; todo &= todo - 1) {
      const int from = __ffsll(static_cast<long long>(todo)) - 1;
      SeenBy s;
      s.q0 = __builtin_amdgcn_readlane(of_lane.q0, from);
      s.q_b = __builtin_amdgcn_readlane(of_lane.q_b, from);
      s.key0 = __builtin_amdgcn_readlane(of_lane.key0, from);
      s.len = __builtin_amdgcn_readlane(of_lane.len, from);
      s.lag = __builtin_amdgcn_readlane(of_lane.lag, from);
      s.first_row = __builtin_amdgcn_readlane(of_lane.first_row, from);
      const int least = s.least(static_cast<int>(t.first - s.key0) + n, n < t.rows);  // first query row that sees this lane's key
      for (int hg = 0; hg < G; ++hg) {
        const int h = t.kvh * G + hg;
        const int64_t stat = static_cast<int64_t>(h) * p.Sq + s.q0;
        for (int i0 = s.first_row / 16 * 16 + 16 * wave; i0 < s.q_b; i0 += 16 * kGradWaves) {
          const int64_t a_off = (static_cast<int64_t>(s.q0 + min(i0 + n, s.q_b - 1)) * p.H + h) * DH + 4 * g;
          float qa[DH / 4], da[DH / 4], lse2[4];
          load_row<DH>(p.Q, a_off, qa);
          load_row<DH>(p.dO, a_off, da);
          floatx4 pr = {0.f, 0.f, 0.f, 0.f}, ds;  // (dP starts from -D, which saves the subtractions)
          int64_t r_off[4];
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int ic = min(i0 + 4 * g + v, s.q_b - 1);
            lse2[v] = p.lse2[stat + ic];
            ds[v] = p.neg_d[stat + ic];
            r_off[v] = (static_cast<int64_t>(s.q0 + ic) * p.H + h) * DH + 4 * n;
          }
          dot_rows<DH>(qa, da, kf, vf, pr, ds);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int i = i0 + 4 * g + v;
            const bool vis = i >= least && i < s.q_b;
            const float w = __builtin_amdgcn_exp2f(fmaf(pr[v], p.scale_log2e, -lse2[v]));
            pr[v] = vis ? w : 0.f;
            ds[v] = vis ? w * ds[v] : 0.f;
          }
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            add_column<DH>(dv, p.dO, r_off[v], pr[v]);
            add_column<DH>(dk, p.Q, r_off[v], ds[v]);
          }
        }
      }
    }
  }
  const bool row_ok = n < t.rows;
  __shared__ float4 lds[2 * kMeetWords<DH>];
  put_sums<DH>(lds, wave, lane, dk);
  put_sums<DH>(lds + kMeetWords<DH>, wave, lane, dv);
  __syncthreads();
  store_sums<DH>(lds, wave, lane, t.dK, off, row_ok, p.scale);
  store_sums<DH>(lds + kMeetWords<DH>, wave, lane, t.dV, off, row_ok, 1.f);
}

template <int DH>
__global__ __launch_bounds__(kGradThreads, 2) void grad_q_plain_kernel(GradParams p, int n_blocks) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id(), n = lane & 15, g = lane >> 4;
  const int blk = blockIdx.x % n_blocks, h = blockIdx.x / n_blocks % p.H, e = blockIdx.x / n_blocks / p.H;
  const Entry s = entry_of(p, e);
  const int i0 = blk * kPlainRows;
  if (i0 >= s.q_b) return;
  const bool row_ok = i0 + n < s.q_b;
  const int i = min(i0 + n, s.q_b - 1);
  const int64_t off = (static_cast<int64_t>(s.q0 + i) * p.H + h) * DH, stat = static_cast<int64_t>(h) * p.Sq + s.q0 + i;
  float qf[DH / 4], df[DH / 4];
  load_row<DH>(p.Q, off + 4 * g, qf);
  load_row<DH>(p.dO, off + 4 * g, df);
  // D and the log-sum-exp in base 2 of the row, here and for the other kernel; a row that sees nothing (-inf) gets +inf: its
  // weights are 0
  float lse2 = p.lse[static_cast<int64_t>(s.q0 + i) * p.H + h] * kLog2e, neg_d = 0.f;
  if (lse2 == -__builtin_inff()) lse2 = __builtin_inff();
  {
    float of[DH / 4];
    load_row<DH>(p.O, off + 4 * g, of);
#pragma unroll
    for (int c = 0; c < DH / 4; ++c) neg_d = fmaf(df[c], of[c], neg_d);
    float lower, upper;
    lane_pair<16>(neg_d, lower, upper);
    neg_d = lower + upper;
    lane_pair<32>(neg_d, lower, upper);
    neg_d = -(lower + upper);
  }
  if (g == 0 && row_ok && wave == 0) {
    p.lse2[stat] = lse2;
    p.neg_d[stat] = neg_d;
  }
  const int kvh = h / (p.H / p.H_kv);
  const int vis = max(0, min(s.m_b, s.m_b - s.q_b + i + 1));  // local rows that this lane's row sees
  const int most = max(0, min(s.m_b, s.m_b - s.q_b + min(i0 + 16, s.q_b)));
  const int n_nug = (s.k_b + 15) / 16, n_tiles = n_nug + (most + 15) / 16;
  OutBlocks<DH> dq;
  clear<DH>(dq);
  for (int tile = wave; tile < n_tiles; tile += kGradWaves) {
    const bool nug = tile < n_nug;
    const int j0 = 16 * (nug ? tile : tile - n_nug), len = nug ? s.k_b : most, seen = nug ? s.k_b : vis;
    const void *K = nug ? p.Kn : p.Kl, *V = nug ? p.Vn : p.Vl;
    const int64_t tok = nug ? p.nug_tok_stride : p.loc_tok_stride;
    const int64_t first = (nug ? s.k0 : s.l0) * tok + kvh * (nug ? p.nug_head_stride : p.loc_head_stride);
    const int64_t a_off = first + min(j0 + n, len - 1) * tok + 4 * g;
    float ka[DH / 4], va[DH / 4];
    load_row<DH>(K, a_off, ka);
    load_row<DH>(V, a_off, va);
    floatx4 sc = {0.f, 0.f, 0.f, 0.f}, dp = {neg_d, neg_d, neg_d, neg_d};  // (dP starts from -D, which saves the subtractions)
    dot_rows<DH>(ka, va, qf, df, sc, dp);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int j = j0 + 4 * g + v;
      const float ds = __builtin_amdgcn_exp2f(fmaf(sc[v], p.scale_log2e, -lse2)) * dp[v];
      add_column<DH>(dq, K, first + min(j, len - 1) * tok + 4 * n, j < seen ? ds : 0.f);
    }
  }
  __shared__ float4 lds[kMeetWords<DH>];
  put_sums<DH>(lds, wave, lane, dq);
  __syncthreads();
  store_sums<DH>(lds, wave, lane, p.dQ, off, row_ok, p.scale);
}

template <int DH>
int launch_plain(const GradParams& p) {
  const int64_t blocks = (static_cast<int64_t>(p.max_q) + kPlainRows - 1) / kPlainRows, rows = blocks * p.H * p.B;
  // keys of every sequence, or of all rows where entries share them
  const int64_t nug_rows = p.shared ? p.Kt : p.max_k, loc_rows = p.shared ? p.Sm : p.max_local;
  const int64_t nug = (nug_rows + kPlainRows - 1) / kPlainRows, loc = (loc_rows + kPlainRows - 1) / kPlainRows;
  const int64_t tiles = (nug + loc) * p.H_kv * (p.shared ? 1 : p.B);
  if (tiles > 0x7fffffffLL || rows > 0x7fffffffLL) return DODO_ERR_UNSUPPORTED;
  if (rows > 0) {  // (first: it makes the rows' statistics)
    hipLaunchKernelGGL(HIP_KERNEL_NAME(grad_q_plain_kernel<DH>), dim3(static_cast<unsigned>(rows)), dim3(kGradThreads), 0, p.stream, p,
                       static_cast<int>(blocks));
    const int rc = launch_status();
    if (rc != DODO_OK) return rc;
  }
  if (tiles == 0) return DODO_OK;
  hipLaunchKernelGGL(HIP_KERNEL_NAME(grad_kv_plain_kernel<DH>), dim3(static_cast<unsigned>(tiles)), dim3(kGradThreads), 0, p.stream, p,
                     static_cast<int>(nug), static_cast<int>(loc));
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
