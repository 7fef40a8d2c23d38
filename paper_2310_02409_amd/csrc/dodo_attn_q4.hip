// dodo_nugget_attention_q4: nugget attention (Eq. 13 / Eq. 9 of the Dodo paper) over a nugget cache held in 4 bits.
//
// Few query rows (bf16): one kernel reads the codes where they are, a quarter of a bf16 cache's bytes, and every one once for
// 16 or 32 query vectors.  A workgroup owns a share of the keys of one (sequence, K/V head, group of query rows); each of its four or eight
// wavefronts takes tiles of 32 keys of it, without a barrier in the loop:
//   K      codes go straight to registers: the sum over channels may run in any order, so a lane takes consecutive channels of
//          its key, whose codes are one load and whose scale is one byte (two bytes for 64 channels), and the query vectors'
//          fragments follow that order.  A conversion turns two codes into two bf16 numbers, scale included, exactly.
//   S^T = K Q^T, online softmax in base 2, O^T += V^T P^T with the weights in two bf16 parts: as in dodo_attn_group.h and .hip
//   V      has to be turned around: its codes are converted as they come (32 channels, one scale a lane), written to LDS and read back
//          through the transposing read.
// Local rows, which are bf16, go through the same LDS by direct loads, K and V in turn, each requested as soon as its half of
// the wavefront's LDS has been read.  The next tile's codes are loaded while a tile is worked on.  Wavefronts merge in LDS; where the
// keys are shared out, every workgroup writes its partial results, counts itself, and the last to come merges all of them in
// order of their shares: nothing waits, and the order of the sums does not depend on who is last.
//
// What bounds it: memory where the cache is large (a decode step of 32 ragged sequences, 64 heads over 8, up to 3277 nuggets: 34.4
// to 35.8 us over fresh caches, 3.4 TB/s; 32 equal ones 40 us, 3.7 TB/s, by heads 33 us, 4.4 TB/s, since token by token a head's codes are half
// a cache line); a chain of latencies where it is small (1 sequence, 32 heads, 410 nuggets 8.3 us: ranges, queries and codes, a tile or
// two, the shares' meeting).
//
// Many query rows, other types: the cache is unpacked into the workspace and attended over from there; bad blocks (scale byte 255) make NaN of
// the same rows there.
#include <algorithm>
#include <type_traits>

#include "dodo_attn_group.h"
#include "dodo_q4.h"

namespace dodo {
namespace {

constexpr int kKeysQ4 = 32;                 // keys per tile
constexpr int kVectorsQ4 = 32;              // query vectors per workgroup at most
constexpr int kMostVectorsQ4 = 128;         // ... and of a K/V head and sequence, where there are many rows
constexpr int kCounters = DODO_Q4_ZEROED_BYTES / 4;  // words at the workspace's start, one per (sequence, K/V head, group of query rows)
constexpr int kMaxSplitsQ4 = 32;

template <int DH, int NV>
struct Q4Dims {
  static constexpr int kRowBytes = DH * 2;            // of a bf16 row in LDS
  static constexpr int kP = kRowBytes / 16;           // 16-byte pieces of it
  static constexpr int kRowShift = DH == 128 ? 0 : 1; // rows of 128 bytes cover half of the banks: swizzles take them in pairs
  static constexpr int kCB = DH / NV;                 // blocks of NV channels, each a granule of 2 NV bytes of a V row
  static constexpr int kGranPieces = NV / 8;
  static constexpr int kGroups = kWave / NV;          // lanes per key: each has a run of DH / kGroups channels
  static constexpr int kRun = DH / kGroups;
  static constexpr int kSteps = kRun / 8;             // products per key block
  static constexpr int kKeyBlocks = kKeysQ4 / NV;
  static constexpr int kPvSteps = NV / 16;
  static constexpr int kRowsPerInstr = 64 / kP;       // rows that a direct load brings
  static constexpr int kInstr = kKeysQ4 / kRowsPerInstr;
  static constexpr int kTensorBytes = kKeysQ4 * kRowBytes;
  static constexpr int kPartStride = DH + 4;          // floats per vector of a partial in LDS (spreads the banks)
  static constexpr int kPartBytes = (NV * kPartStride + 2 * NV) * 4;
  static constexpr int kWaveLds = ((2 * kTensorBytes > kPartBytes ? 2 * kTensorBytes : kPartBytes) + 1023) / 1024 * 1024;
  static constexpr int kQBytes = NV * kRowBytes;
  static constexpr int lds_bytes(int waves) { return waves * kWaveLds + kQBytes; }
  static_assert(2 * lds_bytes(4) <= 160 * 1024 && lds_bytes(8) <= 160 * 1024, "two workgroups of four wavefronts on a compute unit, or one of eight");
  static_assert((2 * NV * kMaxSplitsQ4 + 3 * NV) * 4 <= kWaveLds, "the merge's staging fits into a wavefront's LDS");
};

struct Q4Args {
  const uint16_t *Q, *Kl, *Vl;
  const uint8_t *Kc, *Ks, *Vc, *Vs;
  const int32_t *cu_q, *cu_nuggets, *cu_local;
  int B, H, H_kv, G, max_q, rows_per, n_groups, nsplit;
  int heads_per_unit, n_units;           // K/V heads that go to one XCD together, and the units of so many heads
  FastDiv div_G;
  int nug_cost, loc_cost;                // of a tile, for the shares
  int64_t row_stride, head_stride;       // of the nugget cache, in rows and heads of DH / 2 bytes of codes
  float scale_log2e;
  uint16_t* O;
  float* lse;
  uint32_t* counters;
  uint64_t* records;                     // [pair][vector][split][(DH + 2) / 2] words: m and s, then the channels
};

template <int N>
struct Codes {
  uint32_t w[N];
};
// N words of codes: 8 bytes, or 16 or 32 in pieces of 16, aligned to the piece
template <int N>
__device__ __forceinline__ Codes<N> load_codes(const uint8_t* p) {
  Codes<N> c;
  if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    c.w[0] = v.x; c.w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[i];
      c.w[4 * i] = v.x; c.w[4 * i + 1] = v.y; c.w[4 * i + 2] = v.z; c.w[4 * i + 3] = v.w;
    }
  }
  return c;
}
template <int DH, int NV, int NW>
__global__ __launch_bounds__(NW * kWave, 2) void attention_q4_kernel(Q4Args a) {
  using QD = Q4Dims<DH, NV>;
  using Acc = typename Mfma<NV>::Acc;
  constexpr int kRowBytes = QD::kRowBytes, kP = QD::kP, kRowShift = QD::kRowShift, kCB = QD::kCB, kSteps = QD::kSteps;
  constexpr int kInstr = QD::kInstr, kRowsPerInstr = QD::kRowsPerInstr, kTensorBytes = QD::kTensorBytes, kWaveLds = QD::kWaveLds;
  constexpr int kPartStride = QD::kPartStride, kPARTS = 2;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  // Block i runs on XCD i % 8.  A unit is a share of the keys of some neighbouring K/V heads of a sequence: token by token their codes
  // and scales lie in the same cache lines, which one XCD's L2 then fetches once.
  const int slot = blockIdx.x >> 3, unit = slot / a.heads_per_unit * 8 + (blockIdx.x & 7);
  if (unit >= a.n_units) return;
  const int per_seq = a.H_kv / a.heads_per_unit, rest = unit / per_seq, z = rest / a.B;
  const int kvh = unit % per_seq * a.heads_per_unit + slot % a.heads_per_unit, b = rest % a.B, split = z % a.nsplit, group = z / a.nsplit;
  const int q0 = a.cu_q[b], q_end = a.cu_q[b + 1], k0 = a.cu_nuggets[b], k_end = a.cu_nuggets[b + 1], l0 = a.cu_local[b], l_end = a.cu_local[b + 1];
  asm volatile("" ::"s"(q0), "s"(q_end), "s"(k0), "s"(k_end), "s"(l0), "s"(l_end));  // one round of loads
  const int q_b = min(q_end - q0, a.max_q), k_b = k_end - k0, m_b = l_end - l0, row0 = group * a.rows_per;
  if (q_b <= row0) return;  // uniform over the shares: nothing to write, nobody counts
  const int q_cnt = min(a.rows_per, q_b - row0), G = a.G, nv = q_cnt * G;  // vector v: row row0 + v / G, head kvh * G + v % G

  const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int j = lane % NV, g = lane / NV;
  const int my_i = row0 + static_cast<int>(fast_div(static_cast<uint32_t>(j < nv ? j : 0), a.div_G));
  const int wg_vis = max(0, min(m_b, m_b - q_b + row0 + q_cnt));  // local rows that the group's last row sees
  const int my_vis = max(0, min(m_b, m_b - q_b + my_i + 1));      // (spare lanes: vector 0's)

  // this workgroup's share of the tiles: by cost, the nuggets' first
  const int n_nug = (k_b + kKeysQ4 - 1) / kKeysQ4, n_loc = (wg_vis + kKeysQ4 - 1) / kKeysQ4, n_tiles = n_nug + n_loc;
  const int total = n_nug * a.nug_cost + n_loc * a.loc_cost;
  const auto tile_at = [&](int s) {  // first tile at or behind the cost of s shares
    const int c = static_cast<int>(static_cast<int64_t>(total) * s / a.nsplit);
    return c <= n_nug * a.nug_cost ? (c + a.nug_cost - 1) / a.nug_cost : n_nug + (c - n_nug * a.nug_cost + a.loc_cost - 1) / a.loc_cost;
  };
  const int t0 = a.nsplit == 1 ? 0 : tile_at(split), t1 = a.nsplit == 1 ? n_tiles : tile_at(split + 1);
  const int nug_end = min(t1, n_nug);
  // tiles t0 + wave, t0 + wave + NW, ...: first nuggets, then (from local tile l_first on) local rows
  const int first = t0 + wave;
  const int skip = first < n_nug ? (n_nug - first + NW - 1) / NW * NW : 0;
  const int l_first = first + skip - n_nug, l_end_tile = t1 - n_nug;

  char* const lds_w = lds + wave * kWaveLds;
  const uint32_t lds_addr = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds)), lds_w_addr = lds_addr + static_cast<uint32_t>(wave * kWaveLds);
  const int ld_row0 = lane / kP;
  const uint32_t ld_pos = lane % kP;
  auto k_piece_of = [&](int row) -> uint32_t { return (ld_pos ^ ((row >> kRowShift) & (kP - 1))) * 16u; };
  auto v_piece_of = [&](int row) -> uint32_t {
    return (((ld_pos / QD::kGranPieces) ^ ((row >> kRowShift) & (kCB - 1))) * QD::kGranPieces + ld_pos % QD::kGranPieces) * 16u;
  };
  const uint32_t loc_stride = static_cast<uint32_t>(a.H_kv) * kRowBytes;
  // K (or V) of local tile t into its half of the wavefront's LDS
  auto issue_local = [&](int t, auto v_tag) {
    constexpr bool IS_V = decltype(v_tag)::value;
    const int cnt = min(kKeysQ4, m_b - t * kKeysQ4);
    const uint16_t* from = (IS_V ? a.Vl : a.Kl) + (static_cast<int64_t>(l0 + t * kKeysQ4) * a.H_kv + kvh) * DH;
    const u32x4_t buf = buffer_of(from, static_cast<uint32_t>(cnt - 1) * loc_stride + kRowBytes);
#pragma unroll
    for (int u = 0; u < kInstr; ++u) {
      const int row = ld_row0 + kRowsPerInstr * u;
      dma16_buffer(buf, static_cast<uint32_t>(row) * loc_stride + (IS_V ? v_piece_of(row) : k_piece_of(row)),
                   __builtin_amdgcn_readfirstlane(lds_w_addr + (IS_V ? kTensorBytes : 0) + u * 1024));
    }
  };
  using IsK = std::false_type;
  using IsV = std::true_type;

  // The query vectors go through LDS; every wavefront brings a part of them.
  {
    constexpr int kQInstr = (QD::kQBytes / 1024 + NW - 1) / NW;
    const u32x4_t qbuf = buffer_of(a.Q + (static_cast<int64_t>(q0 + row0) * a.H + kvh * G) * DH, 0xffffffffu);
#pragma unroll
    for (int u = 0; u < kQInstr; ++u) {
      const int chunk = min(wave * kQInstr + u, QD::kQBytes / 1024 - 1);
      const int v = chunk * kRowsPerInstr + ld_row0, jv = v < nv ? v : 0;  // spare rows repeat vector 0; nothing of them is stored
      const int il = static_cast<int>(fast_div(static_cast<uint32_t>(jv), a.div_G));
      dma16_buffer(qbuf, static_cast<uint32_t>(il * a.H + jv - il * G) * kRowBytes + k_piece_of(v),
                   __builtin_amdgcn_readfirstlane(lds_addr + NW * kWaveLds + chunk * 1024));
    }
  }
  if (l_first < l_end_tile) issue_local(l_first, IsK{});  // (nuggets' K does not touch that half)

  // codes and scales of a nugget tile: K of key j (and j + 16), channels kRun g ..; V of row r, block blk
  constexpr int kKWords = QD::kRun / 8, kKScales = QD::kRun >= kBlockQ4 ? QD::kRun / kBlockQ4 : 1;
  constexpr int kBlocks = DH / kBlockQ4, kVRows = kWave / kBlocks, kVPasses = kKeysQ4 / kVRows;
  struct Tile {
    Codes<kKWords> k[QD::kKeyBlocks];
    Codes<4> v[kVPasses];
    uint32_t ks[QD::kKeyBlocks][kKScales], vs[kVPasses];
  };
  const int64_t nug_row0 = static_cast<int64_t>(k0) * a.row_stride + kvh * a.head_stride;
  const int v_blk = lane % kBlocks, v_row = lane / kBlocks;
  auto load_tile = [&](int t) {
    Tile x;
#pragma unroll
    for (int kb = 0; kb < QD::kKeyBlocks; ++kb) {
      const int64_t row = nug_row0 + min(t * kKeysQ4 + NV * kb + j, k_b - 1) * a.row_stride;
      x.k[kb] = load_codes<kKWords>(a.Kc + row * (DH / 2) + g * (QD::kRun / 2));
#pragma unroll
      for (int c = 0; c < kKScales; ++c) x.ks[kb][c] = a.Ks[row * kBlocks + g * QD::kRun / kBlockQ4 + c];
    }
#pragma unroll
    for (int c = 0; c < kVPasses; ++c) {
      const int64_t row = nug_row0 + min(t * kKeysQ4 + kVRows * c + v_row, k_b - 1) * a.row_stride;
      x.v[c] = load_codes<4>(a.Vc + row * (DH / 2) + v_blk * 16);
      x.vs[c] = a.Vs[row * kBlocks + v_blk];
    }
    return x;
  };
  // One tile ahead (2 and 3 are no faster); none where the wide tiles of 128 channels leave no registers for two workgroups on a compute
  // unit with it (8 sequences, 32 rows of 32 heads, 410 nuggets 30.1 -> 22.0 us).
  constexpr int kTilesAhead = DH * NV > 2048 ? 0 : 1;
  Tile buf[kTilesAhead + 1];
#pragma unroll
  for (int c = 0; c < kTilesAhead; ++c)
    if (first + c * NW < nug_end) buf[c] = load_tile(first + c * NW);
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  __syncthreads();  // every wavefront's part of the query vectors has landed
  bf16x8 qf[kSteps];  // lane (j, g): channels kRun g + 8 ds .. + 8 of its vector
  {
    const char* q_lds = lds + NW * kWaveLds + j * kRowBytes;
#pragma unroll
    for (int ds = 0; ds < kSteps; ++ds)
      qf[ds] = *reinterpret_cast<const bf16x8*>(q_lds + (((kSteps * g + ds) ^ ((j >> kRowShift) & (kP - 1))) << 4));
  }

  Acc acc_o[kCB];
#pragma unroll
  for (int cb = 0; cb < kCB; ++cb)
#pragma unroll
    for (int v = 0; v < Mfma<NV>::kRegs; ++v) acc_o[cb][v] = 0.f;
  float m_run = kNegInf, l_run = 0.f;
  const int v_r = 4 * g + ((lane & 15) >> 2);  // V^T through the transposing read: see dodo_attn_group.hip
  const int v_in = (NV == 32 ? 32 * ((lane >> 4) & 1) : 0) + 8 * (lane & 3);
  constexpr int kRegs = QD::kKeyBlocks * Mfma<NV>::kRegs;
  const char *kbuf = lds_w, *vbuf = lds_w + kTensorBytes;
  auto softmax = [&](Acc (&acc_s)[QD::kKeyBlocks], int limit, bf16x8 (&pf)[kPARTS][kRegs / 8]) {
    float sv[kRegs];
#pragma unroll
    for (int v = 0; v < kRegs; ++v) sv[v] = acc_s[v / Mfma<NV>::kRegs][v % Mfma<NV>::kRegs];
    if (__all(limit >= kKeysQ4)) {
      softmax_tile32<false, NV>(sv, limit, g, a.scale_log2e, m_run, l_run, acc_o, pf, 0x1p-126f);
    } else {
      softmax_tile32<true, NV>(sv, limit, g, a.scale_log2e, m_run, l_run, acc_o, pf, 0x1p-126f);
    }
  };
  auto read_v = [&](bf16x8 (&vt)[QD::kPvSteps][kCB]) {
#pragma unroll
    for (int t = 0; t < QD::kPvSteps; ++t)
#pragma unroll
      for (int cb = 0; cb < kCB; ++cb) {
        shortx4 half[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = 16 * t + (NV == 32 ? 8 : 16) * e + v_r;
          const char* p = vbuf + r * kRowBytes + ((cb ^ ((r >> kRowShift) & (kCB - 1))) * (2 * NV)) + v_in;
          half[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shortx4 __attribute__((address_space(3)))*)(p));
        }
        vt[t][cb] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
      }
  };
  auto add_v = [&](const bf16x8 (&vt)[QD::kPvSteps][kCB], const bf16x8 (&pf)[kPARTS][kRegs / 8]) {
#pragma unroll
    for (int part = 0; part < kPARTS; ++part)
#pragma unroll
      for (int t = 0; t < QD::kPvSteps; ++t)
#pragma unroll
        for (int cb = 0; cb < kCB; ++cb) acc_o[cb] = Mfma<NV>::mul(vt[t][cb], pf[part][t], acc_o[cb]);
  };
  auto clear = [&](Acc (&acc_s)[QD::kKeyBlocks]) {
#pragma unroll
    for (int kb = 0; kb < QD::kKeyBlocks; ++kb)
#pragma unroll
      for (int v = 0; v < Mfma<NV>::kRegs; ++v) acc_s[kb][v] = 0.f;
  };

  // ---- nuggets ----
  auto nugget_tile = [&](int t, const Tile& x) {
    // V on its way to be turned around: 32 channels of a row per lane and pass
#pragma unroll
    for (int c = 0; c < kVPasses; ++c) {
      const int r = kVRows * c + v_row;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int piece = 4 * v_blk + i, gran = piece / QD::kGranPieces;
        *reinterpret_cast<uint4*>(lds_w + kTensorBytes + r * kRowBytes +
                                  (((gran ^ ((r >> kRowShift) & (kCB - 1))) * QD::kGranPieces + piece % QD::kGranPieces) << 4)) = unpack8_bf16(x.v[c].w[i], scale_q4(x.vs[c]));
      }
    }
    Acc acc_s[QD::kKeyBlocks];
    clear(acc_s);
#pragma unroll
    for (int ds = 0; ds < kSteps; ++ds)
#pragma unroll
      for (int kb = 0; kb < QD::kKeyBlocks; ++kb)
        acc_s[kb] = Mfma<NV>::mul(__builtin_bit_cast(bf16x8, unpack8_bf16(x.k[kb].w[ds], scale_q4(x.ks[kb][8 * ds / kBlockQ4 % kKScales]))), qf[ds], acc_s[kb]);
    bf16x8 pf[kPARTS][kRegs / 8], vt[QD::kPvSteps][kCB];
    softmax(acc_s, k_b - t * kKeysQ4, pf);
    read_v(vt);
    add_v(vt, pf);
  };
  for (int t = first; t < nug_end; t += (kTilesAhead + 1) * NW) {
#pragma unroll
    for (int c = 0; c <= kTilesAhead; ++c) {  // (every buffer has its registers: a copy would wait for the tile)
      const int now = t + c * NW, then = now + kTilesAhead * NW;
      if (now >= nug_end) break;
      if (then < nug_end) buf[(c + kTilesAhead) % (kTilesAhead + 1)] = load_tile(then);
      nugget_tile(now, buf[c]);
    }
  }
  // ---- local rows ----
  if (l_first < l_end_tile) {
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): V's half has been read
    __builtin_amdgcn_sched_barrier(0);
    issue_local(l_first, IsV{});
  }
  for (int t = l_first; t < l_end_tile; t += NW) {
    const bool more = t + NW < l_end_tile;
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(kInstr));  // K has landed, V may be in flight
    asm volatile("" ::: "memory");
    bf16x8 kf[QD::kKeyBlocks][kSteps];
#pragma unroll
    for (int kb = 0; kb < QD::kKeyBlocks; ++kb)
#pragma unroll
      for (int ds = 0; ds < kSteps; ++ds)
        kf[kb][ds] = *reinterpret_cast<const bf16x8*>(kbuf + (NV * kb + j) * kRowBytes + (((kSteps * g + ds) ^ (((NV * kb + j) >> kRowShift) & (kP - 1))) << 4));
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
    if (more) issue_local(t + NW, IsK{});
    __builtin_amdgcn_sched_barrier(0);
    Acc acc_s[QD::kKeyBlocks];
    clear(acc_s);
#pragma unroll
    for (int ds = 0; ds < kSteps; ++ds)
#pragma unroll
      for (int kb = 0; kb < QD::kKeyBlocks; ++kb) acc_s[kb] = Mfma<NV>::mul(kf[kb][ds], qf[ds], acc_s[kb]);
    bf16x8 pf[kPARTS][kRegs / 8], vt[QD::kPvSteps][kCB];
    softmax(acc_s, my_vis - t * kKeysQ4, pf);
    if (more) {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(kInstr));  // V has landed, the next K may be in flight
    } else {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    }
    asm volatile("" ::: "memory");
    read_v(vt);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
    if (more) issue_local(t + NW, IsV{});
    __builtin_amdgcn_sched_barrier(0);
    add_v(vt, pf);
  }

  // ---- the wavefronts' partials meet in LDS: [vector][channel] floats, then m and l per vector ----
  {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // (a wavefront without local tiles has none in flight)
    float* part = reinterpret_cast<float*>(lds_w);
    const float l_tot = vector_sum<NV>(l_run);
#pragma unroll
    for (int cb = 0; cb < kCB; ++cb)
#pragma unroll
      for (int qd = 0; qd < Mfma<NV>::kRegs / 4; ++qd)
        *reinterpret_cast<float4*>(part + j * kPartStride + NV * cb + 8 * qd + 4 * g) =
            make_float4(acc_o[cb][4 * qd], acc_o[cb][4 * qd + 1], acc_o[cb][4 * qd + 2], acc_o[cb][4 * qd + 3]);
    if (g == 0) {
      part[NV * kPartStride + j] = m_run;
      part[NV * kPartStride + NV + j] = l_tot;
    }
  }
  __syncthreads();
  // Four neighbouring channels of a vector, the wavefronts merged in wavefront order.  A part without keys has m = -inf, a sum of 0 and
  // channels 0; one whose logits are NaN may have m = -inf as well, but its sum is NaN and stays so.
  auto merged = [&](int v, int c, float& M, float& S, float4& o) {
    float mw[NW];
    M = kNegInf;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      mw[w] = reinterpret_cast<const float*>(lds + w * kWaveLds)[NV * kPartStride + v];
      M = fmaxf(M, mw[w]);
    }
    S = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float* part = reinterpret_cast<const float*>(lds + w * kWaveLds);
      const float wgt = exp2_hw(mw[w] - (M == kNegInf ? 0.f : M));
      S = fmaf(part[NV * kPartStride + NV + v], wgt, S);
      const float4 p = *reinterpret_cast<const float4*>(part + v * kPartStride + c);
      o.x = fmaf(p.x, wgt, o.x); o.y = fmaf(p.y, wgt, o.y); o.z = fmaf(p.z, wgt, o.z); o.w = fmaf(p.w, wgt, o.w);
    }
  };
  auto store_out = [&](int v, int c, const float4& o, float S, float M) {
    const int il = static_cast<int>(fast_div(static_cast<uint32_t>(v), a.div_G));
    const int64_t out_row = static_cast<int64_t>(q0 + row0 + il) * a.H + kvh * G + (v - il * G);
    const float inv = S == 0.f ? 0.f : 1.f / S;  // (a row that sees nothing: 0; a NaN stays one)
    *reinterpret_cast<uint2*>(a.O + out_row * DH + c) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    if (a.lse != nullptr && c == 0) a.lse[out_row] = S == 0.f ? kNegInf : ((M == kNegInf ? 0.f : M) + __log2f(S)) * 0.6931471805599453f;
  };
  const int n_quads = nv * (DH / 4);
  if (a.nsplit == 1) {
    for (int e = tid; e < n_quads; e += NW * kWave) {
      const int v = e / (DH / 4), c = 4 * (e % (DH / 4));
      float M, S;
      float4 o;
      merged(v, c, M, S, o);
      store_out(v, c, o, S, M);
    }
    return;
  }
  // ---- shares: every workgroup writes its partial results and counts itself, the last one merges them all ----
  constexpr int kWords = (DH + 2) / 2;
  const int64_t pair = (static_cast<int64_t>(b) * a.H_kv + kvh) * a.n_groups + group;
  uint64_t* const recs = a.records + pair * (min(a.rows_per, a.max_q) * G) * a.nsplit * kWords;
  auto word_of = [](float lo, float hi) -> uint64_t { return static_cast<uint64_t>(__float_as_uint(hi)) << 32 | __float_as_uint(lo); };
  auto lo_of = [](uint64_t w) -> float { return __uint_as_float(static_cast<uint32_t>(w)); };
  auto hi_of = [](uint64_t w) -> float { return __uint_as_float(static_cast<uint32_t>(w >> 32)); };
  for (int e = tid; e < n_quads; e += NW * kWave) {
    const int v = e / (DH / 4), c = 4 * (e % (DH / 4));
    float M, S;
    float4 o;
    merged(v, c, M, S, o);
    uint64_t* rec = recs + (static_cast<int64_t>(v) * a.nsplit + split) * kWords;
    if (c == 0) __hip_atomic_store(rec, word_of(M, S), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(rec + 1 + c / 2, word_of(o.x, o.y), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(rec + 2 + c / 2, word_of(o.z, o.w), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // this thread's stores are acknowledged
  __syncthreads();                            // ... and everyone's; the partials in LDS have been read
  int* const come = reinterpret_cast<int*>(lds);
  if (tid == 0) *come = static_cast<int>(__hip_atomic_fetch_add(a.counters + pair, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  __syncthreads();
  if (*come != a.nsplit - 1) return;
  if (tid == 0) __hip_atomic_store(a.counters + pair, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next call
  float* const st_m = reinterpret_cast<float*>(lds + kWaveLds);  // [vector][split]: exponent offsets, then weights
  float* const st_s = st_m + NV * kMaxSplitsQ4;
  float* const tot_s = st_s + NV * kMaxSplitsQ4;
  float* const tot_m = tot_s + NV;
  for (int f = tid; f < nv * a.nsplit; f += NW * kWave) {
    const uint64_t ms = __hip_atomic_load(recs + static_cast<int64_t>(f) * kWords, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    st_m[f] = lo_of(ms);
    st_s[f] = hi_of(ms);
  }
  __syncthreads();
  if (tid < nv) {
    float M = kNegInf, S = 0.f;
    for (int sp = 0; sp < a.nsplit; ++sp) M = fmaxf(M, st_m[tid * a.nsplit + sp]);
    for (int sp = 0; sp < a.nsplit; ++sp) {
      const float w = exp2_hw(st_m[tid * a.nsplit + sp] - (M == kNegInf ? 0.f : M));
      st_m[tid * a.nsplit + sp] = w;
      S = fmaf(st_s[tid * a.nsplit + sp], w, S);
    }
    tot_s[tid] = S;
    tot_m[tid] = M;
  }
  __syncthreads();
  for (int e = tid; e < n_quads; e += NW * kWave) {
    const int v = e / (DH / 4), c = 4 * (e % (DH / 4));
    const uint64_t* rec = recs + static_cast<int64_t>(v) * a.nsplit * kWords + 1 + c / 2;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kBatch = 8;  // records requested before the first is used
    for (int s0 = 0; s0 < a.nsplit; s0 += kBatch) {
      uint64_t w0[kBatch], w1[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const uint64_t* r = rec + static_cast<int64_t>(min(s0 + u, a.nsplit - 1)) * kWords;
        w0[u] = __hip_atomic_load(r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        w1[u] = __hip_atomic_load(r + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (s0 + u < a.nsplit) {
          const float w = st_m[v * a.nsplit + s0 + u];
          o.x = fmaf(lo_of(w0[u]), w, o.x);
          o.y = fmaf(hi_of(w0[u]), w, o.y);
          o.z = fmaf(lo_of(w1[u]), w, o.z);
          o.w = fmaf(hi_of(w1[u]), w, o.w);
        }
    }
    store_out(v, c, o, tot_s[v], tot_m[v]);
  }
}

__global__ void clear_words_kernel(uint32_t* __restrict__ p, int64_t n) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i < n) p[i] = 0u;
}

// Unpacked caches: the attention kernels know nothing of bad blocks, which the unpacking has put into V, so that their log-sum-exp is made
// NaN afterwards, where the caller asks for it.  A workgroup looks through up to kMarked scales of K of a sequence and K/V head; all that
// find one write the same.  3 us for a sequence of 410 nuggets, 32 heads of 128, 5 for 8 of them or for 32 of 3277, 8 heads.
constexpr int kMarkThreads = 256, kMarked = 4 * kMarkThreads;
template <int BLOCKS>
__global__ __launch_bounds__(kMarkThreads) void mark_lse_kernel(const uint8_t* __restrict__ Ks, const int32_t* __restrict__ cu_q,
                                                                const int32_t* __restrict__ cu_nuggets, int64_t n_items, int n_parts, int H_kv, int G,
                                                                int64_t row_stride, int64_t head_stride, float* __restrict__ lse) {
  for (int64_t item = blockIdx.x; item < n_items; item += gridDim.x) {
    const int64_t part = item % n_parts, pair = item / n_parts, b = pair / H_kv, kvh = pair % H_kv;
    const int64_t q0 = cu_q[b], q_end = cu_q[b + 1], k0 = cu_nuggets[b], k_end = cu_nuggets[b + 1];
    if (q_end <= q0) continue;
    int bad = 0;
#pragma unroll 4
    for (int64_t i = k0 + part * kMarkThreads + threadIdx.x; i < k_end; i += static_cast<int64_t>(n_parts) * kMarkThreads)
      bad |= any_bad_q4(row_scales_q4<BLOCKS>(Ks, i * row_stride + kvh * head_stride)) ? 1 : 0;
    if (!__syncthreads_or(bad)) continue;
    for (int64_t i = threadIdx.x; i < (q_end - q0) * G; i += kMarkThreads) lse[((q0 + i / G) * H_kv + kvh) * G + i % G] = __builtin_nanf("");
  }
}

constexpr int kNugCost = 1, kLocCost = 2;

// How the direct kernel would take a call (bf16, d_h 64 or 128, at most kVectorsQ4 heads per K/V head).
struct Plan {
  bool direct, narrow;  // narrow: groups of up to 16 vectors
  int rows_per, n_groups, nsplit, waves;
  size_t records;  // bytes behind the counters
};
Plan plan_of(int64_t B, int32_t H, int32_t H_kv, int32_t d_h, int32_t max_q, int32_t max_k, int32_t max_local, int dtype) {
  Plan p = {};
  const int64_t G = H / H_kv;
  // Up to 128 vectors a K/V head, and up to 15 rows whatever the heads; beyond, where the vectors read the cache several times, unpacking it
  // once is the faster.  Here / unpacked, us, 257 local rows: 8 sequences, 32 heads over 32, 410 nuggets, 16 rows 13.8 / 33.6, 64 22.6 / 35.7,
  // 128 38.5 / 41.6, 256 68.0 / 46.7; 32 sequences, 32 rows 53 / 120, 64 91 / 126, 128 153 / 136; 64 heads over 8, 3277 nuggets, 16 rows 15.1 /
  // 27.5, 8 sequences of it 44.6 / 63.0.
  if (dtype != DODO_DTYPE_BF16 || G > kVectorsQ4 || (max_q >= DODO_ATTENTION_BLOCK_MIN_Q && max_q * G > kMostVectorsQ4)) return p;
  if (static_cast<int64_t>(B) * H_kv > 1 << 22) return p;  // (the grid, with up to 32 shares and 15 groups of rows)
  if (static_cast<int64_t>(H) * d_h >= 1 << 24) return p;  // (offsets between rows of a tile in 32 bits)
  p.direct = true;
  p.waves = 4;
  // Groups of 16 vectors where that leaves no compute unit with more than two workgroups, else of 32, which read the cache half as often.
  // 16 / 32: 8 sequences, 32 heads, 410 nuggets, 257 local rows: 32 rows 17.3 / 22.0 us, 64 rows 30.6 / 22.6; 32 sequences, 32 rows 77.2 / 54.0;
  // 64 heads over 8, 4 rows, 3277 nuggets, 1 sequence 14.9 / 19.7, 8 22.4 / 24.2.
  const int64_t narrow_groups = (max_q * G + 15) / 16;
  p.narrow = G <= 16 && (max_q * G <= 16 || static_cast<int64_t>(B) * H_kv * narrow_groups <= 2 * compute_units());
  p.rows_per = static_cast<int>((p.narrow ? 16 : kVectorsQ4) / G);
  if (p.rows_per > max_q) p.rows_per = max_q;
  p.n_groups = (max_q + p.rows_per - 1) / p.rows_per;
  const int64_t pairs = static_cast<int64_t>(B) * H_kv * p.n_groups, cus = compute_units(), vectors = p.rows_per * G;
  const int64_t cost = (static_cast<int64_t>(max_k) + kKeysQ4 - 1) / kKeysQ4 * kNugCost + (static_cast<int64_t>(max_local) + kKeysQ4 - 1) / kKeysQ4 * kLocCost;
  // The count of least expected time, in ns: a wavefront takes 900 for a tile of nuggets (twice that in the wide form) and as
  // much again for a local one, half as much again where two workgroups share a compute unit; shares cost 2000, and the last workgroup
  // reads 13 ns worth of records for each share and vector.  64 heads over 8, 3277 nuggets, 257 local rows: 1 sequence 13.5 / 11.4 / 10.9
  // us in 28 / 14 / 16 shares, 2 of them with 1089 local rows 18.3 / 13.3 / 13.6 in 32 / 16 / 8, 8 15.4 / 16.6 in 8 / 4; 32 over 32, 410
  // nuggets, 1 sequence 8.7 / 10.6 in 5 / 2, 8 with 4 rows 13.0 / 14.5 in 1 / 2, 16 22.9 / 28.3 in 1 / 2.
  int64_t n = 1, best = 0;
  for (int64_t s = 1; s <= kMaxSplitsQ4 && (s == 1 || (pairs <= kCounters && s * p.waves <= cost)); ++s) {
    const int64_t workgroups = pairs * s;
    const int64_t tile = (p.narrow ? 900 : 1800) * (workgroups <= cus ? 2 : 3) / 2;
    const int64_t units = std::max<int64_t>((cost + s * p.waves - 1) / (s * p.waves), max_local > 0 ? kLocCost : kNugCost);
    const int64_t ns = std::max(units * tile, units * tile * workgroups / (2 * cus)) + (s == 1 ? 0 : 2000 + 13 * s * vectors);
    if (s == 1 || ns < best) {
      n = s;
      best = ns;
    }
  }
  // Two shares in one workgroup of eight wavefronts, which meet in LDS instead of memory, where there are many records to merge or at least
  // four tiles a wavefront.  Four / eight wavefronts, us (64 heads over 8, 3277 nuggets, 257 local rows, unless said): 32 sequences 42.1 /
  // 40.4, 16 24.8 / 25.0, 8 15.4 / 15.3, of 4 rows 22.6 / 20.3, 2 of 8 rows 17.0 / 15.5; 32 heads over 32 12.6 / 12.0; 2 of 16 rows, 8 heads
  // of 64 over 2 11.9 / 10.3.  Short: 32 heads, 410 nuggets 8.4 / 10.0; 3 sequences of 500 and 500, 32 heads over 8 8.9 / 10.3.
  if (n % 2 == 0 && (vectors * n >= 64 || cost >= 16 * n)) {
    p.waves = 8;
    n /= 2;
  }
  p.nsplit = static_cast<int>(n);
  p.records = n == 1 ? 0 : static_cast<size_t>(pairs) * p.rows_per * G * n * (d_h + 2) * sizeof(float);
  return p;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
constexpr size_t kCounterBytes = kCounters * sizeof(uint32_t);

template <int DH, int NV, int NW>
int launch_direct(const Q4Args& a, hipStream_t stream) {
  constexpr int kLds = Q4Dims<DH, NV>::lds_bytes(NW);
  const auto kern = attention_q4_kernel<DH, NV, NW>;
  const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kern), kLds);
  if (rc != DODO_OK) return rc;
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>((a.n_units + 7) / 8 * 8 * a.heads_per_unit)), dim3(NW * kWave), kLds, stream, a);
  return launch_status();
}
template <int DH>
int launch_direct(const Q4Args& a, const Plan& plan, hipStream_t stream) {
  if (plan.waves == 8) return plan.narrow ? launch_direct<DH, 16, 8>(a, stream) : launch_direct<DH, 32, 8>(a, stream);
  return plan.narrow ? launch_direct<DH, 16, 4>(a, stream) : launch_direct<DH, 32, 4>(a, stream);
}

}  // namespace
}  // namespace dodo

extern "C" size_t dodo_nugget_attention_q4_workspace_bytes(int32_t B, int32_t H, int32_t H_kv, int32_t d_h, int32_t max_q,
                                                           int32_t max_k, int32_t max_local, int64_t Kt, int dtype) {
  using namespace dodo;
  if (B <= 0 || H <= 0 || H_kv <= 0 || H % H_kv != 0 || d_h <= 0 || max_q <= 0 || max_k < 0 || max_local < 0 || Kt < 0 || !dtype_ok(dtype)) return 0;
  const Plan plan = plan_of(B, H, H_kv, d_h, max_q, max_k, max_local, dtype);
  if (plan.direct) return plan.nsplit == 1 ? 0 : kCounterBytes + plan.records;
  const size_t attention = dodo_nugget_attention_workspace_bytes_grouped(B, H, H_kv, d_h, max_q, max_k, max_local, dtype);
  return kCounterBytes + round256(attention) + 2 * round256(static_cast<size_t>(Kt) * H_kv * d_h * elem_bytes(dtype));
}

extern "C" int dodo_nugget_attention_q4(const void* Q, const uint8_t* Kc, const uint8_t* Ks, const uint8_t* Vc, const uint8_t* Vs,
                                        const void* Kl, const void* Vl, const int32_t* cu_q, const int32_t* cu_nuggets,
                                        const int32_t* cu_local, int32_t B, int32_t H, int32_t H_kv, int32_t d_h, int32_t max_q,
                                        int32_t max_k, int32_t max_local, int64_t Kt, float softmax_scale, int dtype, int layout,
                                        void* O, float* lse, void* ws, size_t ws_bytes, void* stream) {
  using namespace dodo;
  if (B < 0 || H <= 0 || H_kv <= 0 || d_h <= 0 || max_q < 0 || max_k < 0 || max_local < 0 || Kt < 0) return DODO_ERR_INVALID_ARG;
  if (H % H_kv != 0) return DODO_ERR_INVALID_ARG;
  if (layout != DODO_LAYOUT_TOKEN_MAJOR && layout != DODO_LAYOUT_HEAD_MAJOR) return DODO_ERR_INVALID_ARG;
  if (!(softmax_scale == softmax_scale)) return DODO_ERR_INVALID_ARG;
  if (B == 0 || max_q == 0) return DODO_OK;
  if (!Q || !O || !cu_q || !cu_nuggets || !cu_local) return DODO_ERR_INVALID_ARG;
  if (Kt > 0 && max_k > 0 && (!Kc || !Ks || !Vc || !Vs)) return DODO_ERR_INVALID_ARG;
  if (max_local > 0 && (!Kl || !Vl)) return DODO_ERR_INVALID_ARG;
  if (!dtype_ok(dtype)) return DODO_ERR_UNSUPPORTED;
  if (d_h != 64 && d_h != 128) return DODO_ERR_UNSUPPORTED;
  if (!aligned16(Q) || !aligned16(O) || !aligned16(Kc) || !aligned16(Vc) || !aligned16(Kl) || !aligned16(Vl) || !aligned16(ws) ||
      ((reinterpret_cast<uintptr_t>(Ks) | reinterpret_cast<uintptr_t>(Vs)) & (d_h / kBlockQ4 - 1)) != 0)  // (2 or 4 scales a row and head)
    return DODO_ERR_UNSUPPORTED;
  const size_t need = dodo_nugget_attention_q4_workspace_bytes(B, H, H_kv, d_h, max_q, max_k, max_local, Kt, dtype);
  if (need > 0 && (!ws || ws_bytes < need)) return DODO_ERR_WORKSPACE_TOO_SMALL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const Plan plan = plan_of(B, H, H_kv, d_h, max_q, max_k, max_local, dtype);
  if (plan.direct) {
    Q4Args a = {};
    a.Q = static_cast<const uint16_t*>(Q); a.Kl = static_cast<const uint16_t*>(Kl); a.Vl = static_cast<const uint16_t*>(Vl);
    a.Kc = Kc; a.Ks = Ks; a.Vc = Vc; a.Vs = Vs;
    a.cu_q = cu_q; a.cu_nuggets = cu_nuggets; a.cu_local = cu_local;
    a.B = B; a.H = H; a.H_kv = H_kv; a.G = H / H_kv; a.max_q = max_q; a.rows_per = plan.rows_per; a.n_groups = plan.n_groups; a.nsplit = plan.nsplit;
    a.div_G = make_fast_div(static_cast<uint32_t>(a.G));
    a.nug_cost = kNugCost; a.loc_cost = kLocCost;
    a.row_stride = layout == DODO_LAYOUT_TOKEN_MAJOR ? H_kv : 1;
    a.head_stride = layout == DODO_LAYOUT_TOKEN_MAJOR ? 1 : Kt;
    a.scale_log2e = softmax_scale * 1.4426950408889634f;
    a.O = static_cast<uint16_t*>(O); a.lse = lse;
    a.counters = static_cast<uint32_t*>(ws);
    a.records = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + kCounterBytes);
    // As many heads to a unit as there are, but units for all of the eight XCDs alike.
    a.heads_per_unit = layout == DODO_LAYOUT_TOKEN_MAJOR ? H_kv : 1;
    const auto units = [&]() { return static_cast<int64_t>(B) * plan.nsplit * plan.n_groups * (H_kv / a.heads_per_unit); };
    while (a.heads_per_unit % 2 == 0 && units() % 8 != 0 && units() < 64) a.heads_per_unit /= 2;
    a.n_units = static_cast<int>(units());
    return d_h == 128 ? launch_direct<128>(a, plan, s) : launch_direct<64>(a, plan, s);
  }
  const size_t attention = dodo_nugget_attention_workspace_bytes_grouped(B, H, H_kv, d_h, max_q, max_k, max_local, dtype);
  const size_t cache = round256(static_cast<size_t>(Kt) * H_kv * d_h * elem_bytes(dtype));
  char* const att_ws = static_cast<char*>(ws) + kCounterBytes;
  char* const Kn = att_ws + round256(attention);
  char* const Vn = Kn + cache;
  if (Kt > 0 && max_k > 0) {
    const int rc = unpack_q4(Kc, Ks, Vc, Vs, Kt * H_kv, d_h, dtype, true, Kn, Vn, stream);
    if (rc != DODO_OK) return rc;
  }
  if (attention > 0 && !(dtype == DODO_DTYPE_BF16 && max_q >= DODO_ATTENTION_BLOCK_MIN_Q)) {  // flags among it, which have to be clear
    const int64_t words = static_cast<int64_t>(attention / 4);
    hipLaunchKernelGGL(clear_words_kernel, dim3(static_cast<unsigned>((words + 255) / 256)), dim3(256), 0, s, reinterpret_cast<uint32_t*>(att_ws), words);
    const int rc = launch_status();
    if (rc != DODO_OK) return rc;
  }
  const int rc = dodo_nugget_attention(Q, Kn, Vn, Kl, Vl, cu_q, cu_nuggets, cu_local, B, H, H_kv, d_h, max_q, max_k, max_local, Kt,
                                       softmax_scale, dtype, layout, O, lse, attention ? att_ws : nullptr, attention, stream);
  if (rc != DODO_OK || lse == nullptr || Kt == 0 || max_k == 0) return rc;
  const int64_t parts = (static_cast<int64_t>(max_k) + kMarked - 1) / kMarked, items = parts * B * H_kv;
  const auto mark = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(std::min<int64_t>(items, 1 << 20))), dim3(kMarkThreads), 0, s, Ks, cu_q, cu_nuggets, items,
                       static_cast<int>(parts), H_kv, H / H_kv, layout == DODO_LAYOUT_TOKEN_MAJOR ? static_cast<int64_t>(H_kv) : int64_t{1},
                       layout == DODO_LAYOUT_TOKEN_MAJOR ? int64_t{1} : Kt, lse);
  };
  if (d_h == 128) mark(mark_lse_kernel<4>); else mark(mark_lse_kernel<2>);
  return launch_status();
}
