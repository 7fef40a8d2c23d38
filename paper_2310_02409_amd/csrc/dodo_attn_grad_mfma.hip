// Gradients of nugget attention for bf16 inputs, on the bf16 matrix instructions (the formulas, and why there are two
// kernels, are in dodo_attn_grad.hip).
//
// Both kernels form 32 x 32 blocks of S and dP with v_mfma_f32_32x32x16_bf16 so that a lane owns a row of what the kernel sums (a key,
// or a query row) and the accumulators run over the rows it walks over.  P and dS, rounded to bf16, are then the right operand of
// the second product as they stand: accumulator v holds walked row 8 (v / 4) + 4 g + v % 4 (g = lane / 32), and the left operand
// takes the walked rows in that order.  The walked tile sits in LDS, 64 rows at a time, and is read in two ways: whole rows (16
// bytes a lane) for S and dP, and columns (transposing reads of 8 bytes) for the second products.  Its 16-byte pieces are
// swizzled so that both are free of bank conflicts.  The owned rows' fragments and the sums stay in registers.
//
// P and dS are rounded to bf16 once before the second products: half a step, 2^-8, of each term, which leaves the gradients
// an error of 2.4e-3 against 64 bits (2-norm; the rounding of the results alone gives 1.7e-3).  With what they lack as a second bf16 part
// the error is 1.7e-3, and the second products are done twice, with 20 to 40 registers more than there are in the kernel for dK and dV.
// Once / twice: 8 sequences of 512 rows, 32 heads, 410 nuggets, 640 local rows 245 / 356 us; 16 of 2048, 40, 103, 2048 2.80 / 4.21 ms; 5 of up to
// 777, 64 over 8 160 / 297 us; segments of 4 texts, 32 690 / 1045 us.
//
// What bounds them: a wavefront with 32 owned rows of 128 channels fills its registers, so every matrix instruction comes with 16 bytes a
// lane from LDS, and a SIMD has two wavefronts to cover the chain LDS, products, exp2, products of each other; in long calls the card lowers its
// clock to 1.75 to 1.9 GHz besides.  16 sequences of 2048 rows, 40 heads of 128 (5 products: 1.89 TFLOP): 2.80 ms, 675 TFLOP/s of the 5 products
// and 945 of the 7 executed, where a large library product reaches 1180 to 1360.  Counters there (dQ; dK, dV): matrix pipes busy in 44 and 54% of
// the cycles, LDS reading in 23 and 36, wavefronts waiting in 23 and 33% of theirs.  8 sequences of 512 rows: pipes 32 and 34%, and
// compute units without any work in 22 and 20%, the start and the end of the launch.  (64 owned rows a wavefront, tiles of 128 rows, or the
// second products one tile later: slower, by spills or by fewer wavefronts.)
#include <type_traits>

#include "dodo_attn_grad.h"

namespace dodo {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short shortx4;
typedef __attribute__((ext_vector_type(8))) float floatx8;
typedef __attribute__((ext_vector_type(16))) float floatx16;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kTile = 64;  // walked rows per tile in LDS

template <int DH>
struct TileDims {
  static constexpr int kRowBytes = DH * 2;
  static constexpr int kPieces = kRowBytes / 16;
  static constexpr int kRowsPerInstr = 64 / kPieces;                       // rows that one direct load brings
  static constexpr int kBytes = kTile * kRowBytes;                         // 16 or 8 KiB
  // Piece p of row r is stored at p ^ swizzle(r).  A transposing read takes 64-byte granules of 4 rows in a row: these go to
  // different granules (of a row, or with 128-byte rows of a pair of rows); a row read takes one piece of 8 or 16 rows, which
  // differ in the granule or inside of it.
  __device__ static __forceinline__ int swizzle(int r) {
    return DH == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
  }
};

// A wavefront's part of the direct loads of a tile of rows `stride` bytes apart: through a buffer that ends with the last
// valid row (rows beyond read as zeros).
template <int DH, int NW = kGradWaves, int ROWS = kTile>
struct TileLoader {
  using TD = TileDims<DH>;
  static constexpr int kInstr = ROWS / TD::kRowsPerInstr / NW;  // direct loads per wavefront, tile and tensor
  uint32_t voff[kInstr], lds_off;
  __device__ __forceinline__ void init(int wave, int lane, uint32_t stride) {
    const int row0 = wave * kInstr * TD::kRowsPerInstr + lane / TD::kPieces, pos = lane % TD::kPieces;
#pragma unroll
    for (int u = 0; u < kInstr; ++u) {
      const int row = row0 + u * TD::kRowsPerInstr;
      voff[u] = static_cast<uint32_t>(row) * stride + static_cast<uint32_t>(pos ^ TD::swizzle(row)) * 16u;
    }
    lds_off = static_cast<uint32_t>(wave) * kInstr * 1024u;
  }
  __device__ __forceinline__ void issue(const uint16_t* first, int rows, uint32_t stride, uint32_t lds_dst) const {
    const u32x4_t buf = buffer_of(first, rows > 0 ? static_cast<uint32_t>(rows - 1) * stride + TD::kRowBytes : 0u);
#pragma unroll
    for (int u = 0; u < kInstr; ++u) dma16_buffer(buf, voff[u], __builtin_amdgcn_readfirstlane(lds_dst + lds_off + u * 1024u));
  }
};

// One direct load of 4 bytes a lane (lane l's land at lds_dst + 4 l), as dma16_buffer.
__device__ __forceinline__ void dma4_buffer(const u32x4_t& buf, uint32_t voff, uint32_t lds_dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff), "s"(buf), "s"(lds_dst) : "memory", "m0");
}

// Reads of a tile in LDS: fragments of rows and of columns of its 32-row half `hf`.
template <int DH>
struct TileReader {
  using TD = TileDims<DH>;
  int row_off, row_sw, col_off[2];
  __device__ __forceinline__ void init(int lane) {
    const int n = lane & 31, g = lane >> 5;
    row_off = n * TD::kRowBytes;
    row_sw = (g ^ TD::swizzle(n)) << 4;
    const int rr = (lane & 15) >> 2;  // row among 4; 8 bytes at channel 32 cb + 16 (lane / 16 % 2) + 4 (lane % 4)
    const int low = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 8 * e + 4 * g + rr;
      col_off[e] = r * TD::kRowBytes + ((low ^ TD::swizzle(r)) << 4) + 8 * (lane & 1);
    }
  }
  // channels 16 ks + 8 g .. + 8 of row n of the half
  __device__ __forceinline__ bf16x8 row(const char* tile, int hf, int ks) const {
    return *reinterpret_cast<const bf16x8*>(tile + hf * 32 * TD::kRowBytes + row_off + (row_sw ^ (ks << 5)));
  }
  // channel 32 cb + lane % 32 of rows 16 t + 8 e + 4 g + r of the half (slot 4 e + r)
  __device__ __forceinline__ bf16x8 column(const char* tile, int hf, int t, int cb) const {
    shortx4 a[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const char* p = tile + (hf * 32 + 16 * t) * TD::kRowBytes + (col_off[e] ^ (cb << 6));
      a[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shortx4 __attribute__((address_space(3)))*)(p));
    }
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a[0], a[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

__device__ __forceinline__ floatx16 zero16() {
  floatx16 z;
#pragma unroll
  for (int v = 0; v < 16; ++v) z[v] = 0.f;
  return z;
}
__device__ __forceinline__ floatx16 mfma(const bf16x8& a, const bf16x8& b, const floatx16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// Accumulators 8 t .. 8 t + 7 as a right operand (hardware round-to-nearest-even).
__device__ __forceinline__ bf16x8 half_bf16(const floatx16& x, int t) {
  floatx8 h;
#pragma unroll
  for (int v = 0; v < 8; ++v) h[v] = x[8 * t + v];
  return __builtin_convertvector(h, bf16x8);
}

// 32 rows of a gradient from a wavefront's transposed blocks (lane (row, g) holds channels 32 cb + 8 v4 + 4 g .. + 4), through LDS, so
// that a store instruction writes whole rows.  `lds` is the wavefront's own, kRowsOut bytes; row r < `rows` goes `stride` bytes after the one before.
template <int DH>
constexpr int kRowsOut = 32 * (DH * 2 + 16);
template <int DH>
__device__ __forceinline__ void store_rows(char* lds, uint16_t* to, uint32_t stride, int rows, const floatx16 (&acc)[DH / 32], float scale) {
  constexpr int kRow = DH * 2 + 16, kPieces = DH / 8, kRows = kWave / kPieces;  // (16 bytes between rows spread them over the banks)
  const int lane = lane_id();
#pragma unroll
  for (int cb = 0; cb < DH / 32; ++cb)
#pragma unroll
    for (int v4 = 0; v4 < 4; ++v4)
      store4<DODO_DTYPE_BF16>(lds + (lane & 31) * kRow, 32 * cb + 8 * v4 + 4 * (lane >> 5), acc[cb][4 * v4] * scale, acc[cb][4 * v4 + 1] * scale,
                              acc[cb][4 * v4 + 2] * scale, acc[cb][4 * v4 + 3] * scale);
#pragma unroll
  for (int u = 0; u < 32 / kRows; ++u) {
    const int r = u * kRows + lane / kPieces, piece = lane % kPieces;
    const uint4 v = *reinterpret_cast<const uint4*>(lds + r * kRow + piece * 16);
    if (r < rows) *reinterpret_cast<uint4*>(reinterpret_cast<char*>(to) + static_cast<uint32_t>(r) * stride + piece * 16) = v;
  }
}

// ---- dK, dV ------------------------------------------------------------------------------------------------------------
// A wavefront owns 32 keys, a workgroup 128 (BLOCKS = 4); its wavefronts walk over the query rows together.  BLOCKS = 2: 64 keys, two or
// four wavefronts (PARTS) per 32, one for either half of a tile's rows, or a quarter of two tiles', whose sums meet in LDS at the end.

template <int PARTS>
constexpr int kWalked = PARTS == 4 ? 2 * kTile : kTile;  // rows in LDS at a time

// A tile of query rows: those from i0 on of an entry, of its K/V head's query head hg.
struct RowTile {
  int q0, q_b, i0, hg, key0, len, lag;
  bool valid;
};

// SHARED: entries may share rows, and those that hold any of the workgroup's keys are looked for, 64 at a time; else the keys are
// those of one entry.
template <int DH, int BLOCKS, int PARTS, bool SHARED>
__global__ __launch_bounds__(BLOCKS * PARTS * kWave, 2) void grad_kv_kernel(GradParams p, int n_nug_tiles, int n_loc_tiles) {
  using TD = TileDims<DH>;
  constexpr int kKeys = 32 * BLOCKS, kRows = kWalked<PARTS>, kTensor = kRows * TD::kRowBytes;
  constexpr int kStage = 2 * kTensor + kRows * 8;  // Q, dO, then log-sum-exp (base 2) and -D of the rows
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
  int* const entries = reinterpret_cast<int*>(lds + 2 * kStage);  // (SHARED)
  // block i runs on XCD i % 8: the key tiles of one (sequence, K/V head) share Q and dO in an XCD's L2.  Shared rows: tile by
  // tile instead, so that the nuggets, which most entries see, come first for every head.
  const int tiles = n_nug_tiles + n_loc_tiles, n_owners = p.H_kv * (SHARED ? 1 : p.B), by_xcd = (n_owners + 7) / 8;
  const unsigned slot = blockIdx.x >> 3;
  const unsigned owner = (SHARED ? slot % by_xcd : slot / tiles) * 8 + (blockIdx.x & 7), tile = SHARED ? slot / by_xcd : slot % tiles;
  if (owner >= static_cast<unsigned>(n_owners)) return;
  const KeyTile t = key_tile(p, owner * tiles + tile, n_nug_tiles, n_loc_tiles, kKeys);
  if (t.rows <= 0) return;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane & 31, g = lane >> 5;
  const int G = p.H / p.H_kv;
  const int blk = wave % BLOCKS, part = wave / BLOCKS;
  const int my_rows = min(32, t.rows - blk * 32);  // of this wavefront
  const bool active = my_rows > 0;
  const int64_t my_first = t.first + blk * 32;

  const uint32_t row_stride = static_cast<uint32_t>(p.H) * TD::kRowBytes;  // bytes between query rows
  TileLoader<DH, BLOCKS * PARTS, kRows> loader;
  loader.init(wave, lane, row_stride);
  TileReader<DH> reader;
  reader.init(lane);

  // fragments of the owned keys: lane (n, g) holds channels 16 ks + 8 g .. + 8 of key n
  bf16x8 kf[DH / 16], vf[DH / 16];
  auto load_keys = [&]() {
    const int64_t first = t.first * t.tok_stride + t.kvh * t.head_stride;
    const char *K = reinterpret_cast<const char*>(static_cast<const uint16_t*>(t.K) + first), *V = reinterpret_cast<const char*>(static_cast<const uint16_t*>(t.V) + first);
    const uint32_t off = static_cast<uint32_t>(min(blk * 32 + n, t.rows - 1)) * static_cast<uint32_t>(t.tok_stride * 2) + 16 * g;
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) {
      kf[ks] = *reinterpret_cast<const bf16x8*>(K + off + 32 * ks);
      vf[ks] = *reinterpret_cast<const bf16x8*>(V + off + 32 * ks);
    }
    // (used here for the compiler's eyes, so that its waits for them stand before the loop)
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) asm volatile("" : "+v"(kf[ks]), "+v"(vf[ks]));
  };
  if (SHARED) load_keys();
  floatx16 dk[DH / 32], dv[DH / 32];
#pragma unroll
  for (int cb = 0; cb < DH / 32; ++cb) dk[cb] = dv[cb] = zero16();

  int e0 = t.entry0;
  do {
    RowTile one = {};
    uint64_t todo = 0;
    if constexpr (SHARED) {  // (of one entry per lane, kept in LDS: registers are what this kernel is short of)
      SeenBy of_lane = {};
      if (e0 + lane < t.entry1) of_lane = seen_by(p, t, e0 + lane, kKeys);
      todo = __ballot(of_lane.any && of_lane.first_row < of_lane.q_b);
      __syncthreads();  // (the chunk of entries before this one has been read)
      if (wave == 0) {
        entries[lane] = of_lane.q0;
        entries[kWave + lane] = of_lane.q_b;
        entries[2 * kWave + lane] = of_lane.len;
        entries[3 * kWave + lane] = of_lane.lag;
        entries[4 * kWave + lane] = of_lane.key0;
        entries[5 * kWave + lane] = of_lane.first_row;
      }
      __syncthreads();
    } else {
      const SeenBy s = seen_by(p, t, e0, kKeys);
      todo = s.any && s.first_row < s.q_b;
      one = RowTile{s.q0, s.q_b, s.first_row, 0, s.key0, s.len, s.lag, todo != 0};
    }
    auto entry_tile = [&]() -> RowTile {  // the first tile of the next entry
      RowTile r = one;
      r.valid = todo != 0;
      if (SHARED && r.valid) {
        const int* of = entries + __ffsll(static_cast<long long>(todo)) - 1;
        r.q0 = __builtin_amdgcn_readfirstlane(of[0]);
        r.q_b = __builtin_amdgcn_readfirstlane(of[kWave]);
        r.len = __builtin_amdgcn_readfirstlane(of[2 * kWave]);
        r.lag = __builtin_amdgcn_readfirstlane(of[3 * kWave]);
        r.key0 = __builtin_amdgcn_readfirstlane(of[4 * kWave]);
        r.i0 = __builtin_amdgcn_readfirstlane(of[5 * kWave]);
      }
      todo &= todo - 1;
      r.i0 = r.i0 / kRows * kRows;
      r.hg = 0;
      return r;
    };
    auto first_tile = [&](const RowTile& r) {  // of the entry, for the next head
      return t.local ? static_cast<int>(max(static_cast<int64_t>(0), max(t.first - r.key0, static_cast<int64_t>(0)) - r.lag)) / kRows * kRows : 0;
    };
    auto advance = [&](RowTile r) -> RowTile {
      r.i0 += kRows;
      if (r.i0 < r.q_b) return r;
      r.i0 = first_tile(r);
      if (++r.hg < G) return r;
      return entry_tile();
    };
    auto issue = [&](const RowTile& r, int stage) {
      const int h = t.kvh * G + r.hg, rows = min(kRows, r.q_b - r.i0);
      const int64_t first = (static_cast<int64_t>(r.q0 + r.i0) * p.H + h) * DH;
      const uint32_t dst = lds_base + stage * kStage;
      loader.issue(static_cast<const uint16_t*>(p.Q) + first, rows, row_stride, dst);
      loader.issue(static_cast<const uint16_t*>(p.dO) + first, rows, row_stride, dst + kTensor);
      if (wave < kRows / 32) {  // 64 of either statistic
        const int of = wave % 2, first_row = kRows > kTile ? wave / 2 * kTile : 0;
        const float* from = (of == 0 ? p.lse2 : p.neg_d) + static_cast<int64_t>(h) * p.Sq + r.q0 + r.i0 + first_row;
        dma4_buffer(buffer_of(from, max(rows - first_row, 0) * 4u), lane * 4u,
                    __builtin_amdgcn_readfirstlane(dst + 2 * kTensor + (of * kRows + first_row) * 4));
      }
    };
    RowTile cur = entry_tile();
    if (cur.valid) issue(cur, 0);
    if (!SHARED) load_keys();  // (behind the first tile's requests)
    for (int stage = 0; cur.valid; stage ^= 1) {
      char* const base = lds + stage * kStage;
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wavefront's part of the tile has landed
      __syncthreads();  // everyone's has, and the other stage has been read
      const RowTile next = advance(cur);
      if (next.valid) issue(next, stage ^ 1);
      // rows [from, ...) see some key of this wavefront; from `all` on they see all of them
      const int j = static_cast<int>(my_first - cur.key0);
      int from = 0, all = 0;
      if (t.local) {
        from = max(0, max(j, 0) - cur.lag);
        all = max(0, j + my_rows - 1 - cur.lag);
      }
      if (SHARED) {
        if (j + my_rows <= 0 || j >= cur.len) from = 0x7fffffff;
        if (j < 0 || j + my_rows > cur.len) all = 0x7fffffff;
      }
      if (active) {
#pragma unroll 1
        for (int hf = part; hf < kRows / 32; hf += PARTS) {
          const int i0 = cur.i0 + 32 * hf;
          if (i0 >= cur.q_b || i0 + 32 <= from) continue;
          const char *qt = base, *dt = base + kTensor;
          const float* lse2 = reinterpret_cast<const float*>(base + 2 * kTensor) + 32 * hf + 4 * g;
          // Fragments are requested one step (two matrix instructions) ahead; the scheduling barriers keep the compiler from
          // requesting them all at once, which would not fit into the registers.
          floatx16 s = zero16(), dp;  // (dP starts from -D, which saves the subtractions)
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4) {
            const float4 d = *reinterpret_cast<const float4*>(lse2 + kRows + 8 * v4);
            dp[4 * v4] = d.x; dp[4 * v4 + 1] = d.y; dp[4 * v4 + 2] = d.z; dp[4 * v4 + 3] = d.w;
          }
          bf16x8 qa[2], da[2];
          qa[0] = reader.row(qt, hf, 0);
          da[0] = reader.row(dt, hf, 0);
#pragma unroll
          for (int ks = 0; ks < DH / 16; ++ks) {
            if (ks + 1 < DH / 16) {
              qa[(ks + 1) & 1] = reader.row(qt, hf, ks + 1);
              da[(ks + 1) & 1] = reader.row(dt, hf, ks + 1);
            }
            s = mfma(qa[ks & 1], kf[ks], s);
            dp = mfma(da[ks & 1], vf[ks], dp);
            __builtin_amdgcn_sched_barrier(0);
          }
          // weights and dS; rows past the entry's last one are zeros with log-sum-exp 0 and D 0: they add nothing
          const bool mask = i0 < all;
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4) {
            const float4 l = *reinterpret_cast<const float4*>(lse2 + 8 * v4);
            const float lv[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int v = 4 * v4 + r;
              s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], p.scale_log2e, -lv[r]));
              dp[v] *= s[v];
            }
          }
          if (mask) {
            const int jk = j + n;
            int least = t.local ? jk - cur.lag : 0;
            if (SHARED && (jk < 0 || jk >= cur.len)) least = 0x7fffffff;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const bool seen = i0 + 8 * (v >> 2) + 4 * g + (v & 3) >= least;
              s[v] = seen ? s[v] : 0.f;
              dp[v] = seen ? dp[v] : 0.f;
            }
          }
          const bf16x8 pf[2] = {half_bf16(s, 0), half_bf16(s, 1)}, sf[2] = {half_bf16(dp, 0), half_bf16(dp, 1)};
          constexpr int kCB = DH / 32, kAhead = 2;
          bf16x8 dc[kAhead + 1], qc[kAhead + 1];
          const auto read = [&](int u) {
            dc[u % (kAhead + 1)] = reader.column(dt, hf, u / kCB, u % kCB);
            qc[u % (kAhead + 1)] = reader.column(qt, hf, u / kCB, u % kCB);
          };
#pragma unroll
          for (int u = 0; u < kAhead; ++u) read(u);
#pragma unroll
          for (int u = 0; u < 2 * kCB; ++u) {
            if (u + kAhead < 2 * kCB) read(u + kAhead);
            dv[u % kCB] = mfma(dc[u % (kAhead + 1)], pf[u / kCB], dv[u % kCB]);
            dk[u % kCB] = mfma(qc[u % (kAhead + 1)], sf[u / kCB], dk[u % kCB]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      cur = next;
    }
    e0 += kWave;
  } while (SHARED && e0 < t.entry1);
  __syncthreads();  // the stages have been read
  constexpr int kRegs = DH / 32 * 16;  // per lane and tensor
  if constexpr (PARTS > 1) {  // dK, then dV: the other parts' sums, added in their order
    float* const meet = reinterpret_cast<float*>(lds) + blk * kRegs * kWave + lane;
    const auto join = [&](floatx16(&acc)[DH / 32]) {
      if (part > 0)
#pragma unroll
        for (int c = 0; c < kRegs; ++c) meet[((part - 1) * BLOCKS * kRegs + c) * kWave] = acc[c / 16][c % 16];
      __syncthreads();
      if (part == 0)
#pragma unroll
        for (int w = 0; w < PARTS - 1; ++w)
#pragma unroll
          for (int c = 0; c < kRegs; ++c) acc[c / 16][c % 16] += meet[(w * BLOCKS * kRegs + c) * kWave];
    };
    join(dk);
    __syncthreads();
    join(dv);
    if (part > 0) return;
  }
  if (!active) return;
  char* out = lds + blk * (PARTS > 1 ? kRegs * kWave * 4 : kRowsOut<DH>);  // (where it met the others' sums, or a part of the stages)
  const int64_t to = my_first * t.tok_stride + t.kvh * t.head_stride;
  store_rows<DH>(out, static_cast<uint16_t*>(t.local ? p.dKl : p.dKn) + to, static_cast<uint32_t>(t.tok_stride * 2), my_rows, dk, p.scale);
  store_rows<DH>(out, static_cast<uint16_t*>(t.local ? p.dVl : p.dVn) + to, static_cast<uint32_t>(t.tok_stride * 2), my_rows, dv, 1.f);
}

// ---- dQ ----------------------------------------------------------------------------------------------------------------
// A wavefront owns 32 query rows of a head, a workgroup 128 (BLOCKS = 4); its wavefronts walk over the keys together: nuggets, then
// local rows up to the last one that the workgroup's last row sees.  BLOCKS = 2: 64 rows, two wavefronts per 32, as above.
template <int DH, int BLOCKS>
__global__ __launch_bounds__(kGradThreads, 2) void grad_q_kernel(GradParams p, int n_blocks) {
  constexpr int kParts = kGradWaves / BLOCKS, kQueryRows = 32 * BLOCKS;
  using TD = TileDims<DH>;
  constexpr int kStage = 2 * TD::kBytes;  // K, V
  constexpr int kAhead = 2;               // steps that fragments are requested ahead
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
  const unsigned slot = blockIdx.x >> 3, owner = slot / n_blocks * 8 + (blockIdx.x & 7);
  if (owner >= static_cast<unsigned>(p.H * p.B)) return;
  const int h = owner % p.H;
  const Entry s = entry_of(p, owner / p.H);
  const int i0 = static_cast<int>(n_blocks - 1 - slot % n_blocks) * kQueryRows;  // the last rows see the most keys: they start first
  if (i0 >= s.q_b) return;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane & 31, g = lane >> 5;
  const int kvh = h / (p.H / p.H_kv);
  const int blk = wave % BLOCKS, part = wave / BLOCKS, w_i0 = i0 + 32 * blk;
  const bool active = w_i0 < s.q_b, row_ok = w_i0 + n < s.q_b;
  const int i = min(w_i0 + n, s.q_b - 1);
  const int64_t off = (static_cast<int64_t>(s.q0 + i) * p.H + h) * DH;
  TileLoader<DH> loader;
  uint32_t loader_stride = 0;
  TileReader<DH> reader;
  reader.init(lane);
  const int lag = s.m_b - s.q_b + 1;  // row i sees local rows [0, i + lag)
  const int vis = max(0, min(s.m_b, i + lag));
  const int w_least = max(0, min(s.m_b, w_i0 + lag)), w_most = max(0, min(s.m_b, min(w_i0 + 32, s.q_b) - 1 + lag));
  const int wg_most = max(0, min(s.m_b, min(i0 + kQueryRows, s.q_b) - 1 + lag));
  const int n_nug = (s.k_b + kTile - 1) / kTile, n_tiles = n_nug + (wg_most + kTile - 1) / kTile;
  const int64_t nug_first = s.k0 * p.nug_tok_stride + kvh * p.nug_head_stride, loc_first = s.l0 * p.loc_tok_stride + kvh * p.loc_head_stride;
  auto issue = [&](int tile, int stage) {
    const bool nug = tile < n_nug;
    const int j0 = kTile * (nug ? tile : tile - n_nug), rows = min(kTile, (nug ? s.k_b : wg_most) - j0);
    const int64_t stride = nug ? p.nug_tok_stride : p.loc_tok_stride, first = (nug ? nug_first : loc_first) + j0 * stride;
    const uint32_t dst = lds_base + stage * kStage;
    if (loader_stride != static_cast<uint32_t>(stride * 2)) {  // (the first tile, and where the cache's stride is not the local rows')
      loader_stride = static_cast<uint32_t>(stride * 2);
      loader.init(wave, lane, loader_stride);
    }
    loader.issue(static_cast<const uint16_t*>(nug ? p.Kn : p.Kl) + first, rows, loader_stride, dst);
    loader.issue(static_cast<const uint16_t*>(nug ? p.Vn : p.Vl) + first, rows, loader_stride, dst + TD::kBytes);
  };
  if (n_tiles > 0) issue(0, 0);
  bf16x8 qf[DH / 16], df[DH / 16];
#pragma unroll
  for (int ks = 0; ks < DH / 16; ++ks) {
    qf[ks] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(p.Q) + off + 16 * ks + 8 * g);
    df[ks] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(p.dO) + off + 16 * ks + 8 * g);
  }
  // D and the log-sum-exp in base 2 of the row, here and for the other kernel; a row that sees nothing (-inf) gets +inf: its
  // weights are 0
  float2 st = make_float2(p.lse[static_cast<int64_t>(s.q0 + i) * p.H + h] * kLog2e, 0.f);
  if (st.x == -__builtin_inff()) st.x = __builtin_inff();
#pragma unroll
  for (int ks = 0; ks < DH / 16; ++ks) {
    const uint4 a = __builtin_bit_cast(uint4, df[ks]), o = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.O) + off + 16 * ks + 8 * g);
    const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, ow[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      st.y = fmaf(bf16_lo(aw[c]), bf16_lo(ow[c]), st.y);
      st.y = fmaf(bf16_hi(aw[c]), bf16_hi(ow[c]), st.y);
    }
  }
  float lower, upper;
  lane_pair<32>(st.y, lower, upper);
  st.y = -(lower + upper);
  if (g == 0 && row_ok && part == 0) {
    p.lse2[static_cast<int64_t>(h) * p.Sq + s.q0 + i] = st.x;
    p.neg_d[static_cast<int64_t>(h) * p.Sq + s.q0 + i] = st.y;
  }
  floatx16 neg_d;  // dP starts from -D, which saves the subtractions
#pragma unroll
  for (int v = 0; v < 16; ++v) neg_d[v] = st.y;
  floatx16 dq[DH / 32];
#pragma unroll
  for (int cb = 0; cb < DH / 32; ++cb) dq[cb] = zero16();
#pragma unroll
  for (int ks = 0; ks < DH / 16; ++ks) asm volatile("" : "+v"(qf[ks]), "+v"(df[ks]));
  asm volatile("" : "+v"(st.x), "+v"(st.y));
  for (int tile = 0; tile < n_tiles; ++tile) {
    const int stage = tile & 1;
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wavefront's part of the tile has landed
    __syncthreads();                      // everyone's has, and the other stage has been read
    if (tile + 1 < n_tiles) issue(tile + 1, stage ^ 1);
    if (!active) continue;
    const bool nug = tile < n_nug;
    const int j0 = kTile * (nug ? tile : tile - n_nug);
    const int limit = (nug ? s.k_b : vis) - j0;  // keys [0, limit) of the tile are seen by this lane's row,
    const int most = (nug ? s.k_b : w_most) - j0, least = (nug ? s.k_b : w_least) - j0;  // ... by some and by all rows of the wavefront
    const char *kt = lds + stage * kStage, *vt = kt + TD::kBytes;
#pragma unroll 1
    for (int hf = part; hf < 2; hf += kParts) {
      if (32 * hf >= most) break;
      floatx16 sc = zero16(), dp = neg_d;
      {
        bf16x8 ka[kAhead + 1], va[kAhead + 1];
        const auto read = [&](int ks) {
          ka[ks % (kAhead + 1)] = reader.row(kt, hf, ks);
          va[ks % (kAhead + 1)] = reader.row(vt, hf, ks);
        };
#pragma unroll
        for (int ks = 0; ks < kAhead; ++ks) read(ks);
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks) {
          if (ks + kAhead < DH / 16) read(ks + kAhead);
          sc = mfma(ka[ks % (kAhead + 1)], qf[ks], sc);
          dp = mfma(va[ks % (kAhead + 1)], df[ks], dp);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      constexpr int kCB = DH / 32;
      bf16x8 kc[2 * kAhead];
#pragma unroll
      for (int u = 0; u < 2 * kAhead - 1; ++u) kc[u] = reader.column(kt, hf, u / kCB, u % kCB);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int v = 0; v < 16; ++v) sc[v] = __builtin_amdgcn_exp2f(fmaf(sc[v], p.scale_log2e, -st.x)) * dp[v];
      if (32 * hf + 32 > least) {
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[v] = 32 * hf + 8 * (v >> 2) + 4 * g + (v & 3) < limit ? sc[v] : 0.f;
      }
      const bf16x8 sf[2] = {half_bf16(sc, 0), half_bf16(sc, 1)};
#pragma unroll
      for (int u = 0; u < 2 * kCB; ++u) {
        const int w = u + 2 * kAhead - 1;
        if (w < 2 * kCB) kc[w % (2 * kAhead)] = reader.column(kt, hf, w / kCB, w % kCB);
        dq[u % kCB] = mfma(kc[u % (2 * kAhead)], sf[u / kCB], dq[u % kCB]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  __syncthreads();  // the stages have been read
  constexpr int kRegs = DH / 32 * 16;  // per lane
  if constexpr (kParts == 2) {
    float* const meet = reinterpret_cast<float*>(lds) + blk * kRegs * kWave + lane;
    if (part == 1)
#pragma unroll
      for (int c = 0; c < kRegs; ++c) meet[c * kWave] = dq[c / 16][c % 16];
    __syncthreads();
    if (part == 1) return;
#pragma unroll
    for (int c = 0; c < kRegs; ++c) dq[c / 16][c % 16] += meet[c * kWave];
  }
  if (!active) return;
  char* const out = lds + blk * (kParts == 2 ? kRegs * kWave * 4 : kRowsOut<DH>);  // (where it met the other's sums, or a part of the stages)
  store_rows<DH>(out, static_cast<uint16_t*>(p.dQ) + (static_cast<int64_t>(s.q0 + w_i0) * p.H + h) * DH,
                 static_cast<uint32_t>(p.H) * TD::kRowBytes, min(32, s.q_b - w_i0), dq, p.scale);
}

static_assert(kGradWaves * kRowsOut<128> <= 2 * 2 * TileDims<128>::kBytes && kGradWaves * kRowsOut<64> <= 2 * 2 * TileDims<64>::kBytes,
              "the stages have room for the rows on their way out");

template <int DH, int BLOCKS, int PARTS, bool SHARED>
int launch_kv(const GradParams& p) {
  constexpr int kKeys = 32 * BLOCKS;
  constexpr int kLds = 2 * kWalked<PARTS> * (2 * TileDims<DH>::kRowBytes + 8) + (SHARED ? 6 * kWave * 4 : 0);
  static_assert((PARTS - 1) * kKeys * DH * 4 <= kLds, "the stages have room for the sums that meet");
  static_assert(kLds * (BLOCKS * PARTS == 8 ? 1 : 2) <= 160 * 1024, "eight wavefronts on a compute unit");
  const int64_t nug_rows = p.shared ? p.Kt : p.max_k, loc_rows = p.shared ? p.Sm : p.max_local;
  const int64_t nug = (nug_rows + kKeys - 1) / kKeys, loc = (loc_rows + kKeys - 1) / kKeys;
  const int64_t owners = (static_cast<int64_t>(p.H_kv) * (p.shared ? 1 : p.B) + 7) / 8 * 8;
  if ((nug + loc) * owners > 0x7fffffffLL) return DODO_ERR_UNSUPPORTED;
  if (nug + loc == 0) return DODO_OK;
  if constexpr (BLOCKS == 4) {
    // 64 keys per workgroup where 128 leave compute units without two of them.  128 / 64 keys, us: 1 sequence of 512 rows, 32 heads, 410
    // nuggets, 640 local rows 37.5 / 28.3; 64 heads over 8 130 / 84, 4 sequences of it 190 / 128, 8 254 / 258; 1 of 2048, 8 heads, 410, 2048
    // 71 / 50; 1 of 1000, 32 heads over 8, 1000, 1000 135 / 88, over 32 62 / 75; 8 of 512, 32 heads, 410, 640 152 / 203; 8 of 16, 100, 32
    // 11 / 20.
    if ((nug + loc) * owners < 2 * compute_units()) {
      if constexpr (!SHARED) {
        // Four wavefronts per 32 keys where the longest walk (of at least 16 tiles) would outlast a compute unit's share of all walks.  Two /
        // four: 1 of 512, 64 heads over 8, 410, 640 84 / 65, 2 of it 90 / 73, 4 128 / 145; 5 of 500, 300, 533 130 / 145, ragged ones up to 777
        // rows 119 / 99; 1 of 2048, 8 heads, 410, 2048 50 / 43; 1 of 128, 64 over 8, 100, 128 26 / 24, of 64 17 / 21; 1 of 512, 32, 410, 640 28 / 47.
        const int64_t G = p.H / p.H_kv, longest = G * ((p.max_q + kTile - 1) / kTile), mean = G * ((p.Sq / p.B + kTile - 1) / kTile);
        const int64_t walks = ((p.Kt + p.Sm) / (2 * 32) + p.B) * p.H_kv;
        if (longest >= 16 && 5 * longest * compute_units() >= 4 * walks * mean) return launch_kv<DH, 2, 4, SHARED>(p);
      }
      return launch_kv<DH, 2, 2, SHARED>(p);
    }
  }
  const auto kern = grad_kv_kernel<DH, BLOCKS, PARTS, SHARED>;
  const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kern), kLds);
  if (rc != DODO_OK) return rc;
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>((nug + loc) * owners)), dim3(BLOCKS * PARTS * kWave), kLds, p.stream, p, static_cast<int>(nug),
                     static_cast<int>(loc));
  return launch_status();
}

template <int DH, int BLOCKS>
int launch_q(const GradParams& p) {
  constexpr int kQueryRows = 32 * BLOCKS;
  constexpr int kLds = 2 * 2 * TileDims<DH>::kBytes;
  static_assert(kQueryRows * DH * 4 <= kLds, "the stages have room for the sums that meet");
  const int64_t blocks = (static_cast<int64_t>(p.max_q) + kQueryRows - 1) / kQueryRows;
  const int64_t owners = (static_cast<int64_t>(p.H) * p.B + 7) / 8 * 8;
  if (blocks * owners > 0x7fffffffLL) return DODO_ERR_UNSUPPORTED;
  if (blocks * owners == 0) return DODO_OK;
  if constexpr (BLOCKS == 4) {
    // 64 rows per workgroup where 128 leave compute units idle or barely fill them.  128 / 64 rows, us: 1 sequence of 512 rows, 32 heads,
    // 410 nuggets, 640 local rows 33 / 24, 64 heads 36 / 36, 2 sequences of 32 heads 36 / 36, of 64 56 / 64; 1 of 2048, 8 heads, 410, 2048
    // 64 / 43; 1 of 64, 32 heads, 3277, 128 81 / 54; 8 of 64, 410, 128 20.9 / 18.8; 8 of 512, 410, 640 115 / 134.
    if (blocks * owners <= compute_units()) return launch_q<DH, 2>(p);
  }
  const auto kern = grad_q_kernel<DH, BLOCKS>;
  const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kern), kLds);
  if (rc != DODO_OK) return rc;
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(blocks * owners)), dim3(kGradThreads), kLds, p.stream, p, static_cast<int>(blocks));
  return launch_status();
}

template <int DH>
int launch_both(const GradParams& p) {
  const int rc = launch_q<DH, 4>(p);  // (first: it makes the rows' statistics)
  if (rc != DODO_OK) return rc;
  return p.shared ? launch_kv<DH, 4, 1, true>(p) : launch_kv<DH, 4, 1, false>(p);
}

}  // namespace

int launch_grad_mfma(const GradParams& p, int32_t d_h) {
  return d_h == 128 ? launch_both<128>(p) : launch_both<64>(p);
}

}  // namespace dodo
