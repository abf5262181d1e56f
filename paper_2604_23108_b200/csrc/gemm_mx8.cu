// The experts in 8 bits: ragged products grouped by expert with block-scaled E4M3 operands, on the
// 5th-generation tensor cores (tcgen05.mma kind::mxf8f6f4, one power-of-two scale per 32 elements of
// the contraction, applied inside the instruction; FP32 accumulators in tensor memory).
//
//   phase 1   A = Xp Wg^T, U = Xp Wu^T, H = mx8(silu(A) U)       rows of an expert x 2 W_g, contraction d
//   phase 2   Yp = H W2^T                                         rows of an expert x d, contraction W_g
//
// Expert segments start at multiples of 128 physical rows, so a 128-row tile belongs to one expert.
// One persistent CTA per SM (a CTA pair per two SMs when the experts see more than 128 rows on average)
// walks the cost-sorted tile list that the BF16 path's list builder makes.  Warp roles:
//   warp 0      TMA producer: per 128 columns of the contraction 16 KiB of A, the pair's half of 256 rows
//               of B (all of them for a single CTA), and the scales, 512 bytes per 128 rows
//   warp 1      tensor memory and MMA issue: copies the scales to tensor memory (tcgen05.cp), then four
//               MMAs of 32 columns; scale byte j of a row's word belongs to the j-th of them
//   warps 2..5  epilogue.  A thread owns a row, so the 32 columns that share a scale of H are its own
//               registers: phase 1 turns a gate chunk and an up chunk into 32 elements and a scale byte
//               without any exchange between threads and writes them where phase 2's operands lie.
// Tensor memory: two accumulators of 256 columns and a set of scales per stage (4 columns for 128 rows
// of A, 8 for 256 rows of B; five stages) need 572 columns of 512.  The accumulators therefore share 60
// columns (0..255 and 196..451, scales at 452): the epilogue reads the shared part first and then lets
// the next tile's MMAs start, so the next tile waits for that read instead of for the whole epilogue.
// With a set per stage, a stage that has been refilled says that its set is free to be rewritten.
//
// Yp is written in BF16, as the 16-bit path's y_perm is, and rounded again after the combine: the error against
// 64 bits is 0.0024 of the outputs' size, 0.0017 if it stayed in FP32, which would cost 8 bytes of traffic per
// routed row and column instead of 4.
//
// What it reaches: 65536 tokens of the large layer (dispatch to combine) 7.9 ms for one call on an idle GPU and
// 9.1-9.6 ms in calls that follow each other, where the power cap holds the SM clock at 1.1 GHz of 1.965 (the first
// product's loop takes 555 clocks per 128 columns, the instructions 512); 256 tokens 376-391 us, 81 % of the
// DRAM's peak in the first product.  Where the contraction is short (d = 1024: eight steps) the 1300 or so
// clocks between tiles count; eight epilogue warps or a list read further ahead did not shorten them.
//
// Every wait is bounded as in the BF16 kernel: after about a second without progress the waiting thread
// records (1 << 24 | site), raises the CTA's abort flag and every role leaves its loop.

#include <string.h>

#include <atomic>

#include "common.cuh"
#include "mx8_math.cuh"
#include "tc_ptx.cuh"

namespace mohge {
namespace {

constexpr int BM = 128;                    // rows of a CTA
constexpr int BK = 128;                    // contraction elements (bytes) per stage
constexpr int BN = 256;                    // MMA N: 128 gate + 128 up columns, or 256 output columns
constexpr int kThreadsMx = 192;
constexpr int kABytes = BM * BK;
constexpr int kSfBytes = 2048;             // 512 for A, 1024 for B, padded so that stages stay 1 KiB aligned
constexpr uint32_t kAcc1 = 196, kSfCol = 452, kSfSet = 12;

template <int CG> struct GeoMx {
  static constexpr int kStages = CG == 2 ? 5 : 4;
  static constexpr int kBBytes = BN / CG * BK;
  static constexpr int kStageBytes = kABytes + kBBytes + kSfBytes;
  static constexpr int kSmemBytes = kStages * kStageBytes + 1024 + 256;
};

struct MxParams {
  CUtensorMap mapA[MOHGE_MAX_GROUPS];      // [cols of the contraction, rows] bytes, 128 x 128 boxes
  CUtensorMap mapA32[MOHGE_MAX_GROUPS];    // the same in boxes of 32 rows, for tiles that are not full
  CUtensorMap mapSA;                       // scales of A: [128 words, k-blocks, row blocks]
  CUtensorMap mapB[MOHGE_MAX_GROUPS];      // [contraction, rows, matrices] bytes
  CUtensorMap mapSB[MOHGE_MAX_GROUPS];     // scales of B: [128 words, k-blocks, row blocks, matrices]
  int W[MOHGE_MAX_GROUPS];
  int Ng, N, d;
  uint8_t* h;                              // phase 1: elements of H [rows, h_pitch]
  int64_t h_pitch;
  __nv_bfloat16* y;                        // phase 2: y_perm [rows, d]
  uint8_t* h_scale;                        // tiled scales of H
  int h_kblocks;                           // its k-blocks per row block (those of the widest group)
  bool sector;                             // rows of this phase's output begin on 32-byte boundaries
  const int32_t* counts;                   // rows of an expert's segment that hold tokens
  const int32_t* aligned;
  const int32_t* tile_count;
  const Tile* tiles;
  int32_t* status;
};

__device__ __forceinline__ uint64_t scale_desc(uint32_t addr) {      // 32 rows of 16 bytes, no swizzle
  return (uint64_t)((addr & 0x3ffffu) >> 4) | (1ull << 16) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
}
template <int CG> __device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint64_t desc) {
  if (CG == 2)
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
template <int CG>
__device__ __forceinline__ void umma_mx8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa,
                                         uint32_t sfb, uint32_t accumulate) {
  if (CG == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}

// 32 bytes of a row, the first `valid` (a multiple of 8) of which exist; sector: the address is a multiple of
// 32, which takes the buffer's own address as well as the row's length (callers promise 16-byte alignment only)
__device__ __forceinline__ void store_sector(uint8_t* p, bool sector, int valid, const uint32_t (&o)[8]) {
  if (sector && valid >= 32) {
    asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]) : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (8 * i < valid) *reinterpret_cast<uint2*>(p + 8 * i) = make_uint2(o[2 * i], o[2 * i + 1]);
  }
}

// PHASE 1 or 2 (see above); CG = CTAs per MMA
template <int PHASE, int CG>
__global__ void __launch_bounds__(kThreadsMx, 1) mx8_grouped_kernel(const __grid_constant__ MxParams p) {
  using G = GeoMx<CG>;
  constexpr int kStages = G::kStages;
  const uint32_t rank = CG == 2 ? cluster_ctarank() : 0u;
  const int unit = blockIdx.x / CG, units = gridDim.x / CG;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar0 = base + kStages * G::kStageBytes;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
  auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * kStages + b); };
  const uint32_t tfree_bar = bar0 + 8u * (2 * kStages + 2);   // shared columns of the current accumulator have been read
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(gen + kStages * G::kStageBytes + 8 * (2 * kStages + 3));
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), CG);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(tfull_bar(0), 1);
    mbar_init(tfull_bar(1), 1);
    mbar_init(tfree_bar, 4 * CG);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  // The rows of A that no box is loaded into are multiplied all the same: as zeros they cost least power
  // (256 tokens against the large layer, 16 of 128 rows used: 400 -> 383 us, the clock holds).
  for (int i = threadIdx.x; i < kStages * (kABytes / 16); i += kThreadsMx)
    *reinterpret_cast<uint4*>(gen + (i / (kABytes / 16)) * G::kStageBytes + (i % (kABytes / 16)) * 16) = make_uint4(0, 0, 0, 0);
  fence_async_smem();
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  // the list is sorted by cost; with unequal costs rounds alternate direction (as in the BF16 kernel)
  const int total = p.tile_count[0];
  const bool zigzag = p.tile_count[1] != 0;
  const int rounds = (total + units - 1) / units;
  auto fetch = [&](int round) -> Tile {
    Tile z;
    z.e = -1; z.m0 = 0; z.n0 = 0; z.ext = 0;
    if (round >= rounds) return z;
    const int ti = round * units + ((zigzag && (round & 1)) ? units - 1 - unit : unit);
    return ti < total ? p.tiles[ti] : z;
  };
  // rows of this CTA's half of a tile that hold tokens (at most 128; none or fewer: nothing to do here)
  auto valid_rows = [&](const Tile& t) { return p.counts[t.e] - (t.m0 - p.aligned[t.e]) - BM * (int)rank; };
  auto kblocks = [&](int e) { return ((PHASE == 1 ? p.d : p.W[e / p.N]) + BK - 1) / BK; };

  if (warp == 0) {
    // ================= producer =================
    if (lane == 0) {
      const uint64_t pol_a = l2_policy_evict_normal(), pol_b = l2_policy_evict_last();
      int stage = 0;
      uint32_t phase = 0;
      bool alive = true;
      constexpr uint32_t kTx = G::kBBytes + 512 + 1024;
      Tile next = fetch(0);
      for (int it = 0; it < rounds && alive; ++it) {
        const Tile t = next;
        next = fetch(it + 1);
        if (t.e < 0) continue;
        const int g = t.e / p.N, i = t.e - g * p.N, nkb = kblocks(t.e);
        const int m0 = t.m0 + BM * (int)rank;
        // Rows of padding are not loaded: an accumulator row depends on its own row of A alone, so what the
        // stage held before may stand there (decode batches fill 16 of 128 rows).
        const int v = valid_rows(t), boxes = v >= BM - 31 ? 4 : v > 0 ? (v + 31) >> 5 : 0;
        const uint32_t tx = kTx + boxes * 32 * BK;
        for (int kb = 0; kb < nkb; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, p.status, 21)) { alive = false; break; }
          const uint32_t sA = base + stage * G::kStageBytes, sB = sA + kABytes, sS = sB + G::kBBytes;
          const uint32_t fb = CG == 2 ? mapa_rank(full_bar(stage), 0) : full_bar(stage);
          if (CG == 2) mbar_expect_tx_cluster(fb, tx); else mbar_expect_tx(fb, tx);
          const int k0 = kb * BK;
          if (boxes == 4) tma_2d<CG>(sA, &p.mapA[PHASE == 1 ? 0 : g], fb, k0, m0, pol_a);
          else
            for (int j = 0; j < boxes; ++j) tma_2d<CG>(sA + j * 32 * BK, &p.mapA32[PHASE == 1 ? 0 : g], fb, k0, m0 + 32 * j, pol_a);
          tma_3d<CG>(sS, &p.mapSA, fb, 0, kb, m0 >> 7, pol_a);
          if (PHASE == 1) {                  // matrices 2 i (gate) and 2 i + 1 (up) of the group
            if (CG == 2) {
              tma_3d<CG>(sB, &p.mapB[g], fb, k0, t.n0, 2 * i + (int)rank, pol_b);
            } else {
              tma_3d<CG>(sB, &p.mapB[g], fb, k0, t.n0, 2 * i, pol_b);
              tma_3d<CG>(sB + G::kBBytes / 2, &p.mapB[g], fb, k0, t.n0, 2 * i + 1, pol_b);
            }
            tma_4d<CG>(sS + 512, &p.mapSB[g], fb, 0, kb, t.n0 >> 7, 2 * i, pol_b);       // box: both matrices
          } else {
            tma_3d<CG>(sB, &p.mapB[g], fb, k0, t.n0 + BN / CG * (int)rank, i, pol_b);
            tma_4d<CG>(sS + 512, &p.mapSB[g], fb, 0, kb, t.n0 >> 7, i, pol_b);           // box: two row blocks
          }
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    // ================= MMA issue =================
    if (rank == 0) {
      // The whole warp walks the loop and one elected lane issues: operands of the tcgen05 instructions
      // are then warp-uniform values.  With one lane alone in the loop the issue took 860-960 clocks per
      // 128 columns, the MMAs take 512.
      const uint64_t desc_a = make_desc(base, 16, 1024), desc_b = make_desc(base + kABytes, 16, 1024);
      const uint64_t desc_s = scale_desc(base + kABytes + G::kBBytes);
      int stage = 0, n_tile = 0;
      uint32_t phase = 0;
      bool alive = true;
      Tile next = fetch(0);
      for (int it = 0; it < rounds && alive; ++it) {
        const Tile t = next;
        next = fetch(it + 1);
        if (t.e < 0) continue;
        const int nkb = kblocks(t.e), buf = n_tile & 1;
        // one arrival round per tile: round n - 1 means that tile n - 1's shared columns, and all of
        // tile n - 2's accumulator, have been read
        if (n_tile > 0 && !mbar_wait(tfree_bar, (uint32_t)(n_tile - 1) & 1u, abort_flag, p.status, 22)) break;
        const uint32_t acc = tmem + (buf ? kAcc1 : 0u);
        for (int kb = 0; kb < nkb; ++kb) {
          if (!mbar_wait(full_bar(stage), phase, abort_flag, p.status, 23)) { alive = false; break; }
          tc_fence_after();
          if (elect_one()) {
            const uint64_t off = (uint64_t)(stage * (G::kStageBytes >> 4));
            const uint32_t sfa = tmem + kSfCol + (uint32_t)stage * kSfSet;
            scales_to_tmem<CG>(sfa, desc_s + off);
            scales_to_tmem<CG>(sfa + 4, desc_s + off + (512 >> 4));
            scales_to_tmem<CG>(sfa + 8, desc_s + off + (1024 >> 4));
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              // E4M3 x E4M3, scales E8M0, byte kk of the scale words
              constexpr uint32_t kIdesc = (1u << 23) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(BM * CG >> 4) << 24);
              umma_mx8<CG>(acc, desc_a + off + 2 * kk, desc_b + off + 2 * kk, kIdesc | (kk << 4) | (kk << 29), sfa, sfa + 4,
                           (kb | kk) ? 1u : 0u);
            }
            if (CG == 2) umma2_commit(empty_bar(stage)); else umma_commit(empty_bar(stage));
            if (kb + 1 == nkb) { if (CG == 2) umma2_commit(tfull_bar(buf)); else umma_commit(tfull_bar(buf)); }
          }
          __syncwarp();
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        ++n_tile;
      }
    }
  } else {
    // ================= epilogue =================
    // Results go from registers to memory, 32 bytes (a sector) per thread and store.  Staged through
    // shared memory for TMA stores instead they cost its bandwidth twice, which the operand tiles need:
    // 512 clocks of MMAs per 128 columns read 64 bytes per clock of the 128 that there are, TMA writes
    // as much, and phase 2 took 714 clocks per 128 columns
    // (at 10 of them per tile) where it takes 630 now, phase 1 560 where it takes 555.
    const int quad = warp & 3;               // the accumulator rows this warp can read
    int n_tile = 0;
    Tile next = fetch(0);
    for (int it = 0; it < rounds; ++it) {
      const Tile t = next;
      next = fetch(it + 1);
      if (t.e < 0) continue;
      const int buf = n_tile & 1, g = t.e / p.N;
      const uint32_t taddr = tmem + ((uint32_t)(quad * 32) << 16) + (buf ? kAcc1 : 0u);
      const int row0 = t.m0 + BM * (int)rank + quad * 32;
      const int64_t row = row0 + lane;
      const bool rows_ok = quad * 32 + lane < valid_rows(t);       // the row holds a token
      const bool got = mbar_wait(tfull_bar(buf), (uint32_t)(n_tile >> 1) & 1u, abort_flag, p.status, 25);
      if (!__all_sync(0xffffffffu, got)) break;
      tc_fence_after();
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (CG == 2) mbar_arrive_cluster(mapa_rank(tfree_bar, 0)); else mbar_arrive(tfree_bar);
        }
      };
      if (PHASE == 1) {
        const int W = p.W[g];
        uint32_t word = 0;
        // the shared columns are the last 60 of accumulator 0 (up columns 68..127) and the first 60 of
        // accumulator 1 (gate columns 0..59): that half of the second chunk is read with the first one
        uint32_t early[32];
#pragma unroll
        for (int ci = 0; ci < 4; ++ci) {
          const int c = buf ? ci : 3 - ci;
          uint32_t ra[32], ru[32];
          if (ci == 1) {
#pragma unroll
            for (int j = 0; j < 32; ++j) { ra[j] = early[j]; ru[j] = early[j]; }
            if (buf) tmem_ld32(taddr + 128 + 32 * c, ru); else tmem_ld32(taddr + 32 * c, ra);
          } else {
            tmem_ld32(taddr + 32 * c, ra);
            tmem_ld32(taddr + 128 + 32 * c, ru);
            if (ci == 0) tmem_ld32(taddr + (buf ? 32 : 128 + 64), early);
          }
          tmem_ld_wait();
          if (ci == 0) release();
          float2 h[16];
          float m = 0.f;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float2 a = make_float2(__uint_as_float(ra[2 * j]), __uint_as_float(ra[2 * j + 1]));
            const float2 u = make_float2(__uint_as_float(ru[2 * j]), __uint_as_float(ru[2 * j + 1]));
            h[j] = __fmul2_rn(__fmul2_rn(a, sigmoid2_fast(a)), u);
            m = fmaxf(m, fmaxf(fabsf(h[j].x), fabsf(h[j].y)));
          }
          const uint32_t byte = mx8_scale_byte(m);
          const float inv = mx8_inv_scale(byte);
          word |= byte << (8 * c);
          const float2 inv2 = make_float2(inv, inv);
          uint32_t o[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 lo = __fmul2_rn(h[2 * j], inv2), hi = __fmul2_rn(h[2 * j + 1], inv2);
            o[j] = mx8_pack4(lo.x, lo.y, hi.x, hi.y);
          }
          const int col = t.n0 + 32 * c;
          if (rows_ok) store_sector(p.h + row * p.h_pitch + col, p.sector, W - col, o);
        }
        if (rows_ok)
          *reinterpret_cast<uint32_t*>(p.h_scale + ((int64_t)(row0 >> 7) * p.h_kblocks + (t.n0 >> 7)) * 512 + lane * 16 + quad * 4) = word;
      } else {
#pragma unroll
        for (int ci = 0; ci < 4; ++ci) {
          const int c = 64 * (buf ? ci : 3 - ci), col = t.n0 + c;
          const bool any = __any_sync(0xffffffffu, rows_ok) && col < p.d;      // the same in the whole warp
          if (ci > 0 && !any) continue;
          uint32_t r0[32], r1[32];
          tmem_ld32(taddr + c, r0);
          tmem_ld32(taddr + c + 32, r1);
          tmem_ld_wait();
          if (ci == 0) release();
          if (!any || !rows_ok) continue;
          uint8_t* const out = reinterpret_cast<uint8_t*>(p.y + row * p.d + col);
          const int left = 2 * (p.d - col);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint32_t lo = q < 2 ? r0[16 * q + 2 * j] : r1[16 * (q - 2) + 2 * j];
              const uint32_t hi = q < 2 ? r0[16 * q + 2 * j + 1] : r1[16 * (q - 2) + 2 * j + 1];
              o[j] = pack2(__uint_as_float(lo), __uint_as_float(hi));
            }
            store_sector(out + 32 * q, p.sector, left - 32 * q, o);
          }
        }
      }
      ++n_tile;
    }
  }

  // ---- teardown
  __syncthreads();
  if (*abort_flag) __nanosleep(200000);      // let copies in flight land before the CTA retires
  if (CG == 2) cluster_sync_all();
  tc_fence_after();
  if (warp == 1) {
    if (CG == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// ---------------------------------------------------------------- rows into expert order, making operands

constexpr int kPermK = 4;                  // 128-column blocks a CTA of the permutation takes

// Rows of x8 (rows layout) into expert order, scales into the tiled layout: a CTA takes one 128-row
// block and kPermK column blocks.  Scale words are gathered through shared memory, so that tiles are
// written whole; rows of padding keep whatever the buffers hold.
__global__ void __launch_bounds__(256)
permute_mx8_kernel(int T, int64_t pitch, int kblocks, const uint8_t* __restrict__ x8, const uint8_t* __restrict__ x8_scale,
                   const int32_t* __restrict__ tok_of_prow, uint8_t* __restrict__ xp8,
                   uint8_t* __restrict__ xp8_scale) {
  __shared__ int s_tok[128];
  __shared__ uint32_t s_w[kPermK][129];
  pdl_enter();
  const int rb = blockIdx.x, kb0 = blockIdx.y * kPermK, tid = threadIdx.x;
  int mine = T;
  if (tid < 128) s_tok[tid] = mine = tok_of_prow[rb * 128 + tid];
  if (!__syncthreads_or(mine >= 0 && mine < T)) return;      // past the last segment
  const int nkb = min(kPermK, kblocks - kb0);
  const int64_t c0 = (int64_t)kb0 * 128;
  const int pieces = (int)(min((int64_t)nkb * 128, pitch - c0) >> 4);        // 16-byte pieces of a row
  uint32_t w[128 * kPermK / 256];                                            // scale words, requested first
#pragma unroll
  for (int j = 0; j < 128 * kPermK / 256; ++j) {
    const int i = tid + 256 * j, k = i % kPermK, tok = s_tok[i / kPermK];
    w[j] = k < nkb && tok >= 0 && tok < T ? __ldg(reinterpret_cast<const uint32_t*>(x8_scale) + (int64_t)tok * kblocks + kb0 + k) : 0u;
  }
  constexpr int kRowsAtOnce = 256 / (kPermK * 8);                            // 8 rows by 32 lanes
  const int r_lo = tid >> 5, piece = tid & 31;
  if (piece < pieces) {
#pragma unroll 8
    for (int r = r_lo; r < 128; r += kRowsAtOnce) {
      const int tok = s_tok[r];
      if (tok >= 0 && tok < T)
        *reinterpret_cast<uint4*>(xp8 + (int64_t)(rb * 128 + r) * pitch + c0 + 16 * piece) =
            __ldg(reinterpret_cast<const uint4*>(x8 + (int64_t)tok * pitch + c0 + 16 * piece));
    }
  }
#pragma unroll
  for (int j = 0; j < 128 * kPermK / 256; ++j) s_w[(tid + 256 * j) % kPermK][(tid + 256 * j) / kPermK] = w[j];
  __syncthreads();
  uint32_t* const out = reinterpret_cast<uint32_t*>(xp8_scale) + ((int64_t)rb * kblocks + kb0) * 128;
  for (int i = tid; i < 128 * nkb; i += 256) {
    const int k = i >> 7, w = i & 127;       // word w of a tile: row 32 (w % 4) + w / 4
    out[i] = s_w[k][32 * (w & 3) + (w >> 2)];
  }
}

// `batch` matrices [rows, K] into the operand layout; a thread per eight columns, four neighbouring
// threads per scale.  Rows up to the next multiple of 128 get zero scales.
template <typename T>
__global__ void __launch_bounds__(256)
quantize_mx8_kernel(int64_t batch, int64_t rows, int K, const T* __restrict__ w, uint8_t* __restrict__ q,
                    uint8_t* __restrict__ scale) {
  pdl_enter();
  const int64_t pitch = mx8_pitch(K), kblocks = mx8_kblocks(K), prows = (rows + 127) / 128 * 128;
  const int64_t per_row = kblocks * 16, total = batch * prows * per_row;     // pieces of eight columns, in whole warps of a row
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t br = i / per_row, b = br / prows, r = br - b * prows;
    const int c = (int)(i - br * per_row) * 8;
    float v[8];
    const bool in = r < rows && c < K;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = in ? (float)w[(b * rows + r) * K + c + j] : 0.f;
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(v[j]));
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const uint32_t byte = mx8_scale_byte(m);
    const float inv = mx8_inv_scale(byte);
    if (r < rows && c < pitch) {
      uint2 o = make_uint2(0u, 0u);
      if (in) {
        o.x = mx8_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
        o.y = mx8_pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
      }
      *reinterpret_cast<uint2*>(q + (b * rows + r) * pitch + c) = o;
    }
    if ((c & 31) == 0) scale[b * (prows / 128) * kblocks * 512 + mx8_tiled_offset(r, c / 32, kblocks)] = (uint8_t)byte;
  }
}

// ---------------------------------------------------------------- host side

int32_t encode_u(CUtensorMap* m, CUtensorMapDataType type, CUtensorMapSwizzle swizzle, const void* base, int rank,
                 const uint64_t* dims, const uint64_t* strides, const uint32_t* box) {
  EncodeFn fn = get_encode();
  if (!fn) {
    set_error("cuTensorMapEncodeTiled is not available from the driver");
    return MOHGE_ERR_UNSUPPORTED;
  }
  cuuint64_t gd[5], gs[5];
  cuuint32_t bx[5], es[5];
  for (int i = 0; i < rank; ++i) {
    gd[i] = dims[i];
    bx[i] = box[i];
    es[i] = 1;
    if (i > 0) gs[i - 1] = strides[i - 1];
  }
  const CUresult r = fn(m, type, (cuuint32_t)rank, const_cast<void*>(base), gd, gs, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    set_error("cuTensorMapEncodeTiled failed with %d (rank %d, dims %llu x %llu, box %u x %u)", (int)r, rank,
              (unsigned long long)dims[0], (unsigned long long)dims[1], box[0], box[1]);
    return MOHGE_ERR_CUDA;
  }
  return MOHGE_OK;
}
// elements: [K, rows(, matrices)] bytes in boxes of 128 columns x box_rows rows
int32_t encode_elements(CUtensorMap* m, const void* p, uint64_t K, uint64_t pitch, uint64_t rows, uint64_t mats, uint32_t box_rows) {
  const uint64_t dims[3] = {K, rows, mats}, str[2] = {pitch, pitch * rows};
  const uint32_t box[3] = {BK, box_rows, 1};
  return encode_u(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, CU_TENSOR_MAP_SWIZZLE_128B, p, mats ? 3 : 2, dims, str, box);
}
// tiled scales: [128 words, k-blocks, row blocks(, matrices)]
int32_t encode_scales(CUtensorMap* m, const void* p, uint64_t kblocks, uint64_t rblocks, uint64_t mats, uint32_t box_r, uint32_t box_m) {
  const uint64_t dims[4] = {128, kblocks, rblocks, mats}, str[3] = {512, 512 * kblocks, 512 * kblocks * rblocks};
  const uint32_t box[4] = {128, 1, box_r, box_m};
  return encode_u(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, CU_TENSOR_MAP_SWIZZLE_NONE, p, mats ? 4 : 3, dims, str, box);
}

template <int PHASE, int CG>
int32_t launch_mx(const MxParams& p, const DeviceInfo& di, cudaStream_t st) {
  static std::atomic<int> clusters[kMaxDevices];      // resident CTA pairs (or CTAs), 0: not yet known
  const auto kernel = mx8_grouped_kernel<PHASE, CG>;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(di.sm_count / CG * CG);
  cfg.blockDim = dim3(kThreadsMx);
  cfg.dynamicSmemBytes = GeoMx<CG>::kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CG;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int mc = clusters[di.ordinal].load(std::memory_order_acquire);
  if (!mc) {
    MOHGE_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, GeoMx<CG>::kSmemBytes));
    mc = di.sm_count;
    if (CG == 2) MOHGE_CUDA(cudaOccupancyMaxActiveClusters(&mc, kernel, &cfg));
    if (mc < 1) mc = 1;
    clusters[di.ordinal].store(mc, std::memory_order_release);
  }
  const int want = di.sm_count / CG < mc ? di.sm_count / CG : mc;
  cfg.gridDim = dim3(want * CG);
  cfg.numAttrs = dependent_launch() ? 2 : 1;
  MOHGE_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
  MOHGE_LAUNCH_CHECK("mx8_grouped_kernel");
  return MOHGE_OK;
}

}  // namespace

int32_t launch_permute_mx8(const Dims& D, const void* x8, const void* x8_scale, const int32_t* tok_of_prow, void* xp8,
                           void* xp8_scale, cudaStream_t st) {
  const int kblocks = (int)mx8_kblocks(D.d);
  launch_dep(permute_mx8_kernel, dim3((unsigned)(D.Rcap / 128), (unsigned)ceil_div(kblocks, kPermK)), dim3(256), st, (int)D.T,
             mx8_pitch(D.d), kblocks, (const uint8_t*)x8, (const uint8_t*)x8_scale, tok_of_prow, (uint8_t*)xp8,
             (uint8_t*)xp8_scale);
  MOHGE_LAUNCH_CHECK("permute_mx8_kernel");
  return MOHGE_OK;
}

int32_t launch_quantize_mx8(int64_t batch, int64_t rows, int K, bool bf16, const void* w, void* q, void* scale, cudaStream_t st) {
  const int64_t blocks = (batch * ((rows + 127) / 128 * 128) * mx8_kblocks(K) * 16 + 255) / 256;
  const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384));
  if (bf16)
    launch_dep(quantize_mx8_kernel<__nv_bfloat16>, grid, dim3(256), st, batch, rows, K, (const __nv_bfloat16*)w, (uint8_t*)q,
               (uint8_t*)scale);
  else
    launch_dep(quantize_mx8_kernel<float>, grid, dim3(256), st, batch, rows, K, (const float*)w, (uint8_t*)q, (uint8_t*)scale);
  MOHGE_LAUNCH_CHECK("quantize_mx8_kernel");
  return MOHGE_OK;
}

int32_t launch_experts_mx8(const Dims& D, const void* xp8, const void* xp8_scale, const int32_t* counts,
                           const int32_t* aligned, const GroupPtrs& P,
                           const GroupPtrs& S, void* h8, void* h8_scale, void* y_perm, int32_t* tile_count, Tile* tiles,
                           int64_t tiles_cap, int32_t* status, cudaStream_t st) {
  DeviceInfo di;
  int32_t rc = current_device(&di);
  if (rc) return rc;
  if (di.cc_major != 10) {
    set_error("the 8-bit experts need an sm_100 device (found sm_%d%d)", di.cc_major, di.cc_minor);
    return MOHGE_ERR_UNSUPPORTED;
  }
  // the BF16 path's rule, pairs above 128 rows per expert: 256 tokens against the large layer take 383 us
  // with single CTAs and 493 with pairs, 8192 tokens of the 1024-wide layer 147 and 140
  const int CG = tc_cta_group_size(D);
  int bn1[MOHGE_MAX_GROUPS], bn2[MOHGE_MAX_GROUPS];
  for (int g = 0; g < MOHGE_MAX_GROUPS; ++g) { bn1[g] = BN / 2; bn2[g] = BN; }
  const TilePlan plans[2] = {make_plan(D, ROLE_FWD1, BM * CG, bn1, true), make_plan(D, ROLE_FWD2, BM * CG, bn2, false)};
  rc = launch_build_tiles_multi(plans, 2, aligned, tile_count, tiles, tiles_cap, status, st);
  if (rc) return rc;

  const uint64_t rows = D.Rcap, rblocks = rows / 128, dp = mx8_pitch(D.d), hp = mx8_pitch(D.Wmax);
  const uint64_t dkb = mx8_kblocks(D.d), hkb = mx8_kblocks(D.Wmax), N = D.N;
  MxParams p;
  memset(&p, 0, sizeof(p));
  p.Ng = D.Ng; p.N = D.N; p.d = D.d; p.status = status; p.counts = counts; p.aligned = aligned;
  p.h = (uint8_t*)h8; p.h_pitch = (int64_t)hp; p.y = (__nv_bfloat16*)y_perm;
  p.h_scale = (uint8_t*)h8_scale; p.h_kblocks = (int)hkb;
  for (int g = 0; g < D.Ng; ++g) p.W[g] = D.W[g];
  // phase 1
  p.tile_count = tile_count; p.tiles = tiles;
  p.sector = (((uintptr_t)h8 | hp) & 31) == 0;
  if ((rc = encode_elements(&p.mapA[0], xp8, D.d, dp, rows, 0, BM))) return rc;
  if ((rc = encode_elements(&p.mapA32[0], xp8, D.d, dp, rows, 0, 32))) return rc;
  if ((rc = encode_scales(&p.mapSA, xp8_scale, dkb, rblocks, 0, 1, 0))) return rc;
  for (int g = 0; g < D.Ng; ++g) {
    const uint64_t W = D.W[g];
    if ((rc = encode_elements(&p.mapB[g], P.w13[g], D.d, dp, W, 2 * N, BN / 2))) return rc;
    if ((rc = encode_scales(&p.mapSB[g], S.w13[g], dkb, (W + 127) / 128, 2 * N, 1, 2))) return rc;
  }
  rc = CG == 2 ? launch_mx<1, 2>(p, di, st) : launch_mx<1, 1>(p, di, st);
  if (rc) return rc;
  // phase 2
  p.tile_count = tile_count + 64; p.tiles = tiles + tiles_cap;
  p.sector = (((uintptr_t)y_perm | (uint64_t)(2 * D.d)) & 31) == 0;
  if ((rc = encode_scales(&p.mapSA, h8_scale, hkb, rblocks, 0, 1, 0))) return rc;
  for (int g = 0; g < D.Ng; ++g) {
    const uint64_t W = D.W[g];
    if ((rc = encode_elements(&p.mapA[g], h8, W, hp, rows, 0, BM))) return rc;
    if ((rc = encode_elements(&p.mapA32[g], h8, W, hp, rows, 0, 32))) return rc;
    if ((rc = encode_elements(&p.mapB[g], P.w2[g], W, mx8_pitch(W), D.d, N, BN / CG))) return rc;
    if ((rc = encode_scales(&p.mapSB[g], S.w2[g], mx8_kblocks(W), (D.d + 127) / 128, N, 2, 1))) return rc;
  }
  return CG == 2 ? launch_mx<2, 2>(p, di, st) : launch_mx<2, 1>(p, di, st);
}

}  // namespace mohge
