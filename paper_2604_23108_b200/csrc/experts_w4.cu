// The routed experts for a handful of tokens, with 4-bit weights and a scale per group of columns.
//
//   y[t] = sum_k gate[t,k] W2_e (silu(Wg_e x_t) * Wu_e x_t),  e = expert_idx[t,k],  w = s_group (q - 8)
//
// With few tokens an expert's weights are used for a handful of dot products each, so the time is that
// of streaming the weights of the experts that were picked, once: 3 W d / 2 bytes each plus the scales.
// Everything below serves that stream:
//   - Weights are packed once (pack_w4_kernel) into tiles of 16 rows x 128 columns stored in the order
//     in which the lanes of a warp hold them as the A operand of mma m16n8k16, scales behind them: a
//     warp reads a tile as two fully coalesced 16-byte loads per lane, and an expert's matrix is one
//     contiguous stream of tiles.  In the gate/up matrix rows 0-7 of a tile are gate rows and rows 8-15
//     the up rows of the same hidden columns, so that both halves of SwiGLU meet in one thread.
//   - The legacy warp-level matrix instruction is used on purpose: its accumulators are registers and
//     its smallest token tile is 8 columns; the tensor memory path would need 128-row operand tiles in
//     shared memory, and at 8 tokens the arithmetic is a few per cent of what either can do.
//   - Unpacking has to keep up with the stream on the integer pipe, which issues at half rate, so a pair
//     of weights costs one three-input logic operation and a word of eight one rotation: with the nibbles
//     placed for it, w & 0x03c003c0 | 0x4c004c00 is the pair of FP16 numbers (16 + q, 16 + q') and
//     w & 0x003c003c | 0x5c005c00 the pair (256 + q, 256 + q'), both exact.  The offsets (and the 8 of
//     q - 8) come off as a whole: the accumulator of a group of columns starts at minus
//     24 sum x + 264 sum x over the columns of either kind, summed once per token when it is staged.
//     With products of at most 271 x and FP32 accumulators that costs some 1e-5 of the group's terms.
//     (Subtracting per pair instead made 72 instructions per tile of 40.)  The group's scale multiplies
//     the FP32 sum of the group, so no rounding is spent on the weights.
//   - Tokens therefore enter as FP16 too, each scaled by the power of two that takes its largest element
//     to 2^14..2^15: the BF16 elements of x are exact down to 2^-29 of the largest (and within 2^-39 of it
//     below), the hidden activations, kept in FP32 between the two products, get 11 significant bits.  One
//     operand, because two parts (16 bits) double the second product's matrix instructions and its tokens'
//     shared memory; an activation is off by at most 2^-12 of itself for it, and the output's error against
//     64 bits is 0.0016-0.0017 of its size, that of rounding y to BF16 (a plain form that keeps the
//     activations in 32 bits has the same two digits).
//   - Work is cut evenly over the SMs by cost: the chunks (expert, up to 8 of its tokens) lie on one
//     line, chunk after chunk, tile row after tile row, and every CTA takes an equal stretch of it (whole
//     tile rows).  Ahead of a chunk's rows the line has what beginning the chunk costs (chunk_cost; one
//     token through the large layer 28.3 -> 20-25 us in calls that repeat, so that its weights are in L2
//     (24-27 from DRAM now), seven through the 1024-wide one 23.1 -> 18.4, 64 242 -> 236).
//     Inside a CTA the 16 warps cut the stretch again into equal runs of tiles, wherever in a row that
//     falls.  A run is contiguous in memory: one lane brings it with untiled bulk copies, four tiles
//     each, into a ring of the warp's own in shared memory, as deep as the tokens leave room (two
//     copies, 130 KB in flight per SM, at eight tokens and d = 4096).  (Loads into registers, six tiles
//     ahead, reached 3.2 TB/s: the hardware tracks too few of them apart.)  A row that lies inside a run
//     is finished by its warp alone, and rows that runs share are added up in warp order after one barrier
//     per chunk.  Nothing depends on timing: the same inputs give the same bits.
//   - At 64 tokens the call takes 233-238 us for 1.05 GB (4.4 TB/s): the integer pipe is busy half of the
//     time and nothing is streamed while a chunk's tokens are staged.
// The second product's results are kept per (token, expert) pair in FP32 and added over a token's
// experts, in slot order, by combine_w4_kernel, which rounds once.

#include <atomic>

#include <cuda_fp16.h>

#include "common.cuh"
#include "tc_ptx.cuh"

namespace mohge {
namespace {

constexpr int kThreadsW4 = 512;
constexpr int kWarpsW4 = kThreadsW4 / 32;
constexpr int kChunk = 8;                        // tokens per chunk: columns of the matrix instruction
constexpr int kTileK = 128;                      // columns of a packed tile
// What beginning a chunk costs a CTA (pair list, staging, an empty ring, the barriers around them), in
// tiles streamed: a line through the clocks of all CTAs has 45-50 clocks per tile, 5000-5900 per chunk and
// 49 per token and 128 columns staged.  Left out, CTAs that had several chunks finished last (64 tokens
// against the large layer: 247k clocks against 221k on average).
constexpr int kChunkTiles = 110;
__device__ __forceinline__ int chunk_cost(int tokens, int steps) { return kChunkTiles + tokens * steps; }

__host__ __device__ constexpr int tile_bytes(int sets) { return 1024 + 32 * sets; }

struct W4Params {
  const uint8_t* w[MOHGE_MAX_GROUPS];            // packed matrices of this phase
  int W[MOHGE_MAX_GROUPS];
  int Ng, N, Ke, d, Wp;                          // Wp: row pitch of the hidden activations
  int pairs;                                     // tokens * K_e of this slab
  int slots;                                     // of a warp's ring
  int chunk, chunk_log;                          // tokens per chunk: a power of two, at most kChunk
  int cs_bytes;                                  // of the starting values
  const __nv_bfloat16* x;                        // [T, d]
  const int32_t* expert_idx;
  const float* gate;
  float* h;                                      // hidden activations [pairs, Wp]
  float* part;                                   // [pairs, d]
  int32_t* status;
};

constexpr int kMaxSlots = 8;
constexpr int kMostSmem = 227 * 1024;            // of a block

// Columns 2 j and 2 j + 1 of a word's eight as FP16 numbers, 16 + q for even j and 256 + q for odd j.  The
// magic numbers are kept in registers so that mask and magic are one instruction.
constexpr float kOffEven = 24.f, kOffOdd = 264.f;        // what has to come off: 16 + 8 and 256 + 8
__device__ __forceinline__ void dequant(uint32_t (&a)[4], uint32_t w, uint32_t magic0, uint32_t magic1) {
  const uint32_t r = __funnelshift_r(w, w, 8);
  asm("lop3.b32 %0, %1, 0x03c003c0, %2, 0xea;" : "=r"(a[0]) : "r"(w), "r"(magic0));
  asm("lop3.b32 %0, %1, 0x003c003c, %2, 0xea;" : "=r"(a[1]) : "r"(w), "r"(magic1));
  asm("lop3.b32 %0, %1, 0x03c003c0, %2, 0xea;" : "=r"(a[2]) : "r"(r), "r"(magic0));
  asm("lop3.b32 %0, %1, 0x003c003c, %2, 0xea;" : "=r"(a[3]) : "r"(r), "r"(magic1));
}
// the bit where the nibble of column c of a word's eight begins (the last ones wrap around)
__device__ __forceinline__ int nibble_bit(int c) {
  const int j = c >> 1;
  return (j == 0 ? 6 : j == 1 ? 2 : j == 2 ? 14 : 10) + 16 * (c & 1);
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same on an accumulator that starts at (c0, c1) in every row
__device__ __forceinline__ void mma_f16_from(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1, float c0, float c1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %10, %11};"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
}

extern __shared__ __align__(128) uint8_t smem[];
__device__ __forceinline__ float2 ld_shared_f2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}

// acc += tile . x for one tile; shared addresses: tl of this lane's 16 bytes of the tile, ts of its scales,
// xa of its (token, 8 t) in the tile's columns, ca of its two tokens' starting values for the tile's groups.
// Left in program order: with everything requested first and two chains of matrix instructions, the
// compiler free to interleave, 64 tokens took 242 us instead of 234.
template <int S>
__device__ __forceinline__ void consume(float (&acc)[4], uint32_t tl, uint32_t ts, uint32_t xa, uint32_t ca,
                                        uint32_t magic0, uint32_t magic1) {
  constexpr int kPer = 4 / S;                    // words per group of columns
  const uint4 fa = ld_shared_v4(tl), fb = ld_shared_v4(tl + 512);
  const uint32_t wa[4] = {fa.x, fa.y, fa.z, fa.w}, wb[4] = {fb.x, fb.y, fb.z, fb.w};
  uint32_t sc[4];                                // (scale of row g, scale of row g + 8) per group
  if constexpr (S == 1) {
    sc[0] = ld_shared_u32(ts);
  } else if constexpr (S == 2) {
    const float2 v = ld_shared_f2(ts);
    sc[0] = __float_as_uint(v.x); sc[1] = __float_as_uint(v.y);
  } else {
    const uint4 v = ld_shared_v4(ts);
    sc[0] = v.x; sc[1] = v.y; sc[2] = v.z; sc[3] = v.w;
  }
  float c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 x = ld_shared_v4(xa + i * 64);
    uint32_t a[4], b[4];
    dequant(a, wa[i], magic0, magic1);
    dequant(b, wb[i], magic0, magic1);
    if (i % kPer == 0) {
      const float2 c0 = ld_shared_f2(ca + (i / kPer) * (kChunk * 4));
      mma_f16_from(c, a[0], b[0], a[1], b[1], x.x, x.y, c0.x, c0.y);
    } else {
      mma_f16(c, a[0], b[0], a[1], b[1], x.x, x.y);
    }
    mma_f16(c, a[2], b[2], a[3], b[3], x.z, x.w);
    if ((i + 1) % kPer == 0) {
      const uint32_t s = sc[i / kPer];
      const float s0 = __uint_as_float(s << 16), s1 = __uint_as_float(s & 0xffff0000u);
      acc[0] = fmaf(s0, c[0], acc[0]);
      acc[1] = fmaf(s0, c[1], acc[1]);
      acc[2] = fmaf(s1, c[2], acc[2]);
      acc[3] = fmaf(s1, c[3], acc[3]);
    }
  }
}

// Exponent a token is scaled by: the largest element goes to 2^14..2^15; 0 for a token of zeros or one
// with an infinity
__device__ __forceinline__ int token_exponent(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23);
  return e == 0 || e == 255 ? 0 : 127 + 14 - e;
}
__device__ __forceinline__ float pow2(int e) {   // -127 < e < 128 in one step, the rest by the caller
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// a / b for 0 <= a < 2^31, 0 < b, quotients below 2^22: the approximate one is off by one at most
__device__ __forceinline__ int quotient(int a, int b) {
  int q = __float2int_rz(__int2float_rn(a) * rcp_approx(__int2float_rn(b)));
  const int r = a - q * b;
  if (r < 0) --q;
  else if (r >= b) ++q;
  return q;
}

struct __align__(128) SmemW4 {
  int32_t idx[kW4MaxPairs];                      // expert of each pair, -1 for an invalid one
  int32_t count[256], unit[256], group[256];     // per expert: pairs, tiles of its matrix, group
  const uint8_t* w[MOHGE_MAX_GROUPS];            // per group, from the parameters (indexing those costs a
  int32_t rows[MOHGE_MAX_GROUPS], steps[MOHGE_MAX_GROUPS], cols[MOHGE_MAX_GROUPS];   // memory round trip)
  int32_t hit[256], start[257];                  // the experts that have pairs, and the cost before each
  int32_t hits, first;                           // how many, and the one in which this CTA's stretch begins
  int32_t pair[kChunk];                          // pairs of the current chunk
  float gate[kChunk];                            // and their gates (phase 2)
  float2 unscale[kChunk];                        // what a token's results are multiplied by, in two steps
  float warp_max[kWarpsW4];                      // largest magnitude of each warp's part of a token
  uint64_t full[kWarpsW4][kMaxSlots];            // a slot's tiles have landed
  int32_t abort;
  // rows that runs share: [0] the end (or the middle) of the row a run begins in, [1] the beginning of
  // the row it ends in
  int32_t part_row[kWarpsW4][2];
  float4 part[kWarpsW4][2][32];
};

// PHASE 1: hidden activations from x; PHASE 2: per-pair outputs from the hidden activations.
// SLOT: tiles per bulk copy
template <int PHASE, int S, int SLOT>
__global__ void __launch_bounds__(kThreadsW4, 1) experts_w4_kernel(const __grid_constant__ W4Params p) {
  constexpr int kTile = tile_bytes(S), kSlotBytes = SLOT * kTile;
  SmemW4& sm = *reinterpret_cast<SmemW4*>(smem);
  // the warps' rings, the tokens' starting values [groups of columns][8], the tokens
  float* const cs = reinterpret_cast<float*>(smem + sizeof(SmemW4) + (size_t)kWarpsW4 * p.slots * SLOT * tile_bytes(S));
  uint8_t* const xs = reinterpret_cast<uint8_t*>(cs) + p.cs_bytes;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int Ne = p.Ng * p.N;
  uint32_t magic0 = 0x4c004c00u, magic1 = 0x5c005c00u;
  asm volatile("" : "+r"(magic0), "+r"(magic1));

  const uint32_t ring = smem_u32(smem) + (uint32_t)sizeof(SmemW4) + warp * p.slots * kSlotBytes;
  if (tid == 0) sm.abort = 0;
  if (lane < p.slots) mbar_init(smem_u32(&sm.full[warp][lane]), 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  const uint32_t full0 = smem_u32(&sm.full[warp][0]);
  int slot = 0;                                  // next slot of the ring, and its phase
  uint32_t phase = 0;

  static_assert(kThreadsW4 >= 256 && kThreadsW4 >= kW4MaxPairs, "one expert and one pair per thread");
  if (tid < 256) {
    const int g = tid < Ne ? tid / p.N : 0, W = p.W[g];
    const int rows = PHASE == 1 ? W >> 3 : (p.d + 15) >> 4, cols = PHASE == 1 ? p.d : W, steps = (cols + kTileK - 1) / kTileK;
    sm.count[tid] = 0;
    sm.unit[tid] = tid < Ne ? rows * steps : 0;
    sm.group[tid] = g;
    if (tid < Ne && g * p.N == tid) {            // the group's first expert
      sm.w[g] = p.w[g];
      sm.rows[g] = rows;
      sm.steps[g] = steps;
      sm.cols[g] = cols;
    }
  }

  // Phase 1 reads what earlier kernels of the stream wrote: it waits first and lets phase 2 be
  // scheduled after that.  So when phase 2 runs, everything before phase 1 is complete: it may read
  // the routing and the weights at once and waits only before it touches the hidden activations.
  if (PHASE == 1) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  } else {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }

  // ---- which experts were picked, and how much work each is
  if (PHASE == 1) {        // x is on its way to L2 meanwhile: every CTA asks for a part
    const int64_t i = ((int64_t)blockIdx.x * kThreadsW4 + tid) * 64;
    if (i < (int64_t)(p.pairs / p.Ke) * p.d) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.x + i));
  }
  __syncthreads();
  if (tid < p.pairs) {
    const int e = p.expert_idx[tid];
    const bool ok = e >= 0 && e < Ne;
    sm.idx[tid] = ok ? e : -1;
    if (ok) atomicAdd(&sm.count[e], 1);
    else if (PHASE == 1 && blockIdx.x == 0) atomicCAS(p.status, 0, (2 << 24) | 40);
  }
  __syncthreads();
  // every CTA's stretch of the cost line: total * b / ctas, in 32 bits
  auto stretch = [&](int total, int b) {
    const int q = quotient(total, gridDim.x);
    return q * b + quotient((total - q * (int)gridDim.x) * b, gridDim.x);
  };
  if (warp == 0) {                               // eight experts per lane: their costs, summed up
    int cost[8], sum = 0, n = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = lane * 8 + j;
      cost[j] = ((sm.count[e] + p.chunk - 1) >> p.chunk_log) *
                (sm.unit[e] + chunk_cost(min(sm.count[e], p.chunk), sm.steps[sm.group[e]]));
      sum += cost[j];
      n += cost[j] > 0;
    }
    int before = sum, place = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, before, o), w = __shfl_up_sync(0xffffffffu, place, o);
      if (lane >= o) { before += u; place += w; }
    }
    const int total = __shfl_sync(0xffffffffu, before, 31), hits = __shfl_sync(0xffffffffu, place, 31);
    before -= sum;
    place -= n;
    const int lo = stretch(total, blockIdx.x);
    if (lane == 0) {
      sm.hits = hits;
      sm.first = hits;
      sm.start[hits] = total;
    }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (cost[j] > 0) {
        sm.hit[place] = lane * 8 + j;
        sm.start[place] = before;
        if (before <= lo && lo < before + cost[j]) sm.first = place;
        before += cost[j];
        ++place;
      }
    }
  }
  __syncthreads();
  const int hits = sm.hits, total = sm.start[hits];
  const int lo_cost = stretch(total, blockIdx.x), hi_cost = stretch(total, blockIdx.x + 1);
  bool waited = PHASE == 1;

  for (int at = sm.first; at < hits && sm.start[at] < hi_cost; ++at) {
    const int e = sm.hit[at], cnt = sm.count[e];
    const int g = sm.group[e], rows = sm.rows[g], steps = sm.steps[g];
    const int chunks = (cnt + p.chunk - 1) >> p.chunk_log;
    const uint8_t* const mat = sm.w[g] + (size_t)(e - g * p.N) * rows * steps * kTile;
    const int K = sm.cols[g];
    const uint32_t pitch = steps * kTileK * 2 + 64;          // 64 mod 128: eight lanes hit all banks

    for (int ch = 0; ch < chunks; ++ch) {
      const int begin = chunk_cost(min(cnt, p.chunk), steps);        // on the line ahead of the chunk's rows
      const int base = sm.start[at] + ch * (rows * steps + begin) + begin;
      const int r0 = lo_cost <= base ? 0 : quotient(lo_cost - base + steps - 1, steps);
      int r1 = hi_cost <= base ? 0 : quotient(hi_cost - base + steps - 1, steps);
      r1 = min(r1, rows);
      if (r0 >= r1) continue;
      const int nrows = r1 - r0;
      // ---- this warp's run of tiles
      const int n = nrows * steps, i_begin = n * warp / kWarpsW4, n_run = n * (warp + 1) / kWarpsW4 - i_begin;
      const int row_first = quotient(i_begin, steps);
      // the next request's source and the tiles still to be requested (lane 0 alone)
      const uint8_t* src = mat + ((size_t)r0 * steps + i_begin) * kTile;
      int ask = n_run;
      auto request = [&](int sl) {
        const uint32_t bytes = ask >= SLOT ? kSlotBytes : ask * kTile, bar = full0 + sl * 8;
        mbar_expect_tx(bar, bytes);
        bulk_load(ring + sl * kSlotBytes, src, bytes, bar);
        src += kSlotBytes;
        ask -= SLOT;
      };
      __syncthreads();                           // the previous chunk's pair list and tokens are done with
      // ---- the chunk's tokens (phase 1) or hidden activations (phase 2), scaled to FP16, zeros up to the
      // end of the last tile.  A token is shared by whole warps.  Loops are kept rolled here and below: a
      // launch of one token runs through this code once, and fetching instructions is what it costs then.
      const int ntok = min(p.chunk, cnt - ch * p.chunk);
      {
        const int vecs = steps * (kTileK / 8);
        const int per_log = 9 - (ntok > 4 ? 3 : ntok > 2 ? 2 : ntok - 1), per = 1 << per_log;
        static_assert(kThreadsW4 == 1 << 9, "threads per token");
        const int nn = tid >> per_log, v0 = tid & (per - 1);
        // its pair: the one of rank nn among this chunk's, pairs in ascending order
        int pr = 0;
        {
          const int rank = ch * p.chunk + nn;
          int seen = 0;
#pragma unroll 1
          for (int i0 = 0; i0 < p.pairs && seen <= rank; i0 += 32) {
            uint32_t m = __ballot_sync(0xffffffffu, i0 + lane < p.pairs && sm.idx[i0 + lane] == e);
            const int in = __popc(m);
            if (rank < seen + in) {
#pragma unroll 1
              for (int k = seen; k < rank; ++k) m &= m - 1;
              pr = i0 + __ffs(m) - 1;
            }
            seen += in;
          }
        }
        const uint4* const src1 = reinterpret_cast<const uint4*>(p.x + (size_t)(pr / p.Ke) * p.d);
        uint4 first = make_uint4(0, 0, 0, 0);
        if (PHASE == 1 && nn < ntok && 8 * v0 < K) first = src1[v0];
        // The ring (empty here) is filled behind the first request for the tokens, which would queue behind
        // it otherwise, but ahead of a wait for phase 1
        if (lane == 0) {
#pragma unroll 1
          for (int k = 0; k < p.slots && ask > 0; ++k) request(slot + k < p.slots ? slot + k : slot + k - p.slots);
        }
        if (!waited) {
          asm volatile("griddepcontrol.wait;" ::: "memory");
          waited = true;
        }
        const float4* const src2 = reinterpret_cast<const float4*>(p.h + (size_t)pr * p.Wp);
        uint8_t* const dst = xs + (size_t)nn * pitch;
        float m = 0.f;
        if (nn < ntok) {
          if (PHASE == 1) {                      // the raw elements wait where their FP16 form will stand
#pragma unroll 4
            for (int v = v0; v < vecs; v += per) {
              const uint4 q = v == v0 ? first : 8 * v < K ? src1[v] : make_uint4(0, 0, 0, 0);
              *reinterpret_cast<uint4*>(dst + 16 * v) = q;
              const __nv_bfloat162* const h = reinterpret_cast<const __nv_bfloat162*>(&q);
              const __nv_bfloat162 a = __hmax2(__hmax2(__habs2(h[0]), __habs2(h[1])), __hmax2(__habs2(h[2]), __habs2(h[3])));
              m = fmaxf(m, fmaxf(__low2float(a), __high2float(a)));
            }
          } else {
#pragma unroll 4
            for (int v = 2 * v0; 4 * v < K; v += 2 * per) {
              const float4 a = src2[v], b = src2[v + 1];
              m = fmaxf(m, fmaxf(fmaxf(fmaxf(fabsf(a.x), fabsf(a.y)), fmaxf(fabsf(a.z), fabsf(a.w))),
                                 fmaxf(fmaxf(fabsf(b.x), fabsf(b.y)), fmaxf(fabsf(b.z), fabsf(b.w)))));
            }
          }
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
          if (lane == 0) sm.warp_max[warp] = m;
        }
        __syncthreads();
        if (nn < ntok) {
          m = 0.f;
#pragma unroll 1
          for (int w = 0; w < per / 32; ++w) m = fmaxf(m, sm.warp_max[nn * (per / 32) + w]);
          const int ex = token_exponent(__float_as_uint(m));
          const float s0 = pow2(ex / 2), s1 = pow2(ex - ex / 2);
          if (v0 == 0) {
            sm.pair[nn] = pr;
            if (PHASE == 2) sm.gate[nn] = p.gate[pr];
            sm.unscale[nn] = make_float2(pow2(-ex / 2), pow2(-ex - -ex / 2));
          }
#pragma unroll 1
          for (int v = v0; v - lane < vecs; v += per) {      // by whole warps: the groups' sums are shuffled
            float2 f[4];
            if (PHASE == 1) {
              const uint4 q = v < vecs ? *reinterpret_cast<const uint4*>(dst + 16 * v) : make_uint4(0, 0, 0, 0);
              const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
              for (int j = 0; j < 4; ++j) f[j] = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
            } else {
              float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
              if (8 * v < K) { a = src2[2 * v]; b = src2[2 * v + 1]; }
              f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w); f[2] = make_float2(b.x, b.y); f[3] = make_float2(b.z, b.w);
            }
            float sum[2] = {0.f, 0.f};
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const __half2 hh = __floats2half2_rn(f[j].x * s0 * s1, f[j].y * s0 * s1);
              o[j] = *reinterpret_cast<const uint32_t*>(&hh);
              const float2 r = __half22float2(hh);
              sum[j & 1] += r.x + r.y;
            }
            float off = -(kOffEven * sum[0] + kOffOdd * sum[1]);
            constexpr int kLanes = kTileK / S / 8;           // lanes per group of columns
#pragma unroll
            for (int k = 1; k < kLanes; k *= 2) off += __shfl_xor_sync(0xffffffffu, off, k);
            if (v < vecs) {
              *reinterpret_cast<uint4*>(dst + 16 * v) = make_uint4(o[0], o[1], o[2], o[3]);
              if ((v & (kLanes - 1)) == 0) cs[v / kLanes * kChunk + nn] = off;
            }
          }
        }
      }
      __syncthreads();

      // ---- stream
      auto finish = [&](int row, float4 v) {     // a complete tile row: (row g, tokens 2 t, 2 t + 1), (row g + 8, same)
        const int gr = lane >> 2;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int tok = 2 * (lane & 3) + j;
          if (tok < ntok) {
            const int pr = sm.pair[tok];
            const float2 u = sm.unscale[tok];
            const float top = (j ? v.y : v.x) * u.x * u.y, bot = (j ? v.w : v.z) * u.x * u.y;
            if (PHASE == 1) {
              p.h[(size_t)pr * p.Wp + (r0 + row) * 8 + gr] = top / (1.0f + __expf(-top)) * bot;
            } else {
              const float gt = sm.gate[tok];
              const int c = (r0 + row) * 16 + gr;
              float* o = p.part + (size_t)pr * p.d + c;
              if (c < p.d) o[0] = gt * top;
              if (c + 8 < p.d) o[8] = gt * bot;
            }
          }
        }
      };
      const uint32_t x0 = smem_u32(xs) + min(lane >> 2, p.chunk - 1) * pitch + (lane & 3) * 16;
      const uint32_t c0 = smem_u32(cs) + (lane & 3) * 8;
      constexpr uint32_t kXStep = kTileK * 2, kCStep = S * kChunk * 4;       // per tile
      int row = row_first, s = i_begin - row_first * steps;
      bool whole = s == 0;                       // the run has the current row from its beginning
      if (lane < 2) sm.part_row[warp][lane] = -1;
      uint32_t xa = x0 + s * kXStep, ca = c0 + s * kCStep;
      float acc[4] = {0.f, 0.f, 0.f, 0.f};
      __syncwarp();
      auto row_end = [&]() {                     // of the row, or of the run inside it
        const float4 v = make_float4(acc[0], acc[1], acc[2], acc[3]);
        if (s == steps && whole) {
          finish(row, v);
        } else {
          sm.part[warp][whole][lane] = v;
          if (lane == 0) sm.part_row[warp][whole] = row;
        }
        ++row;
        s = 0;
        whole = true;
        xa = x0;
        ca = c0;
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[q] = 0.f;
      };
      for (int left = n_run; left > 0; left -= SLOT) {
        (void)mbar_wait(full0 + slot * 8, phase, &sm.abort, p.status, 41);
        const uint32_t tl = ring + slot * kSlotBytes + lane * 16;
        const uint32_t ts = ring + slot * kSlotBytes + 1024 + (lane >> 2) * (S * 4);
#pragma unroll 1
        for (int j = 0; j < SLOT && j < left; ++j) {
          consume<S>(acc, tl + j * kTile, ts + j * kTile, xa, ca, magic0, magic1);
          xa += kXStep;
          ca += kCStep;
          if (++s == steps || j + 1 == left) row_end();
        }
        __syncwarp();                            // every lane has read the slot
        if (lane == 0 && ask > 0) request(slot);
        if (++slot == p.slots) { slot = 0; phase ^= 1u; }
      }
      __syncthreads();
      // a shared row is added up by the warp that has its beginning, in warp order
      const int shared_row = sm.part_row[warp][1];
      if (shared_row >= 0) {
        float4 v = sm.part[warp][1][lane];
#pragma unroll 1
        for (int w = warp + 1; w < kWarpsW4; ++w) {
          const int r = sm.part_row[w][0];
          if (r != shared_row) {
            if (r >= 0 || sm.part_row[w][1] >= 0) break;     // past the row; else a run without tiles, or of whole rows
            continue;
          }
          const float4 u = sm.part[w][0][lane];
          v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
        }
        finish(shared_row, v);
      }
    }
  }
  // every thread of phase 2 has to have waited for phase 1 before the grid ends: what follows in the
  // stream is released by the end of this grid
  if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
  if (*(volatile int32_t*)&sm.abort) __nanosleep(200000);   // a wait gave up: let copies in flight land
}

// y[t] = sum over the token's experts, in slot order (+ y_add), rounded once
__global__ void __launch_bounds__(256)
combine_w4_kernel(int T, int d, int Ke, int Ne, const int32_t* __restrict__ expert_idx, const float* __restrict__ part,
                  const __nv_bfloat16* y_add, __nv_bfloat16* y) {
  pdl_enter();
  const int i = blockIdx.x * 256 + threadIdx.x, np = d >> 2;
  if (i >= T * np) return;
  const int t = i / np, c = (i - t * np) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = 0; k < Ke; ++k) {
    const int e = expert_idx[t * Ke + k];
    if (e < 0 || e >= Ne) continue;
    const float4 v = *reinterpret_cast<const float4*>(part + ((size_t)t * Ke + k) * d + c);
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  if (y_add) {
    const __nv_bfloat162* a = reinterpret_cast<const __nv_bfloat162*>(y_add + (size_t)t * d + c);
    const float2 a0 = __bfloat1622float2(a[0]), a1 = __bfloat1622float2(a[1]);
    s.x += a0.x; s.y += a0.y; s.z += a1.x; s.w += a1.y;
  }
  __nv_bfloat162* o = reinterpret_cast<__nv_bfloat162*>(y + (size_t)t * d + c);
  o[0] = __floats2bfloat162_rn(s.x, s.y);
  o[1] = __floats2bfloat162_rn(s.z, s.w);
}

// ---------------------------------------------------------------- making the weights

// Codes and scales of w [rows, K]: a warp per group of columns.  scale = bf16(max|w| / 7), code =
// nearest integer to w / scale, clipped to -8..7, plus 8; true divisions, so that the codes are those
// of the definition.  A group of zeros has scale 0 and codes 8.
template <typename T>
__global__ void __launch_bounds__(256)
quantize_w4_kernel(int64_t rows, int K, int group, const T* __restrict__ w, uint8_t* __restrict__ q,
                   __nv_bfloat16* __restrict__ scale) {
  pdl_enter();
  const int ng = (K + group - 1) / group, lane = threadIdx.x & 31;
  for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < rows * ng; i += (int64_t)gridDim.x * 8) {
    const int64_t r = i / ng;
    const int k0 = (int)(i - r * ng) * group, k1 = min(K, k0 + group);
    float m = 0.f;
    for (int k = k0 + lane; k < k1; k += 32) m = fmaxf(m, fabsf((float)w[r * K + k]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const __nv_bfloat16 sb = __float2bfloat16_rn(__fdiv_rn(m, 7.0f));
    const float s = __bfloat162float(sb);
    if (lane == 0) scale[i] = sb;
    for (int k = k0 + 2 * lane; k < k1; k += 64) {
      int c[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float v = s != 0.f ? rintf(__fdiv_rn((float)w[r * K + k + j], s)) : 0.f;
        c[j] = (int)fminf(fmaxf(v, -8.f), 7.f) + 8;
      }
      q[(r * K + k) >> 1] = (uint8_t)(c[0] | (c[1] << 4));
    }
  }
}

// Codes [batch, rows, K / 2] (two to a byte, the even column low) and scales [batch, rows, ceil(K / group)]
// into packed tiles.  gate_up: rows 0-7 of tile row r are rows 8 r .. of the first half, rows 8-15 those
// of the second half.  One warp per tile; what lies outside the matrix has code 8 and scale 0.
__global__ void __launch_bounds__(256)
pack_w4_kernel(int64_t batch, int rows, int K, int group, int gate_up, const uint8_t* __restrict__ q,
               const __nv_bfloat16* __restrict__ scale, uint8_t* __restrict__ out) {
  pdl_enter();
  const int S = kTileK / group, steps = (K + kTileK - 1) / kTileK, ng = (K + group - 1) / group;
  const int trows = gate_up ? rows / 16 : (rows + 15) / 16;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t tiles = batch * trows * steps;
  for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < tiles; i += (int64_t)gridDim.x * 8) {
    const int st = (int)(i % steps);
    const int64_t br = i / steps, b = br / trows;
    const int tr = (int)(br - b * trows);
    uint8_t* const o = out + i * tile_bytes(S);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int row = gate_up ? half * (rows / 2) + tr * 8 + g : tr * 16 + half * 8 + g;
      const uint8_t* const src = q + ((b * rows + row) * (int64_t)K >> 1);
      uint32_t w[4];
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const int k = st * kTileK + 32 * i4 + 8 * t;
        uint32_t v = 0x88888888u;
        if (row < rows && k < K) {               // K is a multiple of 8: a word is inside or outside
          v = 0;
          for (int c = 0; c < 8; ++c) {
            const uint32_t q4 = (src[(k + c) >> 1] >> (4 * (c & 1))) & 15;
            v |= __funnelshift_l(q4, q4, nibble_bit(c));
          }
        }
        w[i4] = v;
      }
      *reinterpret_cast<uint4*>(o + half * 512 + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    for (int j = lane; j < 8 * S; j += 32) {
      const int gg = j / S, set = j % S, grp = st * S + set;
      uint32_t v = 0;
      for (int half = 0; half < 2; ++half) {
        const int row = gate_up ? half * (rows / 2) + tr * 8 + gg : tr * 16 + half * 8 + gg;
        if (row < rows && grp < ng)
          v |= (uint32_t)__bfloat16_as_ushort(scale[(b * rows + row) * ng + grp]) << (16 * half);
      }
      reinterpret_cast<uint32_t*>(o + 1024)[j] = v;
    }
  }
}

int xs_bytes(int tokens, int K) { return tokens * ((K + kTileK - 1) / kTileK * kTileK * 2 + 64); }
int cs_bytes(int sets, int K) { return (K + kTileK - 1) / kTileK * sets * kChunk * 4; }

template <int PHASE, int S, int SLOT>
int32_t launch_slot(W4Params p, int fixed, const DeviceInfo& di, cudaStream_t st) {
  constexpr int kSlot = kWarpsW4 * SLOT * tile_bytes(S);
  static std::atomic<bool> set[kMaxDevices];
  const auto kernel = experts_w4_kernel<PHASE, S, SLOT>;
  if (!set[di.ordinal].load(std::memory_order_acquire)) {
    MOHGE_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem));
    set[di.ordinal].store(true, std::memory_order_release);
  }
  p.slots = (kMostSmem - fixed) / kSlot;
  if (p.slots > kMaxSlots) p.slots = kMaxSlots;
  launch_dep_smem(kernel, dim3(di.sm_count), dim3(kThreadsW4), fixed + p.slots * kSlot, st, p);
  MOHGE_LAUNCH_CHECK("experts_w4_kernel");
  return MOHGE_OK;
}

// What the tokens leave of a block's shared memory goes to the rings.  Four tiles per copy where two such
// slots fit (up to eight tokens of 4096 columns), else two: per copy the consumer spends some 30
// instructions on waiting and asking for the next one (64 tokens: 229 against 242 us).  Blocks of half an
// SM, so that phase 2 would be resident beside phase 1, were slower (one token: 45 against 31 us): the
// scheduler puts two blocks of phase 1 on one SM.
template <int PHASE, int S>
int32_t launch_phase(W4Params p, int K, const DeviceInfo& di, cudaStream_t st) {
  constexpr int kWidest = kW4MaxD > kW4MaxW ? kW4MaxD : kW4MaxW, kTwo = kWarpsW4 * 2 * tile_bytes(S);
  static_assert(kMostSmem - (int)sizeof(SmemW4) - kChunk * (kWidest * 2 + 64) - kWidest / kTileK * S * kChunk * 4 >= kTwo, "one slot at least");
  p.cs_bytes = cs_bytes(S, K);
  const int fixed = (int)sizeof(SmemW4) + p.cs_bytes + xs_bytes(p.chunk, K);
  return kMostSmem - fixed >= 4 * kTwo ? launch_slot<PHASE, S, 4>(p, fixed, di, st) : launch_slot<PHASE, S, 2>(p, fixed, di, st);
}

template <int PHASE>
int32_t launch_sets(int sets, const W4Params& p, int K, const DeviceInfo& di, cudaStream_t st) {
  if (sets == 1) return launch_phase<PHASE, 1>(p, K, di, st);
  if (sets == 2) return launch_phase<PHASE, 2>(p, K, di, st);
  return launch_phase<PHASE, 4>(p, K, di, st);
}

}  // namespace

int64_t w4_packed_bytes(int64_t batch, int64_t rows, int64_t K, int group) {
  return batch * ((rows + 15) / 16) * ((K + kTileK - 1) / kTileK) * tile_bytes(kTileK / group);
}

int w4_slab_tokens(const Dims& D) {
  const int most = kW4MaxPairs / D.Ke;
  return most < kW4SlabTokens ? most : kW4SlabTokens;
}

W4Scratch w4_scratch(const Dims& D) {
  W4Scratch s;
  const int64_t tokens = D.T < w4_slab_tokens(D) ? D.T : w4_slab_tokens(D), pairs = tokens * D.Ke;
  s.pitch = (D.Wmax + kTileK - 1) / kTileK * kTileK;
  s.part_off = pairs * s.pitch * 4;
  s.total = s.part_off + pairs * D.d * 4;
  return s;
}

int32_t launch_experts_w4(const Dims& D, int group, const void* x, const int32_t* expert_idx, const float* gate_w,
                          const GroupPtrs& P, const void* y_add, void* scratch, void* y, int32_t* status,
                          cudaStream_t st) {
  DeviceInfo di;
  int32_t rc = current_device(&di);
  if (rc) return rc;
  const W4Scratch L = w4_scratch(D);
  const int slab = w4_slab_tokens(D), sets = kTileK / group;
  for (int64_t t0 = 0; t0 < D.T; t0 += slab) {
    const int tokens = (int)(D.T - t0 < slab ? D.T - t0 : slab);
    W4Params p = {};
    for (int g = 0; g < D.Ng; ++g) p.W[g] = D.W[g];
    p.Ng = D.Ng; p.N = D.N; p.Ke = D.Ke; p.d = D.d; p.Wp = L.pitch;
    p.pairs = tokens * D.Ke;
    // an expert rarely sees a token twice: chunks no longer than the batch leave more room for the rings
    p.chunk_log = tokens >= kChunk ? 3 : tokens > 2 ? 2 : tokens - 1;
    p.chunk = 1 << p.chunk_log;
    p.x = (const __nv_bfloat16*)x + t0 * D.d;
    p.expert_idx = expert_idx + t0 * D.Ke;
    p.gate = gate_w + t0 * D.Ke;
    p.h = (float*)scratch;
    p.part = (float*)((char*)scratch + L.part_off);
    p.status = status;
    for (int g = 0; g < D.Ng; ++g) p.w[g] = (const uint8_t*)P.w13[g];
    rc = launch_sets<1>(sets, p, D.d, di, st);
    if (rc) return rc;
    for (int g = 0; g < D.Ng; ++g) p.w[g] = (const uint8_t*)P.w2[g];
    rc = launch_sets<2>(sets, p, D.Wmax, di, st);
    if (rc) return rc;
    launch_dep(combine_w4_kernel, dim3((unsigned)ceil_div((int64_t)tokens * (D.d >> 2), 256)), dim3(256), st, tokens, D.d,
               D.Ke, D.Ne, p.expert_idx, (const float*)p.part,
               y_add ? (const __nv_bfloat16*)y_add + t0 * D.d : nullptr, (__nv_bfloat16*)y + t0 * D.d);
    MOHGE_LAUNCH_CHECK("combine_w4_kernel");
  }
  return MOHGE_OK;
}

int32_t launch_quantize_w4(int64_t rows, int K, int group, bool bf16, const void* w, void* q, void* scale, cudaStream_t st) {
  const int64_t blocks = (rows * ((K + group - 1) / group) + 7) / 8;
  const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192));
  if (bf16)
    launch_dep(quantize_w4_kernel<__nv_bfloat16>, grid, dim3(256), st, rows, K, group, (const __nv_bfloat16*)w, (uint8_t*)q,
               (__nv_bfloat16*)scale);
  else
    launch_dep(quantize_w4_kernel<float>, grid, dim3(256), st, rows, K, group, (const float*)w, (uint8_t*)q,
               (__nv_bfloat16*)scale);
  MOHGE_LAUNCH_CHECK("quantize_w4_kernel");
  return MOHGE_OK;
}

int32_t launch_pack_w4(int64_t batch, int rows, int K, int group, int gate_up, const void* q, const void* scale, void* out,
                       cudaStream_t st) {
  const int64_t blocks = (batch * ((rows + 15) / 16) * ((K + kTileK - 1) / kTileK) + 7) / 8;
  launch_dep(pack_w4_kernel, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), st, batch, rows, K, group, gate_up,
             (const uint8_t*)q, (const __nv_bfloat16*)scale, (uint8_t*)out);
  MOHGE_LAUNCH_CHECK("pack_w4_kernel");
  return MOHGE_OK;
}

}  // namespace mohge
