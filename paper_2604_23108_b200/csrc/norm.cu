// RMS norm with the residual's addition, forward and backward (sm_100a).
//
//   h = x (+ residual),  rstd = (mean_j h_j^2 + eps)^(-1/2),  y_j = h_j rstd weight_j
//
// Bound by HBM: the forward reads x and the residual and writes h, y and, where asked, y in 8 bits
// (9.03 bytes per element in BF16 with everything on), the backward reads dy, h and the residual
// stream's gradient and writes dx (8 bytes per element).  So a row is read once and kept in registers
// between the sum of squares and the scaling: a row is shared by kTpr threads that hold up to
// kVec pieces of eight columns each, consecutive lanes holding consecutive pieces, so that every
// access is a coalesced 16-byte one and the 32 columns that share an 8-bit scale sit in four
// neighbouring lanes (two shuffles give their maximum).
// At 65536 x 4096 in BF16 the forward takes 357 us (6.8 TB/s, the rate of a copy), the backward 312-317 us; in FP32
// at 16384 x 4096 160 and 174 us (floor 164 each).
// Sums and the statistics are FP32; the statistics come from the unrounded sum x + residual, not from
// the rounded h, so that y is rounded once.

#include <atomic>

#include "common.cuh"
#include "mx8_math.cuh"
#include "tc_ptx.cuh"

namespace mohge {
namespace {

constexpr int kVec = 4;          // pieces of eight columns a thread holds

template <typename T> struct Piece;      // eight consecutive columns as they sit in memory
template <> struct Piece<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = v; }
  __device__ __forceinline__ void get(float2 (&f)[4]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  __device__ __forceinline__ void set(const float2 (&f)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[i].x, f[i].y);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Piece<float> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = a;
    reinterpret_cast<float4*>(p)[1] = b;
  }
  __device__ __forceinline__ void get(float2 (&f)[4]) const {
    f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w); f[2] = make_float2(b.x, b.y); f[3] = make_float2(b.z, b.w);
  }
  __device__ __forceinline__ void set(const float2 (&f)[4]) {
    a = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
    b = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
  }
};
__device__ __forceinline__ float2 two(float v) { return make_float2(v, v); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over the TPR threads of a block that share its row, the same value in each of them, added in a fixed
// order (TPR = 32: one warp of several)
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* slots) {
  v = warp_sum(v);
  if (TPR == 32) return v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) slots[warp] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < TPR / 32; ++w) s += slots[w];
  return s;
}

// barrier of the TPR threads of group g (whole warps)
template <int TPR> __device__ __forceinline__ void group_sync(int g) {
  if (TPR == 32) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "n"(TPR) : "memory");
}

template <int TPR> __host__ __device__ constexpr int block_of() { return TPR < 128 ? 128 : TPR; }

// One row per TPR threads with up to KV pieces each.  HAS_MX8: also y in 8 bits.
template <typename T, int TPR, int KV, bool HAS_MX8>
__global__ void __launch_bounds__(block_of<TPR>())
norm_fwd_kernel(int64_t T_rows, int d, const T* x, const T* residual, const T* __restrict__ weight, float eps, T* h,
                T* y, uint8_t* __restrict__ y8, uint8_t* __restrict__ y8_scale, float* __restrict__ rstd) {
  __shared__ float slots[32];
  pdl_enter();
  const int t = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * (block_of<TPR>() / TPR) + threadIdx.x / TPR;
  if (row >= T_rows) return;                       // whole warps: TPR >= 32
  const int np = d >> 3;                           // pieces in a row
  const int64_t base = row * d;
  float2 v[KV][4];
  Piece<T> pw[KV];
  {
    Piece<T> px[KV], pr[KV];
#pragma unroll
    for (int i = 0; i < KV; ++i) {
      const int p = i * TPR + t;
      px[i].zero();
      pr[i].zero();
      if (p < np) {
        px[i].load(x + base + 8 * p);
        if (residual) pr[i].load(residual + base + 8 * p);
      }
    }
    if (KV == 1) {                                 // the weight's latency hides behind the row's
      pw[0].zero();
      if (t < np) pw[0].load(weight + 8 * t);
    }
#pragma unroll
    for (int i = 0; i < KV; ++i) {
      float2 r[4];
      px[i].get(v[i]);
      pr[i].get(r);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i][j] = __fadd2_rn(v[i][j], r[j]);
    }
  }
  float2 s2 = two(0.f);
#pragma unroll
  for (int i = 0; i < KV; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s2 = __ffma2_rn(v[i][j], v[i][j], s2);
  const float ss = row_sum<TPR>(s2.x + s2.y, slots);
  const float rs = rsqrtf(ss / (float)d + eps);
  if (rstd && t == 0) rstd[row] = rs;
  const int64_t pitch8 = mx8_pitch(d), pitch_s = mx8_scale_pitch(d);
#pragma unroll
  for (int i = 0; i < KV; ++i) {
    const int p = i * TPR + t;
    const bool in = p < np;
    if (h && in) {
      Piece<T> o;
      o.set(v[i]);
      o.store(h + base + 8 * p);
    }
    float2 w[4];
    if (KV > 1) {
      pw[i].zero();
      if (in) pw[i].load(weight + 8 * p);
    }
    pw[i].get(w);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i][j] = __fmul2_rn(__fmul2_rn(v[i][j], two(rs)), w[j]);
    if (y && in) {
      Piece<T> o;
      o.set(v[i]);
      o.store(y + base + 8 * p);
    }
    if (HAS_MX8) {
      // pieces past the row (their h and weight are zero) fill the last block up with zeros
      float m = 0.f;
      if (in) {
#pragma unroll
        for (int j = 0; j < 4; ++j) m = fmaxf(m, fmaxf(fabsf(v[i][j].x), fabsf(v[i][j].y)));
      }
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
      const uint32_t byte = mx8_scale_byte(m);
      const float2 inv = two(mx8_inv_scale(byte));
      // the row's pitch may be 8 bytes more than d: those are written as zeros, and so are the
      // scale bytes up to a whole word
      if (8 * p < pitch8) {
        uint2 o = make_uint2(0u, 0u);
        if (in) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[i][j] = __fmul2_rn(v[i][j], inv);
          o.x = mx8_pack4(v[i][0].x, v[i][0].y, v[i][1].x, v[i][1].y);
          o.y = mx8_pack4(v[i][2].x, v[i][2].y, v[i][3].x, v[i][3].y);
        }
        *reinterpret_cast<uint2*>(y8 + row * pitch8 + 8 * p) = o;
      }
      if ((p & 3) == 0 && (p >> 2) < pitch_s) y8_scale[row * pitch_s + (p >> 2)] = (uint8_t)(in ? byte : 0u);
    }
  }
}

// dx = rstd (g - xhat mean(g xhat)) + dh with g = dy weight, xhat = h rstd.
// One persistent block per SM; kThreads / TPR groups of TPR threads, each with rows of its own and a ring
// of `stages` rows of dy, h and dh in shared memory, filled by untiled bulk copies: what is in flight (up
// to 196 KB per SM) does not depend on registers or on where the threads are in a row.  (Loads into
// registers reached 4.8 TB/s at 65536 x 4096: nothing was in flight during the row's sum and stores.)
// A thread keeps its columns of sum_t dy xhat in registers over all its rows; groups and blocks are added
// in a fixed order (through `parts`, [blocks, d], and dweight_kernel): no atomics, the same bits every time.
constexpr int kMaxStages = 4;
template <typename T> __host__ __device__ constexpr int bwd_threads(int tpr) { return sizeof(T) == 4 && tpr < 512 ? 256 : 512; }

template <typename T, int TPR>
__global__ void __launch_bounds__(bwd_threads<T>(TPR), 1)
norm_bwd_kernel(int64_t T_rows, int d, int stages, const T* dy, const T* dh, const T* __restrict__ h,
                const T* __restrict__ weight, const float* __restrict__ rstd, T* dx, float* __restrict__ parts,
                int32_t* status) {
  constexpr int kGroups = bwd_threads<T>(TPR) / TPR;
  extern __shared__ __align__(128) uint8_t ring_all[];
  __shared__ float slots[kGroups][2][TPR / 32];
  __shared__ uint64_t full[kGroups][kMaxStages];
  __shared__ int abort_flag;
  const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, lane = threadIdx.x & 31;
  const int np = d >> 3;
  const uint32_t row_bytes = (uint32_t)d * sizeof(T), stage_bytes = row_bytes * (dh ? 3 : 2);
  uint8_t* const ring = ring_all + (size_t)g * stages * stage_bytes;
  if (threadIdx.x == 0) abort_flag = 0;
  if (t < stages) mbar_init(smem_u32(&full[g][t]), 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncthreads();
  pdl_enter();
  const int64_t step = (int64_t)gridDim.x * kGroups, first = (int64_t)blockIdx.x * kGroups + g;
  auto request = [&](int64_t row, int st) {
    const uint32_t bar = smem_u32(&full[g][st]), dst = smem_u32(ring + (size_t)st * stage_bytes);
    mbar_expect_tx(bar, stage_bytes);
    bulk_load(dst, dy + row * d, row_bytes, bar);
    bulk_load(dst + row_bytes, h + row * d, row_bytes, bar);
    if (dh) bulk_load(dst + 2 * row_bytes, dh + row * d, row_bytes, bar);
  };
  if (t == 0)
    for (int st = 0; st < stages && first + st * step < T_rows; ++st) request(first + st * step, st);
  float2 dw[kVec][4];
  Piece<T> pw[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    pw[i].zero();
    if (i * TPR + t < np) pw[i].load(weight + 8 * (i * TPR + t));
#pragma unroll
    for (int j = 0; j < 4; ++j) dw[i][j] = two(0.f);
  }
  int st = 0, turn = 0;
  uint32_t phase = 0;
  float rs = first < T_rows ? rstd[first] : 0.f;
  for (int64_t row = first; row < T_rows; row += step, turn ^= 1) {
    const float rs_next = row + step < T_rows ? rstd[row + step] : 0.f;
    (void)mbar_wait(smem_u32(&full[g][st]), phase, &abort_flag, status, 51);
    const T* const s_dy = reinterpret_cast<const T*>(ring + (size_t)st * stage_bytes);
    const T* const s_h = s_dy + d;
    const T* const s_dh = s_h + d;
    float2 dot2 = two(0.f);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int p = i * TPR + t;
      if (p < np) {
        float2 a[4], b[4], w[4];
        Piece<T> q;
        q.load(s_dy + 8 * p);
        q.get(a);
        q.load(s_h + 8 * p);
        q.get(b);
        pw[i].get(w);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          // xhat before its product with dy: h dy leaves FP32's range first, and one such row would be in all of dweight
          const float2 ax = __fmul2_rn(a[j], __fmul2_rn(b[j], two(rs)));
          dot2 = __ffma2_rn(ax, w[j], dot2);
          dw[i][j] = __fadd2_rn(dw[i][j], ax);
        }
      }
    }
    float dot = dot2.x + dot2.y;
    dot = warp_sum(dot);
    if (TPR > 32) {                                 // added in warp order; two turns, so that one barrier is enough
      if (lane == 0) slots[g][turn][t >> 5] = dot;
      group_sync<TPR>(g);
      dot = 0.f;
#pragma unroll
      for (int w = 0; w < TPR / 32; ++w) dot += slots[g][turn][w];
    }
    // dx = rs (a w - (rs mean(g xhat)) b) + dh: without rs^2, which has half of rs's range
    const float2 c = two(-(dot / (float)d) * rs), rs2 = two(rs);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int p = i * TPR + t;
      if (p < np) {
        float2 a[4], b[4], w[4], e[4];
        Piece<T> q;
        q.load(s_dy + 8 * p);
        q.get(a);
        q.load(s_h + 8 * p);
        q.get(b);
        pw[i].get(w);
        if (dh) {
          q.load(s_dh + 8 * p);
          q.get(e);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 g = __ffma2_rn(b[j], c, __fmul2_rn(a[j], w[j]));
          a[j] = dh ? __ffma2_rn(g, rs2, e[j]) : __fmul2_rn(g, rs2);
        }
        q.set(a);
        q.store(dx + row * d + 8 * p);
      }
    }
    group_sync<TPR>(g);                             // the stage has been read
    if (t == 0 && row + stages * step < T_rows) request(row + stages * step, st);
    if (++st == stages) { st = 0; phase ^= 1u; }
    rs = rs_next;
  }
  // the groups of a block, added in ascending order, every thread a few columns; the rings are done with
  float4* const out = reinterpret_cast<float4*>(parts + (int64_t)blockIdx.x * d);
  if (kGroups > 1) {
    float4* const acc = reinterpret_cast<float4*>(ring_all);        // [groups][d / 4]
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int p = i * TPR + t;
      if (p < np) {
        acc[g * (d >> 2) + 2 * p] = make_float4(dw[i][0].x, dw[i][0].y, dw[i][1].x, dw[i][1].y);
        acc[g * (d >> 2) + 2 * p + 1] = make_float4(dw[i][2].x, dw[i][2].y, dw[i][3].x, dw[i][3].y);
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < (d >> 2); c += blockDim.x) {
      float4 s = acc[c];
#pragma unroll
      for (int k = 1; k < kGroups; ++k) {
        const float4 v = acc[k * (d >> 2) + c];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      out[c] = s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int p = i * TPR + t;
      if (p < np) {
        out[2 * p] = make_float4(dw[i][0].x, dw[i][0].y, dw[i][1].x, dw[i][1].y);
        out[2 * p + 1] = make_float4(dw[i][2].x, dw[i][2].y, dw[i][3].x, dw[i][3].y);
      }
    }
  }
  if (*(volatile int*)&abort_flag) __nanosleep(200000);     // a wait gave up: let copies in flight land
}

// dweight[j] (+)= sum over the blocks' partial sums: 32 columns per CTA (eight lanes of four), 32 ranges of
// partial sums side by side, joined in ascending order
__global__ void __launch_bounds__(256)
dweight_kernel(int nparts, int d, const float* __restrict__ parts, float* dweight, int accumulate) {
  __shared__ float4 s[32][8];
  pdl_enter();
  const int q = threadIdx.x & 7, sub = threadIdx.x >> 3;
  const int col = blockIdx.x * 32 + 4 * q;            // d is a multiple of 8: four columns are inside or outside
  const int per = (nparts + 31) / 32;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (col < d) {
    const int end = min(nparts, (sub + 1) * per);
#pragma unroll 8
    for (int i = sub * per; i < end; ++i) {
      const float4 v = *reinterpret_cast<const float4*>(parts + (int64_t)i * d + col);
      a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
    }
  }
  s[sub][q] = a;
  __syncthreads();
  if (threadIdx.x < 32 && blockIdx.x * 32 + (int)threadIdx.x < d) {
    const int c = blockIdx.x * 32 + threadIdx.x;
    float r = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) r += reinterpret_cast<const float*>(&s[i][0])[threadIdx.x];
    dweight[c] = accumulate ? dweight[c] + r : r;
  }
}

template <typename T, int TPR, int KV>
void fwd(const Dims& D, const void* x, const void* residual, const void* weight, float eps, void* h, void* y, void* y8,
         void* y8_scale, float* rstd, cudaStream_t st) {
  const dim3 grid((unsigned)ceil_div(D.T, block_of<TPR>() / TPR)), block(block_of<TPR>());
  const auto kernel = y8 ? norm_fwd_kernel<T, TPR, KV, true> : norm_fwd_kernel<T, TPR, KV, false>;
  launch_dep(kernel, grid, block, st, D.T, D.d, (const T*)x, (const T*)residual, (const T*)weight, eps, (T*)h, (T*)y,
             (uint8_t*)y8, (uint8_t*)y8_scale, rstd);
}

template <typename T, int TPR>
int32_t bwd(const Dims& D, const DeviceInfo& di, const void* dy, const void* dh, const void* h, const void* weight,
            const float* rstd, void* dx, float* parts, int32_t* status, int* nparts, cudaStream_t st) {
  constexpr int kThreads = bwd_threads<T>(TPR), kGroups = kThreads / TPR, kMost = 220 * 1024;
  static_assert(kGroups * 2 * TPR * 8 * kVec * (int)sizeof(T) <= kMost, "one stage of two rows at least");
  const auto kernel = norm_bwd_kernel<T, TPR>;
  static std::atomic<bool> set[kMaxDevices];
  if (!set[di.ordinal].load(std::memory_order_acquire)) {
    MOHGE_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost));
    set[di.ordinal].store(true, std::memory_order_release);
  }
  const int stage_bytes = D.d * (int)sizeof(T) * (dh ? 3 : 2);
  int stages = kMost / (kGroups * stage_bytes);
  if (stages > kMaxStages) stages = kMaxStages;
  int64_t smem = (int64_t)kGroups * stages * stage_bytes;
  const int64_t acc = kGroups > 1 ? (int64_t)kGroups * D.d * 4 : 0;       // the groups' sums reuse the rings
  if (smem < acc) smem = acc;
  const int64_t rows = (D.T + kGroups - 1) / kGroups;
  *nparts = (int)(rows < di.sm_count ? rows : di.sm_count);
  if (*nparts > kNormParts) *nparts = kNormParts;
  launch_dep_smem(kernel, dim3((unsigned)*nparts), dim3(kThreads), (size_t)smem, st, D.T, D.d, stages, (const T*)dy, (const T*)dh,
                  (const T*)h, (const T*)weight, rstd, (T*)dx, parts, status);
  MOHGE_LAUNCH_CHECK("norm_bwd_kernel");
  return MOHGE_OK;
}

// Threads per row: the fewest that hold the row in registers
#define MOHGE_NORM_TPR(d, CALL)                            \
  do {                                                     \
    if ((d) <= 32 * 8 * kVec) { CALL(32, kVec); }          \
    else if ((d) <= 128 * 8 * kVec) { CALL(128, kVec); }   \
    else if ((d) <= 256 * 8 * kVec) { CALL(256, kVec); }   \
    else { CALL(512, kVec); }                              \
  } while (0)
// Small batches: one piece per thread
#define MOHGE_NORM_TPR1(d, CALL)                           \
  do {                                                     \
    if ((d) <= 32 * 8) { CALL(32, 1); }                    \
    else if ((d) <= 128 * 8) { CALL(128, 1); }             \
    else if ((d) <= 256 * 8) { CALL(256, 1); }             \
    else if ((d) <= 512 * 8) { CALL(512, 1); }             \
    else { CALL(1024, 1); }                                \
  } while (0)

}  // namespace

static_assert(kNormMaxD == 512 * 8 * kVec, "widest row that a block keeps in registers");

int32_t launch_norm_fwd(const Dims& D, const void* x, const void* residual, const void* weight, float eps, void* h,
                        void* y, void* y8, void* y8_scale, float* rstd, cudaStream_t st) {
  if (D.T == 0) return MOHGE_OK;
  DeviceInfo di;
  const int32_t rc = current_device(&di);
  if (rc) return rc;
#define CALL(TPR, KV)                                                                                        \
  if (D.bf16) fwd<__nv_bfloat16, TPR, KV>(D, x, residual, weight, eps, h, y, y8, y8_scale, rstd, st);        \
  else fwd<float, TPR, KV>(D, x, residual, weight, eps, h, y, y8, y8_scale, rstd, st)
  // A batch that fits the GPU with one piece per thread is bound by latency: everything is requested at
  // once then (2049 x 1024 FP32: 6.1 us, with four pieces 9.3).  Larger ones run with four pieces per
  // thread, fewer instructions per byte (65536 x 4096 with 8 bits: 357 us, with one piece 406).
  if (D.d <= 1024 * 8 && D.T * (int64_t)(D.d >> 3) <= (int64_t)di.sm_count * 2048) MOHGE_NORM_TPR1(D.d, CALL);
  else MOHGE_NORM_TPR(D.d, CALL);
#undef CALL
  MOHGE_LAUNCH_CHECK("norm_fwd_kernel");
  return MOHGE_OK;
}

int32_t launch_norm_bwd(const Dims& D, const void* dy, const void* dh, const void* h, const void* weight,
                        const float* rstd, void* dx, float* dweight, int accumulate, float* parts, int32_t* status,
                        cudaStream_t st) {
  DeviceInfo di;
  int32_t rc = current_device(&di);
  if (rc) return rc;
  int nparts = 0;
  if (D.T > 0) {
#define CALL(TPR, KV)                                                                                            \
  rc = D.bf16 ? bwd<__nv_bfloat16, TPR>(D, di, dy, dh, h, weight, rstd, dx, parts, status, &nparts, st)          \
              : bwd<float, TPR>(D, di, dy, dh, h, weight, rstd, dx, parts, status, &nparts, st)
    MOHGE_NORM_TPR(D.d, CALL);
#undef CALL
    if (rc) return rc;
  }
  launch_dep(dweight_kernel, dim3((unsigned)ceil_div(D.d, 32)), dim3(256), st, nparts, D.d, (const float*)parts, dweight,
             accumulate);
  MOHGE_LAUNCH_CHECK("dweight_kernel");
  return MOHGE_OK;
}

}  // namespace mohge
