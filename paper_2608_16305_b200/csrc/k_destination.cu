// Softmax cross entropy of a root's target among all rows of a table, and its gradients, without a row of logits in memory.
//
//   z[i, j] = scale q_i . t_j + b_j;   loss_i = log sum_j exp z[i, j] - z[i, y_i]
//   dz[i, j] = g_i (p[i, j] - [j = y_i]);   dq_i = scale sum_j dz[i, j] t_j;   dt_j = scale sum_i dz[i, j] q_i;   db_j = sum_i dz[i, j]
//
// dq_i is g_i scale times the weighted mean of the table's rows less the target's row, whatever g_i turns out to be: an attention over the table
// with the rows as keys and values.  So the forward pass forms it beside the sum (one product more, no second pass over the
// logits), and the backward pass is the gradient of the table alone, an attention the other way round: rows of the table are the queries, roots are
// keys and values, and a weight is exp(z - m_i) w_i with the roots' maxima and factors known.  8 n rows dim operations in all,
// two exponentials per logit, no atomics.
//
// The target is left out of every sum and put in at the end: with r = sum of the others' weights over the target's, loss = log(1 + r),
// 1 - p = r / (1 + r), and dq is (mean of the others - target's row) (1 - p).  What is nearly certain keeps its relative
// accuracy (a loss of 1e-9 is one; a weight rounded to bf16 would leave 2^-8 of it where 1 - p belongs).
//
// One kernel does both directions.  A thread block holds 128 or 256 rows of one matrix (A) in shared memory and walks tiles of 128 (64) rows of the
// other (T): S = A T' on the tensor cores into tensor memory, weights P from S in registers (two threads have a row), P back to
// tensor memory, O += P T with the same tile as the second operand.  Two groups of 128 rows (or two buffers of S) keep the tensor cores busy
// while weights are formed.  All tiles, in order of A's rows, are split over the blocks: a block's first and last group of rows may be
// shared with others and go to scratch as parts, which a last kernel joins.
//
// bf16 rows are operands as they are (copied where a row is no multiple of 16 bytes, or below 64 values), and weights are rounded to bf16 beside them, once (a
// product's operands are of one type; 2^-8 of each, as much as the result's own rounding).  fp32 rows are split into
// two fp16 numbers each, hi + lo, after a multiplication by a power of two that puts the matrix's largest magnitude (of roots that take part and nodes in
// sight) below 2^14: 22 bits for what is within 2^-16 of the largest, 2^-38 of the largest for what is smaller, and a product takes three passes (hi hi,
// hi lo, lo hi).  So a logit is off by 2^-37 scale dim times both largest at most; where that could pass 2^-20 (logits beyond 10^5, which a row or a
// root far larger than all others gives) every product is formed in fp32 instead, by the last kernels, which is slow.  Weights are split the same way, in
// units that put the largest near 2^15.
#include <cuda.h>

#include "tgnn_table.cuh"
#include "tgnn_tensor_map.cuh"

using namespace tgnn_table;

namespace {

constexpr unsigned kSpin = 1u << 22;
constexpr int kMaxBlocks = 160;             // thread blocks of the main kernel, one per multiprocessor
constexpr int kSmem = 220 * 1024;           // dynamic shared memory; the static part is up to 7 KB
constexpr int kMaxParts = 592;              // partial maxima: of fp32 rows, of the bias
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.40282347e38f;
constexpr float kRoom = 60.f;               // a row's sum of weights is trusted within 2^-60 and 2^60 of its reference: sums of rows up to 2^67 fit beside
                                            // it, and gradients down to 2^-66 times its inverse
constexpr float kLeast = 8.6736174e-19f;    // 2^-60
constexpr float kMost = 1.1529215e18f;      // 2^60

enum Mode { LOSS = 0, FORWARD = 1, BACKWARD = 2 };

struct Layout {                              // of the scratch buffer, bytes
  int64_t count, act, parts, qp, tp, cols, slots, full, bytes;
};
struct Shape {
  int64_t n, rows;
  int dim, dp, planes;                       // dp: dim in steps of 64, what a plane of a row takes
  int od;                                    // columns of O, dim in steps of 16
};
__host__ __device__ inline int pitch_of(const Shape& s) { return s.od + 4; }

struct Prep {
  Shape s;
  const void* q;
  const void* table;
  const void* target;
  int index_bits, dtype, copy_table;
  const float* bias;
  const float* dloss;
  const float* kept;
  void* dq;
  float* loss;
  float scale;
  int backward, tile;
  int32_t* count;                            // [0]: roots that take part
  int32_t* act;                              // their indices
  float* parts;                              // largest magnitudes of [q, table, dloss] and the largest bias, [4][kMaxParts], and what the later kernels make of them
  int parts_used;
  uint16_t* qp;
  uint16_t* tp;
  float* cols;                               // what a tile's columns need, tile by tile
  int32_t* status;
};

__device__ __forceinline__ int64_t target_of(const Prep& a, int64_t i) {
  return a.index_bits == 64 ? static_cast<const int64_t*>(a.target)[i] : (int64_t)static_cast<const int32_t*>(a.target)[i];
}
__device__ __forceinline__ float value_of(const void* p, int dtype, int64_t i) {
  return dtype == TGNN_F32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {  // of numbers from 0; a division of 64 bits takes five times as long
  return (((uint64_t)a | (uint64_t)b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// A bias in units of log 2; finite ones stay finite.
__device__ __forceinline__ float bias2(float b) {
  const float x = b * kLog2e;
  return b > -INFINITY ? fmaxf(x, kLowest) : x;
}

// 2^e such that a magnitude up to `top` times it is at most 2^14 (e to 110: of matrices below 2^-97 fewer bits are kept).
__device__ __forceinline__ float unit_of(float top) {
  if (!(top > 0.f)) return 1.f;
  int e;
  frexpf(fminf(top, 3.4e38f), &e);
  return ldexpf(1.f, min(110, 14 - e));
}
// What a product of rows in their units (powers of two, whose reciprocals are exact) is multiplied by to be a logit in units of log 2.  In fp64: a scale beside
// large rows may be subnormal.
__device__ __forceinline__ double factor_of(float scale, float uq, float ut) { return (double)scale * 1.4426950408889634 * __frcp_rn(uq) * __frcp_rn(ut); }
// The largest of the partial maxima of each kind, by a warp; all asked for together.
__device__ __forceinline__ void largest(const float* parts, int used, float (&x)[4]) {
#pragma unroll
  for (int n = 0; n < 4; ++n) x[n] = -INFINITY;
  for (int i0 = threadIdx.x & 31; i0 < used; i0 += 256) {
    float v[4][8];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[n][k] = i0 + 32 * k < used ? parts[n * kMaxParts + i0 + 32 * k] : -INFINITY;
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int k = 0; k < 8; ++k) x[n] = fmaxf(x[n], v[n][k]);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int n = 0; n < 4; ++n) x[n] = fmaxf(x[n], __shfl_xor_sync(FULL, x[n], o));
}

// Roots that take part, in order, by the first block; the others find the largest magnitudes of fp32 rows and the largest bias, and form dq.
__global__ void __launch_bounds__(1024) begin_kernel(const Prep a) {
  chain_wait();
  chain_release();
  __shared__ int s_sum[32];
  __shared__ float s_red[4][32];
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  if (blockIdx.x > 0) {
    const int b = blockIdx.x - 1, nb = gridDim.x - 1;
    float top[4] = {0.f, 0.f, 0.f, -INFINITY};
    const int64_t values = a.s.planes == 2 ? a.s.rows * a.s.dim : 0, stride = (int64_t)nb * 1024;
    if (!a.backward && a.bias)
      for (int64_t i = (int64_t)b * 1024 + t; i < a.s.rows; i += (int64_t)nb * 1024) top[3] = fmaxf(top[3], a.bias[i]);
    if (values > 0) {                                    // (nodes in sight: what a hidden one's row holds is not to cost the others bits)
      const int64_t rows_on = quotient(stride, a.s.dim);
      const int columns_on = (int)(stride - rows_on * a.s.dim);
      int64_t i = (int64_t)b * 1024 + t, row = quotient(i, a.s.dim);
      int column = (int)(i - row * a.s.dim);
      while (i < values) {                               // four at a time, asked for together
        float x[4], hide[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[k] = i < values ? static_cast<const float*>(a.table)[i] : 0.f;
          hide[k] = a.bias && i < values ? a.bias[row] : 0.f;
          i += stride;
          row += rows_on;
          column += columns_on;
          if (column >= a.s.dim) {
            column -= a.s.dim;
            ++row;
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) top[1] = fmaxf(top[1], hide[k] != -INFINITY ? fabsf(x[k]) : 0.f);
      }
    }
    for (int64_t r = (int64_t)b * 32 + warp; r < a.s.n && a.s.planes == 2; r += (int64_t)nb * 32) {
      const int64_t y = target_of(a, r);
      if (y < 0 || y >= a.s.rows) continue;
      for (int c = lane; c < a.s.dim; c += 32) top[0] = fmaxf(top[0], fabsf(static_cast<const float*>(a.q)[r * a.s.dim + c]));
      if (a.backward) top[2] = fmaxf(top[2], fabsf(a.dloss[r]));
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int o = 16; o; o >>= 1) top[k] = fmaxf(top[k], __shfl_xor_sync(FULL, top[k], o));
      if (lane == 0) s_red[k][warp] = top[k];
    }
    __syncthreads();
    if (warp < 4) {
      float x = s_red[warp][lane];
      for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(FULL, x, o));
      if (lane == 0) a.parts[warp * kMaxParts + b] = x;
    }
    if (a.dq) {                                          // dq_i = g_i scale (what the forward pass kept)
      for (int64_t r = (int64_t)b * 32 + warp; r < a.s.n; r += (int64_t)nb * 32) {
        const int64_t y = target_of(a, r);
        const bool in = y >= 0 && y < a.s.rows;
        const double g = in ? (double)a.dloss[r] * a.scale : 0.0;
        for (int c = lane; c < a.s.dim; c += 32) {
          const int64_t x = r * a.s.dim + c;
          const float v = in ? (float)(g * a.kept[3 * a.s.n + x]) : 0.f;
          if (a.dtype == TGNN_F32) static_cast<float*>(a.dq)[x] = v;
          else static_cast<__nv_bfloat16*>(a.dq)[x] = __float2bfloat16_rn(v);
        }
      }
    }
    return;
  }
  if (!a.count) return;                                  // dq alone is wanted
  int done = 0;
  constexpr int K = 4;
  for (int64_t base = 0; base < a.s.n; base += 1024 * K) {
    bool in[K];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t i = base + (int64_t)t * K + k;
      in[k] = false;
      if (i < a.s.n) {
        const int64_t y = target_of(a, i);
        in[k] = y >= 0 && y < a.s.rows;
        if (y >= a.s.rows) *a.status = 4;
        if (!in[k] && !a.backward) a.loss[i] = 0.f;
      }
      mine += in[k];
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(FULL, inc, o);
      if (lane >= o) inc += x;
    }
    if (lane == 31) s_sum[warp] = inc;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < 32; ++w) {
      before += w < warp ? s_sum[w] : 0;
      all += s_sum[w];
    }
    int at = done + before + inc - mine;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (in[k]) a.act[at++] = (int)(base + (int64_t)t * K + k);
    done += all;
    __syncthreads();
  }
  if (t == 0) a.count[0] = done;
}

// Operands and columns: rows of q that take part (and zeros up to a multiple of 128), the table where it is copied, and what the columns of a tile
// need; backward also dq.
__global__ void __launch_bounds__(256) prep_kernel(const Prep a) {
  chain_wait();
  chain_release();
  const int t = threadIdx.x, lane = t & 31;
  const int64_t worker = (int64_t)blockIdx.x * 8 + (t >> 5), workers = (int64_t)gridDim.x * 8;
  const int64_t live = a.count[0], padded = up(live, 128);
  const bool split = a.s.planes == 2;
  float uq = 1.f, ut = 1.f, ug = 1.f;
  float x[4];
  if (split || blockIdx.x == 0) largest(a.parts, a.parts_used, x);
  if (split) {
    uq = unit_of(x[0]);
    ut = unit_of(x[1]);
    if (a.backward) ug = 2.f * unit_of(x[2]);            // |g| up to 2^15
  }
  const int dp = a.s.dp, dim = a.s.dim;
  if (blockIdx.x == 0 && t == 0) {
    const float mark = split && fabsf(a.scale) * x[0] * x[1] * (float)dim > 131072.f ? -1.f : 1.f;      // both below 0: products are to be formed in fp32
    *reinterpret_cast<float4*>(a.parts + 4 * kMaxParts) = make_float4(mark * uq, mark * ut, ug, bias2(x[3]));
  }
  auto operand = [&](const void* src, int64_t row, uint16_t* to, float unit) {     // a row, 2 values at a time
    for (int c = 2 * lane; c < dp; c += 64) {
      float x = 0.f, y = 0.f;
      if (row >= 0) {
        if (c < dim) x = value_of(src, a.dtype, row * dim + c);
        if (c + 1 < dim) y = value_of(src, a.dtype, row * dim + c + 1);
      }
      if (split) {
        x *= unit;
        y *= unit;
        const __half2 h = __floats2half2_rn(x, y);
        const float2 f = __half22float2(h);
        *reinterpret_cast<__half2*>(to + c) = h;
        *reinterpret_cast<__half2*>(to + dp + c) = __floats2half2_rn(x - f.x, y - f.y);
      } else {
        *reinterpret_cast<__nv_bfloat162*>(to + c) = __floats2bfloat162_rn(x, y);  // exact: the values were bf16
      }
    }
  };
  const int64_t wide = (int64_t)a.s.planes * dp;
  for (int64_t i = worker; i < padded; i += workers) operand(a.q, i < live ? a.act[i] : -1, a.qp + i * wide, uq);
  if (a.copy_table)
    for (int64_t i = worker; i < a.s.rows; i += workers) operand(a.table, i, a.tp + i * wide, split && a.bias && a.bias[i] == -INFINITY ? 0.f : ut);
  const int64_t thread = (int64_t)blockIdx.x * 256 + t, threads = (int64_t)gridDim.x * 256;
  if (!a.backward) {
    const int64_t cols = up(a.s.rows, a.tile);
    for (int64_t j = thread; j < cols; j += threads) a.cols[j] = j >= a.s.rows ? -INFINITY : a.bias ? bias2(a.bias[j]) : 0.f;
    return;
  }
  const int64_t cols = up(live, a.tile);
  for (int64_t j = thread; j < cols; j += threads) {
    float* p = a.cols + (j / a.tile) * 4 * a.tile + j % a.tile;
    const int64_t i = j < live ? a.act[j] : -1;
    const float g = i >= 0 ? a.dloss[i] * ug : 0.f;
    p[0] = i >= 0 ? -a.kept[i] : -INFINITY;
    p[a.tile] = i >= 0 ? g * a.kept[a.s.n + i] : 0.f;
    p[2 * a.tile] = i >= 0 ? -g * a.kept[2 * a.s.n + i] : 0.f;
    reinterpret_cast<int32_t*>(p)[3 * a.tile] = i >= 0 ? (int32_t)target_of(a, i) : -1;
  }
}

// -------------------------------------------------------------------------------------------------- the main kernel --
struct Main {
  CUtensorMap a_map, t_map;
  Shape s;
  const int32_t* count;
  const int32_t* act;
  const float* parts;
  const float* cols;
  const void* target;
  int index_bits;
  const float* bias;
  float* slots;              // parts: two per block, [rows of a group / 4][pitch / 4][4 rows][4 columns]: 64 bytes of neighboring rows side by side
  float* full;               // forward, groups of rows that one block has to itself: {m, l, target's z} of every live root
  float* kept;
  void* dtable;
  float* dbias;
  int dtype;
  float scale;
  int chunks, ksteps, stages, ahead, extra;   // chunks of 64 columns in shared memory, steps of 16 of a product over dim
  int32_t* status;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Bounded wait on a phase; gives up early when another role has.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  for (unsigned it = 0; it < kSpin; ++it) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    if (done) return true;
    if ((it & 63) == 63 && *abort_flag) return false;
  }
  return false;
}
// Whether a phase has ended, without waiting for it.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
               "r"(x), "r"(y), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ uint64_t make_desc(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
  return (uint64_t)((saddr >> 4) & 0x3FFF) | (uint64_t)((lbo >> 4) & 0x3FFF) << 16 | (uint64_t)((sbo >> 4) & 0x3FFF) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;                  // the architecture's version, 128-byte swizzle
}
// One lane of a converged warp.  (The compiler knows of it that one lane runs what it guards, and keeps descriptors in uniform registers there:
// 5 % of the kernel's time against lane == 0.)
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
__device__ __forceinline__ void mma(bool on, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"((uint32_t)on)
      : "memory");
}
__device__ __forceinline__ void mma_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {  // A in tensor memory
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
#define REGS32(M, r, o)                                                                                                                  \
  M(r[o + 0]), M(r[o + 1]), M(r[o + 2]), M(r[o + 3]), M(r[o + 4]), M(r[o + 5]), M(r[o + 6]), M(r[o + 7]), M(r[o + 8]), M(r[o + 9]),       \
      M(r[o + 10]), M(r[o + 11]), M(r[o + 12]), M(r[o + 13]), M(r[o + 14]), M(r[o + 15]), M(r[o + 16]), M(r[o + 17]), M(r[o + 18]),       \
      M(r[o + 19]), M(r[o + 20]), M(r[o + 21]), M(r[o + 22]), M(r[o + 23]), M(r[o + 24]), M(r[o + 25]), M(r[o + 26]), M(r[o + 27]),       \
      M(r[o + 28]), M(r[o + 29]), M(r[o + 30]), M(r[o + 31])
#define AS_OUT(x) "=f"(x)
#define AS_BOTH(x) "+f"(x)
#define AS_IN(x) "r"(x)
#define AS_INF(x) "f"(x)
#define REGS16(M, r, o)                                                                                                                  \
  M(r[o + 0]), M(r[o + 1]), M(r[o + 2]), M(r[o + 3]), M(r[o + 4]), M(r[o + 5]), M(r[o + 6]), M(r[o + 7]), M(r[o + 8]), M(r[o + 9]),       \
      M(r[o + 10]), M(r[o + 11]), M(r[o + 12]), M(r[o + 13]), M(r[o + 14]), M(r[o + 15])
#define LIST32                                                                                                                           \
  "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}"
#define LIST32_1                                                                                                                         \
  "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32}"
#define TMEM_LD32(r, o, addr) asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 " LIST32 ", [%32];" : REGS32(AS_OUT, r, o) : "r"(addr))
#define TMEM_ST32(addr, r, o) asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], " LIST32_1 ";" ::"r"(addr), REGS32(AS_IN, r, o) : "memory")
#define TMEM_ST16(addr, r, o)                                                                                                             \
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),      \
               REGS16(AS_IN, r, o)                                                                                                        \
               : "memory")
#define TMEM_ST32F(addr, r, o) asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], " LIST32_1 ";" ::"r"(addr), REGS32(AS_INF, r, o) : "memory")
// the wait, with the loaded registers as its results: nothing that reads them is moved ahead of it
#define WAIT_LD32(r) asm volatile("tcgen05.wait::ld.sync.aligned;" : REGS32(AS_BOTH, r, 0)::"memory")
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// The blocks' shares of the tiles: block c has tiles [begin(c), begin(c + 1)), and tile o of group r belongs to block owner(r, o).  Shares are even with
// `extra` tiles more in front of each group's: what its block needs to write one group and begin the next.
struct Share {
  int64_t tiles, wide, per;                  // of a group, without and with the extra ones; of a block
  int blocks, more;                          // blocks that have a share; the first `more` have per + 1, the others per
  int extra;
  __device__ __forceinline__ Share(int64_t groups, int64_t col_tiles, int extra_tiles, int launched)
      : tiles(col_tiles), wide(col_tiles + extra_tiles), per(0), blocks((int)min(groups * col_tiles, (int64_t)launched)), more(0), extra(extra_tiles) {
    if (blocks > 0) {
      per = quotient(groups * wide, blocks);
      more = (int)(groups * wide - per * blocks);
    }
  }
  __device__ __forceinline__ int64_t begin(int c) const {
    const int64_t x = per * c + min(c, more), r = quotient(x, wide), o = x - r * wide - extra;
    return r * tiles + (o < 0 ? 0 : o);
  }
  __device__ __forceinline__ int owner(int64_t r, int64_t o) const {
    const int64_t x = r * wide + extra + o, edge = more * (per + 1);
    return x < edge ? (int)quotient(x, per + 1) : more + (int)quotient(x - edge, per);
  }
};
// Where block c puts its part of row group r: its first group's place or its last one's.
__device__ __forceinline__ int slot_of(const Share& sh, int64_t col_tiles, int c, int64_t r) {
  const int64_t x = sh.begin(c) - r * col_tiles;           // its first tile is of this group, or of an earlier one
  return x >= 0 ? 2 * c : 2 * c + 1;
}

// Two fp32 values in one register pair: added and multiplied in one instruction.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

template <int PL>
__device__ __forceinline__ uint32_t pack_hi(float x, float y) {
  if (PL == 2) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_lo(float x, float y, uint32_t hi) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  const __half2 l = __floats2half2_rn(x - f.x, y - f.y);
  return *reinterpret_cast<const uint32_t*>(&l);
}

// The meeting of the two warps that share 32 rows, each with half of a unit's columns; false when a role has given up.  A warp that gives up arrives
// once more (pair_leave), behind the flag: its partner is held by no meeting, and leaves at the first that it comes to.
__device__ __forceinline__ bool pair_sync(int id, volatile int* abort_flag) {
  asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory");
  return !__any_sync(FULL, *abort_flag);
}
__device__ __forceinline__ void pair_leave(int id) { asm volatile("bar.arrive %0, 64;" ::"r"(id) : "memory"); }

// MODE; PL planes per operand (2: fp32 rows); NH groups of 128 rows of A; NT rows of T per tile in shared memory; U columns of S at a time, two
// buffers of them per group.
//
// Warps: 0 copies, 1 and 2 issue matrix instructions (one per group of rows, so that neither group waits for the other), the others form weights while the
// other buffer's products run: eight warps per group of rows, two threads per row, each with half of a unit's columns (one thread per row: 4800 roots over
// 200 000 nodes, rows of 128 in bf16, forward 430 us and backward 530; two: 379 and 457, and 365 and 430 with what came after).  P takes the place of the S
// that it was made of.  256 x 128 logits of rows of 128 take the tensor cores 2560 cycles (S is bound by shared memory: 48 cycles for 128 x 64 x 16) and the
// exponentials 2048: the tensor pipe is 72 % active forward and 60 % backward, where groups change five times as often and a weight takes a factor more.
template <int MODE, int PL, int NH, int NT, int U>
__global__ void __launch_bounds__(128 + 256 * NH, 1) destination_kernel(const __grid_constant__ Main g) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t s_full[4], s_empty[4], s_afull, s_aempty, s_sfull[NH][2], s_pfull[NH][2], s_pv[NH][2];
  __shared__ float s_m[2][NH][128], s_l[NH][128], s_zt[NH][128];   // from one half of a row to the other
  __shared__ float s_product[MODE == BACKWARD || (MODE == FORWARD && PL == 2) ? 1 : 2][NH][128];
  __shared__ float s_now[2][MODE == FORWARD && PL == 2 ? 128 : 1];
  __shared__ int s_over[2][2][4];                                  // by unit (even, odd), half and quarter of the rows: a weight has passed what the type holds
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  constexpr int R = 128 * NH, PER = NT / U;            // units per tile
  constexpr int SPLIT = 2, NC = U / SPLIT, CH = NC / 32;   // threads per row, their columns, in steps of 32
  constexpr int KS = NH == 2 || (PL == 2 && NT == 128) ? 8 : 16;   // steps of 16 in dim, at most
  constexpr bool MOVING = MODE == FORWARD && PL == 2;  // the reference of a row's weights can move
  constexpr int COL_BYTES = (MODE == BACKWARD ? 16 : 4) * NT;
  constexpr float SHIFT = PL == 2 ? 7.f : 0.f;         // fp16: weights about 2^7, with 2^-32 of that above its smallest numbers
  constexpr float MOST = 32768.f;                      // a unit's sum that no weight minds
  constexpr uint32_t a_chunk = R * 128, t_chunk = NT * 128;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const uint32_t a_bytes = PL * g.chunks * a_chunk, t_bytes = PL * g.chunks * t_chunk;
  const uint32_t a_base = smem_u32(smem), t_base = a_base + a_bytes;
  unsigned char* col_base = smem + a_bytes + g.stages * t_bytes;

  if (tid == 0) {
    for (int i = 0; i < 4; ++i) {
      mbar_init(smem_u32(&s_full[i]), 1);
      mbar_init(smem_u32(&s_empty[i]), MODE == LOSS ? 4 * SPLIT * NH : NH);
    }
    for (int h = 0; h < NH; ++h)
      for (int i = 0; i < 2; ++i) {
        mbar_init(smem_u32(&s_sfull[h][i]), 1);
        mbar_init(smem_u32(&s_pfull[h][i]), 4 * SPLIT);
        mbar_init(smem_u32(&s_pv[h][i]), 1);
      }
    mbar_init(smem_u32(&s_afull), 1);
    mbar_init(smem_u32(&s_aempty), NH);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = s_tmem;
  volatile int* abort_flag = &s_abort;
  chain_wait();
  chain_release();

  const int64_t live = g.count[0];
  const int64_t a_rows = MODE == BACKWARD ? g.s.rows : live, t_rows = MODE == BACKWARD ? live : g.s.rows;
  const int64_t col_tiles = (t_rows + NT - 1) / NT;
  const Share sh((a_rows + R - 1) / R, col_tiles, g.extra, gridDim.x);
  const int64_t x0 = (int)blockIdx.x >= sh.blocks ? 0 : sh.begin(blockIdx.x), x1 = (int)blockIdx.x >= sh.blocks ? 0 : sh.begin(blockIdx.x + 1);
  const bool idle = x0 == x1;
  const int64_t r0 = idle ? 0 : quotient(x0, col_tiles), j0 = idle ? 0 : x0 - r0 * col_tiles;       // the first tile: group of rows, and tile of columns
  const uint32_t tiles = (uint32_t)(x1 - x0);
  const uint32_t o_base = tmem + 2 * NH * U;

  if (idle) {
    // fewer tiles than blocks (or a share of extra ones)
  } else if (warp == 0) {
    // ---------------------------------------------------------------- copies
    if (lane == 0) {
      bool ok = true;
      uint32_t seg = 0, st = 0, ph = 1;
      int64_t r = r0, j = j0;
      for (uint32_t tile = 0; tile < tiles && ok; ++tile) {
        if (tile == 0 || j == 0) {
          ok = mbar_wait(smem_u32(&s_aempty), (seg & 1) ^ 1, abort_flag);
          if (!ok) break;
          mbar_expect(smem_u32(&s_afull), a_bytes);
          for (int c = 0; c < PL * g.chunks; ++c) tma_2d(a_base + c * a_chunk, &g.a_map, 64 * c, (int)(r * R), smem_u32(&s_afull));
          ++seg;
        }
        ok = mbar_wait(smem_u32(&s_empty[st]), ph, abort_flag);
        if (!ok) break;
        const uint32_t bar = smem_u32(&s_full[st]);
        mbar_expect(bar, t_bytes + COL_BYTES);
        for (int c = 0; c < PL * g.chunks; ++c) tma_2d(t_base + st * t_bytes + c * t_chunk, &g.t_map, 64 * c, (int)(j * NT), bar);
        bulk(smem_u32(col_base + st * COL_BYTES), reinterpret_cast<const char*>(g.cols) + j * COL_BYTES, COL_BYTES, bar);
        if (++st == (uint32_t)g.stages) {
          st = 0;
          ph ^= 1;
        }
        if (++j == col_tiles) {
          j = 0;
          ++r;
        }
      }
      if (!ok) {
        s_abort = 1;
        atomicCAS(g.status, 0, TGNN_ETIMEOUT);
      }
    }
    __syncwarp();
  } else if (warp <= NH) {
    // ---------------------------------------------------------------- matrix instructions of group h
    if (elect_one()) {
      bool ok = true;
      const int h = warp - 1;
      const uint32_t fmt = PL == 2 ? 0u : 1u;            // fp16 or bf16, both operands
      const uint32_t id_s = (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)(U >> 3) << 17) | (8u << 24);
      const uint32_t id_o = (1u << 4) | (fmt << 7) | (fmt << 10) | (1u << 16) | ((uint32_t)(g.s.od >> 3) << 17) | (8u << 24);
      // Descriptors of the operands' first bytes; all others lie a constant further, in units of 16 bytes.
      const uint64_t da = make_desc(a_base + h * 128 * 128, 16, 1024);             // A and, as S's second operand, T: dim side by side
      const uint64_t dt = make_desc(t_base, 16, 1024), dv = make_desc(t_base, t_chunk, 1024);   // T as O's second operand: rows are its sum
      const uint64_t a_plane = g.chunks * (a_chunk >> 4), t_plane = g.chunks * (t_chunk >> 4), t_stage = t_bytes >> 4;
      const uint32_t s_cols = tmem + 2 * h * U, o = o_base + h * 128;
      const uint32_t units = tiles * PER;
      uint32_t s_unit = 0, s_seg = 0, s_st = 0, s_ph = 0, p_st = 0;
      int64_t s_j = j0, p_j = j0;
      auto product_s = [&]() {                           // S of the next unit
        const uint32_t buf = s_unit & 1, use = s_unit >> 1, sub = s_unit % PER;
        if (sub == 0) {
          if (s_unit == 0 || s_j == 0) {
            if (!mbar_wait(smem_u32(&s_afull), s_seg & 1, abort_flag)) return false;
            ++s_seg;
          }
          if (!mbar_wait(smem_u32(&s_full[s_st]), s_ph, abort_flag)) return false;
        }
        // the weights that lie in these columns have been used (without a backward pass: S has been read)
        if (use > 0 && !mbar_wait(MODE == LOSS ? smem_u32(&s_pfull[h][buf]) : smem_u32(&s_pv[h][buf]), (use - 1) & 1, abort_flag)) return false;
        fence_after();
        const uint32_t d = s_cols + buf * U;
        const uint64_t t0 = dt + s_st * t_stage + sub * (U * 128 >> 4);
#pragma unroll
        for (int pr = 0; pr < (PL == 2 ? 3 : 1); ++pr) { // hi hi, hi lo, lo hi
          const uint64_t ap = da + (pr == 2 ? a_plane : 0), tp = t0 + (pr == 1 ? t_plane : 0);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            mma(ks < g.ksteps, d, ap + (ks >> 2) * (a_chunk >> 4) + (ks & 3) * 2, tp + (ks >> 2) * (t_chunk >> 4) + (ks & 3) * 2, id_s, pr > 0 || ks > 0);
          }
        }
        commit(smem_u32(&s_sfull[h][buf]));
        ++s_unit;
        if (sub == PER - 1) {
          if (++s_st == (uint32_t)g.stages) {
            s_st = 0;
            s_ph ^= 1;
          }
          if (++s_j == col_tiles) s_j = 0;
          if (s_j == 0 || s_unit == units) commit(smem_u32(&s_aempty));
        }
        return true;
      };
      const uint32_t ahead = g.ahead;
      for (uint32_t v = 0; v < ahead && v < units && ok; ++v) ok = product_s();
      for (uint32_t u = 0; u < units && ok; ++u) {
        if (MODE != LOSS) {
          const uint32_t buf = u & 1, sub = u % PER;
          ok = mbar_wait(smem_u32(&s_pfull[h][buf]), (u >> 1) & 1, abort_flag);
          if (!ok) break;
          fence_after();
          const bool fresh = sub == 0 && (u == 0 || p_j == 0);
          const uint64_t t0 = dv + p_st * t_stage + sub * (U * 128 >> 4);
#pragma unroll
          for (int pr = 0; pr < (PL == 2 ? 3 : 1); ++pr) {
            const uint32_t p0 = s_cols + buf * U + (pr == 2 ? NC / 2 : 0);
            const uint64_t tp = t0 + (pr == 1 ? t_plane : 0);
#pragma unroll
            for (int ks = 0; ks < U / 16; ++ks)
              mma_ta(o, p0 + ks / (NC / 16) * NC + ks % (NC / 16) * 8, tp + 128 * ks, id_o, pr > 0 || ks > 0 || !fresh);
          }
          commit(smem_u32(&s_pv[h][buf]));
          if (sub == PER - 1) {
            commit(smem_u32(&s_empty[p_st]));
            if (++p_st == (uint32_t)g.stages) p_st = 0;
            if (++p_j == col_tiles) p_j = 0;
          }
        }
        if (u + ahead < units) ok = product_s();
      }
      if (!ok) {
        s_abort = 1;
        atomicCAS(g.status, 0, TGNN_ETIMEOUT);
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    // ---------------------------------------------------------------- weights: two threads have a row of A
    const int grp = (warp - 4) / (4 * SPLIT), part = (warp - 4) / 4 % SPLIT, quarter = warp & 3;
    const int pair = 1 + 4 * grp + quarter;              // the named barrier of the two warps with these rows
    const int lane_row = 32 * quarter + lane, row_in = 128 * grp + lane_row;
    const uint32_t lane_base = (uint32_t)(32 * quarter) << 16;
    const uint32_t o_addr = o_base + grp * 128 + lane_base, s_base = tmem + 2 * grp * U + part * NC + lane_base;
    const uint32_t bar_s = smem_u32(&s_sfull[grp][0]), bar_p = smem_u32(&s_pfull[grp][0]), bar_pv = smem_u32(&s_pv[grp][0]);
    const int pitch = pitch_of(g.s);
    float uq = 1.f, ut = 1.f, ug = 1.f, most_bias = 0.f;
    if (PL == 2 || MODE != BACKWARD) {
      const float4 x = *reinterpret_cast<const float4*>(g.parts + 4 * kMaxParts);
      uq = x.x;
      ut = x.y;
      ug = x.z;
      if (MODE != BACKWARD && !MOVING && g.bias) most_bias = x.w;
    }
    const float factor = (float)factor_of(g.scale, uq, ut);
    const f32x2 factor2 = pack2(factor, factor);
    const bool biased = g.bias != nullptr, summed = g.dbias != nullptr;
    const uint32_t all_cols = (uint32_t)col_tiles, full_tiles = (uint32_t)(t_rows / NT), all_units = tiles * PER;
    uint32_t r = (uint32_t)r0, j = (uint32_t)j0, left = tiles, st = 0, u = 0;
    bool ok = true, have = false;                        // have: the next unit's first columns are in z[0], or on their way
    float z[CH > 1 ? 2 : 1][32];
    while (left > 0 && ok) {
      // ---- the tiles of one group of rows
      const int64_t row = (int64_t)r * R + row_in;
      const bool valid = row < a_rows;
      const uint32_t count = min(left, all_cols - j);
      float m = -INFINITY, l = 0.f, zt = -INFINITY, rb = 0.f;    // backward: l is the row's sum of weights
      int32_t tgt = -1;
      if (MODE == BACKWARD) {
        if (valid && biased) rb = bias2(g.bias[row]);
      } else if (valid) {
        const int i = g.act[row];
        tgt = g.index_bits == 64 ? (int32_t) static_cast<const int64_t*>(g.target)[i] : static_cast<const int32_t*>(g.target)[i];
      }
      for (uint32_t t = 0; t < count && ok; ++t, ++j) {
#pragma unroll
        for (int sub = 0; sub < PER; ++sub, ++u) {
          const uint32_t buf = PER == 2 ? sub : u & 1, use = u >> 1;
          const uint32_t s_addr = s_base + buf * U;
          if (!have) {
            ok = __all_sync(FULL, mbar_wait(bar_s + 8 * buf, use & 1, abort_flag));
            if (!ok) break;
            fence_after();
            TMEM_LD32(z[0], 0, s_addr);
          }
          have = false;
          // the columns' values came with the tile, which S is complete after
          const float* col = reinterpret_cast<const float*>(col_base + st * COL_BYTES) + sub * U + part * NC;
          // While the last columns are worked on, the next unit's first ones are asked for, if they are there.
          auto ask = [&]() {
            const uint32_t next = buf ^ 1, parity = ((u + 1) >> 1) & 1;
            have = u + 1 < all_units && __all_sync(FULL, mbar_test(bar_s + 8 * next, parity));
            if (have) {
              fence_after();
              TMEM_LD32(z[0], 0, s_base + next * U);
            }
          };
          uint32_t hi[NC / 2];
          uint32_t lo[PL == 2 ? NC / 2 : 1];
          if (MODE != BACKWARD) {
            const int hit = tgt - (int32_t)(j * NT + sub * U + part * NC);         // outside [0, NC): not here
            const bool any_hit = __any_sync(FULL, (uint32_t)hit < (uint32_t)NC);
            const bool plain = !biased && j < full_tiles;   // the columns' values are zeros
            // logits of 32 columns less ref in place of S, the target left out
            auto logits = [&](float(&v)[32], int c, float ref) {
              const f32x2 ref2 = pack2(-ref, -ref);
              if (plain) {
#pragma unroll
                for (int k = 0; k < 32; k += 2) unpack2(fma2(pack2(v[k], v[k + 1]), factor2, ref2), v[k], v[k + 1]);
              } else {
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                  const ulonglong2 b = *reinterpret_cast<const ulonglong2*>(col + c + k);
                  unpack2(add2(fma2(pack2(v[k], v[k + 1]), factor2, b.x), ref2), v[k], v[k + 1]);
                  unpack2(add2(fma2(pack2(v[k + 2], v[k + 3]), factor2, b.y), ref2), v[k + 2], v[k + 3]);
                }
              }
              if (any_hit) {
                __syncwarp();                            // keeps this a branch: as predicated instructions it costs 50 a unit
#pragma unroll
                for (int k = 0; k < 32; ++k)
                  if (hit == c + k) {
                    zt = v[k] + ref;
                    v[k] = -INFINITY;
                  }
              }
            };
            auto maximum = [&]() {                       // of the unit's logits; what was asked for is lost
              have = false;
              float top = -INFINITY;
              for (int c = 0; c < NC; c += 32) {
                TMEM_LD32(z[0], 0, s_addr + c);
                WAIT_LD32(z[0]);
                logits(z[0], c, 0.f);
#pragma unroll
                for (int k = 0; k < 32; ++k) top = fmaxf(top, z[0][k]);
              }
              return top;
            };
            // The reference of a row's weights.  Where it can move: the maximum of the first unit in which the row sees anything.  Else, for good, the maximum
            // of the first unit (the target's apart); where biases hide most of that unit it would lie far below the others, and the largest product there plus the
            // largest bias of all is taken: right within the products' spread, whatever the biases hide.  A row for which neither is right is seen by the
            // last kernel, in its sums, and done again there.
            if (MOVING ? (bool)__any_sync(FULL, m == -INFINITY) : t == 0 && sub == 0) {
              WAIT_LD32(z[0]);
              if (MOVING) {
                float top = maximum();
                s_m[part][grp][lane_row] = top;          // one reference for both halves of the row
                ok = pair_sync(pair, abort_flag);
                if (!ok) break;
                top = fmaxf(top, s_m[part ^ 1][grp][lane_row]);
                if (m == -INFINITY) m = top;
              } else {
                have = false;
                float seen = -INFINITY, product = -INFINITY;
                for (int c = 0; c < NC; c += 32) {
                  TMEM_LD32(z[0], 0, s_addr + c);
                  WAIT_LD32(z[0]);
                  if (biased) {                          // (the zeros behind the table's end among them)
#pragma unroll
                    for (int k = 0; k < 32; ++k) product = hit == c + k ? product : fmaxf(product, z[0][k] * factor);
                  }
                  logits(z[0], c, 0.f);
#pragma unroll
                  for (int k = 0; k < 32; ++k) seen = fmaxf(seen, z[0][k]);
                }
                s_m[part][grp][lane_row] = seen;
                s_product[part][grp][lane_row] = product;
                ok = pair_sync(pair, abort_flag);
                if (!ok) break;
                seen = fmaxf(seen, s_m[part ^ 1][grp][lane_row]);
                product = fmaxf(product, s_product[part ^ 1][grp][lane_row]) + most_bias;
                m = !biased || !(seen < product - kRoom / 2) ? seen : product;    // -infinity: the target alone, or nothing at all
              }
              TMEM_LD32(z[0], 0, s_addr);
            }
            float sum;
            auto weights = [&]() {
              const float ref = m == -INFINITY ? 0.f : m;
              const f32x2 shift2 = pack2(SHIFT, SHIFT);
              f32x2 sum2 = pack2(0.f, 0.f), sum3 = sum2;
#pragma unroll
              for (int c = 0; c < CH; ++c) {
                float(&v)[32] = z[CH > 1 ? c & 1 : 0];
                WAIT_LD32(v);
                if (c + 1 < CH) TMEM_LD32(z[CH > 1 ? (c + 1) & 1 : 0], 0, s_addr + 32 * (c + 1));
                else if (CH > 1) ask();
                logits(v, 32 * c, ref);
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                  if (MOVING) {                          // (added to the difference: beside a mask's lowest value it would be lost)
                    unpack2(add2(pack2(v[k], v[k + 1]), shift2), v[k], v[k + 1]);
                    unpack2(add2(pack2(v[k + 2], v[k + 3]), shift2), v[k + 2], v[k + 3]);
                  }
                  const float p0 = tgnn_history::exp2_fast(v[k]), p1 = tgnn_history::exp2_fast(v[k + 1]);
                  const float p2 = tgnn_history::exp2_fast(v[k + 2]), p3 = tgnn_history::exp2_fast(v[k + 3]);
                  sum2 = add2(sum2, pack2(p0, p1));
                  sum3 = add2(sum3, pack2(p2, p3));
                  if (MODE == FORWARD) {
                    const int at = 16 * c + k / 2;
                    hi[at] = pack_hi<PL>(p0, p1);
                    hi[at + 1] = pack_hi<PL>(p2, p3);
                    if (PL == 2) {
                      lo[at] = pack_lo(p0, p1, hi[at]);
                      lo[at + 1] = pack_lo(p2, p3, hi[at + 1]);
                    }
                  }
                }
              }
              float a, b;
              unpack2(add2(sum2, sum3), a, b);
              sum = a + b;
            };
            // The target's own logit apart from a large reference: where a unit's other nodes are hidden that is a mask's value, in which the logit would be lost.
            // (A fixed reference is none, unless all nodes are hidden.)
            float own = 0.f;
            const bool apart = MOVING && any_hit && __any_sync(FULL, fabsf(m) > 64.f);
            if (apart) {
              WAIT_LD32(z[0]);
              for (int c = 0; c < NC; c += 32) {
                TMEM_LD32(z[0], 0, s_addr + c);
                WAIT_LD32(z[0]);
#pragma unroll
                for (int k = 0; k < 32; ++k) own = hit == c + k ? z[0][k] : own;
              }
              if ((uint32_t)hit < (uint32_t)NC) own = fmaf(own, factor, plain ? 0.f : col[hit]);
              TMEM_LD32(z[0], 0, s_addr);
            }
            weights();
            // fp16: the reference is moved when the unit's sum says that a weight may have passed what the type holds.  O has then to be multiplied and the
            // weights are formed again.  (Once: what is too large, or no number, then stays so.)
            // Both halves do it if one has to: O is theirs in common.
            bool over = false;
            if (MOVING) {
              over = __any_sync(FULL, !(sum <= MOST));
              if (lane == 0) s_over[u & 1][part][quarter] = over;
              ok = pair_sync(pair, abort_flag);          // (between two writes to one place lies the meeting of the other parity)
              if (!ok) break;
              over |= s_over[u & 1][part ^ 1][quarter] != 0;
            }
            if (MOVING && __builtin_expect(over, 0)) {
              if (have) WAIT_LD32(z[0]);
              float now = fmaxf(m, maximum());
              s_now[part][lane_row] = now;
              ok = pair_sync(pair, abort_flag);
              if (!ok) break;
              now = fmaxf(now, s_now[part ^ 1][lane_row]);
              const float f = now == -INFINITY ? 1.f : exp2f(m - now);
              l *= f;
              m = now;
              if (t > 0 || sub > 0) {                    // O is at rest once the unit before has been added
                ok = __all_sync(FULL, mbar_wait(bar_pv + 8 * (buf ^ 1), ((u - 1) >> 1) & 1, abort_flag));
                if (!ok) break;
                fence_after();
                for (int c = 32 * part; c < g.s.od; c += 32 * SPLIT) {   // od in steps of 16: the last step may pass it, inside the group's columns
                  TMEM_LD32(z[0], 0, o_addr + c);
                  WAIT_LD32(z[0]);
#pragma unroll
                  for (int k = 0; k < 32; ++k) z[0][k] *= f;
                  TMEM_ST32F(o_addr + c, z[0], 0);
                }
                wait_st();
              }
              TMEM_LD32(z[0], 0, s_addr);
              weights();
            }
            if (apart && (uint32_t)hit < (uint32_t)NC) zt = own;
            l += sum;
          } else {
            // roots whose target is one of this warp's rows: -g (1 - p) in place of their weight
            const int32_t* ct = reinterpret_cast<const int32_t*>(col + 3 * NT);
            const int32_t row0 = (int32_t)(r * R) + 128 * grp + 32 * quarter;
            const f32x2 rb2 = pack2(rb, rb);
            f32x2 sum2 = pack2(0.f, 0.f), sum3 = sum2;
            bool here = false;
#pragma unroll
            for (int c = 0; c < CH; ++c) here |= (uint32_t)(ct[32 * c + lane] - row0) < 32u;
            const bool any_hit = __any_sync(FULL, here);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
              float(&v)[32] = z[CH > 1 ? c & 1 : 0];
              const float* cc = col + 32 * c;
              WAIT_LD32(v);
              if (c + 1 < CH) TMEM_LD32(z[CH > 1 ? (c + 1) & 1 : 0], 0, s_addr + 32 * (c + 1));
              else if (CH > 1) ask();
              if (biased) {
#pragma unroll
                for (int k = 0; k < 32; k += 2) unpack2(fma2(pack2(v[k], v[k + 1]), factor2, rb2), v[k], v[k + 1]);
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                  const ulonglong2 cm = *reinterpret_cast<const ulonglong2*>(cc + k);          // -m
                  unpack2(add2(pack2(v[k], v[k + 1]), cm.x), v[k], v[k + 1]);
                  unpack2(add2(pack2(v[k + 2], v[k + 3]), cm.y), v[k + 2], v[k + 3]);
                }
              } else {
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                  const ulonglong2 cm = *reinterpret_cast<const ulonglong2*>(cc + k);
                  unpack2(fma2(pack2(v[k], v[k + 1]), factor2, cm.x), v[k], v[k + 1]);
                  unpack2(fma2(pack2(v[k + 2], v[k + 3]), factor2, cm.y), v[k + 2], v[k + 3]);
                }
              }
#pragma unroll
              for (int k = 0; k < 32; k += 4) {
                const ulonglong2 cw = *reinterpret_cast<const ulonglong2*>(cc + NT + k);
                const float p0 = tgnn_history::exp2_fast(v[k]), p1 = tgnn_history::exp2_fast(v[k + 1]);
                const float p2 = tgnn_history::exp2_fast(v[k + 2]), p3 = tgnn_history::exp2_fast(v[k + 3]);
                unpack2(mul2(pack2(p0, p1), cw.x), v[k], v[k + 1]);
                unpack2(mul2(pack2(p2, p3), cw.y), v[k + 2], v[k + 3]);
              }
              if (any_hit) {
                const int who = ct[32 * c + lane] - row0;
                for (unsigned more = __ballot_sync(FULL, (uint32_t)who < 32u); more; more &= more - 1) {
                  const int k = __ffs(more) - 1;
                  const int mine = __shfl_sync(FULL, who, k);
                  const float fix = cc[2 * NT + k];
#pragma unroll
                  for (int i = 0; i < 32; ++i)
                    if (i == k && mine == lane) v[i] = fix;
                }
              }
              if (summed) {
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                  sum2 = add2(sum2, pack2(v[k], v[k + 1]));
                  sum3 = add2(sum3, pack2(v[k + 2], v[k + 3]));
                }
              }
#pragma unroll
              for (int k = 0; k < 32; k += 2) {
                const int at = 16 * c + k / 2;
                hi[at] = pack_hi<PL>(v[k], v[k + 1]);
                if (PL == 2) lo[at] = pack_lo(v[k], v[k + 1], hi[at]);
              }
            }
            float a, b;
            unpack2(add2(sum2, sum3), a, b);
            l += a + b;
          }
          if (MODE != LOSS) {
            if (NC == 32) {
              TMEM_ST16(s_addr, hi, 0);
              if constexpr (PL == 2) TMEM_ST16(s_addr + NC / 2, lo, 0);
            } else {
#pragma unroll
              for (int c = 0; c < NC / 2; c += 32) {
                TMEM_ST32(s_addr + c, hi, c);
                if constexpr (PL == 2) TMEM_ST32(s_addr + NC / 2 + c, lo, c);
              }
            }
            wait_st();
          }
          fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar_p + 8 * buf);
            if (MODE == LOSS && sub == PER - 1) mbar_arrive(smem_u32(&s_empty[st]));
          }
        }
        if (++st == (uint32_t)g.stages) st = 0;
      }
      if (!ok) break;
      left -= count;
      // the group's rows are done as far as this block goes
      const bool alone = count == all_cols;
      float* slot = g.slots + ((int64_t)slot_of(sh, col_tiles, blockIdx.x, r) * R + (row_in & ~3)) * pitch + 4 * (row_in & 3);
      if (part == 1) {                                   // what the two halves of a row have is put together
        s_l[grp][lane_row] = l;
        s_zt[grp][lane_row] = zt;
      }
      ok = pair_sync(pair, abort_flag);
      if (!ok) break;
      if (part == 0) {
        const float other = s_zt[grp][lane_row];
        l += s_l[grp][lane_row];
        if (other != -INFINITY) zt = other;
      }
      ok = pair_sync(pair, abort_flag);                  // (the next group's values go to the same places)
      if (!ok) break;
      if (valid && part == 0) {
        if (MODE == BACKWARD) {
          if (!alone) slot[4 * g.s.od] = l;
          else if (summed) g.dbias[row] = l / ug;
        } else {
          float* to = alone ? g.full + 3 * row : slot + 4 * g.s.od;
          to[0] = m;
          to[1] = l;
          to[2] = zt;
        }
      }
      if (MODE != LOSS) {
        ok = __all_sync(FULL, mbar_wait(bar_pv + 8 * ((u - 1) & 1), ((u - 1) >> 1) & 1, abort_flag));
        if (!ok) break;
        fence_after();
        const float out = MODE == BACKWARD ? (float)((double)g.scale * __frcp_rn(ug) * __frcp_rn(uq)) : 1.f;
        const int dim = g.s.dim;
        float* home = MODE == FORWARD && alone && valid ? g.kept + 3 * g.s.n + (int64_t)g.act[row] * dim : nullptr;
        float(&o)[32] = z[CH > 1 ? 1 : 0];               // z[0] may hold what was asked for
        for (int c = 32 * part; c < g.s.od; c += 32 * SPLIT) {
          __syncwarp();                                  // lanes without a row have gone ahead
          TMEM_LD32(o, 0, o_addr + c);
          WAIT_LD32(o);
          if (!valid) {
          } else if (!alone) {
#pragma unroll
            for (int k = 0; k < 32; k += 4)
              if (c + k < g.s.od) *reinterpret_cast<float4*>(slot + 4 * (c + k)) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
          } else if (MODE == FORWARD) {
            if (((uintptr_t)home & 15) == 0 && dim % 4 == 0) {
#pragma unroll
              for (int k = 0; k < 32; k += 4)
                if (c + k < dim) *reinterpret_cast<float4*>(home + c + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
            } else {
#pragma unroll
              for (int k = 0; k < 32; ++k)
                if (c + k < dim) home[c + k] = o[k];
            }
          } else if (g.dtable) {
            if (g.dtype == TGNN_F32) {
              float* to = static_cast<float*>(g.dtable) + row * dim + c;
              if (dim % 4 == 0 && ((uintptr_t)g.dtable & 15) == 0) {
#pragma unroll
                for (int k = 0; k < 32; k += 4)
                  if (c + k < dim) *reinterpret_cast<float4*>(to + k) = make_float4(o[k] * out, o[k + 1] * out, o[k + 2] * out, o[k + 3] * out);
              } else {
#pragma unroll
                for (int k = 0; k < 32; ++k)
                  if (c + k < dim) to[k] = o[k] * out;
              }
            } else {
              __nv_bfloat16* to = static_cast<__nv_bfloat16*>(g.dtable) + row * dim + c;
              if (dim % 8 == 0 && ((uintptr_t)g.dtable & 15) == 0) {
#pragma unroll
                for (int k = 0; k < 32; k += 8)
                  if (c + k < dim)
                    *reinterpret_cast<uint4*>(to + k) = make_uint4(pack_hi<1>(o[k] * out, o[k + 1] * out), pack_hi<1>(o[k + 2] * out, o[k + 3] * out),
                                                                   pack_hi<1>(o[k + 4] * out, o[k + 5] * out), pack_hi<1>(o[k + 6] * out, o[k + 7] * out));
              } else if (dim % 4 == 0 && ((uintptr_t)g.dtable & 7) == 0) {
#pragma unroll
                for (int k = 0; k < 32; k += 4)
                  if (c + k < dim)
                    *reinterpret_cast<uint2*>(to + k) = make_uint2(pack_hi<1>(o[k] * out, o[k + 1] * out), pack_hi<1>(o[k + 2] * out, o[k + 3] * out));
              } else {
#pragma unroll
                for (int k = 0; k < 32; ++k)
                  if (c + k < dim) to[k] = __float2bfloat16_rn(o[k] * out);
              }
            }
          }
        }
        __syncwarp();
        fence_before();
      }
      j = 0;
      ++r;
    }
    if (have) WAIT_LD32(z[0]);
    if (!ok) {
      if (lane == 0) {
        s_abort = 1;
        atomicCAS(g.status, 0, TGNN_ETIMEOUT);
        __threadfence_block();
      }
      __syncwarp();
      pair_leave(pair);
    }
  }
  fence_before();
  __syncthreads();
  if (s_abort && warp == 0)
    for (int i = 0; i < 64; ++i) __nanosleep(2000);       // copies asked for may still be on their way into this block's memory
  __syncthreads();
  if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------------------- joins --
struct Join {
  Shape s;
  const int32_t* count;
  const int32_t* act;
  const float* parts;
  const float* slots;
  const float* full;
  const void* q;
  const void* table;
  const float* bias;
  const float* dloss;
  const void* target;
  int index_bits, dtype, blocks, group, tile;   // blocks of the main kernel, rows of its groups, columns of its tiles (powers of two)
  int group_bits, tile_bits, extra;
  float scale;
  float* loss;
  float* kept;
  void* dtable;
  float* dbias;
};

// Four values of a row from column c on (zeros behind dim), of fp32 or bf16.
__device__ __forceinline__ float4 four_of(const void* base, int dtype, int64_t row, int dim, int c) {
  const int64_t at = row * dim + c;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (dtype == TGNN_F32) {
    const float* p = static_cast<const float*>(base) + at;
    if (c + 4 <= dim && ((uintptr_t)p & 15) == 0) return *reinterpret_cast<const float4*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k < dim) (&v.x)[k] = p[k];
  } else {
    const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(base) + at;
    if (c + 4 <= dim && ((uintptr_t)p & 7) == 0) {
      reinterpret_cast<const Group<__nv_bfloat16, 4>*>(p)->get(&v.x);
      return v;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k < dim) (&v.x)[k] = __bfloat162float(p[k]);
  }
  return v;
}
__device__ __forceinline__ void put_four(void* base, int dtype, int64_t row, int dim, int c, float4 v) {
  const int64_t at = row * dim + c;
  if (dtype == TGNN_F32) {
    float* p = static_cast<float*>(base) + at;
    if (c + 4 <= dim && ((uintptr_t)p & 15) == 0) *reinterpret_cast<float4*>(p) = v;
    else
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < dim) p[k] = (&v.x)[k];
  } else {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(base) + at;
    if (c + 4 <= dim && ((uintptr_t)p & 7) == 0) {
      Group<__nv_bfloat16, 4> g;
      g.set(&v.x);
      *reinterpret_cast<Group<__nv_bfloat16, 4>*>(p) = g;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < dim) p[k] = __float2bfloat16_rn((&v.x)[k]);
    }
  }
}

// What a root's sums make: loss, m, 1 / l, 1 - p.  L counts in units of 2^shift beside M.
struct Outcome {
  float loss, miss, m, inv;
  bool none;
};
__device__ __forceinline__ Outcome outcome_of(float M, float L, float zt, float shift) {
  Outcome v;
  const float d = (M - zt) + (log2f(L) - shift);          // log2 of the others' weight over the target's
  const bool lost = zt == -INFINITY;
  v.none = L == 0.f;
  if (v.none) {                                           // no other node in sight
    v.loss = lost ? INFINITY : zt - zt;
    v.miss = 0.f;
    v.m = lost ? INFINITY : zt;                           // weights of 0 where nothing is in sight
    v.inv = lost ? 0.f : 1.f;
  } else if (lost) {
    v.loss = INFINITY;
    v.miss = 1.f;
    v.m = M;
    v.inv = exp2f(shift) / L;
  } else {
    const float small = exp2f(-fabsf(d));                 // the smaller side over the larger
    v.loss = kLn2 * fmaxf(d, 0.f) + log1pf(small);
    v.miss = (d > 0.f ? 1.f : small) / (1.f + small);
    v.m = fmaxf(M, zt);
    v.inv = 1.f / (exp2f(zt - v.m) + L * exp2f((M - v.m) - shift));
  }
  if (d != d && !v.none && !lost) v.loss = v.miss = v.m = d;   // NaN stays
  return v;
}
__device__ __forceinline__ void put_outcome(const Join& a, int i, const Outcome& v) {
  a.loss[i] = v.loss;
  if (!a.kept) return;
  a.kept[i] = v.m;
  a.kept[a.s.n + i] = v.inv;
  a.kept[2 * a.s.n + i] = v.miss;
}
// Four columns of the direction of dq; o counts in units of those of L and `unit`, own: the target's row.
__device__ __forceinline__ void put_direction(const Join& a, int i, int c, const Outcome& v, float4 o, float L, float unit, float4 own) {
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  if (!v.none) {
    x.x = (o.x / L / unit - own.x) * v.miss;
    x.y = (o.y / L / unit - own.y) * v.miss;
    x.z = (o.z / L / unit - own.z) * v.miss;
    x.w = (o.w / L / unit - own.w) * v.miss;
  }
  put_four(a.kept + 3 * a.s.n, TGNN_F32, i, a.s.dim, c, x);
}

template <int W>
struct RootParts {                                        // of the warps that share a root
  float m[W], l[W], z[W];
  float4 o[W][64];
};

// A root whose weights do not fit beside their references, or whose products want more bits: again, product by product, 32 nodes at a time per warp.
template <int W>
__device__ __noinline__ void redo_root(const Join& a, RootParts<W>* s, int i, int64_t y) {
  const int warp = W == 1 ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31, dim = a.s.dim;
  float M = -INFINITY, l = 0.f, zt = 0.f;
  float4 o[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
  const float2 units = *reinterpret_cast<const float2*>(a.parts + 4 * kMaxParts);      // of equal signs
  const float uq = units.x, ut = units.y;
  const double factor = factor_of(a.scale, uq, ut);     // (beyond fp32 where the largest logits are: others need not be)
  for (int64_t j0 = 32ll * warp; j0 < a.s.rows; j0 += 32 * W) {
    const int64_t j = j0 + lane;
    float x = -INFINITY;
    if (j < a.s.rows) {
      float dot = 0.f;
      for (int c = 0; c < dim; ++c) dot = fmaf(value_of(a.q, a.dtype, (int64_t)i * dim + c) * uq, value_of(a.table, a.dtype, j * dim + c) * ut, dot);
      const float b = a.bias ? bias2(a.bias[j]) : 0.f;
      x = b == -INFINITY ? b : (float)(dot * factor + b);
      if (j == y) {
        zt = x;
        x = -INFINITY;
      }
    }
    float top = x;
    for (int e = 16; e; e >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, e));
    const float now = fmaxf(M, top), ref = now == -INFINITY ? 0.f : now, f = exp2f(M - ref), p = exp2f(x - ref);
    M = now;
    l = l * f + p;
    for (int k = 0; k < 8; ++k) (&o[0].x)[k] *= f;
    for (int e = 0; e < 32 && j0 + e < a.s.rows && a.kept; ++e) {
      const float pe = __shfl_sync(FULL, p, e);
      for (int h = 0; h < 2; ++h)
        if (128 * h + 4 * lane < dim) {
          const float4 t = four_of(a.table, a.dtype, j0 + e, dim, 128 * h + 4 * lane);
          for (int k = 0; k < 4; ++k) (&o[h].x)[k] = fmaf(pe, (&t.x)[k], (&o[h].x)[k]);
        }
    }
  }
  for (int e = 16; e; e >>= 1) {
    l += __shfl_xor_sync(FULL, l, e);
    zt += __shfl_xor_sync(FULL, zt, e);                   // 0 but in one lane
  }
  if (W > 1) {
    __syncthreads();
    if (lane == 0) {
      s->m[warp] = M;
      s->z[warp] = zt;
    }
    __syncthreads();
    const float mine = M;
    zt = 0.f;
    for (int w = 0; w < W; ++w) {
      M = fmaxf(M, s->m[w]);
      zt += s->z[w];
    }
    const float f = exp2f(mine - (M == -INFINITY ? 0.f : M));
    if (lane == 0) s->l[warp] = l * f;
    for (int k = 0; k < 8; ++k) (&s->o[warp][lane + 32 * (k >> 2)].x)[k & 3] = (&o[0].x)[k] * f;
    __syncthreads();
    l = 0.f;
    for (int w = 0; w < W; ++w) l += s->l[w];
    for (int k = 0; k < 8; ++k) {
      float v = 0.f;
      for (int w = 0; w < W; ++w) v += (&s->o[w][lane + 32 * (k >> 2)].x)[k & 3];
      (&o[0].x)[k] = v;
    }
    __syncthreads();
  }
  if (warp != 0) return;
  const Outcome v = outcome_of(M, l, zt, 0.f);
  if (lane == 0) put_outcome(a, i, v);
  if (!a.kept) return;
  for (int h = 0; h < 2; ++h) {
    const int c = 128 * h + 4 * lane;
    if (c < dim) put_direction(a, i, c, v, o[h], l, 1.f, four_of(a.table, a.dtype, y, dim, c));
  }
}

// W warps (8: a block, where the parts of a root are many) take the parts of four neighboring roots in turn, a few at a time: a lane has one of the roots
// and every eighth four of its columns.  H: halves of 128 columns, 0 where the loss alone is wanted.
template <int W, int H>
__global__ void __launch_bounds__(256, 2) join_roots_kernel(const __grid_constant__ Join a) {
  chain_wait();
  chain_release();
  constexpr int AHEAD = H == 0 ? 4 : 2 / H, K = 4 * H;     // (four parts ahead leave no room in registers: 600 roots 38 us in place of 36)
  constexpr bool dir = H > 0;
  __shared__ RootParts<W> s_root;
  __shared__ float s_m[W][4], s_l[W][4], s_high[W][4];
  __shared__ unsigned s_again;
  __shared__ float4 s_o[W > 1 ? W : 1][W > 1 && H > 0 ? K : 1][32];
  const int warp = W == 1 ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31, which = lane & 3, c_first = lane >> 2 << 2;
  const int64_t live = a.count[0];
  const int64_t col_tiles = (a.s.rows + a.tile - 1) >> a.tile_bits;
  const Share sh((live + a.group - 1) >> a.group_bits, col_tiles, a.extra, a.blocks);
  const int pitch = pitch_of(a.s), dim = a.s.dim, od = a.s.od;
  const int64_t step = W == 1 ? (int64_t)gridDim.x * 8 : gridDim.x;
  const float unit = a.parts[4 * kMaxParts + 1];
  const bool plain = unit < 0.f;
  const float shift = a.s.planes == 2 && dir ? 7.f : 0.f;
  for (int64_t four = W == 1 ? (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x; 4 * four < live; four += step) {
    const int64_t row = 4 * four + which, r = 4 * four >> a.group_bits, in = 4 * four - (r << a.group_bits);
    const bool valid = row < live;
    const int i = valid ? a.act[row] : 0;
    const int c0 = sh.owner(r, 0), c1 = sh.owner(r, col_tiles - 1);
    float M = -INFINITY, L = 0.f, zt = 0.f;
    float high = -INFINITY;                               // the highest reference beside which there is nothing; +infinity: a sum that is not trusted
    auto look = [&](float& m, float l) {                  // a part of no weight does not count with its reference
      if (l == 0.f) {
        high = fmaxf(high, m);
        m = -INFINITY;
      } else if (l < kLeast || l > kMost) {
        high = INFINITY;
      }
    };
    float4 o[dir ? K : 1], own[dir ? K : 1];
#pragma unroll
    for (int k = 0; k < K; ++k) o[k] = own[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    int64_t y = 0;
    auto targets_row = [&]() {
      if (valid) y = a.index_bits == 64 ? static_cast<const int64_t*>(a.target)[i] : static_cast<const int32_t*>(a.target)[i];
      if (dir && warp == 0)
#pragma unroll
        for (int k = 0; k < K; ++k)
          if (c_first + 32 * k < dim) own[k] = four_of(a.table, a.dtype, y, dim, c_first + 32 * k);
    };
    if (c0 == c1) {
      targets_row();
      if (valid) {
        M = a.full[3 * row];
        L = a.full[3 * row + 1];
        zt = a.full[3 * row + 2];
        look(M, L);
        if (dir && warp == 0)
#pragma unroll
          for (int k = 0; k < K; ++k)
            if (c_first + 32 * k < dim) o[k] = four_of(a.kept + 3 * a.s.n, TGNN_F32, i, dim, c_first + 32 * k);
      }
    } else {
      // parts lie two places apart, but for the first, which may be its block's last
      const float* first = a.slots + ((int64_t)slot_of(sh, col_tiles, c0, r) * a.group + in) * pitch + 4 * which;
      const float* rest = a.slots + ((int64_t)2 * c0 * a.group + in) * pitch + 4 * which;
      const int64_t apart = 2ll * a.group * pitch;
      const int parts = c1 - c0 + 1;
      auto part = [&](int k) { return k == 0 ? first : rest + k * apart; };
      if (warp >= parts) targets_row();
      for (int j0 = warp; j0 < parts; j0 += W * AHEAD) {
        float4 tail[AHEAD], v[AHEAD][dir ? K : 1];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          const int j = j0 + u * W;
          tail[u] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
          if (j >= parts) continue;
          const float* p = part(j);
          tail[u] = *reinterpret_cast<const float4*>(p + 4 * od);
          if (dir)
#pragma unroll
            for (int k = 0; k < K; ++k)
              if (c_first + 32 * k < od) v[u][k] = *reinterpret_cast<const float4*>(p + 4 * (c_first + 32 * k));
        }
        if (j0 == warp) {                                 // (asked for behind the first parts)
          targets_row();
          zt = part(sh.owner(r, y >> a.tile_bits) - c0)[4 * od + 2];
        }
        float top = M;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          look(tail[u].x, tail[u].y);
          top = fmaxf(top, tail[u].x);
        }
        const float ref = top == -INFINITY ? 0.f : top, before = exp2f(M - ref);
        M = top;
        L *= before;
#pragma unroll
        for (int k = 0; k < K; ++k) o[k] = make_float4(o[k].x * before, o[k].y * before, o[k].z * before, o[k].w * before);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          if (j0 + u * W >= parts) break;
          const float f = exp2f(tail[u].x - ref);
          L = fmaf(tail[u].y, f, L);
          if (dir)
#pragma unroll
            for (int k = 0; k < K; ++k)
              if (c_first + 32 * k < od) {
                o[k].x = fmaf(v[u][k].x, f, o[k].x);
                o[k].y = fmaf(v[u][k].y, f, o[k].y);
                o[k].z = fmaf(v[u][k].z, f, o[k].z);
                o[k].w = fmaf(v[u][k].w, f, o[k].w);
              }
        }
      }
      if (W > 1) {
        if (lane < 4) {
          s_m[warp][lane] = M;
          s_l[warp][lane] = L;
          s_high[warp][lane] = high;
        }
#pragma unroll
        for (int k = 0; k < K; ++k) s_o[warp][k][lane] = o[k];
        __syncthreads();
        for (int w = 0; w < W; ++w) {
          M = fmaxf(M, s_m[w][which]);
          high = fmaxf(high, s_high[w][which]);
        }
        const float ref = M == -INFINITY ? 0.f : M;
        L = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = 0; w < W; ++w) {
          const float f = exp2f(s_m[w][which] - ref);
          L = fmaf(s_l[w][which], f, L);
          if (warp == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) {
              const float4 x = s_o[w][k][lane];
              o[k].x = fmaf(x.x, f, o[k].x);
              o[k].y = fmaf(x.y, f, o[k].y);
              o[k].z = fmaf(x.z, f, o[k].z);
              o[k].w = fmaf(x.w, f, o[k].w);
            }
        }
        __syncthreads();
      }
    }
    // Done again: where weights below 2^-126 of a reference, which were left out, lie so near the root's sum that they may count; where sums are not trusted,
    // those of the table's rows among them, which can pass fp32 before the weights' do.  (What is no number stays so.)
    bool lost = plain || high == INFINITY || high > M + log2f(L) + kRoom;
    if (dir && warp == 0 && L == L) {
      float size = 0.f;
#pragma unroll
      for (int k = 0; k < K; ++k) size += fabsf(o[k].x) + fabsf(o[k].y) + fabsf(o[k].z) + fabsf(o[k].w);
      lost |= !(size < INFINITY);
    }
    unsigned again = __ballot_sync(FULL, valid && lost);
    again |= again >> 16;
    again |= again >> 8;
    again = (again | again >> 4) & 15u;                   // of the four roots
    if (W > 1) {
      if (threadIdx.x == 0) s_again = again;
      __syncthreads();
      again = s_again;
      __syncthreads();
    }
    if (warp == 0 && valid && !(again >> which & 1)) {
      const Outcome v = outcome_of(M, L, zt, shift);
      if (lane < 4) put_outcome(a, i, v);
      if (dir)
#pragma unroll
        for (int k = 0; k < K; ++k)
          if (c_first + 32 * k < dim) put_direction(a, i, c_first + 32 * k, v, o[k], L, unit, own[k]);
    }
    __syncwarp();
    for (; again; again &= again - 1) {
      const int x = __ffs(again) - 1;
      redo_root<W>(a, &s_root, __shfl_sync(FULL, i, x), __shfl_sync(FULL, y, x));
    }
  }
}

// Gradients of table rows whose products want more bits than the operands have: product by product, a warp per row, 32 roots at a time.
__device__ __noinline__ void plain_table(const Join& a, int64_t live, float uq, float ut) {
  const int lane = threadIdx.x & 31, dim = a.s.dim;
  const int64_t warps = (int64_t)gridDim.x * gridDim.y * 8, first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 8 + (threadIdx.x >> 5);
  const float* table = static_cast<const float*>(a.table);
  const double factor = factor_of(a.scale, uq, ut);
  for (int64_t j = first; j < a.s.rows; j += warps) {
    const float b = a.bias ? bias2(a.bias[j]) : 0.f;
    float t[8], sum[8], all = 0.f;
    for (int k = 0; k < 8; ++k) {
      t[k] = lane + 32 * k < dim && b != -INFINITY ? table[j * dim + lane + 32 * k] * ut : 0.f;
      sum[k] = 0.f;
    }
    for (int64_t x0 = 0; x0 < live; x0 += 32) {
      float part[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, part_all = 0.f;
      for (int64_t x = x0; x < min(live, x0 + 32); ++x) {
        const int64_t i = a.act[x];
        float q[8], dot = 0.f;
        for (int k = 0; k < 8; ++k) {
          q[k] = lane + 32 * k < dim ? static_cast<const float*>(a.q)[i * dim + lane + 32 * k] * uq : 0.f;
          dot = fmaf(q[k], t[k], dot);
        }
        for (int e = 16; e; e >>= 1) dot += __shfl_xor_sync(FULL, dot, e);
        const int64_t y = a.index_bits == 64 ? static_cast<const int64_t*>(a.target)[i] : static_cast<const int32_t*>(a.target)[i];
        const float g = a.dloss[i];
        const float w = y == j ? -g * a.kept[2 * a.s.n + i] : g * (exp2f((float)(dot * factor + b) - a.kept[i]) * a.kept[a.s.n + i]);
        part_all += w;
        for (int k = 0; k < 8; ++k) part[k] = fmaf(w, q[k], part[k]);
      }
      all += part_all;
      for (int k = 0; k < 8; ++k) sum[k] += part[k];
    }
    if (a.dtable)
      for (int k = 0; k < 8; ++k)
        if (lane + 32 * k < dim) static_cast<float*>(a.dtable)[j * dim + lane + 32 * k] = (float)((double)sum[k] * a.scale * __frcp_rn(uq));
    if (a.dbias && lane == 0) a.dbias[j] = all;
  }
}

// Groups of table rows that several blocks share: block b takes the group that begins before the boundary between blocks b - 1 and b, if that is the
// group's first one; grid.y parts of its rows.  Without any live root, zeros everywhere.
template <bool FP32>
__global__ void __launch_bounds__(256, 4) join_table_kernel(const __grid_constant__ Join a) {
  chain_wait();
  chain_release();
  const int64_t live = a.count[0];
  const int dim = a.s.dim, pitch = pitch_of(a.s);
  auto put = [&](int64_t x, float v) {
    if (a.dtype == TGNN_F32) static_cast<float*>(a.dtable)[x] = v;
    else static_cast<__nv_bfloat16*>(a.dtable)[x] = __float2bfloat16_rn(v);
  };
  if (live == 0) {
    const int64_t t = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x, all = (int64_t)gridDim.x * gridDim.y * 256;
    if (a.dtable)
      for (int64_t x = t; x < a.s.rows * dim; x += all) put(x, 0.f);
    if (a.dbias)
      for (int64_t x = t; x < a.s.rows; x += all) a.dbias[x] = 0.f;
    return;
  }
  const float4 units = *reinterpret_cast<const float4*>(a.parts + 4 * kMaxParts);
  const float uq = units.x, ug = units.z, out = (float)((double)a.scale * __frcp_rn(ug) * __frcp_rn(uq));
  if (FP32 && uq < 0.f) {
    plain_table(a, live, uq, units.y);
    return;
  }
  const int64_t col_tiles = (live + a.tile - 1) / a.tile;
  const Share sh((a.s.rows + a.group - 1) / a.group, col_tiles, a.extra, a.blocks);
  const int b = blockIdx.x + 1;
  if (b >= sh.blocks) return;
  const int64_t x = sh.begin(b), r = quotient(x, col_tiles);
  if (x == r * col_tiles) return;
  const int c0 = sh.owner(r, 0), c1 = sh.owner(r, col_tiles - 1);
  if (b != c0 + 1) return;
  const int od = a.s.od, chunks = pitch / 4, all = a.group * chunks;
  // the others than the first part are their blocks' first; all in the order in which they lie
  const float4* first = reinterpret_cast<const float4*>(a.slots + (int64_t)slot_of(sh, col_tiles, c0, r) * a.group * pitch);
  const float4* rest = reinterpret_cast<const float4*>(a.slots + (int64_t)2 * c0 * a.group * pitch);
  const int64_t apart = (int64_t)a.group * pitch / 2;
  const int stride = gridDim.y * 256;
  for (int e0 = blockIdx.y * 256 + threadIdx.x; e0 < all; e0 += 4 * stride) {               // four at a time
    float4 v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = e0 + q * stride < all ? first[e0 + q * stride] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int k = 1; k <= c1 - c0; ++k) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (e0 + q * stride >= all) continue;
        const float4 w = rest[k * apart + e0 + q * stride];
        v[q].x += w.x;
        v[q].y += w.y;
        v[q].z += w.z;
        v[q].w += w.w;
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int e = e0 + q * stride, fours = e / 4 / chunks, c = 4 * (e / 4 - fours * chunks);
      const int64_t row = r * a.group + 4 * fours + (e & 3);
      if (e >= all || row >= a.s.rows) continue;
      if (c == od) {
        if (a.dbias) a.dbias[row] = v[q].x / ug;
      } else if (a.dtable) {
        put_four(a.dtable, a.dtype, row, dim, c, make_float4(v[q].x * out, v[q].y * out, v[q].z * out, v[q].w * out));
      }
    }
  }
}

// --------------------------------------------------------------------------------------------------------- host side --
struct Form {
  int planes, group, tile;                    // of the main kernel
};
Form form_of(int dim, int dtype) {
  if (dtype == TGNN_F32) return {2, 128, dim <= 128 ? 128 : 64};
  return {1, dim <= 128 ? 256 : 128, 128};
}
Shape shape_of(int64_t n, int64_t rows, int dim, int dtype) {
  Shape s;
  s.n = n;
  s.rows = rows;
  s.dim = dim;
  s.dp = (dim + 63) / 64 * 64;
  s.planes = dtype == TGNN_F32 ? 2 : 1;
  s.od = (dim + 15) / 16 * 16;
  return s;
}
Layout layout(const Shape& s, int dtype) {
  const Form f = form_of(s.dim, dtype);
  Layout l;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t p = at;
    at += up(bytes, 256);
    return p;
  };
  l.count = take(4);
  l.act = take(4 * s.n);
  l.parts = take(4ll * (4 * kMaxParts + 4));
  l.qp = take(2ll * up(s.n, 128) * s.planes * s.dp);
  l.tp = take(2ll * s.rows * s.planes * s.dp);
  const int64_t forward = 4ll * up(s.rows, f.tile), backward = 16ll * up(s.n, f.tile);
  l.cols = take(forward > backward ? forward : backward);
  const int64_t tiles = (up(s.n, 128) / 128 + 1) * (up(s.rows, 64) / 64 + 1);   // of either direction, at most
  l.slots = take(4ll * 2 * (tiles < kMaxBlocks ? tiles : kMaxBlocks) * f.group * pitch_of(s));
  l.full = take(12ll * s.n);
  l.bytes = at;
  return l;
}

bool encode(CUtensorMap* map, const void* base, int64_t width, int64_t rows, int64_t pitch_bytes, int box_rows) {
  const tgnn::TensorMapEncodeFn enc = tgnn::tensor_map_encoder();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch_bytes};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, step[2] = {1, 1};
  auto made = [&] {
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (made()) return true;
  // The encoder wants a context, and a thread that has made no call to the runtime so far (a backward pass's first one) has none: the device is set.
  int device;
  return cudaGetDevice(&device) == cudaSuccess && cudaSetDevice(device) == cudaSuccess && made();
}

template <int MODE>
void launch_main(Chain& c, const Main& m, int blocks, size_t smem) {
  auto go = [&](auto kernel, int threads) {
    if (c.e == cudaSuccess) c.e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    c(kernel, dim3(blocks), dim3(threads), smem, m);
  };
  if (m.s.planes == 2) {
    if (m.s.dim <= 128) go(destination_kernel<MODE, 2, 1, 128, 128>, 384);
    else go(destination_kernel<MODE, 2, 1, 64, 64>, 384);
  } else {
    if (m.s.dim <= 128) go(destination_kernel<MODE, 1, 2, 128, 64>, 640);
    else go(destination_kernel<MODE, 1, 1, 128, 128>, 384);
  }
}

struct Call {
  const char* who;
  const void *q, *table;
  int dtype;
  int64_t n, rows;
  int dim;
  const void* target;
  int index_bits;
  const float* bias;
  float scale;
  void* scratch;
  int32_t* status;
  void* stream;
  char* err;
  int64_t err_size;
};

bool sizes_ok(int64_t n, int64_t rows, int dim) {
  return n >= 0 && n < 0x7fff0000ll && rows >= 0 && rows <= 0x7fff0000ll && dim >= 1 && dim <= 256;
}

int check(const Call& a) {
  if (a.dtype != TGNN_F32 && a.dtype != TGNN_BF16) return fail(a.err, a.err_size, TGNN_EINVAL, "%s: rows are fp32 or bf16", a.who);
  if (a.index_bits != 32 && a.index_bits != 64) return fail(a.err, a.err_size, TGNN_EINVAL, "%s: index_bits is 32 or 64", a.who);
  if (!sizes_ok(a.n, a.rows, a.dim) || a.rows < 1)
    return fail(a.err, a.err_size, TGNN_EINVAL, "%s: size out of range (dim 1 to 256, rows from 1, n and rows to 2^31 - 2^16)", a.who);
  if (!(a.scale - a.scale == 0)) return fail(a.err, a.err_size, TGNN_EINVAL, "%s: scale is not finite", a.who);
  if (!a.table || !a.status || !a.scratch || (a.n > 0 && (!a.q || !a.target))) return fail(a.err, a.err_size, TGNN_EINVAL, "%s: null pointer", a.who);
  if ((((uintptr_t)a.q | (uintptr_t)a.table) & (elem_bytes(a.dtype) - 1)) || ((uintptr_t)a.target & (a.index_bits / 8 - 1)) ||
      (((uintptr_t)a.bias | (uintptr_t)a.status) & 3) || ((uintptr_t)a.scratch & 255))
    return fail(a.err, a.err_size, TGNN_EINVAL, "%s: a pointer is not aligned (scratch to 256 bytes, the others to their elements)", a.who);
  return TGNN_OK;
}

// begin, prep and main kernels of one direction
template <int MODE>
int run(const Call& a, Chain& c, float* loss, float* kept, const float* dloss, void* dq, void* dtable, float* dbias, Join* j) {
  const Shape s = shape_of(a.n, a.rows, a.dim, a.dtype);
  const Form f = form_of(a.dim, a.dtype);
  const Layout l = layout(s, a.dtype);
  char* base = static_cast<char*>(a.scratch);
  const int sms = num_sms() < kMaxBlocks ? num_sms() : kMaxBlocks;
  const bool direct = a.dtype == TGNN_BF16 && a.dim >= 64 && a.dim % 8 == 0 && ((uintptr_t)a.table & 15) == 0;
  Prep p = {};
  p.s = s;
  p.q = a.q;
  p.table = a.table;
  p.target = a.target;
  p.index_bits = a.index_bits;
  p.dtype = a.dtype;
  p.copy_table = !direct;
  p.bias = a.bias;
  p.dloss = dloss;
  p.kept = kept;
  p.loss = loss;
  p.scale = a.scale;
  p.backward = MODE == BACKWARD;
  p.tile = f.tile;
  p.count = reinterpret_cast<int32_t*>(base + l.count);
  p.act = reinterpret_cast<int32_t*>(base + l.act);
  p.parts = reinterpret_cast<float*>(base + l.parts);
  p.qp = reinterpret_cast<uint16_t*>(base + l.qp);
  p.tp = reinterpret_cast<uint16_t*>(base + l.tp);
  p.cols = reinterpret_cast<float*>(base + l.cols);
  p.status = a.status;
  p.dq = dq;
  Main m = {};
  m.s = s;
  m.count = p.count;
  m.act = p.act;
  m.parts = p.parts;
  m.cols = p.cols;
  m.target = a.target;
  m.index_bits = a.index_bits;
  m.bias = a.bias;
  m.slots = reinterpret_cast<float*>(base + l.slots);
  m.full = reinterpret_cast<float*>(base + l.full);
  m.kept = kept;
  m.dtable = dtable;
  m.dbias = dbias;
  m.dtype = a.dtype;
  m.scale = a.scale;
  m.chunks = s.dp / 64;
  m.ksteps = s.od / 16;
  m.status = a.status;
  const int64_t pitch = 2ll * s.planes * s.dp;
  const void* rows = direct ? a.table : p.tp;
  const int64_t width = direct ? a.dim : s.planes * s.dp, t_pitch = direct ? 2ll * a.dim : pitch;
  const int q_box = MODE == BACKWARD ? f.tile : f.group, t_box = MODE == BACKWARD ? f.group : f.tile;
  if (!encode(MODE == BACKWARD ? &m.t_map : &m.a_map, p.qp, s.planes * s.dp, up(s.n, 128), pitch, q_box) ||
      !encode(MODE == BACKWARD ? &m.a_map : &m.t_map, rows, width, s.rows, t_pitch, t_box))
    return fail(a.err, a.err_size, TGNN_ECUDA, "%s: a tensor map could not be made", a.who);
  const int a_bytes = s.planes * m.chunks * f.group * 128, t_bytes = s.planes * m.chunks * f.tile * 128 + (MODE == BACKWARD ? 16 : 4) * f.tile;
  m.stages = (kSmem - 1024 - a_bytes) / t_bytes;
  if (m.stages > 4) m.stages = 4;
  m.ahead = m.stages > 1 ? 2 : 1;
  const size_t smem = 1024 + a_bytes + (size_t)m.stages * t_bytes;
  // blocks beside the first one: some 4096 values each
  const int64_t beside = s.planes == 2 ? a.rows * a.dim + (dq ? a.n * a.dim : 0) : dq ? a.n * a.dim : MODE != BACKWARD && a.bias ? a.rows : 0;
  const int blocks_of_parts = beside == 0 ? 0 : (int)(beside >> 12 >= kMaxParts - 1 ? kMaxParts - 1 : (beside >> 12) + 1);
  p.parts_used = blocks_of_parts;
  c(begin_kernel, dim3(1 + blocks_of_parts), dim3(1024), 0, p);
  const int64_t work = (direct ? 0 : a.rows) + a.n + (MODE == BACKWARD ? a.n : a.rows) / 32;
  c(prep_kernel, dim3((unsigned)(work / 16 >= 8 * sms ? 8 * sms : work / 16 + 1)), dim3(256), 0, p);
  const int64_t r_tiles = ((MODE == BACKWARD ? a.rows : a.n) + f.group - 1) / f.group, c_tiles = ((MODE == BACKWARD ? a.n : a.rows) + f.tile - 1) / f.tile;
  const int blocks = (int)(r_tiles * c_tiles < sms ? r_tiles * c_tiles : sms);
  // Extra tiles of a group, where a block has several tiles.  Us of the forward pass with 0 / 1 / 2 / 3 / 4 of them, rows of 100 in bf16: 4000 roots over 17 000
  // nodes 58.1 / 56.0 / 54.0 / 54.3 / 54.2, 12 000 roots 124 / 117 / 116 / 112 / 112, 30 000 roots over 2000 nodes 93 / 92 / 93 / 92 / 102; fp32, 2000 roots over
  // 50 000 nodes, both passes 312 / 309 / 309 / 312 / 315.
  m.extra = r_tiles * c_tiles < 8 * blocks ? 0 : s.planes == 2 ? 2 : 3;
  launch_main<MODE>(c, m, blocks, smem);
  *j = Join{};
  j->s = s;
  j->count = p.count;
  j->act = p.act;
  j->parts = p.parts;
  j->slots = m.slots;
  j->full = m.full;
  j->q = a.q;
  j->table = a.table;
  j->bias = a.bias;
  j->dloss = dloss;
  j->target = a.target;
  j->index_bits = a.index_bits;
  j->dtype = a.dtype;
  j->blocks = blocks;
  j->group = f.group;
  j->tile = f.tile;
  j->group_bits = f.group == 256 ? 8 : 7;
  j->tile_bits = f.tile == 128 ? 7 : 6;
  j->extra = m.extra;
  j->scale = a.scale;
  j->loss = loss;
  j->kept = kept;
  j->dtable = dtable;
  j->dbias = dbias;
  return TGNN_OK;
}

}  // namespace

extern "C" TGNN_API int64_t tgnn_destination_loss_kept(int64_t n, int dim) { return n < 0 || dim < 1 || dim > 256 ? -1 : n * (3 + dim); }

extern "C" TGNN_API int64_t tgnn_destination_loss_scratch(int64_t n, int64_t rows, int dim, int dtype) {
  if (!sizes_ok(n, rows, dim) || (dtype != TGNN_F32 && dtype != TGNN_BF16)) return -1;
  return layout(shape_of(n, rows, dim, dtype), dtype).bytes;
}

extern "C" TGNN_API int tgnn_destination_loss(const void* q, const void* table, int dtype, int64_t n, int64_t rows, int dim, const void* target,
                                              int index_bits, const float* bias, float scale, float* loss, float* kept, void* scratch,
                                              int32_t* status, void* stream, char* err, int64_t err_size) {
  const Call a = {"tgnn_destination_loss", q, table, dtype, n, rows, dim, target, index_bits, bias, scale, scratch, status, stream, err, err_size};
  if (int rc = check(a)) return rc;
  if (n == 0) return TGNN_OK;
  if (!loss || (((uintptr_t)loss | (uintptr_t)kept) & 3)) return fail(err, err_size, TGNN_EINVAL, "%s: loss is null, or loss or kept not aligned", a.who);
  Chain c(stream);
  Join j;
  const int rc = kept ? run<FORWARD>(a, c, loss, kept, nullptr, nullptr, nullptr, nullptr, &j) : run<LOSS>(a, c, loss, kept, nullptr, nullptr, nullptr, nullptr, &j);
  if (rc) return rc;
  // 16 parts of a root and more: a block for four roots, else a warp.  Us of a loss with what the backward pass needs, a warp and a block, rows of 100: 49 parts
  // (600 roots, 9000 nodes, bf16) 50 and 31, 29 (the same in fp32) 46 and 36, 18 (2000 roots, bf16) 39 and 40, (1024 roots, 100 000 nodes, fp32) 181 and 174,
  // 9 (2000 roots, 9000 nodes, fp32) 52 and 55, 8 (4800 roots, 17 000 nodes, bf16) 61 and 81
  const int64_t groups = (n + j.group - 1) / j.group, most = 8 * num_sms();
  const bool many = j.blocks >= 16 * groups;
  const int64_t blocks = many ? (n + 3) / 4 : (n + 31) / 32;
  auto go = [&](auto kernel) { c(kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, j); };
  if (!kept) many ? go(join_roots_kernel<8, 0>) : go(join_roots_kernel<1, 0>);
  else if (dim <= 128) many ? go(join_roots_kernel<8, 1>) : go(join_roots_kernel<1, 1>);
  else many ? go(join_roots_kernel<8, 2>) : go(join_roots_kernel<1, 2>);
  return c.end(a.who, err, err_size);
}

extern "C" TGNN_API int tgnn_destination_loss_backward(const void* q, const void* table, int dtype, int64_t n, int64_t rows, int dim,
                                                       const void* target, int index_bits, const float* bias, float scale, const float* kept,
                                                       const float* dloss, void* dq, void* dtable, float* dbias, void* scratch, int32_t* status,
                                                       void* stream, char* err, int64_t err_size) {
  const Call a = {"tgnn_destination_loss_backward", q, table, dtype, n, rows, dim, target, index_bits, bias, scale, scratch, status, stream, err,
                  err_size};
  if (int rc = check(a)) return rc;
  if (n > 0 && (!kept || !dloss)) return fail(err, err_size, TGNN_EINVAL, "%s: null pointer", a.who);
  if ((((uintptr_t)dq | (uintptr_t)dtable) & (elem_bytes(dtype) - 1)) || (((uintptr_t)kept | (uintptr_t)dloss | (uintptr_t)dbias) & 3))
    return fail(err, err_size, TGNN_EINVAL, "%s: a pointer is not aligned to its element", a.who);
  cudaStream_t s = (cudaStream_t)stream;
  if (n == 0) {
    cudaError_t e = dtable ? cudaMemsetAsync(dtable, 0, (size_t)(rows * dim * elem_bytes(dtype)), s) : cudaSuccess;
    if (e == cudaSuccess && dbias) e = cudaMemsetAsync(dbias, 0, (size_t)(4 * rows), s);
    if (e != cudaSuccess) {
      cudaGetLastError();
      return fail(err, err_size, TGNN_ECUDA, "%s: %s", a.who, cudaGetErrorString(e));
    }
    return TGNN_OK;
  }
  Chain c(stream);
  if (dtable || dbias) {
    Join j;
    if (int rc = run<BACKWARD>(a, c, nullptr, const_cast<float*>(kept), dloss, dq, dtable, dbias, &j)) return rc;
    c(dtype == TGNN_F32 ? join_table_kernel<true> : join_table_kernel<false>, dim3((unsigned)j.blocks, 8), dim3(256), 0, j);
  } else if (dq) {
    Prep p = {};
    p.s = shape_of(n, rows, dim, TGNN_BF16);              // no maxima of rows
    p.target = target;
    p.index_bits = index_bits;
    p.dtype = dtype;
    p.dloss = dloss;
    p.kept = kept;
    p.dq = dq;
    p.scale = scale;
    p.backward = 1;
    const Layout l = layout(shape_of(n, rows, dim, dtype), dtype);
    p.parts = reinterpret_cast<float*>(static_cast<char*>(scratch) + l.parts);
    const int64_t blocks = n * dim >> 12;
    c(begin_kernel, dim3((unsigned)(2 + (blocks < kMaxParts - 1 ? blocks : kMaxParts - 2))), dim3(1024), 0, p);
  }
  return c.end(a.who, err, err_size);
}
