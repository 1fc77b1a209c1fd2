// Attention of one query per root and head over the window and the sinks of the root's history, keys and values in a row cache
// of 4 or 8 bits, with a learned bias by buckets of the time difference.
//
//   s_j = scale * q . k_j + bias[h, bucket_j],   k_j = ks_j * c_j   (c_j: integer codes, one scale per row and head)
//   out = sum_j p_j v_j / l,   p_j = exp(s_j - m),  l = sum_j p_j    (m = running maximum)
// (Logits stay in natural units, and log2(e) goes into the difference: a bias of the type's lowest value is then still finite.)
//
// Both products run on the tensor cores (m16n8k16, fp16 operands, fp32 sums) although a root has a single query: what they save is not
// the multiplications but the conversion of every code to fp32 and the sums across lanes.  The codes go in as they are, as fp16
// integers (exact), and the scales are applied to the other side: ks_j to the finished logits, vs_j to the weights.  The other operand
// is kept to fp32's accuracy by splitting it in two fp16 terms (x = hi + lo / 2048, 22 bits): a tile has 16 rows, the terms of 8
// query heads that share a cached head take all of them (hi in rows 0-7, lo in rows 8-15), so the split costs nothing.  Both terms of
// a row end up in one thread.  fp16's range is no limit: a query is divided by a power of two at its largest value, and
// weights w_j = p_j vs_j are divided by a running bound sc of w.  The output is held in units of sc at maximum m; when a weight
// passes sc it is rescaled.
//
// The sum over dim may be taken in any order, so a lane reads neighbouring words of a key's codes with one wide load and the query
// is laid out to match; likewise for the values' columns.  tcgen05's 128-row tiles would be filled to 1/16 by one root's
// heads, and roots see different rows.
//
// Work: a unit is a root, a cached head and up to 8 of its query heads.  Units are handled by a warp, by a block of 4 warps
// or by a cluster of 2 to 8 blocks whose partial results meet in distributed shared memory (no workspace, no atomics, sums in
// a fixed order); the launch takes more warps per unit while the units alone would leave SMs idle and each warp still has a few
// tiles to walk.
//
// Bound by the codes' bytes for long windows, by the chain of dependent loads (length, then rows) for short ones.
#include <cooperative_groups.h>

#include "tgnn_history.cuh"

using namespace tgnn_history;
namespace cg = cooperative_groups;

namespace {

constexpr int WARPS = 4;
constexpr int GH = 8;                     // query heads of a unit
constexpr float kLo = 2048.f;             // lo terms are held times 2^11, clear of fp16's subnormals

struct AttendArgs {
  const void* q;
  void* out;
  int dtype;
  const uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
  int k_code_stride, v_code_stride, k_scale_stride, v_scale_stride;
  int64_t rows;
  uint32_t units;
  int heads, kv_heads, group, passes, dim;    // group = heads / kv_heads, passes = ceil(group / 8)
  const int64_t* first;
  const int32_t* len;
  const float* bias;
  const double *bounds, *times, *ts;
  int buckets, window, sinks;
  float scale;
  int32_t* status;
};

__device__ __forceinline__ uint32_t h2u(__half2 x) { return *reinterpret_cast<uint32_t*>(&x); }
__device__ __forceinline__ __half2 u2h(uint32_t x) { return *reinterpret_cast<__half2*>(&x); }

// (a & mask) | bits
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(a), "r"(mask), "r"(bits));
  return r;
}

// The four pairs of codes whose nibbles lie in the low and the high half of t: out[j] = (nibble j, nibble j + 4) - 8 as fp16.  A nibble
// under the exponent of 1024 reads as 1024 + n, four bits further up as 1024 + 16 n.
__device__ __forceinline__ void nibbles(uint32_t t, uint32_t (&out)[4]) {
  const __half2 one = u2h(0x64086408u);                                 // 1032
  const __half2 sixteenth = u2h(0x2c002c00u), off = u2h(0xd480d480u);   // 1 / 16, -72
  out[0] = h2u(__hsub2(u2h(and_or(t, 0x000f000fu, 0x64006400u)), one));
  out[1] = h2u(__hfma2(u2h(and_or(t, 0x00f000f0u, 0x64006400u)), sixteenth, off));
  t >>= 8;
  out[2] = h2u(__hsub2(u2h(and_or(t, 0x000f000fu, 0x64006400u)), one));
  out[3] = h2u(__hfma2(u2h(and_or(t, 0x00f000f0u, 0x64006400u)), sixteenth, off));
}

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// x0, x1 as fp16 pairs hi and lo with x = hi + lo / 2048
__device__ __forceinline__ void split2(float x0, float x1, uint32_t* hi, uint32_t* lo) {
  const __half2 h = __floats2half2_rn(x0, x1);
  const float2 f = __half22float2(h);
  *hi = h2u(h);
  *lo = h2u(__floats2half2_rn((x0 - f.x) * kLo, (x1 - f.y) * kLo));
}

template <int N>
struct Words { uint32_t w[N]; };
// N words that start on a multiple of their size (16 bytes at most)
template <int N>
__device__ __forceinline__ Words<N> load_words(const uint8_t* p) {
  Words<N> r;
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(p) + i);
      r.w[4 * i] = x.x;
      r.w[4 * i + 1] = x.y;
      r.w[4 * i + 2] = x.z;
      r.w[4 * i + 3] = x.w;
    }
  } else if constexpr (N == 2) {
    const uint2 x = __ldg(reinterpret_cast<const uint2*>(p));
    r.w[0] = x.x;
    r.w[1] = x.y;
  } else {
    static_assert(N == 1, "");
    r.w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
  }
  return r;
}
// B bytes: 2, or whole words
template <int B>
__device__ __forceinline__ Words<(B + 3) / 4> load_piece(const uint8_t* p) {
  if constexpr (B == 2) {
    Words<1> r;
    r.w[0] = __ldg(reinterpret_cast<const uint16_t*>(p));
    return r;
  } else {
    return load_words<B / 4>(p);
  }
}

__device__ __forceinline__ float load_q(const void* q, int dtype, int64_t i) {
  if (dtype == TGNN_F32) return __ldg(reinterpret_cast<const float*>(q) + i);
  if (dtype == TGNN_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(q)[i]);
  return __half2float(reinterpret_cast<const __half*>(q)[i]);
}
__device__ __forceinline__ void store_out(void* o, int dtype, int64_t i, float x) {
  if (dtype == TGNN_F32) reinterpret_cast<float*>(o)[i] = x;
  else if (dtype == TGNN_BF16) reinterpret_cast<__nv_bfloat16*>(o)[i] = __float2bfloat16_rn(x);
  else reinterpret_cast<__half*>(o)[i] = __float2half_rn(x);
}

// Keys that a warp takes at a time: 32, or 16 where 32 rows of codes would not fit into registers.
template <int BITS, int DP>
struct Tile {
  static constexpr int TK = (BITS == 8 && DP == 128) ? 16 : 32;
  static constexpr int NT = TK / 8;                 // key tiles of 8 columns
  static constexpr int KW = DP * BITS / 128;        // words of a key that a lane reads (a quarter of the row)
  static constexpr int VD = DP / 8;                 // columns of a value that a lane reads
  static constexpr int VB = VD * BITS / 8;          // bytes of them: 2 to 16
};

// One warp's walk over tiles w, w + workers, ... of the unit's visible entries.  Results: o[VD][4] in units of sc, m, l, sc; the rows
// of a lane are the hi and lo terms of head `lane / 4` of the unit, its columns [2 c VD, 2 c VD + 2 VD) with c = lane % 4.
template <int BITS, int DP>
struct Walk {
  using T = Tile<BITS, DP>;
  float o[T::VD][4];
  float m, l, sc;

  __device__ __forceinline__ void run(const AttendArgs& a, const double* s_bounds, int64_t root, int kv, int head0, int64_t first, int lo,
                                      int ns, int n, int worker, int workers) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    constexpr int KS = DP / 16;
    m = -INFINITY;
    l = 0.f;
    sc = 0.f;
#pragma unroll
    for (int i = 0; i < T::VD; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    const int tiles = (n + T::TK - 1) / T::TK;
    if (worker >= tiles) return;
    const bool mine = head0 + g < (kv + 1) * a.group;               // a query head of this unit

    // the query: a lane holds columns [c * DP / 4, (c + 1) * DP / 4) of head g, divided by a power of two
    uint32_t qa[KS][4];
    float qfac;
    {
      float x[DP / 4];
      const int64_t base = (root * a.heads + head0 + g) * a.dim;
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < DP / 4; ++i) {
        const int e = c * (DP / 4) + i;
        x[i] = mine && e < a.dim ? load_q(a.q, a.dtype, base + e) : 0.f;
        top = fmaxf(top, fabsf(x[i]));
      }
      top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
      top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
      // 2^e <= top < 2^(e + 1): scaled queries lie below 2 (infinities and NaN stay what they are)
      const int e = min(max((int)(__float_as_uint(top) >> 23), 2), 252);
      const float down = __uint_as_float((uint32_t)(254 - e) << 23);
      qfac = a.scale * __uint_as_float((uint32_t)e << 23);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        // BITS 4: the columns of a step in the order in which nibbles() pairs them
        const int b = BITS == 4 ? 8 * (s >> 1) + 2 * (s & 1) : 4 * s;
        const int i1 = BITS == 4 ? b + 4 : b + 1, i2 = BITS == 4 ? b + 1 : b + 2, i3 = BITS == 4 ? b + 5 : b + 3;
        split2(x[b] * down, x[i1] * down, &qa[s][0], &qa[s][1]);
        split2(x[i2] * down, x[i3] * down, &qa[s][2], &qa[s][3]);
      }
    }

    const double t_root = a.bias ? a.times[root] : 0.0;
    const uint8_t* kp = a.k_codes + first * a.k_code_stride + kv * (DP * BITS / 8) + c * (DP * BITS / 32);
    const uint8_t* vp = a.v_codes + first * a.v_code_stride + kv * (DP * BITS / 8) + g * T::VB;
    const uint8_t* ksp = a.k_scales + first * a.k_scale_stride + 2 * kv;
    const uint8_t* vsp = a.v_scales + first * a.v_scale_stride + 2 * kv;
    const float* bias = a.bias ? a.bias + (int64_t)min(head0 + g, a.heads - 1) * a.buckets : nullptr;
    const int skip = lo - ns;
    // entry of the u-th visible one; beyond the last: the last (its weight is set to 0)
    auto entry = [&](int u) { u = min(u, n - 1); return u < ns ? u : u + skip; };

    for (int tile = worker; tile < tiles; tile += workers) {
      const int u0 = tile * T::TK;
      Words<T::KW> kw[T::NT];
      Words<(T::VB + 3) / 4> vw[T::TK / 4];
#pragma unroll
      for (int j = 0; j < T::NT; ++j) kw[j] = load_words<T::KW>(kp + (int64_t)entry(u0 + 8 * j + g) * a.k_code_stride);
      uint32_t scales;
      int bucket = 0;
      {
        const int e = entry(u0 + (lane & (T::TK - 1)));
        scales = __ldg(reinterpret_cast<const uint16_t*>(ksp + (int64_t)e * a.k_scale_stride)) |
                 (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(vsp + (int64_t)e * a.v_scale_stride)) << 16;
        if (bias) bucket = bucket_of(s_bounds, a.buckets - 1, t_root - __ldg(a.ts + first + e));
      }
#pragma unroll
      for (int i = 0; i < T::TK / 4; ++i)            // pieces 4 t + {0, 1, 2, 3}: keys 16 t + 2 c + {0, 1, 8, 9}
        vw[i] = load_piece<T::VB>(vp + (int64_t)entry(u0 + 16 * (i >> 2) + 2 * c + (i & 1) + 8 * ((i >> 1) & 1)) * a.v_code_stride);

      // logits
      float s[T::NT][2];
#pragma unroll
      for (int j = 0; j < T::NT; ++j) {
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < T::KW; ++w) {
          if constexpr (BITS == 4) {
            uint32_t b[4];
            nibbles(kw[j].w[w], b);
            mma(acc, qa[2 * w], b[0], b[1]);
            mma(acc, qa[2 * w + 1], b[2], b[3]);
          } else {
            const __half2 off = u2h(0x64806480u);    // 1152: a byte under the exponent of 1024, minus the offset of 128
            const uint32_t b0 = h2u(__hsub2(u2h(__byte_perm(kw[j].w[w], 0x64646464u, 0x4140)), off));
            const uint32_t b1 = h2u(__hsub2(u2h(__byte_perm(kw[j].w[w], 0x64646464u, 0x4342)), off));
            mma(acc, qa[w], b0, b1);
          }
        }
        s[j][0] = fmaf(acc[2], 1.f / kLo, acc[0]);
        s[j][1] = fmaf(acc[3], 1.f / kLo, acc[1]);
      }
      float vs[T::NT][2], top = m;
#pragma unroll
      for (int j = 0; j < T::NT; ++j) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int key = 8 * j + 2 * c + e;
          const uint32_t two = __shfl_sync(FULL, scales, key);
          vs[j][e] = __uint_as_float(two & 0xffff0000u);
          float x = s[j][e] * (qfac * __uint_as_float(two << 16));
          if (bias) x += __ldg(bias + __shfl_sync(FULL, bucket, key));
          s[j][e] = u0 + key < n ? x : -INFINITY;
          top = fmaxf(top, s[j][e]);
        }
      }
      top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
      top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
      const float base = top == -INFINITY ? 0.f : top;               // nothing but -infinity so far: weights are 0
      const float corr = exp2_fast((m - base) * kLog2e);                  // m = -infinity: 0
      m = top;
      float wmax = 0.f, sum = 0.f;
#pragma unroll
      for (int j = 0; j < T::NT; ++j) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float p = exp2_fast((s[j][e] - base) * kLog2e);
          sum += p;
          const float w = u0 + 8 * j + 2 * c + e < n ? p * vs[j][e] : 0.f;
          s[j][e] = w;
          wmax = fmaxf(wmax, w);
        }
      }
      l = fmaf(l, corr, sum);
      wmax = fmaxf(wmax, __shfl_xor_sync(FULL, wmax, 1));
      wmax = fmaxf(wmax, __shfl_xor_sync(FULL, wmax, 2));
      // a larger maximum m shrinks the unit of the sums, not the sums; they are rescaled where a weight passes the unit
      const float old = sc * corr;
      const float need = __uint_as_float(min(max((__float_as_uint(wmax) >> 23) + 1u, 2u), 252u) << 23);   // 2^e > wmax
      const bool grow = need > old;
      sc = grow ? need : old;
      const float inv = __frcp_rn(sc);
      if (__any_sync(FULL, grow)) {
        const float f = grow ? old * inv : 1.f;
#pragma unroll
        for (int i = 0; i < T::VD; ++i) { o[i][0] *= f; o[i][1] *= f; o[i][2] *= f; o[i][3] *= f; }
      }
      // output: 16 keys at a time
#pragma unroll
      for (int t = 0; t < T::TK / 16; ++t) {
        uint32_t pa[4];
        split2(s[2 * t][0] * inv, s[2 * t][1] * inv, &pa[0], &pa[1]);
        split2(s[2 * t + 1][0] * inv, s[2 * t + 1][1] * inv, &pa[2], &pa[3]);
        const auto &v0 = vw[4 * t], &v1 = vw[4 * t + 1], &v2 = vw[4 * t + 2], &v3 = vw[4 * t + 3];
        if constexpr (BITS == 4) {
#pragma unroll
          for (int h = 0; h < T::VD / 4; ++h) {                      // four columns of two keys share a word
            uint32_t b0[4], b1[4];
            nibbles(__byte_perm(v0.w[h >> 1], v1.w[h >> 1], (h & 1) ? 0x7632 : 0x5410), b0);
            nibbles(__byte_perm(v2.w[h >> 1], v3.w[h >> 1], (h & 1) ? 0x7632 : 0x5410), b1);
#pragma unroll
            for (int j = 0; j < 4; ++j) mma(o[4 * h + j], pa, b0[j], b1[j]);
          }
        } else {
          const __half2 off = u2h(0x64806480u);
#pragma unroll
          for (int i = 0; i < T::VD; ++i) {
            const uint32_t sel = (uint32_t)(i & 3) | (uint32_t)(4 + (i & 3)) << 8;     // byte i of both words, to bytes 0 and 2
            const uint32_t x0 = __byte_perm(v0.w[i >> 2], v1.w[i >> 2], sel), x1 = __byte_perm(v2.w[i >> 2], v3.w[i >> 2], sel);
            mma(o[i], pa, h2u(__hsub2(u2h(and_or(x0, 0x00ff00ffu, 0x64006400u)), off)),
                h2u(__hsub2(u2h(and_or(x1, 0x00ff00ffu, 0x64006400u)), off)));
          }
        }
      }
    }
    l += __shfl_xor_sync(FULL, l, 1);
    l += __shfl_xor_sync(FULL, l, 2);
  }
};

// BY_BLOCK false: a warp per unit.  true: all warps of a cluster (of one block or more) work on one unit.
template <int BITS, int DP, bool BY_BLOCK>
__global__ void __launch_bounds__(32 * WARPS) cached_attend_kernel(const AttendArgs a) {
  using T = Tile<BITS, DP>;
  __shared__ double s_bounds[kMaxBuckets];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
  if (a.bias) {
    for (int i = threadIdx.x; i < a.buckets - 1; i += 32 * WARPS) s_bounds[i] = a.bounds[i];
    __syncthreads();
  }
  int ranks = 1, rank = 0;
  if (BY_BLOCK) {
    ranks = (int)cg::this_cluster().num_blocks();
    rank = (int)cg::this_cluster().block_rank();
  }
  const uint32_t unit = BY_BLOCK ? blockIdx.x / (uint32_t)ranks : blockIdx.x * WARPS + wid;
  if (unit >= a.units) return;                                      // (by warp: no barrier follows; by block: the grid fits)
  const uint32_t pass = unit % (uint32_t)a.passes, rest = unit / (uint32_t)a.passes;
  const int kv = (int)(rest % (uint32_t)a.kv_heads);
  const int64_t root = rest / (uint32_t)a.kv_heads;
  const int head0 = kv * a.group + (int)pass * GH;
  const int nh = min(GH, (kv + 1) * a.group - head0);
  const int64_t first = a.first[root];
  int len = a.len[root];
  if (first < 0 || len < 0 || first > a.rows - len) {
    if (lane == 0) atomicMax(a.status, 4);
    len = 0;
  }
  const int lo = len > a.window ? len - a.window : 0;
  const int ns = min(a.sinks, lo);
  const int n = len - lo + ns;
  Walk<BITS, DP> w;
  w.run(a, s_bounds, root, kv, head0, first, lo, ns, n, BY_BLOCK ? rank * WARPS + wid : 0, BY_BLOCK ? ranks * WARPS : 1);

  if constexpr (!BY_BLOCK) {
    const float f = w.l == 0.f ? 0.f : w.sc / w.l;                   // nothing seen, or nothing but -infinity: zeros
    const int64_t base = (root * a.heads + head0 + g) * a.dim;
    if (g < nh) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < T::VD; ++i) {
          const int e = (2 * c + h) * T::VD + i;
          if (e < a.dim) store_out(a.out, a.dtype, base + e, fmaf(w.o[i][2 + h], 1.f / kLo, w.o[i][h]) * f);
        }
      }
    }
  } else {
    __shared__ float s_o[WARPS][GH][DP + 4], s_m[WARPS][GH], s_l[WARPS][GH], b_m[GH], b_l[GH];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < T::VD; ++i) s_o[wid][g][(2 * c + h) * T::VD + i] = fmaf(w.o[i][2 + h], 1.f / kLo, w.o[i][h]) * w.sc;
    }
    if (c == 0) { s_m[wid][g] = w.m; s_l[wid][g] = w.l; }
    __syncthreads();
    // the block's sums, at the block's maximum
    for (int i = threadIdx.x; i < nh * DP; i += 32 * WARPS) {
      const int h = i / DP, e = i - h * DP;
      float top = -INFINITY;
#pragma unroll
      for (int x = 0; x < WARPS; ++x) top = fmaxf(top, s_m[x][h]);
      const float base = top == -INFINITY ? 0.f : top;
      float o = 0.f, l = 0.f;
#pragma unroll
      for (int x = 0; x < WARPS; ++x) {
        const float f = exp2_fast((s_m[x][h] - base) * kLog2e);
        o = fmaf(s_o[x][h][e], f, o);
        l = fmaf(s_l[x][h], f, l);
      }
      if (ranks == 1) {
        if (e < a.dim) store_out(a.out, a.dtype, (root * a.heads + head0 + h) * a.dim + e, l == 0.f ? 0.f : o / l);
      } else {
        s_o[0][h][e] = o;                                            // this thread alone reads and writes column e of head h
        if (e == 0) { b_m[h] = top; b_l[h] = l; }
      }
    }
    if (ranks == 1) return;
    cg::cluster_group cl = cg::this_cluster();
    cl.sync();
    // every block finishes a part of the columns from all blocks' sums, in the order of their ranks
    for (int i = rank * (32 * WARPS) + threadIdx.x; i < nh * DP; i += ranks * (32 * WARPS)) {
      const int h = i / DP, e = i - h * DP;
      if (e >= a.dim) continue;
      float top = -INFINITY;
      for (int r = 0; r < ranks; ++r) top = fmaxf(top, *cl.map_shared_rank(&b_m[h], r));
      const float base = top == -INFINITY ? 0.f : top;
      float o = 0.f, l = 0.f;
      for (int r = 0; r < ranks; ++r) {
        const float f = exp2_fast((*cl.map_shared_rank(&b_m[h], r) - base) * kLog2e);
        o = fmaf(*cl.map_shared_rank(&s_o[0][h][e], r), f, o);
        l = fmaf(*cl.map_shared_rank(&b_l[h], r), f, l);
      }
      store_out(a.out, a.dtype, (root * a.heads + head0 + h) * a.dim + e, l == 0.f ? 0.f : o / l);
    }
    cl.sync();                                                       // no block leaves while its memory is read
  }
}

// Warps on one unit: by warp, unless the units leave most of the machine's warps without work and a unit has more tiles than
// a warp should walk alone.
struct Shape {
  bool by_block;
  int ranks;
};
Shape choose(int64_t units, int64_t tiles) {
  Shape s = {false, 1};
  const int64_t machine = (int64_t)num_sms() * 12;                   // warps that are resident together
  if (tiles <= 2 || units >= 2 * machine) return s;
  s.by_block = true;
  while (s.ranks < 8 && units * WARPS * s.ranks * 2 <= machine && tiles >= 2 * WARPS * s.ranks * 2) s.ranks *= 2;
  return s;
}

template <int BITS, int DP>
cudaError_t launch(const AttendArgs& a, const Shape& sh, cudaStream_t s) {
  if (!sh.by_block) {
    cached_attend_kernel<BITS, DP, false><<<(a.units + WARPS - 1) / WARPS, 32 * WARPS, 0, s>>>(a);
    return cudaGetLastError();
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.units * (unsigned)sh.ranks);
  cfg.blockDim = dim3(32 * WARPS);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)sh.ranks;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, cached_attend_kernel<BITS, DP, true>, a);
}

template <int BITS>
cudaError_t launch_dim(const AttendArgs& a, const Shape& sh, cudaStream_t s) {
  switch (padded_dim(a.dim)) {
    case 32: return launch<BITS, 32>(a, sh, s);
    case 64: return launch<BITS, 64>(a, sh, s);
    default: return launch<BITS, 128>(a, sh, s);
  }
}

}  // namespace

extern "C" int tgnn_cached_attend(const void* q, int dtype, const tgnn_cache* k_host, const tgnn_cache* v_host, int64_t n, int heads,
                                  const int64_t* first, const int32_t* len, const float* bias, int num_buckets, const double* bounds,
                                  const double* times, const double* ts, int window, int sinks, int max_len, float scale, void* out,
                                  int32_t* status, void* stream, char* err_host, int64_t err_size) {
  const char* who = "tgnn_cached_attend";
  CacheView k, v;
  int rc = check_cache(who, "k", k_host, &k, err_host, err_size);
  if (!rc) rc = check_cache(who, "v", v_host, &v, err_host, err_size);
  if (rc) return rc;
  if (k.rows != v.rows || k.heads != v.heads || k.dim != v.dim || k.bits != v.bits)
    return fail(err_host, err_size, TGNN_ESHAPE, "%s: k and v differ in rows, heads, dim or bits", who);
  if (!known_dtype(dtype)) return fail(err_host, err_size, TGNN_EINVAL, "%s: unknown type %d", who, dtype);
  if (n < 0 || window < 0 || sinks < 0 || (int64_t)window + sinks < 1 || max_len < 0)
    return fail(err_host, err_size, TGNN_EINVAL, "%s: size out of range (window and sinks see one entry at least)", who);
  if (heads < 1 || heads > 1024 || heads % k.heads)
    return fail(err_host, err_size, TGNN_EINVAL, "%s: %d heads over %d cached ones", who, heads, k.heads);
  if (!status || (n > 0 && (!q || !out || !first || !len))) return fail(err_host, err_size, TGNN_EINVAL, "%s: null pointer", who);
  if (bias && (num_buckets < 1 || num_buckets > kMaxBuckets))
    return fail(err_host, err_size, TGNN_EINVAL, "%s: %d buckets (1 to %d)", who, num_buckets, kMaxBuckets);
  if (bias && n > 0 && ((num_buckets > 1 && !bounds) || !times || (k.rows > 0 && !ts)))
    return fail(err_host, err_size, TGNN_EINVAL, "%s: a bias needs bounds, times and ts", who);
  const int es = elem_bytes(dtype) - 1;
  if ((((uintptr_t)q | (uintptr_t)out) & es) || (((uintptr_t)first | (uintptr_t)bounds | (uintptr_t)times | (uintptr_t)ts) & 7) ||
      (((uintptr_t)len | (uintptr_t)bias | (uintptr_t)status) & 3))
    return fail(err_host, err_size, TGNN_EINVAL, "%s: a pointer is not aligned to its element", who);
  AttendArgs a = {};
  a.group = heads / k.heads;
  a.passes = (a.group + GH - 1) / GH;
  if (n > 0x0fffffff / ((int64_t)k.heads * a.passes)) return fail(err_host, err_size, TGNN_ECAPACITY, "%s: n * heads above 2^28", who);
  if (n == 0) return TGNN_OK;
  a.q = q;
  a.out = out;
  a.dtype = dtype;
  a.k_codes = k.codes;
  a.v_codes = v.codes;
  a.k_scales = k.scales;
  a.v_scales = v.scales;
  a.k_code_stride = (int)k.code_stride;
  a.v_code_stride = (int)v.code_stride;
  a.k_scale_stride = (int)k.scale_stride;
  a.v_scale_stride = (int)v.scale_stride;
  a.rows = k.rows;
  a.heads = heads;
  a.kv_heads = k.heads;
  a.dim = k.dim;
  a.units = (uint32_t)(n * k.heads * a.passes);
  a.first = first;
  a.len = len;
  a.bias = bias;
  a.bounds = bounds;
  a.times = times;
  a.ts = ts;
  a.buckets = num_buckets;
  a.window = window;
  a.sinks = sinks;
  a.scale = scale;
  a.status = status;
  int64_t see = (int64_t)window + sinks;
  if (max_len > 0 && max_len < see) see = max_len;
  if (k.rows < see) see = k.rows;
  const int tk = k.bits == 8 && padded_dim(k.dim) == 128 ? 16 : 32;
  const Shape sh = choose(a.units, (see + tk - 1) / tk);
  const cudaError_t e = k.bits == 4 ? launch_dim<4>(a, sh, (cudaStream_t)stream) : launch_dim<8>(a, sh, (cudaStream_t)stream);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return fail(err_host, err_size, TGNN_ECUDA, "%s: %s", who, cudaGetErrorString(e));
  }
  return TGNN_OK;
}
