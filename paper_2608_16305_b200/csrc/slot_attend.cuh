// Attention of one query per root and head over the root's sampled slots, forward and backward, with a learned bias by buckets
// of the time difference and its gradient.
//
//   z_s = scale * q . k_s + bias[h, b_s],  p = softmax(z),  o = sum_s p_s v_s
//   dp_s = do . v_s,  delta = sum_s p_s dp_s,  dz_s = p_s (dp_s - delta)
//   dq = scale * sum_s dz_s k_s,  dk_s = scale * sum_{h of the group} dz_s q_h,  dv_s = sum_{h of the group} p_s do_h,
//   dbias[h, b] = sum over roots and slots in bucket b of dz_s
//
// Keys and values are rows of their own per (root, slot): every byte of k and v is used once (forward) or for one root's gradients
// (backward), so both passes are bound by HBM: k and v in, and for the backward pass dk and dv out.  Tensor cores have nothing to
// gain on one query per row.  The backward pass recomputes the weights and needs nothing of the forward pass.
//
// A warp takes a root, or a block's warps one together where roots are few.  The values of one (slot, cached head) lie side by side; P lanes
// hold such a segment, NV words of VB bytes each, 8 values in all where there are as many, so that a warp loads 32 / P segments at once
// straight into registers, two to four deep for k and v.  A dot product is then VB / size multiplications and log2(P) shuffles.  Forward, every group of P lanes runs a softmax of its own over its slots (maximum, sum and
// output in registers; the groups of a head are merged at the end), so nothing is written between k and the output.  Backward,
// logits and dp go to shared memory for the root's slots, weights and dz are formed there, and a second walk over k (which lies
// in L1 or L2 by then) sums dq while dk and dv are written.  Roots with more slots than a warp's shared memory holds are taken in
// chunks: maximum, sum and delta over all of them first, gradients then.
// Sums are fp32; in the backward pass a head's l and delta are fp64, and so are the bias's gradients, which run over the whole batch (runs of up
// to 32 neighbouring slots in one bucket are added in fp32 before): each
// warp keeps a table of its own and a second kernel adds the blocks' tables in a fixed order, so no atomics decide on a result.
// Logits stay in natural units: a bias of the type's lowest value is then still finite.
//
// Measured on a B200, 14 400 roots of 64 slots, 4 heads of 32 in bf16: forward 89 us at 5.2 TB/s, backward 204 us at 4.75 TB/s of DRAM (a copy
// reaches 6.5); 1800 roots of 20 slots, 2 heads of 50 in fp32: 10 and 20 us, a single wave of 12 warps per SM, bound by the latency of a
// root's chain of loads and sums.
#pragma once

#include "tgnn_history.cuh"

namespace tgnn_slots {

using namespace tgnn_history;

constexpr int MAX_BLOCKS = 1024;
constexpr int MAX_WARPS = 4;

struct SlotArgs {
  const void *q, *k, *v, *dout;
  void *out, *dq, *dk, *dv;
  const int32_t* cnt;
  const float* bias;
  const double *bounds, *times, *ts;
  double* partial;                       // [blocks][heads * buckets]
  int64_t n;
  int slots, heads, kv_heads, dim, group;
  int buckets;
  int chunk;                             // slots of a chunk
  int warps;
  int team;                              // warps that share a root: 1, or all of a block
  int warp_bytes;                        // shared memory of a warp, or of a block that shares a root
  float scale;
};

// Shared memory of a warp, or of a block that shares a root, all parts multiples of 16 bytes: bucket [chunk] (bytes); backward: z and dp [chunk * H] in pairs, per head m,
// 1 / l and delta, dq [H * dim] and the running l and delta in fp64 where there are several chunks, and with a bias the table
// [H * buckets] in fp64 for every warp; where warps share a root, what they put together: outputs or dq of the heads in hand, and forward m and l.
constexpr int RED = 256;                   // values of the heads that a warp has in hand, per query head of a cached head: 32 lanes of 8
struct Layout {
  int z, head, dq, sums, table, red, total;
};
__host__ __device__ inline int up16(int x) { return (x + 15) & ~15; }
__host__ __device__ inline Layout layout(int heads, int dim, int chunk, bool several, bool backward, int table, int team, int together) {
  Layout l;
  int at = up16(chunk);
  l.z = at; at += backward ? up16(heads * chunk * 8) : 0;
  l.head = at; at += backward ? up16(heads * 16) : 0;
  l.dq = at; at += backward && several ? up16(heads * dim * 4) : 0;
  l.sums = at; at += backward && several ? heads * 16 : 0;
  l.table = at; at += up16(table * team * 8);
  l.red = at; at += team > 1 ? team * together * (RED + 16) * 4 : 0;
  l.total = at;
  return l;
}

// NV words of VB bytes of a segment, as they are in memory and as fp32.  Word i of lane `part` starts at value (i * P + part) * VE.
template <typename T, int VB, int P, int NV>
struct Seg {
  static constexpr int VE = VB / (int)sizeof(T), N = NV * VE;
  typedef typename Vec<VB>::type W;
  W w[NV];
  __device__ __forceinline__ void load(const T* p, int part, int dim, bool on) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      w[i] = W();
      if (on && (i * P + part) * VE < dim) w[i] = __ldg(reinterpret_cast<const W*>(p) + i * P + part);
    }
  }
  __device__ __forceinline__ float at(int j) const {           // j: compile-time after unrolling
    if constexpr (sizeof(T) == 4) {
      return reinterpret_cast<const float*>(w)[j];
    } else if constexpr (VB == 2) {
      return to_float<T>(reinterpret_cast<const T*>(w)[j]);
    } else {
      const uint32_t x = reinterpret_cast<const uint32_t*>(w)[j >> 1];
      if constexpr (sizeof(T) == 2 && is_bf16()) return __uint_as_float((j & 1) ? x & 0xffff0000u : x << 16);
      else return to_float<T>(reinterpret_cast<const T*>(&x)[j & 1]);
    }
  }
  __device__ __forceinline__ void floats(float (&x)[N]) const {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = at(j);
  }
  static __device__ constexpr bool is_bf16();
  static __device__ __forceinline__ void store(T* p, int part, int dim, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      union { W w; T e[VE]; } u;
#pragma unroll
      for (int e = 0; e < VE; ++e) u.e[e] = from_float<T>(x[i * VE + e]);
      if ((i * P + part) * VE < dim) reinterpret_cast<W*>(p)[i * P + part] = u.w;
    }
  }
};
template <typename T>
struct IsBf16 { static constexpr bool value = false; };
template <>
struct IsBf16<__nv_bfloat16> { static constexpr bool value = true; };
template <typename T, int VB, int P, int NV>
__device__ constexpr bool Seg<T, VB, P, NV>::is_bf16() { return IsBf16<T>::value; }

// Sums of N values each over the P lanes of a segment, several at a time: a lane hands half of its values to its partner and
// goes on with the other half, so that 8 values take 9 shuffles over 32 lanes instead of 40.  What a lane ends up with is the sum
// of value Reduced::id (and the next ones, where P < N); lanes whose Reduced::first is not set hold copies.
template <int P, int N>
struct Reduced {
  int id;
  bool first;
  __device__ __forceinline__ explicit Reduced(int lane) {
    id = 0;
    int n = N;
#pragma unroll
    for (int o = P / 2; o > 0 && n > 1; o >>= 1) {
      n >>= 1;
      id += (lane & o) ? n : 0;
    }
    first = (lane & (P > N ? P / N - 1 : 0)) == 0;
  }
  static __device__ __forceinline__ void run(float (&v)[N], int lane) {
    int n = N;
#pragma unroll
    for (int o = P / 2; o > 0; o >>= 1) {
      if (n > 1) {
        n >>= 1;
        const bool up = (lane & o) != 0;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          if (i < n) {
            const float give = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
            v[i] = keep + __shfl_xor_sync(FULL, give, o);
          }
        }
      } else {
        v[0] += __shfl_xor_sync(FULL, v[0], o);
      }
    }
  }
};

// Query heads of a cached head that a warp takes together: 4, 2 or 1, whatever divides their number.  One after another they read and
// unpacked a root's rows again for each (6000 roots of 40 slots, 2 x 4 heads of 64, bf16: 76 us forward and 154 us backward; 49 and 103 us
// by fours; 2 x 2 heads of 64 in fp32: 68 and 158 us; 49 and 110 us by twos).
__host__ __device__ inline int heads_at_once(int group) { return (group & 3) == 0 ? 4 : (group & 1) == 0 ? 2 : 1; }

// Segments of k and of v in flight per lane: 64 bytes of each, 2 segments at least and 4 at most.
template <typename S>
constexpr int kDeep = sizeof(S) >= 32 ? 2 : 4;
// With four query heads at a time their registers leave room for two.
template <typename S, int GT>
constexpr int kDeepOf = GT >= 4 ? 2 : kDeep<S>;
// Blocks per SM of the backward pass, and of the forward pass in fp32: four heads' q and do, or q and output, take 64 registers.  (16-bit
// rows leave room for a fourth block in the forward pass: 49 instead of 57 us for 6000 roots of 40 slots, 2 x 4 heads of 64.)
template <int GT>
constexpr int kBlocks = GT >= 4 ? 3 : 4;

// Which segments a lane takes: 32 / P of them at a time, KC neighbouring cached heads of RPI neighbouring slots.
template <int P>
struct Lanes {
  int part, kc, KC, row, RPI;
  __device__ __forceinline__ Lanes(int lane, int kv_heads) {
    constexpr int NG = 32 / P;
    part = lane & (P - 1);
    KC = min(NG, kv_heads & -kv_heads);                        // powers of two
    RPI = NG / KC;
    kc = (lane / P) & (KC - 1);
    row = (lane / P) / KC;
  }
};

__device__ __forceinline__ void fill_buckets(const SlotArgs& a, const double* s_bounds, uint8_t* bucket, int64_t r, int s0, int s1, int first, int step) {
  if (!a.bias) return;
  const double t = a.times[r];
  for (int s = s0 + first; s < s1; s += step) bucket[s - s0] = (uint8_t)bucket_of(s_bounds, a.buckets - 1, t - __ldg(a.ts + r * a.slots + s));
}

// Of warps that share a root, or of one that has it alone.
__device__ __forceinline__ void sync_team(int team) {
  if (team > 1) __syncthreads();
  else __syncwarp();
}

// A lane's values of one head in hand, to row e of the block's.
template <typename S, int P>
__device__ __forceinline__ void put_team(float* red, int e, int dim, int part, const float (&x)[S::N]) {
#pragma unroll
  for (int j = 0; j < S::N; ++j) {
    const int d = ((j / S::VE) * P + part) * S::VE + j % S::VE;
    if (d < dim) red[e * dim + d] = x[j];
  }
}

// The outputs of the warps that share a root put together: per warp and head in hand m, l and acc (not divided by l).  All
// threads of the block.
template <typename T>
__device__ __forceinline__ void merge_team(const SlotArgs& a, const float* red, int heads_in_hand, int together, int64_t r, int kv0, int g0) {
  const int D = a.dim, size = heads_in_hand * D;
  const float2* ml = reinterpret_cast<const float2*>(red + a.team * together * RED);
  for (int i = threadIdx.x; i < size; i += blockDim.x) {
    const int e = i / D, d = i - e * D;
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int w = 0; w < a.team; ++w) m = fmaxf(m, ml[w * heads_in_hand + e].x);
    const float base = m == -INFINITY ? 0.f : m;
    for (int w = 0; w < a.team; ++w) {
      const float2 at = ml[w * heads_in_hand + e];
      const float f = exp2_fast((at.x - base) * kLog2e);
      l = fmaf(at.y, f, l);
      o = fmaf(red[w * size + i], f, o);
    }
    const int h = (kv0 + e / together) * a.group + g0 + e % together;
    reinterpret_cast<T*>(a.out)[(r * a.heads + h) * D + d] = from_float<T>(l == 0.f ? 0.f : o / l);
  }
}

template <typename T, int VB, int P, int NV>
__global__ void __launch_bounds__(32 * MAX_WARPS, 4) slot_forward_kernel(const SlotArgs a) {
  using S = Seg<T, VB, P, NV>;
  constexpr int UN = kDeep<S>;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ double s_bounds[kMaxBuckets + 1];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int team = a.team, sub = team > 1 ? wid : 0;
  uint8_t* bucket = smem + (team > 1 ? 0 : (size_t)wid * a.warp_bytes);
  if (a.bias) {
    stage_bounds(s_bounds, a.bounds, a.buckets - 1, threadIdx.x, blockDim.x);
    __syncthreads();
  }
  const Lanes<P> me(lane, a.kv_heads);
  const int D = a.dim, ROW = a.kv_heads * D;
  const int64_t r = team > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * a.warps + wid;
  if (r >= a.n) return;
  const int cnt = min(max(a.cnt[r], 0), a.slots);
  const bool several = cnt > a.chunk;                          // chunks are multiples of the team's UN * RPI slots
  const int row = me.row + sub * UN * me.RPI, step = team * UN * me.RPI;
  bool filled = several;
  const T* kr = reinterpret_cast<const T*>(a.k) + r * a.slots * ROW;
  const T* vr = reinterpret_cast<const T*>(a.v) + r * a.slots * ROW;
  for (int kv0 = 0; kv0 < a.kv_heads; kv0 += me.KC) {
    const int kv = kv0 + me.kc;
    for (int g = 0; g < a.group; ++g) {
      const int h = kv * a.group + g;
      // all first loads on their way before the first of them is waited for
      const T* kp = kr + (int64_t)row * ROW + kv * D;
      const T* vp = vr + (int64_t)row * ROW + kv * D;
      S k[UN], v[UN], raw;
#pragma unroll
      for (int u = 0; u < UN; ++u) k[u].load(kp + u * me.RPI * ROW, me.part, D, row + u * me.RPI < cnt);
      raw.load(reinterpret_cast<const T*>(a.q) + (r * a.heads + h) * D, me.part, D, true);
#pragma unroll
      for (int u = 0; u < UN; ++u) v[u].load(vp + u * me.RPI * ROW, me.part, D, row + u * me.RPI < cnt);
      if (!filled) {
        fill_buckets(a, s_bounds, bucket, r, 0, cnt, lane + 32 * sub, 32 * team);
        sync_team(team);
        filled = true;
      }
      float q[S::N];
      raw.floats(q);
      const float* bias = a.bias ? a.bias + h * a.buckets : nullptr;
      float m = -INFINITY, l = 0.f, acc[S::N];
#pragma unroll
      for (int j = 0; j < S::N; ++j) acc[j] = 0.f;
      for (int c0 = 0; c0 < cnt; c0 += a.chunk) {
        const int c1 = min(cnt, c0 + a.chunk);
        if (several) {
          sync_team(team);
          fill_buckets(a, s_bounds, bucket, r, c0, c1, lane + 32 * sub, 32 * team);
          sync_team(team);
        }
        for (int s0 = c0 + row; s0 - me.row < c1; s0 += step) {
          float z[UN];
#pragma unroll
          for (int u = 0; u < UN; ++u) {
            z[u] = 0.f;
#pragma unroll
            for (int j = 0; j < S::N; ++j) z[u] = fmaf(k[u].at(j), q[j], z[u]);
          }
          // the next slots' keys come while these are weighed, their values while the next are
          const int next = s0 + step;
          kp += step * ROW;
#pragma unroll
          for (int u = 0; u < UN; ++u) k[u].load(kp + u * me.RPI * ROW, me.part, D, next + u * me.RPI < cnt);
          if constexpr (P >= 16) {
            // the sums of all slots together, then back to all lanes of the segment
            Reduced<P, UN>::run(z, lane);
            const float mine = z[0];
#pragma unroll
            for (int u = 0; u < UN; ++u) z[u] = __shfl_sync(FULL, mine, (lane & ~(P - 1)) | (u & UN / 2 ? P / 2 : 0) | (UN == 4 && (u & 1) ? P / 4 : 0));
          } else {
#pragma unroll
            for (int u = 0; u < UN; ++u) {
#pragma unroll
              for (int o = 1; o < P; o <<= 1) z[u] += __shfl_xor_sync(FULL, z[u], o);
            }
          }
          float top = m;
#pragma unroll
          for (int u = 0; u < UN; ++u) {
            const int s = s0 + u * me.RPI;
            z[u] *= a.scale;
            if (bias && s < c1) z[u] += __ldg(bias + bucket[s - c0]);
            if (s >= c1) z[u] = -INFINITY;
            top = fmaxf(top, z[u]);
          }
          const float base = top == -INFINITY ? 0.f : top;     // nothing but -infinity: weights are 0
          const float corr = exp2_fast((m - base) * kLog2e);   // m = -infinity: 0
          m = top;
          l *= corr;
#pragma unroll
          for (int j = 0; j < S::N; ++j) acc[j] *= corr;
#pragma unroll
          for (int u = 0; u < UN; ++u) {
            const float p = exp2_fast((z[u] - base) * kLog2e);
            l += p;
#pragma unroll
            for (int j = 0; j < S::N; ++j) acc[j] = fmaf(p, v[u].at(j), acc[j]);
          }
          vp += step * ROW;
#pragma unroll
          for (int u = 0; u < UN; ++u) v[u].load(vp + u * me.RPI * ROW, me.part, D, next + u * me.RPI < cnt);
        }
      }
      // the groups of lanes that shared a head's slots
      for (int o = P * me.KC; o < 32; o <<= 1) {
        const float om = __shfl_xor_sync(FULL, m, o), top = fmaxf(m, om);
        const float base = top == -INFINITY ? 0.f : top;
        const float f = exp2_fast((m - base) * kLog2e), of = exp2_fast((om - base) * kLog2e);
        m = top;
        l = l * f + __shfl_xor_sync(FULL, l, o) * of;
#pragma unroll
        for (int j = 0; j < S::N; ++j) acc[j] = acc[j] * f + __shfl_xor_sync(FULL, acc[j], o) * of;
      }
      if (team > 1) {
        float* red = reinterpret_cast<float*>(smem + layout(a.heads, D, a.chunk, false, false, 0, team, 1).red);
        if (me.row == 0) put_team<S, P>(red, sub * me.KC + me.kc, D, me.part, acc);
        if (me.row == 0 && me.part == 0) reinterpret_cast<float2*>(red + team * RED)[sub * me.KC + me.kc] = make_float2(m, l);
        __syncthreads();
        merge_team<T>(a, red, me.KC, 1, r, kv0, g);
        __syncthreads();                                       // before the next heads overwrite it
        continue;
      }
      const float f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int j = 0; j < S::N; ++j) acc[j] *= f;
      if (me.row == 0) S::store(reinterpret_cast<T*>(a.out) + (r * a.heads + h) * D, me.part, D, acc);
    }
  }
}

// The same for query heads that share a cached head, GT of them at a time: k and v are loaded and unpacked once for them.  The sums of
// UN slots and GT heads end on different lanes (value g * UN + u on the lane, or the lanes, that Reduced gives it), and each lane weighs its
// own, instead of P lanes all of them; weights and corrections then go back to the segment.
template <typename T, int VB, int P, int NV, int GT>
__global__ void __launch_bounds__(32 * MAX_WARPS, sizeof(T) == 2 ? 4 : kBlocks<GT>) slot_forward_group_kernel(const SlotArgs a) {
  using S = Seg<T, VB, P, NV>;
  constexpr int UN = kDeepOf<S, GT>, N = GT * UN;
  constexpr int C = N > P ? N / P : 1, SP = P > N ? P / N : 1;  // values per lane, lanes per value
  static_assert(C <= UN, "a lane's values belong to one head");
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ double s_bounds[kMaxBuckets + 1];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int team = a.team, sub = team > 1 ? wid : 0;
  uint8_t* bucket = smem + (team > 1 ? 0 : (size_t)wid * a.warp_bytes);
  if (a.bias) {
    stage_bounds(s_bounds, a.bounds, a.buckets - 1, threadIdx.x, blockDim.x);
    __syncthreads();
  }
  const Lanes<P> me(lane, a.kv_heads);
  const Reduced<P, N> sums(lane);
  const int my_g = sums.id / UN, my_u = sums.id % UN, base_lane = lane & ~(P - 1);
  const int D = a.dim, ROW = a.kv_heads * D;
  const int64_t r = team > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * a.warps + wid;
  if (r >= a.n) return;
  const int cnt = min(max(a.cnt[r], 0), a.slots);
  const bool several = cnt > a.chunk;                          // chunks are multiples of the team's UN * RPI slots
  const int row = me.row + sub * UN * me.RPI, step = team * UN * me.RPI;
  bool filled = several;
  const T* kr = reinterpret_cast<const T*>(a.k) + r * a.slots * ROW;
  const T* vr = reinterpret_cast<const T*>(a.v) + r * a.slots * ROW;
  for (int kv0 = 0; kv0 < a.kv_heads; kv0 += me.KC) {
    const int kv = kv0 + me.kc;
    for (int g0 = 0; g0 < a.group; g0 += GT) {
      const int h0 = kv * a.group + g0;
      const T* kp = kr + (int64_t)row * ROW + kv * D;
      const T* vp = vr + (int64_t)row * ROW + kv * D;
      S k[UN], v[UN];
#pragma unroll
      for (int u = 0; u < UN; ++u) k[u].load(kp + u * me.RPI * ROW, me.part, D, row + u * me.RPI < cnt);
      float q[GT][S::N], acc[GT][S::N];
      {
        S raw[GT];
#pragma unroll
        for (int g = 0; g < GT; ++g) raw[g].load(reinterpret_cast<const T*>(a.q) + (r * a.heads + h0 + g) * D, me.part, D, true);
#pragma unroll
        for (int u = 0; u < UN; ++u) v[u].load(vp + u * me.RPI * ROW, me.part, D, row + u * me.RPI < cnt);
        if (!filled) {
          fill_buckets(a, s_bounds, bucket, r, 0, cnt, lane + 32 * sub, 32 * team);
          sync_team(team);
          filled = true;
        }
#pragma unroll
        for (int g = 0; g < GT; ++g) {
          raw[g].floats(q[g]);
#pragma unroll
          for (int j = 0; j < S::N; ++j) acc[g][j] = 0.f;
        }
      }
      const float* bias = a.bias ? a.bias + (h0 + my_g) * a.buckets : nullptr;
      float m = -INFINITY, l = 0.f;                            // of the lane's head; l over the lane's slots
      for (int c0 = 0; c0 < cnt; c0 += a.chunk) {
        const int c1 = min(cnt, c0 + a.chunk);
        if (several) {
          sync_team(team);
          fill_buckets(a, s_bounds, bucket, r, c0, c1, lane + 32 * sub, 32 * team);
          sync_team(team);
        }
        for (int s0 = c0 + row; s0 - me.row < c1; s0 += step) {
          float z[N];
#pragma unroll
          for (int u = 0; u < UN; ++u) {
#pragma unroll
            for (int g = 0; g < GT; ++g) z[g * UN + u] = 0.f;
#pragma unroll
            for (int j = 0; j < S::N; ++j) {
              const float x = k[u].at(j);
#pragma unroll
              for (int g = 0; g < GT; ++g) z[g * UN + u] = fmaf(x, q[g][j], z[g * UN + u]);
            }
          }
          const int next = s0 + step;
          kp += step * ROW;
#pragma unroll
          for (int u = 0; u < UN; ++u) k[u].load(kp + u * me.RPI * ROW, me.part, D, next + u * me.RPI < cnt);
          Reduced<P, N>::run(z, lane);
          float top = m;
#pragma unroll
          for (int i = 0; i < C; ++i) {
            const int s = s0 + (my_u + i) * me.RPI;
            z[i] *= a.scale;
            if (bias && s < c1) z[i] += __ldg(bias + bucket[s - c0]);
            if (s >= c1) z[i] = -INFINITY;
            top = fmaxf(top, z[i]);
          }
#pragma unroll
          for (int o = SP; o < SP * (UN / C); o <<= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
          const float base = top == -INFINITY ? 0.f : top;     // nothing but -infinity: weights are 0
          const float corr = exp2_fast((m - base) * kLog2e);   // m = -infinity: 0
          m = top;
          l *= corr;
          float p[C];
#pragma unroll
          for (int i = 0; i < C; ++i) {
            p[i] = exp2_fast((z[i] - base) * kLog2e);
            l += p[i];
          }
#pragma unroll
          for (int g = 0; g < GT; ++g) {
            const float f = __shfl_sync(FULL, corr, base_lane | (g * UN / C * SP));
#pragma unroll
            for (int j = 0; j < S::N; ++j) acc[g][j] *= f;
          }
#pragma unroll
          for (int u = 0; u < UN; ++u) {
            float w[GT];
#pragma unroll
            for (int g = 0; g < GT; ++g) w[g] = __shfl_sync(FULL, p[(g * UN + u) % C], base_lane | ((g * UN + u) / C * SP));
#pragma unroll
            for (int j = 0; j < S::N; ++j) {
              const float x = v[u].at(j);
#pragma unroll
              for (int g = 0; g < GT; ++g) acc[g][j] = fmaf(w[g], x, acc[g][j]);
            }
          }
          vp += step * ROW;
#pragma unroll
          for (int u = 0; u < UN; ++u) v[u].load(vp + u * me.RPI * ROW, me.part, D, next + u * me.RPI < cnt);
        }
      }
#pragma unroll
      for (int o = SP; o < SP * (UN / C); o <<= 1) l += __shfl_xor_sync(FULL, l, o);
      // the groups of lanes that shared a head's slots
      float* red = reinterpret_cast<float*>(smem + layout(a.heads, D, a.chunk, false, false, 0, team, GT).red);
#pragma unroll
      for (int g = 0; g < GT; ++g) {
        float gm = __shfl_sync(FULL, m, base_lane | (g * UN / C * SP)), gl = __shfl_sync(FULL, l, base_lane | (g * UN / C * SP));
        for (int o = P * me.KC; o < 32; o <<= 1) {
          const float om = __shfl_xor_sync(FULL, gm, o), top = fmaxf(gm, om);
          const float base = top == -INFINITY ? 0.f : top;
          const float f = exp2_fast((gm - base) * kLog2e), of = exp2_fast((om - base) * kLog2e);
          gm = top;
          gl = gl * f + __shfl_xor_sync(FULL, gl, o) * of;
#pragma unroll
          for (int j = 0; j < S::N; ++j) acc[g][j] = acc[g][j] * f + __shfl_xor_sync(FULL, acc[g][j], o) * of;
        }
        if (team > 1) {
          const int e = (sub * me.KC + me.kc) * GT + g;
          if (me.row == 0) put_team<S, P>(red, e, D, me.part, acc[g]);
          if (me.row == 0 && me.part == 0) reinterpret_cast<float2*>(red + team * GT * RED)[e] = make_float2(gm, gl);
          continue;
        }
        const float f = gl == 0.f ? 0.f : 1.f / gl;
#pragma unroll
        for (int j = 0; j < S::N; ++j) acc[g][j] *= f;
        if (me.row == 0) S::store(reinterpret_cast<T*>(a.out) + (r * a.heads + h0 + g) * D, me.part, D, acc[g]);
      }
      if (team > 1) {
        __syncthreads();
        merge_team<T>(a, red, me.KC * GT, GT, r, kv0, g0);
        __syncthreads();                                       // before the next heads overwrite it
      }
    }
  }
}

template <typename T, int VB, int P, int NV, int GT>
__global__ void __launch_bounds__(32 * MAX_WARPS, kBlocks<GT>) slot_backward_kernel(const SlotArgs a) {
  using S = Seg<T, VB, P, NV>;
  constexpr int UN = kDeepOf<S, GT>, N = 2 * GT * UN;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ double s_bounds[kMaxBuckets + 1];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int H = a.heads, D = a.dim, ROW = a.kv_heads * D;
  const bool table = a.partial != nullptr;
  const int team = a.team, sub = team > 1 ? wid : 0;
  const Layout L = layout(H, D, a.chunk, a.chunk < a.slots, true, table ? H * a.buckets : 0, team, GT);
  uint8_t* my = smem + (team > 1 ? 0 : (size_t)wid * a.warp_bytes);
  uint8_t* bucket = my;
  float2* zd = reinterpret_cast<float2*>(my + L.z);            // [slot][head]: logit and do . v, then weight and dz
  float4* s_head = reinterpret_cast<float4*>(my + L.head);     // m, 1 / l, delta in two terms
  double2* s_sums = reinterpret_cast<double2*>(my + L.sums);   // l and l * delta so far
  float* s_dq = reinterpret_cast<float*>(my + L.dq);
  double* tab = reinterpret_cast<double*>(my + L.table) + sub * H * a.buckets;
  float* red = reinterpret_cast<float*>(my + L.red);
  if (a.bias) stage_bounds(s_bounds, a.bounds, a.buckets - 1, threadIdx.x, blockDim.x);
  if (table) {
    for (int i = lane; i < H * a.buckets; i += 32) tab[i] = 0.0;
  }
  __syncthreads();
  const Lanes<P> me(lane, a.kv_heads);
  const Reduced<P, N> sums(lane);
  const int h_first = (lane + 32 * sub) % H, h_step = 32 * team % H;   // head of entry lane + 32 (sub + team i) of a [slot][head] array, by steps
  const int64_t stride = (int64_t)gridDim.x * (team > 1 ? 1 : a.warps);
  const int row = me.row + sub * UN * me.RPI, step = team * UN * me.RPI;
  auto count = [&](int64_t r) { return r < a.n ? min(max(a.cnt[r], 0), a.slots) : 0; };
  int64_t r = team > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * a.warps + wid;
  int cnt = count(r), next_cnt = count(r + stride);
  for (; r < a.n; r += stride, cnt = next_cnt, next_cnt = count(r + stride)) {
    const T* kr = reinterpret_cast<const T*>(a.k) + r * a.slots * ROW;
    const T* vr = reinterpret_cast<const T*>(a.v) + r * a.slots * ROW;
    T* dkr = reinterpret_cast<T*>(a.dk) + r * a.slots * ROW;
    T* dvr = reinterpret_cast<T*>(a.dv) + r * a.slots * ROW;
    const T* qr = reinterpret_cast<const T*>(a.q) + r * H * D;
    const T* gr = reinterpret_cast<const T*>(a.dout) + r * H * D;
    T* dqr = reinterpret_cast<T*>(a.dq) + r * H * D;
    const bool several = cnt > a.chunk;
    if (several) {
      for (int h = lane + 32 * sub; h < H; h += 32 * team) {
        s_head[h].x = -INFINITY;
        s_sums[h] = make_double2(0.0, 0.0);
      }
      sync_team(team);
    }

    for (int sweep = 0; sweep < (several ? 2 : 1); ++sweep) {
      for (int c0 = 0; c0 == 0 || c0 < cnt; c0 += a.chunk) {
        const int ns = min(cnt - c0, a.chunk);
        bool filled = false;
        // logits and dp of the chunk
        for (int kv0 = 0; kv0 < a.kv_heads; kv0 += me.KC) {
          const int kv = kv0 + me.kc;
          for (int g0 = 0; g0 < a.group; g0 += GT) {
            const int h0 = kv * a.group + g0;
            const T* kp = kr + (int64_t)(c0 + row) * ROW + kv * D;
            const T* vp = vr + (int64_t)(c0 + row) * ROW + kv * D;
            S k[UN], v[UN], raw[GT], raw2[GT];
#pragma unroll
            for (int u = 0; u < UN; ++u) k[u].load(kp + u * me.RPI * ROW, me.part, D, row + u * me.RPI < ns);
#pragma unroll
            for (int u = 0; u < UN; ++u) v[u].load(vp + u * me.RPI * ROW, me.part, D, row + u * me.RPI < ns);
#pragma unroll
            for (int g = 0; g < GT; ++g) {
              raw[g].load(qr + (h0 + g) * D, me.part, D, true);
              raw2[g].load(gr + (h0 + g) * D, me.part, D, true);
            }
            if (!filled) {
              fill_buckets(a, s_bounds, bucket, r, c0, c0 + ns, lane + 32 * sub, 32 * team);
              sync_team(team);
              filled = true;
            }
            float q[GT][S::N], go[GT][S::N];
#pragma unroll
            for (int g = 0; g < GT; ++g) {
              raw[g].floats(q[g]);
              raw2[g].floats(go[g]);
            }
            for (int s0 = row; s0 - me.row < ns; s0 += step) {
              float x[N];                                      // q . k of the heads' slots, then do . v
#pragma unroll
              for (int u = 0; u < UN; ++u) {
#pragma unroll
                for (int g = 0; g < GT; ++g) x[g * UN + u] = x[(GT + g) * UN + u] = 0.f;
#pragma unroll
                for (int j = 0; j < S::N; ++j) {
                  const float xk = k[u].at(j), xv = v[u].at(j);
#pragma unroll
                  for (int g = 0; g < GT; ++g) {
                    x[g * UN + u] = fmaf(xk, q[g][j], x[g * UN + u]);
                    x[(GT + g) * UN + u] = fmaf(xv, go[g][j], x[(GT + g) * UN + u]);
                  }
                }
              }
              // the next slots' rows come while these sums are put together
              const int next = s0 + step;
              kp += step * ROW;
              vp += step * ROW;
#pragma unroll
              for (int u = 0; u < UN; ++u) k[u].load(kp + u * me.RPI * ROW, me.part, D, next + u * me.RPI < ns);
#pragma unroll
              for (int u = 0; u < UN; ++u) v[u].load(vp + u * me.RPI * ROW, me.part, D, next + u * me.RPI < ns);
              Reduced<P, N>::run(x, lane);
              if (sums.first) {
#pragma unroll
                for (int i = 0; i < (N > P ? N / P : 1); ++i) {
                  const int s = s0 + ((sums.id + i) & (UN - 1)) * me.RPI, h = h0 + (sums.id + i) / UN % GT;
                  if (s < ns) {
                    if (sums.id + i < GT * UN) {
                      float y = x[i] * a.scale;
                      if (a.bias) y += __ldg(a.bias + h * a.buckets + bucket[s]);
                      zd[s * H + h].x = y;
                    } else {
                      zd[s * H + h].y = x[i];
                    }
                  }
                }
              }
            }
          }
        }
        sync_team(team);
        if (sweep == 0) {
          // Maximum, sum and delta: 2^lg lanes per head, 32 / 2^lg heads at a time.  Sum and delta in fp64, delta kept in two terms:
          // a root's dz sum to 0, and what delta is off by falls on all of them with one sign.  In fp32 that decided the bias's gradient where
          // nearly all slots lie in one bucket and the rest cancels (2 buckets, 3751 roots of 52 slots: 1.9e-5 of it off, 1.7e-6 this way, in the same time).
          int lg = 5;
          while (lg > 0 && (H << lg) > 32) --lg;
          const int per = 32 >> lg, part = lane & ((1 << lg) - 1);
          for (int h0 = sub * per; h0 < H; h0 += team * per) {
            const int h = h0 + (lane >> lg);
            const bool in = h < H;
            const float was = several && in ? s_head[h].x : -INFINITY;
            float top = was;
            for (int s = part; in && s < ns; s += 1 << lg) top = fmaxf(top, zd[s * H + h].x);
            for (int w = 1; w < (1 << lg); w <<= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, w));
            const float base = top == -INFINITY ? 0.f : top;   // nothing but -infinity: weights are 0
            double sum = 0.0, del = 0.0;
            for (int s = part; in && s < ns; s += 1 << lg) {
              const float2 at = zd[s * H + h];
              const float p = exp2_fast((at.x - base) * kLog2e);
              if (!several) zd[s * H + h].x = p;
              sum += p;
              del = fma((double)p, (double)at.y, del);
            }
            for (int w = 1; w < (1 << lg); w <<= 1) {
              sum += __shfl_xor_sync(FULL, sum, w);
              del += __shfl_xor_sync(FULL, del, w);
            }
            __syncwarp();
            if (in && part == 0) {
              if (several) {
                const double corr = exp2_fast((was - base) * kLog2e);     // was = -infinity: 0
                const double2 so = s_sums[h];
                sum = fma(so.x, corr, sum);
                del = fma(so.y, corr, del);
                s_sums[h] = make_double2(sum, del);
              }
              // 1 / l by one Newton step from its fp32 value; both are used after the last chunk only
              const float rl = sum == 0.0 ? 0.f : 1.f / (float)sum;
              del *= (double)rl * fma(-sum, (double)rl, 2.0);
              const float hi = (float)del;
              s_head[h] = make_float4(top, rl, hi, isfinite(hi) ? (float)(del - (double)hi) : 0.f);
            }
          }
          sync_team(team);
          if (several) continue;
        }
        // weights and dz
        for (int i = lane + 32 * sub, h = h_first; i < ns * H; i += 32 * team) {
          const float2 at = zd[i];
          const float4 head = s_head[h];
          float p = at.x;
          if (several) {
            p = exp2_fast((p - (head.x == -INFINITY ? 0.f : head.x)) * kLog2e);
          }
          p *= head.y;
          zd[i] = make_float2(p, p * ((at.y - head.z) - head.w));
          h += h_step;
          if (h >= H) h -= H;
        }
        sync_team(team);
        if (table) {
          // 32 slots at a time.  Slots in time order have neighbouring buckets: runs of one bucket are summed by a segmented scan and each
          // run's last lane adds to its bucket, all different ones.  Otherwise a lane per head goes through them.
          for (int t0 = 32 * sub; t0 < ns; t0 += 32 * team) {
            const int s = t0 + lane, b = bucket[min(s, ns - 1)];
            const int below = __shfl_up_sync(FULL, b, 1), above = __shfl_down_sync(FULL, b, 1);
            if (__all_sync(FULL, lane == 31 || b <= above) || __all_sync(FULL, lane == 31 || b >= above)) {
              const unsigned starts = __ballot_sync(FULL, lane == 0 || b != below);
              const int back = lane - (31 - __clz(starts & (0xffffffffu >> (31 - lane))));   // lanes to the run's first
              const bool end = lane == 31 || b != above;
              for (int h = 0; h < H; ++h) {
                float v = s < ns ? zd[s * H + h].y : 0.f;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                  const float w = __shfl_up_sync(FULL, v, o);
                  if (back >= o) v += w;
                }
                if (end) tab[h * a.buckets + b] += (double)v;
              }
            } else {
              for (int h = lane; h < H; h += 32) {
                for (int u = t0; u < min(t0 + 32, ns); ++u) tab[h * a.buckets + bucket[u]] += (double)zd[u * H + h].y;
              }
            }
            __syncwarp();
          }
        }
        const bool final_chunk = c0 + a.chunk >= cnt;
        for (int kv0 = 0; kv0 < a.kv_heads; kv0 += me.KC) {
          const int kv = kv0 + me.kc;
          for (int g0 = 0; g0 < a.group; g0 += GT) {
            const int h0 = kv * a.group + g0;
            float acc[GT][S::N];
#pragma unroll
            for (int g = 0; g < GT; ++g) {
#pragma unroll
              for (int j = 0; j < S::N; ++j) acc[g][j] = 0.f;
            }
            const T* kp = kr + (int64_t)(c0 + row) * ROW + kv * D;
            const float2* wz = zd + row * H + h0;
            S k[UN];
#pragma unroll
            for (int u = 0; u < UN; ++u) k[u].load(kp + u * me.RPI * ROW, me.part, D, row + u * me.RPI < ns);
            for (int s0 = row; s0 - me.row < ns; s0 += step) {
              const int next = s0 + step;
              kp += step * ROW;
#pragma unroll
              for (int u = 0; u < UN; ++u) {
                float w[GT];
#pragma unroll
                for (int g = 0; g < GT; ++g) w[g] = s0 + u * me.RPI < ns ? wz[u * me.RPI * H + g].y : 0.f;
#pragma unroll
                for (int j = 0; j < S::N; ++j) {
                  const float x = k[u].at(j);
#pragma unroll
                  for (int g = 0; g < GT; ++g) acc[g][j] = fmaf(w[g], x, acc[g][j]);
                }
                k[u].load(kp + u * me.RPI * ROW, me.part, D, next + u * me.RPI < ns);
              }
              wz += step * H;
            }
#pragma unroll
            for (int g = 0; g < GT; ++g) {
              for (int o = P * me.KC; o < 32; o <<= 1) {
#pragma unroll
                for (int j = 0; j < S::N; ++j) acc[g][j] += __shfl_xor_sync(FULL, acc[g][j], o);
              }
              if (team > 1) {
                if (me.row == 0) put_team<S, P>(red, (sub * me.KC + me.kc) * GT + g, D, me.part, acc[g]);
                continue;
              }
              if (several && me.row == 0) {                    // carried from chunk to chunk
#pragma unroll
                for (int j = 0; j < S::N; ++j) {
                  const int e = ((j / S::VE) * P + me.part) * S::VE + j % S::VE;
                  if (e < D) {
                    if (c0 > 0) acc[g][j] += s_dq[(h0 + g) * D + e];
                    if (!final_chunk) s_dq[(h0 + g) * D + e] = acc[g][j];
                  }
                }
              }
              if (final_chunk && me.row == 0) {
#pragma unroll
                for (int j = 0; j < S::N; ++j) acc[g][j] *= a.scale;
                S::store(dqr + (h0 + g) * D, me.part, D, acc[g]);
              }
            }
            if (team > 1) {
              __syncthreads();
              const int size = me.KC * GT * D;
              for (int i = threadIdx.x; i < size; i += blockDim.x) {
                const int e = i / D, at = ((kv0 + e / GT) * a.group + g0 + e % GT) * D + (i - e * D);
                float x = 0.f;
                for (int w = 0; w < team; ++w) x += red[w * size + i];
                if (c0 > 0) x += s_dq[at];
                if (!final_chunk) s_dq[at] = x;
                else dqr[at] = from_float<T>(x * a.scale);
              }
              __syncthreads();                                 // before the next heads overwrite it
            }
          }
          const int own = me.row + sub * me.RPI, each = team * me.RPI;
          T* dkp = dkr + (int64_t)(c0 + own) * ROW + kv * D;
          T* dvp = dvr + (int64_t)(c0 + own) * ROW + kv * D;
          int s = own;
          if (a.group == GT) {
            float q[GT][S::N], go[GT][S::N];
            {
              S raw[GT], raw2[GT];
#pragma unroll
              for (int g = 0; g < GT; ++g) {
                raw[g].load(qr + (kv * GT + g) * D, me.part, D, true);
                raw2[g].load(gr + (kv * GT + g) * D, me.part, D, true);
              }
#pragma unroll
              for (int g = 0; g < GT; ++g) {
                raw[g].floats(q[g]);
                raw2[g].floats(go[g]);
#pragma unroll
                for (int j = 0; j < S::N; ++j) q[g][j] *= a.scale;
              }
            }
            const float2* at = zd + s * H + kv * GT;
#pragma unroll 2
            for (; s < ns; s += each) {
              float xk[S::N], xv[S::N];
#pragma unroll
              for (int g = 0; g < GT; ++g) {
                const float p = at[g].x, y = at[g].y;
#pragma unroll
                for (int j = 0; j < S::N; ++j) {
                  xk[j] = g == 0 ? y * q[g][j] : fmaf(y, q[g][j], xk[j]);
                  xv[j] = g == 0 ? p * go[g][j] : fmaf(p, go[g][j], xv[j]);
                }
              }
              S::store(dkp, me.part, D, xk);
              S::store(dvp, me.part, D, xv);
              dkp += each * ROW;
              dvp += each * ROW;
              at += each * H;
            }
          } else {
            for (; s < ns; s += each) {
              float xk[S::N], xv[S::N];
#pragma unroll
              for (int j = 0; j < S::N; ++j) xk[j] = xv[j] = 0.f;
              for (int h = kv * a.group; h < (kv + 1) * a.group; ++h) {
                S q, go;
                q.load(qr + h * D, me.part, D, true);
                go.load(gr + h * D, me.part, D, true);
                const float p = zd[s * H + h].x, y = zd[s * H + h].y * a.scale;
#pragma unroll
                for (int j = 0; j < S::N; ++j) {
                  xk[j] = fmaf(y, q.at(j), xk[j]);
                  xv[j] = fmaf(p, go.at(j), xv[j]);
                }
              }
              S::store(dkp, me.part, D, xk);
              S::store(dvp, me.part, D, xv);
              dkp += each * ROW;
              dvp += each * ROW;
            }
          }
          if (final_chunk) {                                   // behind the last slot that counts: zeros
            float zero[S::N];
#pragma unroll
            for (int j = 0; j < S::N; ++j) zero[j] = 0.f;
            for (; s < a.slots - c0; s += each) {
              S::store(dkp, me.part, D, zero);
              S::store(dvp, me.part, D, zero);
              dkp += each * ROW;
              dvp += each * ROW;
            }
          }
        }
        sync_team(team);                                       // before the next chunk or root overwrites what was read
      }
    }
  }
  if (table) {
    __syncthreads();
    for (int i = threadIdx.x; i < H * a.buckets; i += blockDim.x) {
      double sum = 0.0;
      for (int w = 0; w < a.warps; ++w) sum += reinterpret_cast<const double*>(smem + L.table + (size_t)w * (team > 1 ? H * a.buckets * 8 : a.warp_bytes))[i];
      a.partial[(int64_t)blockIdx.x * H * a.buckets + i] = sum;
    }
  }
}

// dbias[i] = sum of the blocks' partial sums, in a fixed order: four entries (a sector) by 256 threads each, so that every thread's
// loads are on their way at once.  (A warp per entry spent 10 us on the tables of a thousand blocks.)
static __global__ void __launch_bounds__(1024) bias_sum_kernel(const double* __restrict__ partial, int blocks, int entries, float* __restrict__ dbias) {
  __shared__ double s_sum[32][4];
  const int i = blockIdx.x * 4 + (threadIdx.x & 3), lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.wait;" ::: "memory");           // its launch is prepared while the blocks' kernel runs
  double x[MAX_BLOCKS / 256];
#pragma unroll
  for (int j = 0; j < MAX_BLOCKS / 256; ++j) {
    const int b = (threadIdx.x >> 2) + 256 * j;
    x[j] = b < blocks && i < entries ? partial[(int64_t)b * entries + i] : 0.0;
  }
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < MAX_BLOCKS / 256; ++j) sum += x[j];
  for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(FULL, sum, o);
  if (lane < 4) s_sum[threadIdx.x >> 5][lane] = sum;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  sum = 0.0;
#pragma unroll
  for (int j = 0; j < 4; ++j) sum += s_sum[(lane >> 2) + 8 * j][lane & 3];
  for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(FULL, sum, o);
  if (lane < 4 && i < entries) dbias[i] = (float)sum;
}

template <bool BACKWARD, typename T, int VB, int P, int NV, int GT>
auto kernel_of() {
  if constexpr (BACKWARD) return slot_backward_kernel<T, VB, P, NV, GT>;
  else if constexpr (GT > 1) return slot_forward_group_kernel<T, VB, P, NV, GT>;
  else return slot_forward_kernel<T, VB, P, NV>;
}

constexpr int SMEM_BLOCK = 200 * 1024;     // of an SM's 227 KB, beside the bounds and what the system keeps

// Slots of a chunk, warps of a block and warps per root.  Forward a slot takes a byte: chunks of 4096.  Backward logits and dp of a chunk take
// 8 * heads bytes a slot: 12 KB of them, so that 16 warps have room on an SM.  `step`: slots that a warp has in flight.  A block's warps
// share a root where they all fit on the GPU at once and each has a step of its own (500 roots of 100 slots, 2 heads of 64 in fp32: 16
// us forward and 41 us backward with a warp per root, 10 and 26 us with four; 60 roots of 100 slots, 2 x 4 heads of 64 in bf16: 19 and 42, 11 and
// 21 us; with fewer slots than a step per warp nothing is gained).  0: a warp's share exceeds shared memory.
inline int plan(SlotArgs* a, bool backward, int step) {
  const int table = backward && a->partial ? a->heads * a->buckets : 0, together = heads_at_once(a->group);
  int chunk = backward ? 12 * 1024 / (8 * a->heads) : 4096;
  if (chunk > a->slots) chunk = a->slots;
  a->chunk = chunk;
  auto bytes = [&](int team) { return layout(a->heads, a->dim, chunk, chunk < a->slots, backward, table, team, together).total; };
  const int room = num_sms() * (together == 4 ? 4 * kBlocks<4> : 4 * kBlocks<1>);
  int team = MAX_WARPS;
  while (team > 1 && (team * a->n > room || (backward && a->n > MAX_BLOCKS) || team * step > a->slots || bytes(team) > SMEM_BLOCK / 4)) team >>= 1;
  a->team = team;
  a->warp_bytes = bytes(team);
  if (team > 1) {
    a->warps = team;
    return team;
  }
  int w = MAX_WARPS;
  while (w > 1 && (w * a->warp_bytes > SMEM_BLOCK / 4 || w * (int64_t)num_sms() > a->n)) w >>= 1;   // four blocks to an SM; few roots: over all SMs
  a->warps = w;
  return w * a->warp_bytes <= SMEM_BLOCK ? w : 0;
}

inline int grid_of(const SlotArgs& a, bool backward) {
  const int roots = a.team > 1 ? 1 : a.warps, bytes = roots * a.warp_bytes;   // of a block
  const int64_t want = (a.n + roots - 1) / roots;
  if (!backward) return (int)want;
  int resident = (220 * 1024) / (bytes + 2048);
  if (resident < 1) resident = 1;
  const int warps = 4 * (heads_at_once(a.group) == 4 ? kBlocks<4> : kBlocks<1>);
  if (resident > warps / a.warps) resident = warps / a.warps;
  int64_t most = (int64_t)num_sms() * resident;
  if (most > MAX_BLOCKS) most = MAX_BLOCKS;
  return (int)(want < most ? want : most);
}

template <bool BACKWARD, typename T, int VB, int P, int NV>
cudaError_t launch_kernel(SlotArgs& a, int* blocks, cudaStream_t s) {
  const int gt = heads_at_once(a.group);
  const int kc = a.kv_heads & -a.kv_heads, deep = gt == 4 ? kDeepOf<Seg<T, VB, P, NV>, 4> : kDeepOf<Seg<T, VB, P, NV>, 1>;
  if (!plan(&a, BACKWARD, deep * (32 / P) / (kc < 32 / P ? kc : 32 / P))) return cudaErrorInvalidConfiguration;
  *blocks = grid_of(a, BACKWARD);
  const auto kernel = gt == 4   ? kernel_of<BACKWARD, T, VB, P, NV, 4>()
                      : gt == 2 ? kernel_of<BACKWARD, T, VB, P, NV, 2>()
                                : kernel_of<BACKWARD, T, VB, P, NV, 1>();
  const int bytes = (a.team > 1 ? 1 : a.warps) * a.warp_bytes;
  if (bytes > 46 * 1024) {
    // More than a kernel has without asking for it.  What is asked for is kept per kernel and device, and another thread's call may ask between
    // this one's question and its launch: so it is always the most that any plan takes, never this call's bytes.  (Asking again costs little.)
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BLOCK);
    if (e != cudaSuccess) return e;
  }
  kernel<<<*blocks, 32 * a.warps, bytes, s>>>(a);
  return cudaGetLastError();
}

// Words of 16 bytes where every head of every row starts on one, pairs of values (heads of 50) or single ones (odd heads, odd
// bases) otherwise; as many lanes per segment as 8 values each (4 single ones) need.  (Heads of 50 in fp32 over a whole warp, a pair
// per lane: forward 12.4 and backward 22.7 us for 1800 roots of 20 slots, 2 heads, 85 and 155 us for 14 400; this way 8.2 and 20.7, 56 and 109: the
// sums' and weights' instructions serve four segments.)
template <bool BACKWARD, typename T>
cudaError_t launch_type(SlotArgs& a, int* blocks, cudaStream_t s) {
  constexpr int ES = (int)sizeof(T), N16 = ES / 2;             // words of 16 bytes for 8 values
  const uint64_t at = (uint64_t)(uintptr_t)a.k | (uint64_t)(uintptr_t)a.v | (uint64_t)(uintptr_t)a.q | (uint64_t)(uintptr_t)a.out |
                      (uint64_t)(uintptr_t)a.dout | (uint64_t)(uintptr_t)a.dq | (uint64_t)(uintptr_t)a.dk | (uint64_t)(uintptr_t)a.dv |
                      (uint64_t)(a.dim * ES);
  if ((at & 15) == 0) {
    if (a.dim <= 32) return launch_kernel<BACKWARD, T, 16, 4, N16>(a, blocks, s);
    if (a.dim <= 64) return launch_kernel<BACKWARD, T, 16, 8, N16>(a, blocks, s);
    return launch_kernel<BACKWARD, T, 16, 16, N16>(a, blocks, s);
  }
  if ((at & (2 * ES - 1)) == 0) {
    if (a.dim <= 32) return launch_kernel<BACKWARD, T, 2 * ES, 4, 4>(a, blocks, s);
    if (a.dim <= 64) return launch_kernel<BACKWARD, T, 2 * ES, 8, 4>(a, blocks, s);
    return launch_kernel<BACKWARD, T, 2 * ES, 16, 4>(a, blocks, s);
  }
  if (a.dim <= 32) return launch_kernel<BACKWARD, T, ES, 8, 4>(a, blocks, s);
  return launch_kernel<BACKWARD, T, ES, 32, 4>(a, blocks, s);
}

// The backward pass's kernels of each type are compiled in a file of their own.
extern template cudaError_t launch_type<true, float>(SlotArgs&, int*, cudaStream_t);
extern template cudaError_t launch_type<true, __nv_bfloat16>(SlotArgs&, int*, cudaStream_t);
extern template cudaError_t launch_type<true, __half>(SlotArgs&, int*, cudaStream_t);

template <bool BACKWARD>
int run(const char* who, SlotArgs& a, int dtype, const void* out_like, float* dbias, float* scratch, void* stream, char* err, int64_t size) {
  if (!known_dtype(dtype)) return fail(err, size, TGNN_EINVAL, "%s: unknown type %d", who, dtype);
  if (a.n < 0 || a.slots < 1 || a.slots > 65536 || a.heads < 1 || a.heads > 256 || a.kv_heads < 1 || a.dim < 1 || a.dim > 128)
    return fail(err, size, TGNN_EINVAL, "%s: size out of range (slots 1 to 65536, heads to 256, dim 1 to 128)", who);
  if (a.heads % a.kv_heads) return fail(err, size, TGNN_EINVAL, "%s: %d heads over %d key and value heads", who, a.heads, a.kv_heads);
  if (a.heads * a.dim > 2048) return fail(err, size, TGNN_ECAPACITY, "%s: heads * dim above 2048", who);
  if (a.n > 0x7fffffff) return fail(err, size, TGNN_ECAPACITY, "%s: n beyond int32", who);
  if (a.bias && (a.buckets < 1 || a.buckets > kMaxBuckets))
    return fail(err, size, TGNN_EINVAL, "%s: %d buckets (1 to %d)", who, a.buckets, kMaxBuckets);
  if (a.bias && a.heads * a.buckets > 16384) return fail(err, size, TGNN_ECAPACITY, "%s: heads * num_buckets above 16384", who);
  if (a.n > 0 && (!a.q || !a.k || !a.v || !a.cnt || !out_like || (BACKWARD && (!a.dout || !a.dk || !a.dv))))
    return fail(err, size, TGNN_EINVAL, "%s: null pointer", who);
  if (a.bias && a.n > 0 && ((a.buckets > 1 && !a.bounds) || !a.times || !a.ts))
    return fail(err, size, TGNN_EINVAL, "%s: a bias needs bounds, times and ts", who);
  if (BACKWARD && ((a.bias != nullptr) != (dbias != nullptr) || (dbias && a.n > 0 && !scratch)))
    return fail(err, size, TGNN_EINVAL, "%s: dbias and scratch belong to a bias", who);
  const int elem = elem_bytes(dtype);
  if ((((uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.dout | (uintptr_t)out_like | (uintptr_t)a.dk | (uintptr_t)a.dv) &
       (elem - 1)) ||
      (((uintptr_t)a.bounds | (uintptr_t)a.times | (uintptr_t)a.ts | (uintptr_t)scratch) & 7) ||
      (((uintptr_t)a.cnt | (uintptr_t)a.bias | (uintptr_t)dbias) & 3))
    return fail(err, size, TGNN_EINVAL, "%s: a pointer is not aligned to its element", who);
  cudaStream_t s = (cudaStream_t)stream;
  if (a.n == 0) {
    if (dbias && cudaMemsetAsync(dbias, 0, sizeof(float) * (size_t)a.heads * a.buckets, s) != cudaSuccess)
      return fail(err, size, TGNN_ECUDA, "%s: %s", who, cudaGetErrorString(cudaGetLastError()));
    return TGNN_OK;
  }
  a.group = a.heads / a.kv_heads;
  a.partial = dbias ? reinterpret_cast<double*>(scratch) : nullptr;
  int blocks = 0;
  cudaError_t e;
  if (dtype == TGNN_F32) e = launch_type<BACKWARD, float>(a, &blocks, s);
  else if (dtype == TGNN_BF16) e = launch_type<BACKWARD, __nv_bfloat16>(a, &blocks, s);
  else e = launch_type<BACKWARD, __half>(a, &blocks, s);
  if (blocks == 0)
    return fail(err, size, TGNN_ECAPACITY, "%s: %d heads with %d buckets exceed shared memory", who, a.heads, a.buckets);
  if (e == cudaSuccess && BACKWARD && a.partial) {
    const int entries = a.heads * a.buckets;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(entries + 3) / 4);
    cfg.blockDim = dim3(1024);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, bias_sum_kernel, (const double*)a.partial, blocks, entries, dbias);
  }
  if (e != cudaSuccess) {
    cudaGetLastError();
    return fail(err, size, TGNN_ECUDA, "%s: %s", who, cudaGetErrorString(e));
  }
  return TGNN_OK;
}

inline SlotArgs args_of(const void* q, const void* k, const void* v, int64_t n, int slots, int heads, int kv_heads, int dim, const int32_t* cnt,
                 const float* bias, int buckets, const double* bounds, const double* times, const double* ts, float scale) {
  SlotArgs a = {};
  a.q = q;
  a.k = k;
  a.v = v;
  a.n = n;
  a.slots = slots;
  a.heads = heads;
  a.kv_heads = kv_heads;
  a.dim = dim;
  a.cnt = cnt;
  a.bias = bias;
  a.buckets = bias ? buckets : 0;
  a.bounds = bounds;
  a.times = times;
  a.ts = ts;
  a.scale = scale;
  return a;
}

}  // namespace tgnn_slots
