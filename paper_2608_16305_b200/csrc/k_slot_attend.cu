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
// gain on one query per row.  The backward pass recomputes the weights, which costs no traffic while a root's rows stay in
// shared memory, and needs nothing of the forward pass.
//
// A warp takes one root after another.  The rows of a root lie side by side; they are staged in the warp's own shared memory by
// asynchronous copies in chunks of slots, the next chunk (of this root or the next) while one is worked on, so that two chunks
// per warp are in flight or in use.  Roots with more slots than a chunk are walked twice by the backward pass: maximum, sum
// and delta first, gradients then.  All sums are fp32; those of the bias, which run over the whole batch, fp64: each warp
// keeps a table of its own and a second kernel adds the blocks' tables in a fixed order, so no atomics decide on a result.
// Logits stay in natural units: a bias of the type's lowest value is then still finite.
#include "tgnn_history.cuh"

using namespace tgnn_history;

namespace {

constexpr int MAX_BLOCKS = 1024;
constexpr int MAX_WARPS = 8;

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
  int warp_bytes;                        // shared memory of a warp
  float scale;
};

// A warp's shared memory, all parts multiples of 16 bytes: two stages of (K chunk, V chunk), then floats:
// query [H * dim], output or dq [H * dim], (backward: dout [H * dim]), z [H * chunk], (backward: dp [H * chunk]),
// per head m, l, corr, delta; bucket [chunk]; (backward with bias: table [H * buckets] fp64)
__host__ __device__ inline int up16(int x) { return (x + 15) & ~15; }
struct Layout {
  int row, stage, q, o, g, z, dp, head, bucket, table, total;
};
__host__ __device__ inline Layout layout(int heads, int kv_heads, int dim, int chunk, int elem, bool backward, int table) {
  Layout l;
  l.row = kv_heads * dim * elem;
  l.stage = up16(l.row * chunk);
  int at = 4 * l.stage;
  const int vec = up16(heads * dim * 4), hc = up16(heads * chunk * 4);
  l.q = at; at += vec;
  l.o = at; at += vec;
  l.g = at; at += backward ? vec : 0;
  l.z = at; at += hc;
  l.dp = at; at += backward ? hc : 0;
  l.head = at; at += up16(heads * 16);
  l.bucket = at; at += up16(chunk * 4);
  l.table = at; at += up16(table * 8);
  l.total = at;
  return l;
}

template <int VB>
__device__ __forceinline__ void copy_async(uint8_t* dst, const uint8_t* src) {
  if constexpr (VB >= 4) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    if constexpr (VB == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
    else if constexpr (VB == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(d), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d), "l"(src) : "memory");
  } else {
    *reinterpret_cast<uint16_t*>(dst) = __ldg(reinterpret_cast<const uint16_t*>(src));
  }
}

// E neighbouring values as fp32
template <typename T, int E>
__device__ __forceinline__ void load_e(const T* p, float (&x)[E]) {
  if constexpr (E == 1) {
    x[0] = to_float<T>(*p);
  } else if constexpr (sizeof(T) == 4) {
    const float2 f = *reinterpret_cast<const float2*>(p);
    x[0] = f.x;
    x[1] = f.y;
  } else {
    union { uint32_t w; T e[2]; } u;
    u.w = *reinterpret_cast<const uint32_t*>(p);
    x[0] = to_float<T>(u.e[0]);
    x[1] = to_float<T>(u.e[1]);
  }
}
template <typename T, int E>
__device__ __forceinline__ void store_e(T* p, const float (&x)[E]) {
  if constexpr (E == 1) {
    *p = from_float<T>(x[0]);
  } else if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]);
  } else {
    union { uint32_t w; T e[2]; } u;
    u.e[0] = from_float<T>(x[0]);
    u.e[1] = from_float<T>(x[1]);
    *reinterpret_cast<uint32_t*>(p) = u.w;
  }
}

// What a warp works on: chunk `c` of root `r`, in sweep 0 (maximum, sum, delta) or 1 (gradients; backward passes over several
// chunks only).  A root without slots is one empty chunk.
struct Item {
  int64_t r;
  int c, sweep, cnt;
};

// One root's slots against one vector per head: out[h * chunk + s] = x[h] . rows[s][h / group], s < ns.
// A lane takes a (slot, head) pair, or a part of one where there are fewer pairs than lanes.  Lanes start at different columns, so that
// rows a multiple of 128 bytes long do not meet in one bank.
template <typename T, int E>
__device__ __forceinline__ void dots(const SlotArgs& a, const T* rows, const float* x, float* out, int ns, int lane) {
  const int pairs = ns * a.heads, row = a.kv_heads * a.dim, steps = a.dim / E;
  int lg = 0;                                                  // 2^lg lanes per pair
  while (lg < 3 && (pairs << (lg + 1)) <= 32) ++lg;
  const int part = lane & ((1 << lg) - 1), per = 32 >> lg;
  for (int p0 = 0; p0 < pairs; p0 += per) {
    const int p = p0 + (lane >> lg);
    float acc = 0.f;
    int h = 0, s = 0;
    if (p < pairs) {
      s = p / a.heads;
      h = p - s * a.heads;
      const T* kr = rows + s * row + (h / a.group) * a.dim;
      const float* xr = x + h * a.dim;
      const int mine = (steps - part + (1 << lg) - 1) >> lg;   // steps part, part + 2^lg, ...
      if (mine > 0) {
        int i = (lane >> lg) % mine;
        for (int j = 0; j < mine; ++j) {
          const int e = (part + (i << lg)) * E;
          float kx[E], xx[E];
          load_e<T, E>(kr + e, kx);
          load_e<float, E>(xr + e, xx);
#pragma unroll
          for (int q = 0; q < E; ++q) acc = fmaf(kx[q], xx[q], acc);
          if (++i == mine) i = 0;
        }
      }
    }
    for (int o = 1; o < (1 << lg); o <<= 1) acc += __shfl_xor_sync(FULL, acc, o);
    if (p < pairs && part == 0) out[h * a.chunk + s] = acc;
  }
}

template <typename T, int VB, int E, bool BACKWARD>
__global__ void __launch_bounds__(32 * MAX_WARPS) slot_attend_kernel(const SlotArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ double s_bounds[kMaxBuckets];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const int H = a.heads, D = a.dim, HD = H * D, ROW = a.kv_heads * D;
  const bool table = BACKWARD && a.partial != nullptr;
  const Layout L = layout(H, a.kv_heads, D, a.chunk, (int)sizeof(T), BACKWARD, table ? H * a.buckets : 0);
  uint8_t* my = smem + (size_t)wid * a.warp_bytes;
  float* q = reinterpret_cast<float*>(my + L.q);
  float* o = reinterpret_cast<float*>(my + L.o);
  float* g = reinterpret_cast<float*>(my + L.g);
  float* z = reinterpret_cast<float*>(my + L.z);
  float* dp = reinterpret_cast<float*>(my + L.dp);
  float* s_m = reinterpret_cast<float*>(my + L.head);
  float *s_l = s_m + H, *s_c = s_m + 2 * H, *s_d = s_m + 3 * H;
  int* bucket = reinterpret_cast<int*>(my + L.bucket);
  double* tab = reinterpret_cast<double*>(my + L.table);
  if (a.bias) {
    for (int i = threadIdx.x; i < a.buckets - 1; i += blockDim.x) s_bounds[i] = a.bounds[i];
  }
  if (table) {
    for (int i = lane; i < H * a.buckets; i += 32) tab[i] = 0.0;
  }
  __syncthreads();

  const int64_t stride = (int64_t)gridDim.x * a.warps;
  auto count = [&](int64_t r) { return r < a.n ? min(max(a.cnt[r], 0), a.slots) : 0; };
  int64_t next_r = (int64_t)blockIdx.x * a.warps + wid;        // the root behind the item's
  int next_cnt = count(next_r);
  auto advance = [&](Item it) {
    const int chunks = it.cnt > 0 ? (it.cnt + a.chunk - 1) / a.chunk : 1;
    if (++it.c < chunks) return it;
    it.c = 0;
    if (BACKWARD && it.sweep == 0 && chunks > 1) { it.sweep = 1; return it; }
    it.sweep = 0;
    it.r = next_r;
    it.cnt = next_cnt;
    next_r += stride;
    next_cnt = count(next_r);
    return it;
  };
  auto stage = [&](const Item& it, int buf) {
    if (it.r < a.n) {
      const int s0 = it.c * a.chunk, ns = min(a.chunk, it.cnt - s0);
      const int64_t at = (it.r * a.slots + s0) * ROW * (int64_t)sizeof(T);
      const uint8_t* kp = reinterpret_cast<const uint8_t*>(a.k) + at;
      const uint8_t* vp = reinterpret_cast<const uint8_t*>(a.v) + at;
      uint8_t* ks = my + 2 * buf * L.stage;
      uint8_t* vs = ks + L.stage;
      const int bytes = max(ns, 0) * L.row;                    // a last word may reach into the root's next slot, never beyond its rows
      for (int i = lane * VB; i < bytes; i += 32 * VB) copy_async<VB>(ks + i, kp + i);
      for (int i = lane * VB; i < bytes; i += 32 * VB) copy_async<VB>(vs + i, vp + i);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  Item cur;
  cur.r = next_r;
  cur.cnt = next_cnt;
  cur.c = cur.sweep = 0;
  next_r += stride;
  next_cnt = count(next_r);
  int buf = 0;
  stage(cur, 0);
  while (cur.r < a.n) {
    const Item nxt = advance(cur);
    stage(nxt, buf ^ 1);
    const int64_t r = cur.r;
    const int s0 = cur.c * a.chunk, ns = max(min(a.chunk, cur.cnt - s0), 0);
    const int chunks = cur.cnt > 0 ? (cur.cnt + a.chunk - 1) / a.chunk : 1;
    const bool last = cur.c == chunks - 1;
    if (cur.c == 0 && cur.sweep == 0) {                        // a new root
      const T* qg = reinterpret_cast<const T*>(a.q) + r * HD;
      for (int i = lane * E; i < HD; i += 32 * E) {
        float x[E];
        load_e<T, E>(qg + i, x);
#pragma unroll
        for (int e = 0; e < E; ++e) { q[i + e] = x[e]; o[i + e] = 0.f; }
      }
      if (BACKWARD) {
        const T* gg = reinterpret_cast<const T*>(a.dout) + r * HD;
        for (int i = lane * E; i < HD; i += 32 * E) {
          float x[E];
          load_e<T, E>(gg + i, x);
#pragma unroll
          for (int e = 0; e < E; ++e) g[i + e] = x[e];
        }
      }
      for (int h = lane; h < H; h += 32) { s_m[h] = -INFINITY; s_l[h] = 0.f; s_d[h] = 0.f; }
    }
    if (a.bias) {
      const double t = a.times[r];
      for (int s = lane; s < ns; s += 32) bucket[s] = bucket_of(s_bounds, a.buckets - 1, t - __ldg(a.ts + r * a.slots + s0 + s));
    }
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncwarp();
    const T* ks = reinterpret_cast<const T*>(my + 2 * buf * L.stage);
    const T* vs = reinterpret_cast<const T*>(my + 2 * buf * L.stage + L.stage);
    dots<T, E>(a, ks, q, z, ns, lane);
    if (BACKWARD) dots<T, E>(a, vs, g, dp, ns, lane);
    __syncwarp();

    // softmax of the chunk: 2^lg lanes per head, 32 / 2^lg heads at a time
    {
      int lg = 5;
      while (lg > 0 && (H << lg) > 32) --lg;
      const int per = 32 >> lg, part = lane & ((1 << lg) - 1);
      for (int h0 = 0; h0 < H; h0 += per) {
        const int h = h0 + (lane >> lg);
        const bool in = h < H;
        float* zh = z + h * a.chunk;
        float top = in ? s_m[h] : -INFINITY;
        const float was = top;
        if (in) {
          for (int s = part; s < ns; s += 1 << lg) {
            float x = zh[s] * a.scale;
            if (a.bias) x += __ldg(a.bias + h * a.buckets + bucket[s]);
            zh[s] = x;
            top = fmaxf(top, x);
          }
        }
        if (cur.sweep == 0) {
          for (int w = 1; w < (1 << lg); w <<= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, w));
        }
        const float base = top == -INFINITY ? 0.f : top;       // nothing but -infinity: weights are 0
        float sum = 0.f, del = 0.f;
        const float inv = in && cur.sweep ? s_c[h] : 1.f;
        if (in) {
          for (int s = part; s < ns; s += 1 << lg) {
            const float p = exp2_fast((zh[s] - base) * kLog2e) * inv;
            zh[s] = p;
            sum += p;
            if (BACKWARD) del = fmaf(p, dp[h * a.chunk + s], del);
          }
        }
        if (cur.sweep == 0) {
          for (int w = 1; w < (1 << lg); w <<= 1) {
            sum += __shfl_xor_sync(FULL, sum, w);
            if (BACKWARD) del += __shfl_xor_sync(FULL, del, w);
          }
          __syncwarp();
          if (in && part == 0) {
            const float corr = exp2_fast((was - base) * kLog2e);          // was = -infinity: 0
            const float l = fmaf(s_l[h], corr, sum);
            s_m[h] = top;
            s_l[h] = l;
            if (BACKWARD) {
              const float d = fmaf(s_d[h], corr, del);
              const float il = l == 0.f ? 0.f : 1.f / l;
              s_d[h] = last ? d * il : d;
              s_c[h] = il;                                     // the weights' factor, final at the last chunk
            } else {
              s_c[h] = corr;
            }
          }
        }
      }
    }
    __syncwarp();

    if (!BACKWARD) {
      // o = o * corr + sum_s p_s v_s
      T* og = reinterpret_cast<T*>(a.out) + r * HD;
      for (int i = lane * E; i < HD; i += 32 * E) {
        const int h = i / D, col = (h / a.group) * D + (i - h * D);
        const float corr = s_c[h];
        const float* p = z + h * a.chunk;
        float acc[E];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = o[i + e] * corr;
        for (int s = 0; s < ns; ++s) {
          float x[E];
          load_e<T, E>(vs + s * ROW + col, x);
          const float w = p[s];
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] = fmaf(w, x[e], acc[e]);
        }
        if (last) {
          const float l = s_l[h], f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] *= f;
          store_e<T, E>(og + i, acc);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) o[i + e] = acc[e];
        }
      }
    } else if (chunks == 1 || cur.sweep == 1) {
      // weights and dz of the chunk; the bias's sums: a lane per head, so that no two lanes add to one bucket
      const bool single = cur.sweep == 0;
      for (int i = lane; i < ns * H; i += 32) {
        const int s = i / H, h = i - s * H;
        const float p = single ? z[h * a.chunk + s] * s_c[h] : z[h * a.chunk + s];
        z[h * a.chunk + s] = p;
        dp[h * a.chunk + s] = p * (dp[h * a.chunk + s] - s_d[h]);
      }
      __syncwarp();
      if (table) {
        for (int h = lane; h < H; h += 32) {
          for (int s = 0; s < ns; ++s) tab[h * a.buckets + bucket[s]] += (double)dp[h * a.chunk + s];
        }
      }
      const int64_t row0 = (r * a.slots + s0) * (int64_t)ROW;
      T* dkg = reinterpret_cast<T*>(a.dk) + row0;
      T* dvg = reinterpret_cast<T*>(a.dv) + row0;
      T* dqg = reinterpret_cast<T*>(a.dq) + r * HD;
      for (int i = lane * E; i < HD; i += 32 * E) {
        const int h = i / D, col = (h / a.group) * D + (i - h * D);
        const float* dz = dp + h * a.chunk;
        float acc[E];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = o[i + e];
        for (int s = 0; s < ns; ++s) {
          float x[E];
          load_e<T, E>(ks + s * ROW + col, x);
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] = fmaf(dz[s], x[e], acc[e]);
        }
        if (last) {
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] *= a.scale;
          store_e<T, E>(dqg + i, acc);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) o[i + e] = acc[e];
        }
      }
      for (int i = lane * E; i < ROW; i += 32 * E) {
        const int kv = i / D, h0 = kv * a.group, col = i - kv * D;
        for (int s = 0; s < ns; ++s) {
          float xk[E], xv[E];
#pragma unroll
          for (int e = 0; e < E; ++e) xk[e] = xv[e] = 0.f;
          for (int h = h0; h < h0 + a.group; ++h) {
            const float dz = dp[h * a.chunk + s] * a.scale, p = z[h * a.chunk + s];
#pragma unroll
            for (int e = 0; e < E; ++e) {
              xk[e] = fmaf(dz, q[h * D + col + e], xk[e]);
              xv[e] = fmaf(p, g[h * D + col + e], xv[e]);
            }
          }
          store_e<T, E>(dkg + (int64_t)s * ROW + i, xk);
          store_e<T, E>(dvg + (int64_t)s * ROW + i, xv);
        }
        if (last) {                                            // slots that do not count
          float zero[E];
#pragma unroll
          for (int e = 0; e < E; ++e) zero[e] = 0.f;
          for (int s = ns; s < a.slots - s0; ++s) {
            store_e<T, E>(dkg + (int64_t)s * ROW + i, zero);
            store_e<T, E>(dvg + (int64_t)s * ROW + i, zero);
          }
        }
      }
    }
    __syncwarp();                                              // the stage may be filled again
    cur = nxt;
    buf ^= 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (table) {
    __syncthreads();
    for (int i = threadIdx.x; i < H * a.buckets; i += blockDim.x) {
      double sum = 0.0;
      for (int w = 0; w < a.warps; ++w) sum += reinterpret_cast<const double*>(smem + (size_t)w * a.warp_bytes + L.table)[i];
      a.partial[(int64_t)blockIdx.x * H * a.buckets + i] = sum;
    }
  }
}

// dbias[i] = sum of the blocks' partial sums: a warp per entry, lanes and shuffles in a fixed order.
__global__ void __launch_bounds__(256) bias_sum_kernel(const double* __restrict__ partial, int blocks, int entries, float* __restrict__ dbias) {
  const int i = (blockIdx.x * 256 + threadIdx.x) >> 5, lane = threadIdx.x & 31;
  if (i >= entries) return;
  double sum = 0.0;
  for (int b = lane; b < blocks; b += 32) sum += partial[(int64_t)b * entries + i];
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
  if (lane == 0) dbias[i] = (float)sum;
}

template <typename T, int VB, int E, bool BACKWARD>
cudaError_t launch_kernel(const SlotArgs& a, int blocks, cudaStream_t s) {
  const int bytes = a.warps * a.warp_bytes;
  // more dynamic shared memory than 48 KB has to be asked for, per device; asking again costs less than a microsecond
  const cudaError_t e = cudaFuncSetAttribute(slot_attend_kernel<T, VB, E, BACKWARD>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) return e;
  slot_attend_kernel<T, VB, E, BACKWARD><<<blocks, 32 * a.warps, bytes, s>>>(a);
  return cudaGetLastError();
}

// Chunks are copied in words of 16, 8, 4 or 2 bytes: the widest on which k, v, a root's rows and a chunk's rows all start.  Even
// head sizes are worked on two values at a time.
template <typename T, bool BACKWARD>
cudaError_t launch_type(const SlotArgs& a, int blocks, cudaStream_t s) {
  const int64_t row = (int64_t)a.kv_heads * a.dim * (int64_t)sizeof(T);
  uint64_t at = (uint64_t)(uintptr_t)a.k | (uint64_t)(uintptr_t)a.v | (uint64_t)(row * a.slots);
  if (a.chunk < a.slots) at |= (uint64_t)(row * a.chunk);
  const bool even = a.dim % 2 == 0 &&
                    ((((uintptr_t)a.q | (uintptr_t)a.out | (uintptr_t)a.dout | (uintptr_t)a.dq | (uintptr_t)a.dk | (uintptr_t)a.dv) &
                      (2 * sizeof(T) - 1)) == 0);
  if (even) {
    if ((at & 15) == 0) return launch_kernel<T, 16, 2, BACKWARD>(a, blocks, s);
    if ((at & 7) == 0) return launch_kernel<T, 8, 2, BACKWARD>(a, blocks, s);
    if ((at & 3) == 0) return launch_kernel<T, 4, 2, BACKWARD>(a, blocks, s);
    return launch_kernel<T, (int)sizeof(T), 2, BACKWARD>(a, blocks, s);
  }
  if ((at & 15) == 0) return launch_kernel<T, 16, 1, BACKWARD>(a, blocks, s);
  if ((at & 3) == 0) return launch_kernel<T, 4, 1, BACKWARD>(a, blocks, s);
  return launch_kernel<T, (int)sizeof(T), 1, BACKWARD>(a, blocks, s);
}

constexpr int SMEM_BLOCK = 200 * 1024;     // of an SM's 227 KB, beside the bounds and what the system keeps
constexpr int WANT_WARP = 24 * 1024;

// Slots of a chunk and warps of a block: chunks as large as WANT_WARP allows for a warp, all slots if they fit; multiples of 4 slots
// otherwise, which keeps chunks on word boundaries.  false: not even one slot fits.
bool plan(SlotArgs* a, int elem, bool backward) {
  const int table = backward && a->partial ? a->heads * a->buckets : 0;
  auto bytes = [&](int chunk) { return layout(a->heads, a->kv_heads, a->dim, chunk, elem, backward, table).total; };
  const int fixed = bytes(1), per = bytes(9) - fixed;           // of 8 slots
  int chunk = a->slots < 2048 ? a->slots : 2048;
  if (bytes(chunk) > WANT_WARP) {
    const int fit = fixed < WANT_WARP ? 1 + (WANT_WARP - fixed) * 8 / (per > 0 ? per : 1) : 1;
    chunk = fit < chunk ? fit : chunk;
    chunk = chunk >= 4 ? chunk & ~3 : chunk;
    while (chunk > 1 && bytes(chunk) > SMEM_BLOCK) chunk = chunk > 4 ? (chunk - 1) & ~3 : chunk - 1;
  }
  a->chunk = chunk;
  a->warp_bytes = bytes(chunk);
  int w = SMEM_BLOCK / a->warp_bytes;
  const int64_t per_sm = (a->n + num_sms() - 1) / num_sms();    // few roots: over all SMs
  if (w > MAX_WARPS) w = MAX_WARPS;
  if (w > per_sm) w = (int)per_sm;
  a->warps = w;
  return w >= 1;
}

int grid_of(const SlotArgs& a) {
  const int64_t want = (a.n + a.warps - 1) / a.warps;
  int resident = (int)((220 * 1024) / ((int64_t)a.warps * a.warp_bytes + 2048));
  if (resident < 1) resident = 1;
  if (resident > 64 / a.warps) resident = 64 / a.warps;
  int64_t most = (int64_t)num_sms() * resident;
  if (most > MAX_BLOCKS) most = MAX_BLOCKS;
  return (int)(want < most ? want : most);
}

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
  if (!plan(&a, elem, BACKWARD))
    return fail(err, size, TGNN_ECAPACITY, "%s: one slot of %d heads of %d with %d buckets exceeds shared memory", who, a.heads, a.dim, a.buckets);
  const int blocks = grid_of(a);
  cudaError_t e;
  if (dtype == TGNN_F32) e = launch_type<float, BACKWARD>(a, blocks, s);
  else if (dtype == TGNN_BF16) e = launch_type<__nv_bfloat16, BACKWARD>(a, blocks, s);
  else e = launch_type<__half, BACKWARD>(a, blocks, s);
  if (e == cudaSuccess && BACKWARD && a.partial) {
    const int entries = a.heads * a.buckets;
    bias_sum_kernel<<<(entries + 7) / 8, 256, 0, s>>>(a.partial, blocks, entries, dbias);
    e = cudaGetLastError();
  }
  if (e != cudaSuccess) {
    cudaGetLastError();
    return fail(err, size, TGNN_ECUDA, "%s: %s", who, cudaGetErrorString(e));
  }
  return TGNN_OK;
}

SlotArgs args_of(const void* q, const void* k, const void* v, int64_t n, int slots, int heads, int kv_heads, int dim, const int32_t* cnt,
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

}  // namespace

extern "C" {

int tgnn_slot_attend(const void* q, const void* k, const void* v, int dtype, int64_t n, int slots, int heads, int kv_heads, int dim,
                     const int32_t* cnt, const float* bias, int num_buckets, const double* bounds, const double* times, const double* ts,
                     float scale, void* out, void* stream, char* err_host, int64_t err_size) {
  SlotArgs a = args_of(q, k, v, n, slots, heads, kv_heads, dim, cnt, bias, num_buckets, bounds, times, ts, scale);
  a.out = out;
  return run<false>("tgnn_slot_attend", a, dtype, out, nullptr, nullptr, stream, err_host, err_size);
}

int64_t tgnn_slot_attend_scratch(int64_t n, int heads, int num_buckets) {
  if (n < 0 || heads < 1 || heads > 256 || num_buckets < 0 || num_buckets > kMaxBuckets) return -1;
  return 2 * (n < MAX_BLOCKS ? n : (int64_t)MAX_BLOCKS) * heads * num_buckets;
}

int tgnn_slot_attend_backward(const void* q, const void* k, const void* v, int dtype, int64_t n, int slots, int heads, int kv_heads, int dim,
                              const int32_t* cnt, const float* bias, int num_buckets, const double* bounds, const double* times,
                              const double* ts, float scale, const void* dout, void* dq, void* dk, void* dv, float* dbias, float* scratch,
                              void* stream, char* err_host, int64_t err_size) {
  SlotArgs a = args_of(q, k, v, n, slots, heads, kv_heads, dim, cnt, bias, num_buckets, bounds, times, ts, scale);
  a.dout = dout;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  return run<true>("tgnn_slot_attend_backward", a, dtype, dq, dbias, scratch, stream, err_host, err_size);
}

}  // extern "C"
