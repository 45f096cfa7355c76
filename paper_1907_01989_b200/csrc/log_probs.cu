// What a row of logits says: log probabilities of given classes, the entropy, and the most probable classes with theirs.
//
//   m = max x,  d_i = (x_i - m) / T,  S = sum e^d_i:   log p_i = d_i - ln S,   H = ln S - (sum e^d_i d_i) / S
//
// One pass over the logits (what bounds it: their bytes, where there are enough of them to fill the memory's pipe): every thread
// keeps the running maximum m of what it has seen, S and the sum of e^d d relative to it, rescaled when the maximum grows, and its
// largest element.  (x - m) is formed first, so that logits of any size, the type's lowest value among them, lose nothing; minus
// infinity gives e^d = 0, and where nothing else is left in a row S stays 0.
//
// The `top` largest elements, ties to the lower class: with `top` groups of threads whose largest elements lead, the least of those
// bounds the answer from below, and only these groups' elements can reach it: they alone are read again (out of L1 or L2), the few
// that do reach it are collected in shared memory and ranked by counting.  An element is a whole number of 64 bits, the value's
// ordered bits above the inverted class, so that all are different and no order of execution shows.
//
// Three shapes: a thread a row for a handful of classes (every pixel of a segmentation), a warp a row, a CTA a row - or a cluster
// of up to 16 CTAs, where rows are few: they read one row together and join through distributed shared memory, in a fixed order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "kernels.h"
#include "pdl.cuh"
#include "sm100_ptx.cuh"

namespace gi {
namespace {

using namespace ptx;

typedef unsigned long long u64;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.402823466e38f;
constexpr int kMaxTop = GI_MAX_TOP;

struct Params {
  const void* x;
  const int* given;
  float* given_lp;
  float* entropy;
  int* top_ids;
  float* top_lp;
  long long ld;
  int rows, classes, n_given, top;
  float inv_t, c;  // 1 / T, and that in units of log2
  int ks;          // CTAs of a row
};

template <int XT>
struct Elem;
template <>
struct Elem<GI_F16> {
  typedef __half type;
  static constexpr int kVec = 8;
  static __device__ __forceinline__ float f32(__half v) { return __half2float(v); }
};
template <>
struct Elem<GI_BF16> {
  typedef __nv_bfloat16 type;
  static constexpr int kVec = 8;
  static __device__ __forceinline__ float f32(__nv_bfloat16 v) { return __bfloat162float(v); }
};
template <>
struct Elem<GI_F32> {
  typedef float type;
  static constexpr int kVec = 4;
  static __device__ __forceinline__ float f32(float v) { return v; }
};

// ordered bits of a value above the inverted class: larger values first, then lower classes; a NaN above all, -0 as 0
__device__ __forceinline__ u64 key_of(float v, int i) {
  int b = __float_as_int(v + 0.0f);
  if (v != v) b = 0x7fffffff;
  const unsigned o = static_cast<unsigned>(b ^ ((b >> 31) & 0x7fffffff)) ^ 0x80000000u;
  return (static_cast<u64>(o) << 32) | (0xffffffffu - static_cast<unsigned>(i));
}
__device__ __forceinline__ int class_of(u64 k) { return static_cast<int>(0xffffffffu - static_cast<unsigned>(k)); }
__device__ __forceinline__ float value_of(u64 k) {
  const int o = static_cast<int>(static_cast<unsigned>(k >> 32) ^ 0x80000000u);
  return __int_as_float(o ^ ((o >> 31) & 0x7fffffff));
}
__device__ __forceinline__ u64 max64(u64 a, u64 b) { return a > b ? a : b; }
__device__ __forceinline__ u64 shfl_xor64(u64 v, int m) { return __shfl_xor_sync(0xffffffffu, v, m); }

__device__ __forceinline__ float ex2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// the larger; a NaN stays one
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Running sums relative to a maximum m: s = sum 2^d, t = sum 2^d d with d = (x - m) c.
struct Stat {
  float m, s, t;
  __device__ __forceinline__ void clear() {
    m = kLowest;
    s = t = 0.0f;
  }
  // to a new maximum: every d grows by e = (m - to) c <= 0
  __device__ __forceinline__ void rebase(float to, float c) {
    const float e = fmaxf((m - to) * c, -1.0e30f), f = ex2(e);
    t = f * (t + e * s);  // (s = 0 where nothing was seen: 0 again)
    s *= f;
    m = to;
  }
  // d bounded from below, where 2^d is 0: nothing is multiplied by infinity.  A NaN comes through.
  __device__ __forceinline__ void add(float v, float c) {
    const float d = max_nan((v - m) * c, -1000.0f), e = ex2(d);
    s += e;
    t = fmaf(e, d, t);
  }
  __device__ __forceinline__ void merge(Stat o, float c) {
    const float to = fmaxf(m, o.m);
    rebase(to, c);
    o.rebase(to, c);
    s += o.s;
    t += o.t;
  }
};

__device__ __forceinline__ Stat warp_merge(Stat st, float c, int width) {
  for (int o = 1; o < width; o <<= 1) {
    Stat other;
    other.m = __shfl_xor_sync(0xffffffffu, st.m, o);
    other.s = __shfl_xor_sync(0xffffffffu, st.s, o);
    other.t = __shfl_xor_sync(0xffffffffu, st.t, o);
    // both lanes of a pair add the same two in the same order
    const bool low = (threadIdx.x & o) == 0;
    Stat a = low ? st : other;
    const Stat b = low ? other : st;
    a.merge(b, c);
    st = a;
  }
  return st;
}

// log p of a logit, given a row's sums: minus infinity in a row in which nothing is left
__device__ __forceinline__ float log_prob(float v, const Stat& st, float log_s, float inv_t) {
  return st.s == 0.0f ? -INFINITY : (v - st.m) * inv_t - log_s;
}
__device__ __forceinline__ float entropy_of(const Stat& st, float log_s) { return st.s == 0.0f ? 0.0f : log_s - st.t * kLn2 / st.s; }

// ---------------------------------------------------------------- a row in 16-byte pieces
// Piece i of a row covers the elements that lie in one aligned unit of 16 bytes; `lead` of the first piece's lie in front of the row.
template <int XT>
struct Row {
  static constexpr int V = Elem<XT>::kVec;
  typedef typename Elem<XT>::type T;
  const T* x;
  int lead, classes, pieces;
  __device__ __forceinline__ Row(const Params& p, long long row) {
    x = static_cast<const T*>(p.x) + row * p.ld;
    lead = static_cast<int>(reinterpret_cast<unsigned long long>(x) / sizeof(T) % V);
    classes = p.classes;
    pieces = (lead + classes + V - 1) / V;
  }
  __device__ __forceinline__ bool whole(int i) const { return i * V >= lead && (i + 1) * V - lead <= classes; }
  __device__ __forceinline__ uint4 raw(int i) const { return __ldg(reinterpret_cast<const uint4*>(x + (i * V - lead))); }
  static __device__ __forceinline__ void convert(const uint4& w, float (&v)[V]) {
    const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = Elem<XT>::f32(e[j]);
  }
  __device__ __forceinline__ float at(int c) const { return Elem<XT>::f32(x[c]); }
};

// What a thread has seen of a row: sums, and its largest element.
template <int XT>
struct Seen {
  static constexpr int V = Elem<XT>::kVec;
  Stat st;
  u64 best;
  float best_v;  // NaN: every element is looked at
  __device__ __forceinline__ void clear() {
    st.clear();
    best = 0;
    best_v = __int_as_float(0x7fffffff);
  }
  __device__ __forceinline__ void piece(const float (&v)[V], int c0, float c) {
    float pm = v[0];
#pragma unroll
    for (int j = 1; j < V; ++j) pm = max_nan(pm, v[j]);
    if (!(pm <= best_v)) {
#pragma unroll
      for (int j = 0; j < V; ++j) best = max64(best, key_of(v[j], c0 + j));
      best_v = value_of(best);
    }
    if (pm > st.m) st.rebase(pm, c);
#pragma unroll
    for (int j = 0; j < V; ++j) st.add(v[j], c);
  }
  __device__ __forceinline__ void one(float v, int cl, float c) {
    best = max64(best, key_of(v, cl));
    best_v = value_of(best);
    if (v > st.m) st.rebase(v, c);
    st.add(v, c);
  }
  // piece i of a row, if there is one
  __device__ __forceinline__ void edge(const Row<XT>& row, int i, float c) {
    for (int j = 0; j < V; ++j) {
      const int cl = i * V - row.lead + j;
      if (cl >= 0 && cl < row.classes) one(row.at(cl), cl, c);
    }
  }
};

__device__ __forceinline__ void write_given(const Params& p, long long row, int j, const Stat& st, float log_s, float v, int id) {
  // (the logit is read by the caller where the class is one of the row's)
  p.given_lp[row * p.n_given + j] = id < 0 ? 0.0f : id >= p.classes ? __int_as_float(0x7fffffff) : log_prob(v, st, log_s, p.inv_t);
}
__device__ __forceinline__ void write_top(const Params& p, long long row, int j, u64 key, const Stat& st, float log_s) {
  p.top_ids[row * p.top + j] = class_of(key);
  p.top_lp[row * p.top + j] = log_prob(value_of(key), st, log_s, p.inv_t);
}

// ---------------------------------------------------------------- a CTA, or a cluster of them, for a row
constexpr int kThreads = 256, kWarps = 8;
constexpr int kGroups = 64;    // groups of 4 threads, whose largest elements bound the answer
constexpr int kFound = 1024;   // elements collected at a time

struct Shared {
  u64 group[kGroups];
  u64 found[kFound];
  u64 best[kMaxTop];     // this CTA's answer, largest first; 0: none
  Stat warp[kWarps], st;
  u64 bound;
  int n_win, n_found;
  int win[kMaxTop];
};

template <int XT>
__global__ void __launch_bounds__(kThreads) row_kernel(const Params p) {
  constexpr int V = Elem<XT>::kVec;
  extern __shared__ __align__(16) unsigned char raw_smem[];
  Shared& sh = *reinterpret_cast<Shared*>(raw_smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long r = blockIdx.x / p.ks;
  const int rank = blockIdx.x % p.ks;
  pdl_launch_dependents();
  pdl_wait();
  const Row<XT> row(p, r);
  const int stride = kThreads * p.ks, first = rank * kThreads + tid;
  // pieces of this thread: first, first + stride, ...; the row's first and last may be cut
  Seen<XT> seen;
  seen.clear();
  int i = first;
  if (i < row.pieces && !row.whole(i)) {
    seen.edge(row, i, p.c);
    i += stride;
  }
  for (; i + 3 * stride < row.pieces && row.whole(i + 3 * stride); i += 4 * stride) {
    uint4 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = row.raw(i + j * stride);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v[V];
      Row<XT>::convert(w[j], v);
      seen.piece(v, (i + j * stride) * V - row.lead, p.c);
    }
  }
  for (; i < row.pieces; i += stride) {
    if (row.whole(i)) {
      float v[V];
      Row<XT>::convert(row.raw(i), v);
      seen.piece(v, i * V - row.lead, p.c);
    } else {
      seen.edge(row, i, p.c);
    }
  }

  {
    const Stat st = warp_merge(seen.st, p.c, 32);
    if (lane == 0) sh.warp[warp] = st;
  }
  if (p.top) {
    u64 g = max64(seen.best, shfl_xor64(seen.best, 1));
    g = max64(g, shfl_xor64(g, 2));
    if ((tid & 3) == 0) sh.group[tid >> 2] = g;
    if (tid == 0) {
      sh.n_win = 0;
      sh.bound = 0;
    }
    if (tid < kMaxTop) sh.best[tid] = 0;
  }
  __syncthreads();
  if (tid == 0) {
    Stat st = sh.warp[0];
    for (int k = 1; k < kWarps; ++k) st.merge(sh.warp[k], p.c);
    sh.st = st;
  }
  if (p.top) {
    // the `top` groups whose largest elements lead (all with elements, where these are fewer), and the least of those
    if (tid < kGroups) {
      const u64 mine = sh.group[tid];
      int above = 0;
      for (int k = 0; k < kGroups; ++k) above += sh.group[k] > mine;
      if (mine && above < p.top) sh.win[atomicAdd(&sh.n_win, 1)] = tid;
      if (mine && above == p.top - 1) sh.bound = mine;
    }
    __syncthreads();
    u64 bound = sh.bound;
    for (;;) {
      if (tid == 0) sh.n_found = 0;
      __syncthreads();
      const float bound_v = value_of(bound);
      for (int k = warp; k < sh.n_win; k += kWarps) {
        // this group's pieces again: lane l takes those of thread l % 4
        for (int q = rank * kThreads + sh.win[k] * 4 + (lane & 3) + (lane >> 2) * stride; q < row.pieces; q += 8 * stride) {
          const int c0 = q * V - row.lead;
          if (row.whole(q)) {
            float v[V];
            Row<XT>::convert(row.raw(q), v);
#pragma unroll
            for (int j = 0; j < V; ++j) {
              if (bound && v[j] < bound_v) continue;
              const u64 key = key_of(v[j], c0 + j);
              if (key >= bound) {
                const int at = atomicAdd(&sh.n_found, 1);
                if (at < kFound) sh.found[at] = key;
              }
            }
          } else {
            for (int j = 0; j < V; ++j) {
              if (c0 + j < 0 || c0 + j >= row.classes) continue;
              const u64 key = key_of(row.at(c0 + j), c0 + j);
              if (key >= bound) {
                const int at = atomicAdd(&sh.n_found, 1);
                if (at < kFound) sh.found[at] = key;
              }
            }
          }
        }
      }
      __syncthreads();
      const int found = sh.n_found, n = min(found, kFound);
      // their order: an element's place is the number of larger ones
      for (int k = tid; k < n; k += kThreads) {
        const u64 mine = sh.found[k];
        int above = 0;
        for (int j = 0; j < n; ++j) above += sh.found[j] > mine;
        if (above < p.top) sh.best[above] = mine;
      }
      __syncthreads();
      if (found <= kFound) break;
      // more than fit (large elements at the same places of many pieces): the least of the leading ones found so far bounds the answer
      // more closely, and leaves out all but `top` of what was collected
      bound = sh.best[p.top - 1];
    }
  }
  if (p.ks > 1) {
    cluster_sync();
    if (rank == 0) {
      // the other CTAs' sums and answers, in the order of the CTAs
      const unsigned at = smem_u32(&sh);
      if (tid == 0) {
        Stat st = sh.st;
        for (int k = 1; k < p.ks; ++k) {
          const unsigned from = mapa_shared(at + static_cast<unsigned>(reinterpret_cast<unsigned char*>(&sh.st) - raw_smem), k);
          Stat o;
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o.m) : "r"(from) : "memory");
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o.s) : "r"(from + 4) : "memory");
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o.t) : "r"(from + 8) : "memory");
          st.merge(o, p.c);
        }
        sh.st = st;
      }
      const int n = p.ks * p.top;
      for (int k = tid; k < n; k += kThreads) {
        const unsigned from = mapa_shared(at + static_cast<unsigned>(reinterpret_cast<unsigned char*>(sh.best) - raw_smem) + (k % p.top) * 8, k / p.top);
        u64 v;
        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(from) : "memory");
        sh.found[k] = v;
      }
      __syncthreads();
      for (int k = tid; k < n; k += kThreads) {
        const u64 mine = sh.found[k];
        int above = 0;
        for (int j = 0; j < n; ++j) above += sh.found[j] > mine;
        if (mine && above < p.top) sh.best[above] = mine;
      }
      __syncthreads();
    }
  } else {
    __syncthreads();
  }
  if (rank == 0) {
    const Stat st = sh.st;
    const float log_s = logf(st.s);
    if (tid == 0 && p.entropy) p.entropy[r] = entropy_of(st, log_s);
    if (tid < p.top) write_top(p, r, tid, sh.best[tid], st, log_s);
    for (int j = tid; j < p.n_given; j += kThreads) {
      const int id = p.given[r * p.n_given + j];
      write_given(p, r, j, st, log_s, id >= 0 && id < p.classes ? row.at(id) : 0.0f, id);
    }
  }
  if (p.ks > 1) cluster_sync();  // nobody leaves while its shared memory is read
}

// ---------------------------------------------------------------- a warp for a row
constexpr int kWarpFound = 128;

template <int XT>
__global__ void __launch_bounds__(kThreads) warp_kernel(const Params p) {
  constexpr int V = Elem<XT>::kVec;
  __shared__ u64 found_all[kWarps][kWarpFound];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long r = static_cast<long long>(blockIdx.x) * kWarps + warp;
  pdl_launch_dependents();
  pdl_wait();
  if (r >= p.rows) return;
  u64* found = found_all[warp];
  const Row<XT> row(p, r);
  Seen<XT> seen;
  seen.clear();
  for (int i = lane; i < row.pieces; i += 32) {
    if (row.whole(i)) {
      float v[V];
      Row<XT>::convert(row.raw(i), v);
      seen.piece(v, i * V - row.lead, p.c);
    } else {
      seen.edge(row, i, p.c);
    }
  }
  const Stat st = warp_merge(seen.st, p.c, 32);
  const float log_s = logf(st.s);
  if (lane == 0 && p.entropy) p.entropy[r] = entropy_of(st, log_s);
  for (int j = lane; j < p.n_given; j += 32) {
    const int id = p.given[r * p.n_given + j];
    write_given(p, r, j, st, log_s, id >= 0 && id < p.classes ? row.at(id) : 0.0f, id);
  }
  if (p.top == 0) return;
  u64 mine = seen.best;
  if (p.top == 1) {
#pragma unroll
    for (int o = 16; o; o >>= 1) mine = max64(mine, shfl_xor64(mine, o));
    if (lane == 0) write_top(p, r, 0, mine, st, log_s);
    return;
  }
  // the least of the `top` leading lanes' largest elements bounds the answer
  int above = 0;
#pragma unroll
  for (int k = 0; k < 32; ++k) above += __shfl_sync(0xffffffffu, mine, k) > mine;
  const unsigned edge = __ballot_sync(0xffffffffu, mine != 0 && above == p.top - 1);
  const u64 bound = edge ? __shfl_sync(0xffffffffu, mine, __ffs(edge) - 1) : 0;
  // every lane's elements that reach it, lane by lane; as many as fit
  int n = 0;
  const bool look = mine != 0 && mine >= bound;
  const float bound_v = value_of(bound);
  for (int i = lane; __any_sync(0xffffffffu, i < row.pieces); i += 32) {
    const int c0 = i * V - row.lead;
    unsigned hits = 0;
    float v[V];
    if (look && i < row.pieces) {
      if (row.whole(i)) {
        Row<XT>::convert(row.raw(i), v);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (!(bound && v[j] < bound_v) && key_of(v[j], c0 + j) >= bound) hits |= 1u << j;
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (c0 + j >= 0 && c0 + j < row.classes) {
            v[j] = row.at(c0 + j);
            if (key_of(v[j], c0 + j) >= bound) hits |= 1u << j;
          }
      }
    }
    if (!__any_sync(0xffffffffu, hits != 0)) continue;
    // places for this round's, in the order of the lanes
    const int count = __popc(hits);
    int upto = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += u;
    }
    int at = n + upto - count;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (hits >> j & 1u) {
        if (at < kWarpFound) found[at] = key_of(v[j], c0 + j);
        ++at;
      }
    n += __shfl_sync(0xffffffffu, upto, 31);
  }
  __syncwarp();
  if (n <= kWarpFound) {
    for (int k = lane; k < n; k += 32) {
      const u64 key = found[k];
      int place = 0;
      for (int j = 0; j < n; ++j) place += found[j] > key;
      if (place < p.top) write_top(p, r, place, key, st, log_s);
    }
    return;
  }
  // more than fit: one after the other, each lane's largest element below the last one
  u64 last = ~0ull;
  for (int k = 0; k < p.top; ++k) {
    u64 best = 0;
    for (int i = lane; i < row.pieces; i += 32)
      for (int j = 0; j < V; ++j) {
        const int cl = i * V - row.lead + j;
        if (cl < 0 || cl >= row.classes) continue;
        const u64 key = key_of(row.at(cl), cl);
        if (key < last) best = max64(best, key);
      }
#pragma unroll
    for (int o = 16; o; o >>= 1) best = max64(best, shfl_xor64(best, o));
    if (lane == 0) write_top(p, r, k, best, st, log_s);
    last = best;
  }
}

// ---------------------------------------------------------------- a thread for a row of few classes
constexpr int kFew = 64;         // classes
constexpr int kThreadRows = 128; // rows of a CTA

template <int XT>
__global__ void __launch_bounds__(kThreadRows) thread_kernel(const Params p) {
  typedef typename Elem<XT>::type T;
  constexpr int V = Elem<XT>::kVec;
  extern __shared__ __align__(16) unsigned char raw_smem[];
  T* xs = reinterpret_cast<T*>(raw_smem);
  pdl_launch_dependents();
  pdl_wait();
  const long long r0 = static_cast<long long>(blockIdx.x) * kThreadRows;
  const int n = static_cast<int>(min(static_cast<long long>(kThreadRows), p.rows - r0));
  const T* x = static_cast<const T*>(p.x) + r0 * p.ld;
  int lead = 0;
  if (p.ld == p.classes) {
    // the rows are one run of memory: whole pieces of it, and what lies at its ends by elements
    lead = static_cast<int>(reinterpret_cast<unsigned long long>(x) / sizeof(T) % V);
    const int total = n * p.classes, pieces = (lead + total + V - 1) / V;
    for (int i = threadIdx.x; i < pieces; i += kThreadRows) {
      const int e = i * V - lead;
      if (e >= 0 && e + V <= total) {
        *reinterpret_cast<uint4*>(xs + i * V) = __ldg(reinterpret_cast<const uint4*>(x + e));
      } else {
        for (int j = 0; j < V; ++j)
          if (e + j >= 0 && e + j < total) xs[i * V + j] = x[e + j];
      }
    }
  } else {
    for (int k = threadIdx.x; k < n * p.classes; k += kThreadRows) {
      const int row = k / p.classes;
      xs[k] = x[row * p.ld + (k - row * p.classes)];
    }
  }
  __syncthreads();
  if (static_cast<int>(threadIdx.x) >= n) return;
  const T* mine = xs + lead + threadIdx.x * p.classes;
  const long long r = r0 + threadIdx.x;
  Stat st;
  st.clear();
  float high = Elem<XT>::f32(mine[0]);
  int where = 0;
  bool nan = high != high;
  for (int j = 1; j < p.classes; ++j) {
    const float v = Elem<XT>::f32(mine[j]);
    if (v > high || (v != v && !nan)) {  // the first NaN leads, as in key_of
      high = v;
      where = j;
      nan = v != v;
    }
  }
  st.m = high > kLowest ? high : kLowest;  // (also where it is a NaN: the sums become one)
  for (int j = 0; j < p.classes; ++j) st.add(Elem<XT>::f32(mine[j]), p.c);
  const float log_s = logf(st.s);
  if (p.entropy) p.entropy[r] = entropy_of(st, log_s);
  for (int j = 0; j < p.n_given; ++j) {
    const int id = p.given[r * p.n_given + j];
    write_given(p, r, j, st, log_s, id >= 0 && id < p.classes ? Elem<XT>::f32(mine[id]) : 0.0f, id);
  }
  if (p.top == 0) return;
  u64 last = key_of(high, where);
  write_top(p, r, 0, last, st, log_s);
  for (int k = 1; k < p.top; ++k) {
    u64 best = 0;
    for (int j = 0; j < p.classes; ++j) {
      const u64 key = key_of(Elem<XT>::f32(mine[j]), j);
      if (key < last) best = max64(best, key);
    }
    write_top(p, r, k, best, st, log_s);
    last = best;
  }
}

template <int XT>
cudaError_t launch_type(Params& p, cudaStream_t stream) {
  constexpr int V = Elem<XT>::kVec;
  const int sms = device_sm_count();
  if (p.classes <= kFew && p.rows >= 4096) {
    const unsigned grid = static_cast<unsigned>((static_cast<long long>(p.rows) + kThreadRows - 1) / kThreadRows);
    return launch_pdl(thread_kernel<XT>, dim3(grid), dim3(kThreadRows), (kThreadRows * p.classes + 2 * V) * sizeof(typename Elem<XT>::type), stream, p);
  }
  if (p.classes <= 2048) {
    const unsigned grid = static_cast<unsigned>((static_cast<long long>(p.rows) + kWarps - 1) / kWarps);
    return launch_pdl(warp_kernel<XT>, dim3(grid), dim3(kThreads), 0, stream, p);
  }
  p.ks = 1;
  while (p.ks < 16 && static_cast<long long>(p.rows) * p.ks < 4 * sms && p.classes / V >= 2 * kThreads * p.ks) p.ks *= 2;
  static bool raised[kMaxDevices] = {};
  bool& done = raised[current_device_slot()];
  if (!done) {
    const cudaError_t err = cudaFuncSetAttribute(row_kernel<XT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (err != cudaSuccess) return err;
    done = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(static_cast<long long>(p.rows) * p.ks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Shared);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(p.ks);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.ks > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, row_kernel<XT>, static_cast<const Params>(p));
}

}  // namespace

int launch_log_probs(const LogProbsCall& c, void* stream) {
  if (c.rows <= 0) return 0;
  Params p{};
  p.x = c.x;
  p.given = c.given;
  p.given_lp = c.given_lp;
  p.entropy = c.entropy;
  p.top_ids = c.top_ids;
  p.top_lp = c.top_lp;
  p.ld = c.ld;
  p.rows = c.rows;
  p.classes = c.classes;
  p.n_given = c.n_given;
  p.top = c.top;
  p.inv_t = 1.0f / c.temperature;
  p.c = p.inv_t * kLog2e;
  p.ks = 1;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (c.dtype) {
    case GI_F16: return static_cast<int>(launch_type<GI_F16>(p, st));
    case GI_BF16: return static_cast<int>(launch_type<GI_BF16>(p, st));
    default: return static_cast<int>(launch_type<GI_F32>(p, st));
  }
}

}  // namespace gi
