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
// Measured (B200): 2048 x 131072 fp16 125 us (4.3 TB/s), without `top` 111 us (4.9); 50000 x 3000 152 us, without `top` 74; 4.2 M rows of
// 21 classes 87 us (3.0), of 16 97, of 32 299, of 64 1017 (rows an even number of 32-bit words apart meet in the same banks of shared
// memory); 1 x 262144 fp32 10 us, 1 x 1001 5 us.
//
// Three shapes: a thread a row for a handful of classes (every pixel of a segmentation), a warp a row (few classes, or many rows), a CTA a row - or a cluster
// of up to 8 CTAs, where rows are few: they read one row together and join through distributed shared memory, in a fixed order.
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
// d is bounded from below, where 2^d is 0, so that no infinity is multiplied by it; a NaN comes through
constexpr float kNothing = -1000.0f;
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

template <int XT>
struct Elem;
template <>
struct Elem<GI_F16> {
  typedef __half type;
  static constexpr int kVec = 8;
  static __device__ __forceinline__ __half none() { return __ushort_as_half(0xfc00); }
  static __device__ __forceinline__ float f32(__half v) { return __half2float(v); }
  static __device__ __forceinline__ float most(const uint4& w) {  // the largest of 16 bytes, a NaN if there is one
    const __half2* h = reinterpret_cast<const __half2*>(&w);
    const float2 m = __half22float2(__hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
    return max_nan(m.x, m.y);
  }
};
template <>
struct Elem<GI_BF16> {
  typedef __nv_bfloat16 type;
  static constexpr int kVec = 8;
  static __device__ __forceinline__ __nv_bfloat16 none() { return __ushort_as_bfloat16(0xff80); }
  static __device__ __forceinline__ float f32(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ float most(const uint4& w) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&w);
    const float2 m = __bfloat1622float2(__hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
    return max_nan(m.x, m.y);
  }
};
template <>
struct Elem<GI_F32> {
  typedef float type;
  static constexpr int kVec = 4;
  static __device__ __forceinline__ float none() { return -INFINITY; }
  static __device__ __forceinline__ float f32(float v) { return v; }
  static __device__ __forceinline__ float most(const uint4& w) {
    return max_nan(max_nan(__uint_as_float(w.x), __uint_as_float(w.y)), max_nan(__uint_as_float(w.z), __uint_as_float(w.w)));
  }
};

// A value's bits as a whole number of the same order; a NaN above all values, -0 as 0.  (One NaN's bits stand for all: with a class
// beside them they are still below the whole numbers that a search for the next smaller key starts from.)
__device__ __forceinline__ int ordered(float v) {
  int b = __float_as_int(v + 0.0f);
  if (v != v) b = 0x7fc00000;
  return b ^ ((b >> 31) & 0x7fffffff);
}
// that above the inverted class: larger values first, then lower classes
__device__ __forceinline__ u64 key_of(float v, int i) {
  return (static_cast<u64>(static_cast<unsigned>(ordered(v)) ^ 0x80000000u) << 32) | (0xffffffffu - static_cast<unsigned>(i));
}
__device__ __forceinline__ int class_of(u64 k) { return static_cast<int>(0xffffffffu - static_cast<unsigned>(k)); }
__device__ __forceinline__ float value_of(u64 k) {
  const int o = static_cast<int>(static_cast<unsigned>(k >> 32) ^ 0x80000000u);
  return __int_as_float(o ^ ((o >> 31) & 0x7fffffff));
}
__device__ __forceinline__ u64 max64(u64 a, u64 b) { return a > b ? a : b; }
__device__ __forceinline__ u64 shfl_xor64(u64 v, int m) { return __shfl_xor_sync(0xffffffffu, v, m); }

// two fp32 numbers in a register pair: one instruction for both
__device__ __forceinline__ u64 pack2(float a, float b) {
  u64 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(u64 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ u64 add2(u64 a, u64 b) {
  u64 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ u64 mul2(u64 a, u64 b) {
  u64 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) {
  u64 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// Sums relative to a maximum m: s = sum 2^d, t = sum 2^d d with d = (x - m) c.
struct Stat {
  float m, s, t;
  // to a new maximum: every d grows by e = (m - to) c <= 0
  __device__ __forceinline__ void rebase(float to, float c) {
    const float e = fmaxf((m - to) * c, -1.0e30f), f = ex2(e);
    t = f * (t + e * s);  // (s = 0 where nothing was seen: 0 again)
    s *= f;
    m = to;
  }
};

// the sums of the lanes of every group of `width`: one change of maximum, then sums that come out the same in every lane
__device__ __forceinline__ Stat warp_merge(Stat st, float c, int width) {
  float m = st.m;
  for (int o = 1; o < width; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  st.rebase(m, c);
  for (int o = 1; o < width; o <<= 1) {
    st.s += __shfl_xor_sync(0xffffffffu, st.s, o);
    st.t += __shfl_xor_sync(0xffffffffu, st.t, o);
  }
  return st;
}

// log p of a logit, given a row's sums: minus infinity in a row in which nothing is left
template <int XT>
__device__ __forceinline__ float log_prob(float v, const Stat& st, float log_s, float inv_t) {
  if (st.s == 0.0f) return -INFINITY;
  float d = (v - st.m) * inv_t;
  // two numbers whose difference is none in fp32: halves of them, which the temperature may bring back into its range
  if (XT != GI_F16 && d == -INFINITY) d = 2.0f * ((0.5f * v - 0.5f * st.m) * inv_t);
  return d - log_s;
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
  // piece i; beside the row, and where there is no such piece, minus infinity: that adds nothing to a sum
  __device__ __forceinline__ uint4 piece(int i) const {
    if (whole(i)) return raw(i);
    uint4 w;
    T* e = reinterpret_cast<T*>(&w);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int cl = i * V - lead + j;
      e[j] = cl >= 0 && cl < classes ? x[cl] : Elem<XT>::none();
    }
    return w;
  }
};

// What a thread has seen of a row: sums, two at a time, and its largest element - as the first of the 16-byte pieces that hold a
// largest one (looking for the element at every new maximum, which some lane of a warp meets at almost every piece, took two thirds
// of the instructions).
template <int XT>
struct Seen {
  static constexpr int V = Elem<XT>::kVec;
  float m;
  u64 s, t;
  int most;    // ordered bits of the largest element of whole pieces; below all of them at first
  uint4 where; // it
  int at;      // class of its first element
  __device__ __forceinline__ void clear() {
    m = kLowest;
    s = t = 0;
    most = static_cast<int>(0x80000000u);
    where = make_uint4(0u, 0u, 0u, 0u);
    at = 0;
  }
  __device__ __forceinline__ void grow(float to, float c) {
    if (!(to > m)) return;
    const float e = fmaxf((m - to) * c, -1.0e30f), f = ex2(e);
    t = mul2(fma2(pack2(e, e), s, t), pack2(f, f));
    s = mul2(s, pack2(f, f));
    m = to;
  }
  // N pieces, their first elements' classes `step` apart
  template <int N>
  __device__ __forceinline__ void pieces(const uint4 (&w)[N], int c0, int step, float c) {
    float pm[N], top;
#pragma unroll
    for (int j = 0; j < N; ++j) pm[j] = Elem<XT>::most(w[j]);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int o = ordered(pm[j]);
      if (o > most) {
        most = o;
        where = w[j];
        at = c0 + j * step;
      }
    }
    top = pm[0];
#pragma unroll
    for (int j = 1; j < N; ++j) top = max_nan(top, pm[j]);
    grow(top, c);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float v[V];
      Row<XT>::convert(w[j], v);
      add(v, c);
    }
  }
  __device__ __forceinline__ void add(const float (&v)[V], float c) {
    const u64 minus = pack2(-m, -m), c2 = pack2(c, c);
#pragma unroll
    for (int k = 0; k < V; k += 2) {
      float d0, d1;
      unpack2(mul2(add2(pack2(v[k], v[k + 1]), minus), c2), d0, d1);
      d0 = max_nan(d0, kNothing);
      d1 = max_nan(d1, kNothing);
      const u64 e = pack2(ex2(d0), ex2(d1));
      s = add2(s, e);
      t = fma2(e, pack2(d0, d1), t);
    }
  }
  // the pieces first, first + stride, ... of a row, N requested at a time
  template <int N>
  __device__ __forceinline__ void walk(const Row<XT>& row, int first, int stride, float c) {
    for (int i = first; i < row.pieces; i += N * stride) {
      uint4 w[N];
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = row.piece(i + j * stride);
      pieces(w, i * V - row.lead, stride * V, c);
    }
  }
  __device__ __forceinline__ Stat stat() const {
    Stat st;
    float a, b;
    st.m = m;
    unpack2(s, a, b);
    st.s = a + b;
    unpack2(t, a, b);
    st.t = a + b;
    return st;
  }
  __device__ __forceinline__ u64 best(const Row<XT>& row) const {
    u64 k = 0;
    if (most != static_cast<int>(0x80000000u)) {
      float v[V];
      Row<XT>::convert(where, v);
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (at + j >= 0 && at + j < row.classes) k = max64(k, key_of(v[j], at + j));
    }
    return k;
  }
};

template <int XT>
__device__ __forceinline__ void write_given(const Params& p, long long row, int j, const Stat& st, float log_s, float v, int id) {
  // (the logit is read by the caller where the class is one of the row's)
  p.given_lp[row * p.n_given + j] = id < 0 ? 0.0f : id >= p.classes ? __int_as_float(0x7fffffff) : log_prob<XT>(v, st, log_s, p.inv_t);
}
template <int XT>
__device__ __forceinline__ void write_top(const Params& p, long long row, int j, u64 key, const Stat& st, float log_s) {
  p.top_ids[row * p.top + j] = class_of(key);
  p.top_lp[row * p.top + j] = log_prob<XT>(value_of(key), st, log_s, p.inv_t);
}

// ---------------------------------------------------------------- a CTA, or a cluster of them, for a row
constexpr int kGroups = 64;    // groups of threads, whose largest elements bound the answer
constexpr int kFound = 1024;   // elements collected at a time
constexpr int kMostWarps = 32;

struct Shared {
  alignas(16) u64 group[kGroups];
  u64 found[kFound];
  u64 kept[kMaxTop * (kFound / kGroups)];  // the ones that a second bound leaves of them
  u64 best[kMaxTop];     // this CTA's answer, largest first; 0: none
  Stat warp[kMostWarps], st;
  u64 bound;
  int n_win, n_found, n_kept;
  int win[kMaxTop];
};

// T: threads of a CTA.
template <int XT, int T>
__global__ void __launch_bounds__(T) row_kernel(const Params p) {
  constexpr int kThreads = T, kWarps = T / 32, kWidth = T / kGroups;
  constexpr int V = Elem<XT>::kVec;
  extern __shared__ __align__(16) unsigned char raw_smem[];
  Shared& sh = *reinterpret_cast<Shared*>(raw_smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = blockIdx.x % p.ks;
  const long long r = blockIdx.x / p.ks;
  const int stride = kThreads * p.ks, first = rank * kThreads + tid;
  pdl_launch_dependents();
  pdl_wait();
  const Row<XT> row(p, r);
  // the classes asked for, and their logits: two requests one after the other, answered while the row is read
  int id0 = -1;
  float given0 = 0.0f;
  if (rank == 0 && tid < p.n_given) {
    id0 = p.given[r * p.n_given + tid];
    if (id0 >= 0 && id0 < p.classes) given0 = row.at(id0);
  }
  // pieces of this thread: first, first + stride, ...; the row's first and last may be cut
  Seen<XT> seen;
  seen.clear();
  seen.template walk<4>(row, first, stride, p.c);
  {
    const Stat st = warp_merge(seen.stat(), p.c, 32);
    if (lane == 0) sh.warp[warp] = st;
  }
  if (p.top) {
    u64 g = seen.best(row);
#pragma unroll
    for (int o = 1; o < kWidth; o <<= 1) g = max64(g, shfl_xor64(g, o));
    if (tid % kWidth == 0) sh.group[tid / kWidth] = g;
    if (tid == 0) {
      sh.n_win = sh.n_found = 0;
      sh.bound = 0;
    }
    if (tid < kMaxTop) sh.best[tid] = 0;
  }
  __syncthreads();
  if (warp == kWarps - 1) {
    const Stat st = warp_merge(sh.warp[lane % kWarps], p.c, kWarps);
    if (lane == 0) sh.st = st;
  }
  if (p.top) {
    // the `top` groups whose largest elements lead (all with elements, where these are fewer), and the least of those
    if (tid < kGroups) {
      const u64 mine = sh.group[tid];
      int above = 0;
#pragma unroll 8
      for (int k = 0; k < kGroups; k += 2) {
        const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(&sh.group[k]);
        above += (two.x > mine) + (two.y > mine);
      }
      if (mine && above < p.top) sh.win[atomicAdd(&sh.n_win, 1)] = tid;
      if (mine && above == p.top - 1) sh.bound = mine;
    }
    __syncthreads();
    u64 bound = sh.bound;
    for (;;) {
      const float bound_v = value_of(bound);
      for (int k = warp; k < sh.n_win; k += kWarps) {
        // this group's pieces again, its threads' side by side
        for (int q = rank * kThreads + sh.win[k] * kWidth + lane % kWidth + lane / kWidth * stride; q < row.pieces; q += 32 / kWidth * stride) {
          const int c0 = q * V - row.lead;
          float v[V];
          Row<XT>::convert(row.piece(q), v);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            if ((bound && v[j] < bound_v) || c0 + j < 0 || c0 + j >= row.classes) continue;
            const u64 key = key_of(v[j], c0 + j);
            if (key >= bound) {
              const int at = atomicAdd(&sh.n_found, 1);
              if (at < kFound) sh.found[at] = key;
            }
          }
        }
      }
      __syncthreads();
      const int found = sh.n_found;
      int n = min(found, kFound);
      const u64* list = sh.found;
      if (n > 2 * kGroups) {
        // many (equal ones, as in a row of which nothing is left): the same bound once more, from 64 shares of what was found
        if (tid < kGroups) {
          u64 m = 0;
          for (int k = tid; k < n; k += kGroups) m = max64(m, sh.found[k]);
          sh.group[tid] = m;
        }
        if (tid == 0) sh.n_kept = 0;
        __syncthreads();
        if (tid < kGroups) {
          const u64 mine = sh.group[tid];
          int above = 0;
          for (int k = 0; k < kGroups; ++k) above += sh.group[k] > mine;
          if (above == p.top - 1) sh.bound = mine;
        }
        __syncthreads();
        for (int k = tid; k < n; k += kThreads)
          if (sh.found[k] >= sh.bound) sh.kept[atomicAdd(&sh.n_kept, 1)] = sh.found[k];
        __syncthreads();
        n = sh.n_kept;
        list = sh.kept;
      }
      // their order: an element's place is the number of larger ones
      for (int k = tid; k < n; k += kThreads) {
        const u64 mine = list[k];
        int above = 0;
        for (int j = 0; j < n; ++j) above += list[j] > mine;
        if (above < p.top) sh.best[above] = mine;
      }
      __syncthreads();
      if (found <= kFound) break;
      // more than fit (large elements at the same places of many pieces): the least of the leading ones found so far bounds the answer
      // more closely, and leaves out all but `top` of what was collected
      bound = sh.best[p.top - 1];
      __syncthreads();
      if (tid == 0) sh.n_found = 0;
      __syncthreads();
    }
  }
  if (p.ks > 1) {
    cluster_sync();
    if (rank == 0) {
      // the other CTAs' sums and answers, in the order of the CTAs
      const unsigned at = smem_u32(&sh);
      if (warp == kWarps - 1) {
        const unsigned from = mapa_shared(at + static_cast<unsigned>(reinterpret_cast<unsigned char*>(&sh.st) - raw_smem), lane % p.ks);
        Stat st;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(st.m) : "r"(from) : "memory");
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(st.s) : "r"(from + 4) : "memory");
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(st.t) : "r"(from + 8) : "memory");
        st = warp_merge(st, p.c, p.ks);
        __syncwarp();
        if (lane == 0) sh.st = st;  // (nobody else reads this CTA's)
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
    if (tid < p.top) write_top<XT>(p, r, tid, sh.best[tid], st, log_s);
    if (tid < p.n_given) write_given<XT>(p, r, tid, st, log_s, given0, id0);
    for (int j = tid + kThreads; j < p.n_given; j += kThreads) {
      const int id = p.given[r * p.n_given + j];
      write_given<XT>(p, r, j, st, log_s, id >= 0 && id < p.classes ? row.at(id) : 0.0f, id);
    }
  }
  if (p.ks > 1) cluster_sync();  // nobody leaves while its shared memory is read
}

// ---------------------------------------------------------------- a warp for a row
constexpr int kThreads = 256, kWarps = 8;
constexpr int kWarpFound = 256;  // (fewer pieces than lanes, all of whose elements may have to be looked at, hold at most 248)

// N: pieces that a lane requests at a time.
template <int XT, int N>
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
  int id0 = -1;
  float given0 = 0.0f;
  if (lane < p.n_given) {
    id0 = p.given[r * p.n_given + lane];
    if (id0 >= 0 && id0 < p.classes) given0 = row.at(id0);
  }
  Seen<XT> seen;
  seen.clear();
  seen.template walk<N>(row, lane, 32, p.c);
  const Stat st = warp_merge(seen.stat(), p.c, 32);
  const float log_s = logf(st.s);
  if (lane == 0 && p.entropy) p.entropy[r] = entropy_of(st, log_s);
  if (lane < p.n_given) write_given<XT>(p, r, lane, st, log_s, given0, id0);
  for (int j = lane + 32; j < p.n_given; j += 32) {
    const int id = p.given[r * p.n_given + j];
    write_given<XT>(p, r, j, st, log_s, id >= 0 && id < p.classes ? row.at(id) : 0.0f, id);
  }
  if (p.top == 0) return;
  if (p.top == 1) {
    u64 mine = seen.best(row);
#pragma unroll
    for (int o = 16; o; o >>= 1) mine = max64(mine, shfl_xor64(mine, o));
    if (lane == 0) write_top<XT>(p, r, 0, mine, st, log_s);
    return;
  }
  // The least of the `top` leading lanes' largest values bounds the answer from below (equal values count together); a lane without
  // elements has the least of all, which every element reaches.
  int above = 0;
#pragma unroll
  for (int k = 0; k < 32; ++k) above += __shfl_sync(0xffffffffu, seen.most, k) > seen.most;
  const int bound = __reduce_min_sync(0xffffffffu, above < p.top ? seen.most : 0x7fffffff);
  // every lane's elements that reach it; as many as fit
  int n = 0;
  const unsigned before = (1u << lane) - 1u;
  for (int i = lane; __any_sync(0xffffffffu, i < row.pieces); i += 32) {
    const int c0 = i * V - row.lead;
    bool look = i < row.pieces && seen.most >= bound;
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (look) {
      w = row.piece(i);
      look = ordered(Elem<XT>::most(w)) >= bound;
    }
    if (!__any_sync(0xffffffffu, look)) continue;  // (most pieces)
    float v[V];
    Row<XT>::convert(w, v);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const bool hit = look && ordered(v[j]) >= bound && c0 + j >= 0 && c0 + j < row.classes;
      const unsigned hits = __ballot_sync(0xffffffffu, hit);
      if (!hits) continue;
      const int at = n + __popc(hits & before);
      if (hit && at < kWarpFound) found[at] = key_of(v[j], c0 + j);
      n += __popc(hits);
    }
  }
  __syncwarp();
  if (n <= kWarpFound) {
    // an element's place is the number of larger ones
    for (int k = lane; k < n; k += 32) {
      const u64 key = found[k];
      int place = 0;
      for (int j = 0; j < n; ++j) place += found[j] > key;
      if (place < p.top) write_top<XT>(p, r, place, key, st, log_s);
    }
    return;
  }
  // more than fit (many equal ones): one after the other, each lane's largest element below the last one
  u64 last = ~0ull;
  for (int k = 0; k < p.top; ++k) {
    u64 best = 0;
    for (int i = lane; i < row.pieces; i += 32) {
      float v[V];
      Row<XT>::convert(row.piece(i), v);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int cl = i * V - row.lead + j;
        const u64 key = key_of(v[j], cl);
        if (cl >= 0 && cl < row.classes && key < last) best = max64(best, key);
      }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) best = max64(best, shfl_xor64(best, o));
    if (lane == 0) write_top<XT>(p, r, k, best, st, log_s);
    last = best;
  }
}

// ---------------------------------------------------------------- a thread for a row of few classes
constexpr int kFew = 64;         // classes
constexpr int kThreadRows = 128; // rows of a CTA

// LEAST, MOST: the fewest and the most classes.
template <int XT, int LEAST, int MOST>
__global__ void __launch_bounds__(kThreadRows) thread_kernel(const Params p) {
  typedef typename Elem<XT>::type T;
  constexpr int V = Elem<XT>::kVec;
  extern __shared__ __align__(16) unsigned char raw_smem[];
  const int buffer = kThreadRows * p.classes + 2 * V;  // elements
  const long long tiles = (static_cast<long long>(p.rows) + kThreadRows - 1) / kThreadRows;
  // the rows of a tile into one of two buffers; the elements in front of the first one's, where they are copied by whole pieces
  auto fetch = [&](long long tile, int which) {
    T* xs = reinterpret_cast<T*>(raw_smem) + which * buffer;
    const long long r0 = tile * kThreadRows;
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
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(xs + i * V)), "l"(x + e) : "memory");
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
    asm volatile("cp.async.commit_group;" ::: "memory");
    return lead;
  };
  pdl_launch_dependents();
  pdl_wait();
  int lead = fetch(blockIdx.x, 0);
  int id = -1;  // the first class asked for
  if (p.n_given && static_cast<long long>(blockIdx.x) * kThreadRows + threadIdx.x < p.rows)
    id = p.given[(static_cast<long long>(blockIdx.x) * kThreadRows + threadIdx.x) * p.n_given];
  for (long long tile = blockIdx.x, which = 0; tile < tiles; tile += gridDim.x, which ^= 1) {
  const long long next = tile + gridDim.x, r = tile * kThreadRows + threadIdx.x;
  int next_lead = 0, next_id = -1;
  __syncthreads();  // the other buffer has been read
  if (next < tiles) {
    next_lead = fetch(next, static_cast<int>(which ^ 1));
    if (p.n_given && next * kThreadRows + threadIdx.x < p.rows) next_id = p.given[(next * kThreadRows + threadIdx.x) * p.n_given];
    asm volatile("cp.async.wait_group 1;" ::: "memory");
  } else {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  }
  __syncthreads();
  if (r < p.rows) {
  const T* mine = reinterpret_cast<const T*>(raw_smem) + which * buffer + lead + threadIdx.x * p.classes;
  // the row in registers; behind its last class minus infinity, which adds nothing and, as a later class, leads nothing
  float v[MOST];
#pragma unroll
  for (int j = 0; j < MOST; ++j) v[j] = j < LEAST || j < p.classes ? Elem<XT>::f32(mine[j]) : -INFINITY;
  float high = v[0];
#pragma unroll
  for (int j = 1; j < MOST; ++j) high = max_nan(high, v[j]);
  Stat st;
  st.m = high > kLowest ? high : kLowest;  // (also where it is a NaN: the sums become one)
  u64 s = 0, t = 0;
  const u64 minus = pack2(-st.m, -st.m), c2 = pack2(p.c, p.c);
#pragma unroll
  for (int j = 0; j < MOST; j += 2) {
    float d0, d1;
    unpack2(mul2(add2(pack2(v[j], v[j + 1]), minus), c2), d0, d1);
    d0 = max_nan(d0, kNothing);
    d1 = max_nan(d1, kNothing);
    const u64 e = pack2(ex2(d0), ex2(d1));
    s = add2(s, e);
    t = fma2(e, pack2(d0, d1), t);
  }
  float a, b;
  unpack2(s, a, b);
  st.s = a + b;
  unpack2(t, a, b);
  st.t = a + b;
  const float log_s = logf(st.s);
  if (p.entropy) p.entropy[r] = entropy_of(st, log_s);
  for (int j = 0; j < p.n_given; ++j) {
    if (j) id = p.given[r * p.n_given + j];
    write_given<XT>(p, r, j, st, log_s, id >= 0 && id < p.classes ? Elem<XT>::f32(mine[id]) : 0.0f, id);
  }
  if (p.top) {
  int where = 0;  // the first of the largest
#pragma unroll
  for (int j = MOST - 1; j >= 0; --j) where = v[j] == high ? j : where;
  if (high != high) {  // or the first NaN
#pragma unroll
    for (int j = MOST - 1; j >= 0; --j) where = v[j] != v[j] ? j : where;
  }
  p.top_ids[r * p.top] = where;
  p.top_lp[r * p.top] = log_prob<XT>(high, st, log_s, p.inv_t);
  if (p.top > 1) {
  if (XT != GI_F32) {
    // the ordered bits of a value of 16 bits leave at least 13 low ones to themselves: the class goes there
    int key[MOST];
#pragma unroll
    for (int j = 0; j < MOST; ++j) key[j] = j < p.classes ? (ordered(v[j]) & ~(kFew - 1)) | (kFew - 1 - j) : static_cast<int>(0x80000000u);
    int last = 0x7fffffff;
    for (int k = 0; k < p.top; ++k) {
      int best = static_cast<int>(0x80000000u);
#pragma unroll
      for (int j = 0; j < MOST; ++j) best = max(best, key[j] < last ? key[j] : static_cast<int>(0x80000000u));
      const int id = kFew - 1 - (best & (kFew - 1));
      p.top_ids[r * p.top + k] = id;
      p.top_lp[r * p.top + k] = log_prob<XT>(Elem<XT>::f32(mine[id]), st, log_s, p.inv_t);
      last = best;
    }
  } else {
    u64 last = key_of(high, where);
    for (int k = 1; k < p.top; ++k) {
      u64 best = 0;
      for (int j = 0; j < p.classes; ++j) {
        const u64 key = key_of(Elem<XT>::f32(mine[j]), j);
        if (key < last) best = max64(best, key);
      }
      write_top<XT>(p, r, k, best, st, log_s);
      last = best;
    }
  }
  }
  }
  }
  lead = next_lead;
  id = next_id;
  }
}

template <int XT>
cudaError_t launch_type(Params& p, cudaStream_t stream) {
  constexpr int V = Elem<XT>::kVec;
  const int sms = device_sm_count();
  if (p.classes <= kFew && p.rows >= 4096) {
    const unsigned grid = static_cast<unsigned>(std::min<long long>((static_cast<long long>(p.rows) + kThreadRows - 1) / kThreadRows, 8 * sms));
    const size_t smem = 2 * (kThreadRows * p.classes + 2 * V) * sizeof(typename Elem<XT>::type);
    void (*k)(const Params) = p.classes <= 8    ? thread_kernel<XT, 1, 8>
                              : p.classes <= 16 ? thread_kernel<XT, 9, 16>
                              : p.classes <= 24 ? thread_kernel<XT, 17, 24>
                              : p.classes <= 40 ? thread_kernel<XT, 25, 40>
                                                : thread_kernel<XT, 41, kFew>;
    if (smem > 48 * 1024) {
      // (only the kernel of the most classes comes here.  Its limit is raised once, to the most that any call needs: other threads' calls
      // of other sizes may lie between this line and the launch.)
      static bool raised[kMaxDevices] = {};
      bool& done = raised[current_device_slot()];
      if (!done) {
        const cudaError_t err = cudaFuncSetAttribute(thread_kernel<XT, 41, kFew>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                     static_cast<int>(2 * (kThreadRows * kFew + 2 * V) * sizeof(typename Elem<XT>::type)));
        if (err != cudaSuccess) return err;
        done = true;
      }
    }
    return launch_pdl(k, dim3(grid), dim3(kThreadRows), smem, stream, static_cast<const Params>(p));
  }
  // A warp a row: few classes, or enough rows to fill the GPU with warps (fp16, top 5: 5000 x 5000 31 us, with a CTA a row 45; 50000 x
  // 3000 146 and 452; but 1200 x 5000 17 and 14, 20000 x 10000 fp32 340 and 220).
  if (p.classes <= 2048 || (p.classes / V <= 1024 && p.rows >= 16 * sms)) {
    const unsigned grid = static_cast<unsigned>((static_cast<long long>(p.rows) + kWarps - 1) / kWarps);
    void (*k)(const Params) = p.classes <= 32 * V ? warp_kernel<XT, 1> : p.classes <= 64 * V ? warp_kernel<XT, 2> : warp_kernel<XT, 4>;
    return launch_pdl(k, dim3(grid), dim3(kThreads), 0, stream, static_cast<const Params>(p));
  }
  // Few rows of many classes: CTAs of 1024 threads, and clusters of CTAs, as long as a thread has three pieces to read (1 x 262144
  // fp32 9.7 us with 8 CTAs of 1024, 13.4 of 256; 64 x 50257 bf16 9.2 with 2, 10.6 with 8 of 256; 16 x 131072 fp16 8.6 with 4, 16.0
  // with 8; 1 x 32000 5.2 with 4 of 256, 6.4 with one, 8.5 with 4 of 1024; 2048 x 131072 124 with one of 256, 205 of 1024).
  const int pieces = p.classes / V;
  const bool few = p.rows * 2 <= sms && pieces >= 6 * 1024;
  const int threads = few ? 1024 : 256;
  void (*k)(const Params) = few ? row_kernel<XT, 1024> : row_kernel<XT, 256>;
  p.ks = 1;
  while (p.ks < 8 && static_cast<long long>(p.rows) * p.ks * 2 <= (few ? sms : 2 * sms) && pieces >= 3 * threads * p.ks * 2) p.ks *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(static_cast<long long>(p.rows) * p.ks));
  cfg.blockDim = dim3(threads);
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
  return cudaLaunchKernelEx(&cfg, k, static_cast<const Params>(p));
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
