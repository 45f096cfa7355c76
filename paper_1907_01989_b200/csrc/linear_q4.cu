// Fully connected layer (1x1 convolution) with 4-bit weights: y = act(x w^T + bias), w[o, k] = s[o, k / group] (q[o, k] - z[o, k / group]),
// q and z whole numbers of 0 .. 15.
//
// What bounds it: for few rows of x the bytes of the weights, half a byte each - so the kernel is built around reading them once, in
// whole 512-byte warp loads that are requested a batch ahead, and around spending less than the 2.8 instructions a weight that an SM
// has at the rate at which its share of the memory's bandwidth delivers them.  q - z is exact in fp16 and in bf16: eight weights are
// taken out of a word by five logical operations (q becomes the low digits of 1024 or 128) and four subtractions, and go into
// mma.sync.m16n8k16 as the A operand, the rows of x being the 8 columns.  Sums are fp32 for each group of input channels and are
// scaled in fp32: nothing of a weight is rounded.  tcgen05 wants 128 x 8 tiles with A in shared or tensor memory: here one store
// and one transfer more for each weight, for products that take a tenth of the time the weights' bytes take.
//
// x in 32 bits: a value is the exact sum of three bf16 numbers (8 + 8 + 8 digits), so a row of x becomes three columns of the product.
//
// Layout of the packed weights (host: linear_q4_pack): units of 16 outputs x 64 input channels, 512 bytes, lane l = 4 g + t of a
// warp reads 16 of them: rows g and g + 8, channels 32 h + 8 t + 0 .. 7 of both halves h; the units of 16 outputs follow one
// another along the input channels.  A lane's eight channels are contiguous in x, so x needs no rearrangement either.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstring>

#include "kernels.h"
#include "mma_frag.cuh"
#include "pdl.cuh"
#include "sm100_ptx.cuh"

namespace gi {
namespace {

using namespace ptx;
using namespace frag;

constexpr int kWarps = 8, kThreads = kWarps * 32;
// units of a block that a warp has in flight (with 32 columns there are registers for two only)
int depth_of(int nt) { return nt == 4 ? 2 : 8; }
constexpr int kUnitBytes = 512, kUnitK = 64;
constexpr int kXBytes = 72 * 1024;        // most shared memory for staged rows of x: two CTAs on an SM, or three

struct Params {
  const unsigned char *wts, *scales, *zeros;
  const float* bias;
  const void* x;
  const void* res;
  void* y;
  long long x_row, x_slice;   // elements between rows; between slices of 4 channels (0: channels are contiguous)
  long long y_row, y_slice;
  int rows, cin, cout;
  int n_units, n_groups;      // units along the input channels; groups of a row
  int scale_dtype;
  unsigned mul_group;         // division by group / 32
  int group32;
  int tiles, kw, ks;          // tiles of output blocks; warps and CTAs that share a tile's sum
  int row_tile, x_vec;
  int chunk;                  // units of x staged at a time
  int act_pre, has_res, act_post;
  int plane, real;            // > 0: stored and real pixels of a plane, padding pixels are not written
};

__device__ __forceinline__ uint4 ldg_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// What is subtracted from the digits of a word's rows g and g + 8.
template <bool BF>
struct Zero {
  unsigned lo, hi;
};
template <bool BF>
__device__ __forceinline__ Zero<BF> zero_of(unsigned z_lo, unsigned z_hi) {
  Zero<BF> z;
  if (BF) {
    z.lo = 0x43004300u | z_lo * 0x10001u;          // 128 + z
    z.hi = 0x43004300u | z_hi * 0x10001u;
  } else {
    z.lo = 0x64006400u | z_lo * 0x10001u;          // 1024 + z
    z.hi = 0xd400d400u | z_hi * 0x100010u;         // -(64 + z)
  }
  return z;
}

// Eight weights of a word as the A operand: q - z, exact.
template <bool BF>
__device__ __forceinline__ void expand(unsigned w, const Zero<BF>& z, unsigned (&a)[4]) {
  if (BF) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned v = ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u;  // 128 + q
      const unsigned c = i & 1 ? z.hi : z.lo;
      const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&c));
      a[i] = *reinterpret_cast<const unsigned*>(&d);
    }
  } else {
    const unsigned sixteenth = 0x2c002c00u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned u = i ? w >> 8 : w;
      const unsigned lo = (u & 0x000f000fu) | 0x64006400u;  // 1024 + q
      const unsigned hi = (u & 0x00f000f0u) | 0x64006400u;  // 1024 + 16 q
      const __half2 d0 = __hsub2(*reinterpret_cast<const __half2*>(&lo), *reinterpret_cast<const __half2*>(&z.lo));
      const __half2 d1 = __hfma2(*reinterpret_cast<const __half2*>(&hi), *reinterpret_cast<const __half2*>(&sixteenth),
                                 *reinterpret_cast<const __half2*>(&z.hi));
      a[2 * i] = *reinterpret_cast<const unsigned*>(&d0);
      a[2 * i + 1] = *reinterpret_cast<const unsigned*>(&d1);
    }
  }
}

// Scales of rows g and g + 8, neighbours in memory, as they are stored: converting them where they are loaded would wait for them.
__device__ __forceinline__ uint2 load_scales(const Params& p, size_t at) {
  if (p.scale_dtype == GI_F32) return *reinterpret_cast<const uint2*>(p.scales + at * 8);
  return make_uint2(*reinterpret_cast<const unsigned*>(p.scales + at * 4), 0u);
}
__device__ __forceinline__ float2 scales_f32(const Params& p, uint2 v) {
  if (p.scale_dtype == GI_F32) return make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
  if (p.scale_dtype == GI_BF16) return make_float2(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&v.x));
}

// Eight channels k .. k + 7 of row r of x (16-bit types), zero behind the last one.
__device__ __forceinline__ uint4 load_x8(const Params& p, int r, int k) {
  const unsigned short* x = static_cast<const unsigned short*>(p.x);
  if (p.x_slice) {  // slices of 4 channels: the lanes behind the last channel hold zeros
    const unsigned short* s = x + (k >> 2) * p.x_slice + r * 4ll;
    uint2 a = make_uint2(0u, 0u), b = a;
    if (k < p.cin) a = *reinterpret_cast<const uint2*>(s);
    if (k + 4 < p.cin) b = *reinterpret_cast<const uint2*>(s + p.x_slice);
    return make_uint4(a.x, a.y, b.x, b.y);
  }
  const unsigned short* row = x + r * p.x_row + k;
  if (p.x_vec && k + 8 <= p.cin) return *reinterpret_cast<const uint4*>(row);
  unsigned v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = k + i < p.cin ? row[i] : 0u;
  return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

// The three bf16 numbers whose sum is v: its digits cut off after 8, 16 and 24.  What is not finite stays in the first.
__device__ __forceinline__ void split3(float v, unsigned (&s)[3]) {
  const unsigned b = __float_as_uint(v), h = b & 0xffff0000u;
  s[0] = h >> 16;
  if ((b & 0x7f800000u) == 0x7f800000u) {
    if (b & 0x7fffffu) s[0] |= 0x40u;  // a NaN whose digits were all cut off
    s[1] = s[2] = 0u;
    return;
  }
  const float rest = v - __uint_as_float(h);
  const unsigned m = __float_as_uint(rest) & 0xffff0000u;
  s[1] = m >> 16;
  s[2] = __float_as_uint(rest - __uint_as_float(m)) >> 16;
}

// Rows of x for units [u0, u0 + n) into shared memory, `pitch` bytes a row.
template <int XT>
__device__ __forceinline__ void stage_x(const Params& p, unsigned char* xs, int pitch, int row0, int nrows, int u0, int n) {
  const int per_row = n * 8;  // eights of channels
  for (int i = threadIdx.x; i < per_row * nrows; i += kThreads) {
    const int r = i / per_row, c = i - r * per_row, k = u0 * kUnitK + c * 8;
    if (XT != GI_F32) {
      *reinterpret_cast<uint4*>(xs + r * pitch + c * 16) = load_x8(p, row0 + r, k);
    } else {
      const float* x = static_cast<const float*>(p.x) + (row0 + r) * p.x_row + k;
      float v[8];
      if (p.x_vec && k + 8 <= p.cin) {
        *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(x);
        *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(x + 4);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = k + j < p.cin ? x[j] : 0.0f;
      }
      unsigned s[8][3];
#pragma unroll
      for (int j = 0; j < 8; ++j) split3(v[j], s[j]);
#pragma unroll
      for (int q = 0; q < 3; ++q)
        *reinterpret_cast<uint4*>(xs + (3 * r + q) * pitch + c * 16) =
            make_uint4(s[0][q] | s[1][q] << 16, s[2][q] | s[3][q] << 16, s[4][q] | s[5][q] << 16, s[6][q] | s[7][q] << 16);
    }
  }
}

template <int XT>
__device__ __forceinline__ void store_y(const Params& p, int r, int o, float v) {
  v = act_f(v, p.act_pre);
  long long at;
  if (p.y_slice) {
    at = (o >> 2) * p.y_slice + r * 4ll + (o & 3);
  } else {
    long long row = r;
    if (p.plane) {
      const int img = r / p.plane, in = r - img * p.plane;
      if (in >= p.real) return;
      row = static_cast<long long>(img) * p.real + in;
    }
    at = row * p.y_row + o;
  }
  if (p.has_res) v = act_f(v + __half2float(static_cast<const __half*>(p.res)[(o >> 2) * p.y_slice + r * 4ll + (o & 3)]), p.act_post);
  if (XT == GI_F16) static_cast<__half*>(p.y)[at] = __float2half_rn(v);
  else if (XT == GI_BF16) static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(v);
  else static_cast<float*>(p.y)[at] = v;
}

// XT: type of x and y.  NT: eights of columns (rows of x, three for a row of 32 bits).  RB: blocks of 16 outputs of a warp.
// G32: a group may end inside a unit.  ZP: zero points of the groups (else 8 everywhere).
template <int XT, int NT, int RB, bool G32, bool ZP>
__global__ void __launch_bounds__(kThreads, 2) linear_q4_kernel(const Params p) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr bool BF = XT != GI_F16;
  constexpr int kCols = XT == GI_F32 ? 3 : 1;  // columns of a row of x
  constexpr int HG = G32 ? 2 : 1;              // groups of a unit
  constexpr int kDepth = NT == 4 ? 2 : 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank = blockIdx.x % p.ks, tile = blockIdx.x / p.ks % p.tiles, row0 = blockIdx.x / p.ks / p.tiles * p.row_tile;
  const int nrows = min(p.row_tile, p.rows - row0), cols = nrows * kCols;
  const int kwi = warp % p.kw, blocks = (kWarps / p.kw) * RB;
  const int n_blocks = (p.cout + 15) / 16;
  const int block0 = tile * blocks + warp / p.kw * RB;  // this warp's blocks; those behind the last one are computed as the last
  // this CTA's units, and how many of them this warp takes: kwi, kwi + kw, ...
  const int ua = static_cast<int>(static_cast<long long>(p.n_units) * rank / p.ks), ub = static_cast<int>(static_cast<long long>(p.n_units) * (rank + 1) / p.ks);
  const int mine = ub - ua > kwi ? (ub - ua - kwi + p.kw - 1) / p.kw : 0;

  // units in flight: a slot is asked for again as soon as it has been used
  uint4 w[RB][kDepth];
  uint2 sc[RB][kDepth][HG];
  unsigned zp[RB][kDepth][HG];
  const unsigned char* wp[RB];
  size_t gp[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const size_t block = min(block0 + b, n_blocks - 1);
    wp[b] = p.wts + (block * p.n_units + ua + kwi) * kUnitBytes + lane * 16;
    gp[b] = block * p.n_groups * 8 + g;
  }
  auto load = [&](int j, int i) {
    const int u = ua + kwi + i * p.kw;
    size_t pair[HG];
#pragma unroll
    for (int h = 0; h < HG; ++h) {
      const int half = 2 * u + h;
      pair[h] = min(G32 && p.group32 == 1 ? half : div_by(half, p.mul_group), p.n_groups - 1) * 8;
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      w[b][j] = ldg_stream(wp[b] + static_cast<size_t>(i) * (p.kw * kUnitBytes));
#pragma unroll
      for (int h = 0; h < HG; ++h) {
        sc[b][j][h] = load_scales(p, gp[b] + pair[h]);
        if (ZP) zp[b][j][h] = *reinterpret_cast<const unsigned short*>(p.zeros + (gp[b] + pair[h]) * 2);
      }
    }
  };

  pdl_launch_dependents();
  // What the first units bring is asked for while the kernel in front of this one ends: into L2 only, so that a blob that this very
  // kernel's predecessor wrote is read as it left it.
#pragma unroll
  for (int j = 0; j < kDepth; ++j)
    if (j < mine && (lane & 1) == 0) asm volatile("prefetch.global.L2 [%0];" ::"l"(wp[0] + static_cast<size_t>(j) * (p.kw * kUnitBytes)));
  pdl_wait();
#pragma unroll
  for (int j = 0; j < kDepth; ++j)
    if (j < mine) load(j, j);

  float acc[RB][NT][4];
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[b][n][i] = 0.0f;

  const int pitch = p.chunk * kUnitK * 2 + 64;  // 64 modulo 128: the eight columns of a fragment lie in different banks
  const unsigned xs = smem_u32(smem);

  auto compute = [&](int j, unsigned at) {  // the unit in slot j; `at`: its channels of the first column of x
    uint4 xb[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int col = n * 8 + g;
      if (col < cols) {
        xb[n][0] = lds128(at + col * pitch);
        xb[n][1] = lds128(at + col * pitch + 64);
      } else {
        xb[n][0] = xb[n][1] = make_uint4(0u, 0u, 0u, 0u);
      }
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const unsigned word[4] = {w[b][j].x, w[b][j].y, w[b][j].z, w[b][j].w};
      float part[NT][4];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int h = G32 ? s >> 1 : 0;
        const Zero<BF> z = ZP ? zero_of<BF>(zp[b][j][h] & 255u, zp[b][j][h] >> 8) : zero_of<BF>(8u, 8u);
        unsigned a[4];
        expand<BF>(word[s], z, a);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint4& v = xb[n][s >> 1];
          const unsigned b0 = s & 1 ? v.z : v.x, b1 = s & 1 ? v.w : v.y;
          if (s == 0 || (G32 && s == 2)) part[n][0] = part[n][1] = part[n][2] = part[n][3] = 0.0f;
          if (BF) mma_bf16(part[n], a, b0, b1);
          else mma16816(part[n], a, b0, b1);
        }
        if (s == 3 || (G32 && s == 1)) {
          const float2 f = scales_f32(p, sc[b][j][h]);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            acc[b][n][0] = fmaf(f.x, part[n][0], acc[b][n][0]);
            acc[b][n][1] = fmaf(f.x, part[n][1], acc[b][n][1]);
            acc[b][n][2] = fmaf(f.y, part[n][2], acc[b][n][2]);
            acc[b][n][3] = fmaf(f.y, part[n][3], acc[b][n][3]);
          }
        }
      }
    }
  };

  const int per_chunk = p.chunk / p.kw;  // units of a warp in a chunk: whole rounds of slots
  for (int c = 0; c * p.chunk < ub - ua; ++c) {
    if (c) __syncthreads();  // every warp is done with the chunk before
    stage_x<XT>(p, smem, pitch, row0, nrows, ua + c * p.chunk, min(p.chunk, ub - ua - c * p.chunk));
    __syncthreads();
    unsigned at = xs + kwi * (kUnitK * 2) + t * 16;
    const int i1 = min((c + 1) * per_chunk, mine);
    for (int i = c * per_chunk; i < i1; i += kDepth) {
#pragma unroll
      for (int j = 0; j < kDepth; ++j) {
        if (i + j < i1) {
          compute(j, at);
          at += p.kw * (kUnitK * 2);
          if (i + j + kDepth < mine) load(j, i + j + kDepth);
        }
      }
    }
  }

  // The warps' sums meet in shared memory, [warp][block][column][16 outputs], and are added in a fixed order.
  __syncthreads();
  float* red = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = n * 8 + 2 * t + (i & 1);
        if (col < cols) red[((warp * RB + b) * (NT * 8) + col) * 16 + g + (i >> 1) * 8] = acc[b][n][i];
      }
  if (p.ks > 1) cluster_sync();
  else __syncthreads();
  // the CTAs of a cluster share the outputs out among themselves
  const int total = blocks * 16 * nrows;
  for (int i = threadIdx.x + rank * kThreads; i < total; i += kThreads * p.ks) {
    const int r = i / (blocks * 16), ol = i - r * (blocks * 16), o = tile * blocks * 16 + ol;
    if (o >= p.cout) continue;
    const int bl = ol >> 4, wr = bl / RB * p.kw;
    float v = p.bias[o];
    for (int k = 0; k < p.ks; ++k) {
      const unsigned base = p.ks > 1 ? mapa_shared(xs, k) : 0u;
      for (int j = 0; j < p.kw; ++j) {
        const int at = (((wr + j) * RB + bl % RB) * (NT * 8) + r * kCols) * 16 + (ol & 15);
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
          if (p.ks > 1) {
            float s;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(s) : "r"(base + (at + c * 16) * 4) : "memory");
            v += s;
          } else {
            v += red[at + c * 16];
          }
        }
      }
    }
    store_y<XT>(p, row0 + r, o, v);
  }
  if (p.ks > 1) cluster_sync();  // nobody leaves while its shared memory is read
}

template <int XT, int NT, int RB>
cudaError_t launch_shape(const Params& p, bool zeros, unsigned grid, size_t smem, cudaStream_t stream) {
  const bool g32 = p.group32 % 2 != 0;
  void (*k)(const Params) = g32 ? (zeros ? linear_q4_kernel<XT, NT, RB, true, true> : linear_q4_kernel<XT, NT, RB, true, false>)
                                : (zeros ? linear_q4_kernel<XT, NT, RB, false, true> : linear_q4_kernel<XT, NT, RB, false, false>);
  static bool raised[2][2][kMaxDevices] = {};
  bool& done = raised[g32][zeros][current_device_slot()];
  if (!done) {
    const cudaError_t err = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kXBytes);
    if (err != cudaSuccess) return err;
    done = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(p.ks);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.ks > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k, p);
}

struct Shape {
  int nt, rb, kw, ks, row_tile;
};

// Which shape of the kernel runs a product: columns a CTA takes at once, warps (kw) and CTAs (ks) that share an output's sum.
Shape choose_shape(int rows, int cols_per_row, int n_blocks, int n_units, int sms) {
  Shape s{};
  const int fit = 32 / cols_per_row;
  s.row_tile = std::min(rows, fit);
  const int cols = s.row_tile * cols_per_row;
  s.nt = cols <= 8 ? 1 : cols <= 16 ? 2 : 4;
  s.rb = s.nt == 4 ? 2 : 1;
  s.kw = 8;
  while (s.kw > 1 && s.kw * cols > 64) s.kw /= 2;
  while (s.kw > 1 && s.kw * depth_of(s.nt) > 2 * n_units) s.kw /= 2;
  const int tiles = (n_blocks + kWarps / s.kw * s.rb - 1) / (kWarps / s.kw * s.rb);
  const long long ctas = static_cast<long long>(tiles) * ((rows + s.row_tile - 1) / s.row_tile);
  s.ks = 1;
  while (s.ks < 8 && ctas * s.ks * 2 <= 2 * sms && s.ks * s.kw * depth_of(s.nt) <= n_units) s.ks *= 2;
  return s;
}

template <int XT>
cudaError_t launch_type(const Params& p, const Shape& s, bool zeros, unsigned grid, size_t smem, cudaStream_t stream) {
  switch (s.nt) {
    case 1: return launch_shape<XT, 1, 1>(p, zeros, grid, smem, stream);
    case 2: return launch_shape<XT, 2, 1>(p, zeros, grid, smem, stream);
    default: return launch_shape<XT, 4, 2>(p, zeros, grid, smem, stream);
  }
}

int scale_bytes(int dtype) { return dtype == GI_F32 ? 4 : 2; }

}  // namespace

LinearQ4Layout linear_q4_layout(int cin, int cout, int group, int scale_dtype, bool zeros) {
  LinearQ4Layout l;
  l.n_blocks = (cout + 15) / 16;
  l.n_units = (cin + kUnitK - 1) / kUnitK;
  l.n_groups = static_cast<int>((static_cast<int64_t>(cin) + group - 1) / group);
  const uint64_t per_group = static_cast<uint64_t>(l.n_blocks) * l.n_groups * 16;
  l.scales = round_up_u64(static_cast<uint64_t>(l.n_blocks) * l.n_units * kUnitBytes, 256);
  l.zeros = round_up_u64(l.scales + per_group * scale_bytes(scale_dtype), 256);
  l.bias = round_up_u64(l.zeros + (zeros ? per_group : 0), 256);
  l.bytes = round_up_u64(l.bias + static_cast<uint64_t>(l.n_blocks) * 16 * sizeof(float), 256);
  return l;
}

void linear_q4_pack(const LinearQ4Weights& w, const float* bias, uint8_t* blob) {
  const LinearQ4Layout l = linear_q4_layout(w.cin, w.cout, w.group, w.scale_dtype, w.zeros != nullptr);
  std::memset(blob, 0, l.bytes);
  const int64_t pitch = (static_cast<int64_t>(w.cin) + 1) / 2;  // bytes of a row of the caller's
  uint32_t* out = reinterpret_cast<uint32_t*>(blob);
  for (int b = 0; b < l.n_blocks; ++b)
    for (int u = 0; u < l.n_units; ++u)
      for (int g = 0; g < 8; ++g) {
        // two rows' 32 bytes of this unit, zero behind the last channel and the last output
        uint8_t row[2][kUnitK / 2] = {};
        for (int i = 0; i < 2; ++i) {
          const int o = b * 16 + g + 8 * i;
          const int64_t at = static_cast<int64_t>(u) * (kUnitK / 2), n = std::min<int64_t>(kUnitK / 2, pitch - at);
          if (o < w.cout) std::memcpy(row[i], w.q + o * pitch + at, static_cast<size_t>(n));
        }
        for (int t = 0; t < 4; ++t)
          for (int s = 0; s < 4; ++s) {
            const int at = (s >> 1) * 16 + t * 4 + (s & 1) * 2;  // byte of channel 32 (s / 2) + 8 t + 4 (s % 2)
            const uint32_t a0 = row[0][at], a1 = row[0][at + 1], c0 = row[1][at], c1 = row[1][at + 1];
            out[((static_cast<size_t>(b) * l.n_units + u) * 32 + g * 4 + t) * 4 + s] =
                (a0 & 15u) | (c0 & 15u) << 4 | (a1 & 15u) << 8 | (c1 & 15u) << 12 | (a0 >> 4) << 16 | (c0 >> 4) << 20 | (a1 >> 4) << 24 | (c1 >> 4) << 28;
          }
      }
  // scales and zero points: [block of 16 outputs][group][8][2], outputs g and g + 8 side by side
  const int sb = scale_bytes(w.scale_dtype);
  for (int o = 0; o < w.cout; ++o)
    for (int gr = 0; gr < l.n_groups; ++gr) {
      const size_t to = (static_cast<size_t>(o / 16) * l.n_groups + gr) * 16 + (o % 8) * 2 + o % 16 / 8, from = static_cast<size_t>(o) * l.n_groups + gr;
      std::memcpy(blob + l.scales + to * sb, static_cast<const uint8_t*>(w.scales) + from * sb, sb);
      if (w.zeros) blob[l.zeros + to] = w.zeros[from] & 15u;
    }
  if (bias) std::memcpy(blob + l.bias, bias, static_cast<size_t>(w.cout) * sizeof(float));
}

int launch_linear_q4(const LinearQ4Call& c, void* stream) {
  if (c.rows <= 0) return 0;
  const LinearQ4Layout l = linear_q4_layout(c.cin, c.cout, c.group, c.scale_dtype, c.zeros);
  const int cols_per_row = c.dtype == GI_F32 ? 3 : 1;
  const Shape s = choose_shape(c.rows, cols_per_row, l.n_blocks, l.n_units, device_sm_count());
  Params p{};
  const unsigned char* blob = static_cast<const unsigned char*>(c.blob);
  p.wts = blob;
  p.scales = blob + l.scales;
  p.zeros = blob + l.zeros;
  p.bias = reinterpret_cast<const float*>(blob + l.bias);
  p.x = c.x;
  p.res = c.res;
  p.y = c.y;
  p.x_row = c.x_row;
  p.x_slice = c.x_slice;
  p.y_row = c.y_row;
  p.y_slice = c.y_slice;
  p.rows = c.rows;
  p.cin = c.cin;
  p.cout = c.cout;
  p.n_units = l.n_units;
  p.n_groups = l.n_groups;
  p.scale_dtype = c.scale_dtype;
  p.group32 = std::min(c.group / 32, 2 * l.n_units);  // one group: as many halves of units as there are
  p.mul_group = p.group32 > 1 ? magic(static_cast<uint64_t>(p.group32)) : 0u;
  p.kw = s.kw;
  p.ks = s.ks;
  p.row_tile = s.row_tile;
  const int blocks = kWarps / s.kw * s.rb, elem = c.dtype == GI_F32 ? 4 : 2, cols = s.row_tile * cols_per_row;
  p.tiles = (l.n_blocks + blocks - 1) / blocks;
  p.x_vec = c.x_slice == 0 && reinterpret_cast<uintptr_t>(c.x) % 16 == 0 && (c.rows == 1 || c.x_row * elem % 16 == 0);
  // units staged at a time: whole rounds of slots of every warp
  const int step = s.kw * depth_of(s.nt);
  const int fit = (kXBytes / cols - 64) / (kUnitK * 2);
  const int need = (l.n_units + s.ks - 1) / s.ks;
  p.chunk = std::max(step, std::min(fit / step * step, (need + step - 1) / step * step));
  p.act_pre = c.ep.act_pre;
  p.has_res = c.ep.has_res;
  p.act_post = c.ep.act_post;
  p.plane = c.plane;
  p.real = c.real;
  const size_t smem = std::max<size_t>(static_cast<size_t>(cols) * (p.chunk * kUnitK * 2 + 64), static_cast<size_t>(kWarps) * s.rb * s.nt * 8 * 16 * 4);
  const long long grid = static_cast<long long>(p.tiles) * s.ks * ((c.rows + s.row_tile - 1) / s.row_tile);
  if (grid > 0x7fffffffll || smem > kXBytes) return static_cast<int>(cudaErrorInvalidConfiguration);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const unsigned n = static_cast<unsigned>(grid);
  switch (c.dtype) {
    case GI_F16: return static_cast<int>(launch_type<GI_F16>(p, s, c.zeros, n, smem, st));
    case GI_BF16: return static_cast<int>(launch_type<GI_BF16>(p, s, c.zeros, n, smem, st));
    default: return static_cast<int>(launch_type<GI_F32>(p, s, c.zeros, n, smem, st));
  }
}

}  // namespace gi
