// Fully connected layer (1x1 convolution) with 4-bit weights: y = act(x w^T + bias), w[o, k] = s[o, k / group] (q[o, k] - z[o, k / group]),
// q and z whole numbers of 0 .. 15.
//
// What bounds it: for few rows of x the bytes of the weights, half a byte each - so the kernel is built around reading them once,
// in copies that are under way long before they are needed, and around spending less than the 2.8 issue slots a weight that an SM has
// at the rate at which its share of the memory's bandwidth delivers them (it spends 2.2, and the ALU's half-rate pipe 0.9 of 1.4).
// q - z is exact in fp16 and in bf16: eight weights are taken out of a word by five logical operations (q becomes the low digits of
// 1024 or 128) and four subtractions, and go into mma.sync.m16n8k16 as the A operand, the rows of x being the 8 columns.  Sums are
// fp32 for each group of input channels and are scaled in fp32: nothing of a weight is rounded.  For so few columns tcgen05 would
// only add a store to shared memory for every weight; from 17 rows on it wins (linear_q4_tc.cu).
//
// Measured (B200): one row 8192 -> 28672 32 us, 3.7 TB/s (its copies alone 23 us, its arithmetic alone 27), one row 4096 -> 4096
// 5.9 us, 8 rows 4096 -> 12288 13.5 us, 16 rows 5120 -> 13824 with zero points 23.5 us.
//
// x in 32 bits: a value is the exact sum of three bf16 numbers (8 + 8 + 8 digits), so a row of x becomes three columns of the product.
// Ten rows are a tile, and every tile reads and expands all weights: 5 rows 4096 -> 12288 17 us, 10 47, 32 124, 256 755.
//
// Layout of the packed weights (linear_q4_pack): records of 16 outputs x 128 input channels, those of 16 outputs one after another.
// A record is 1024 bytes of weights - lane l = 4 g + t of a warp reads bytes 16 l .. and 512 + 16 l .., which are rows g and g + 8,
// channels 64 i + 32 h + 8 t + 0 .. 7 - and behind them the scales and zero points of the groups it touches ([group][8][2], rows g
// and g + 8 side by side), so that one address leads to all that a lane needs and nothing is computed to find it.  A lane's eight
// channels are contiguous in x too, so x needs no rearrangement.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "kernels.h"
#include "mma_frag.cuh"
#include "pdl.cuh"
#include "q4_record.cuh"
#include "sm100_ptx.cuh"

namespace gi {
namespace {

using namespace ptx;
using namespace frag;
using namespace q4;

// One CTA an SM: two of 8 warps would each stage x (8 rows 4096 -> 12288 13.0 us, two CTAs 15.2; 16 rows 8192 -> 8192 22.8 and 27.3;
// one row 8192 -> 28672 31.4 and 33.1, 4096 -> 4096 5.9 and 5.5).  That leaves 128 registers a thread: of the 48 variants of more than 8
// columns 33 spill, by 32 bytes at most and by 108 where there are more than 16.
constexpr int kWarps = 16, kThreads = kWarps * 32;
// A warp's ring of copies: slots of two records (neighbours of one block, or one of each of two blocks).  16 warps keep 128 KB of
// requests open.
constexpr int kSlots = 4;
constexpr int kSmem = 226 * 1024;         // one CTA on an SM
constexpr int kSumBytes = 16384;          // most for the items' sums: with the rings (records of up to 1344 bytes) and one step of x inside that

struct Params {
  const unsigned char* wts;
  const float* bias;
  const void* x;
  const void* res;
  void* y;
  long long x_row, x_slice;   // elements between rows; between slices of 4 channels (0: channels are contiguous)
  long long y_row, y_slice, res_slice;
  int rows, cin, cout;
  int n_units;                // records along the input channels
  int tiles, kw, ks;          // tiles of output blocks, a cluster of ks CTAs each; parts of a block's sum in a CTA
  int row_tile, x_vec;
  int chunk;                  // records of x staged at a time
  int ring_at, red_at;        // where the rings of copies, and the items' sums, begin in shared memory
  q4::Masks q;
  int act_pre, has_res, act_post;
  int plane, real;            // > 0: stored and real pixels of a plane, padding pixels are not written
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the same with the sum started from zero (as an operand: cleared registers cost four instructions more)
__device__ __forceinline__ void mma_bf16z(float (&d)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
template <bool BF, bool FIRST>
__device__ __forceinline__ void mma(float (&d)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  if (BF && FIRST) mma_bf16z(d, a, b0, b1);
  else if (BF) mma_bf16(d, a, b0, b1);
  else if (FIRST) mma16816z(d, a, b0, b1);
  else mma16816(d, a, b0, b1);
}

// Eight channels k .. k + 7 of row r of x (16-bit types), zero behind the last one.  GR: as an operator
// of a graph - x and y may lie in slices of 4 channels, y may be joined with a residual; fp16 and up to 8 columns only.
template <bool GR>
__device__ __forceinline__ uint4 load_x8(const Params& p, int r, int k) {
  const unsigned short* x = static_cast<const unsigned short*>(p.x);
  if (GR && p.x_slice) {  // the lanes behind the last channel hold zeros
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
template <int XT, bool GR>
__device__ __forceinline__ void stage_x(const Params& p, unsigned char* xs, int pitch, int row0, int nrows, int u0, int n) {
  const int per_row = n * (kUnitK / 8);
  for (int i = threadIdx.x; i < per_row * nrows; i += kThreads) {
    int r = i / per_row, c = i - r * per_row;
    if (GR && p.x_slice) {  // the pixels of a slice are neighbours
      c = i / nrows;
      r = i - c * nrows;
    }
    const int k = u0 * kUnitK + c * 8;
    if (XT != GI_F32) {
      *reinterpret_cast<uint4*>(xs + r * pitch + c * 16) = load_x8<GR>(p, row0 + r, k);
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

// the activation; a NaN stays one
__device__ __forceinline__ float act_nan(float v, int act) {
  if (act != GI_ACT_NONE && v < 0.0f) v = 0.0f;
  if (act == GI_ACT_RELU6 && v > 6.0f) v = 6.0f;
  return v;
}

template <int XT, bool GR>
__device__ __forceinline__ void store_y(const Params& p, int r, int o, float v) {
  v = act_nan(v, p.act_pre);
  long long at;
  if (GR && p.y_slice) {
    at = (o >> 2) * p.y_slice + r * 4ll + (o & 3);
  } else {
    long long row = r;
    if (GR && p.plane) {
      const int img = r / p.plane, in = r - img * p.plane;
      if (in >= p.real) return;
      row = static_cast<long long>(img) * p.real + in;
    }
    at = row * p.y_row + o;
  }
  if (GR && p.has_res) v = act_nan(v + __half2float(static_cast<const __half*>(p.res)[(o >> 2) * p.res_slice + r * 4ll + (o & 3)]), p.act_post);
  if (XT == GI_F16) static_cast<__half*>(p.y)[at] = __float2half_rn(v);
  else if (XT == GI_BF16) static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(v);
  else static_cast<float*>(p.y)[at] = v;
}

// XT: type of x and y.  NT: eights of columns (rows of x, three for a row of 32 bits).  RB: blocks of 16 outputs of a warp.
// HG: groups that a record may touch, 1, 2 or 4 parts of it.  ZP: zero points of the groups (else 8 everywhere).  S32: scales in 32 bits.
template <int XT, int NT, int RB, int HG, bool ZP, bool S32>
__global__ void __launch_bounds__(kThreads, 1) linear_q4_kernel(const Params p) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr bool BF = XT != GI_F16, kGraph = XT == GI_F16 && NT == 1;
  constexpr int kCols = XT == GI_F32 ? 3 : 1;  // columns of a row of x
  constexpr int kZerosAt = zeros_at(HG, S32), kRecord = record_bytes(HG, S32, ZP), kBehind = kRecord - kUnitWeights;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank = blockIdx.x % p.ks, tile = blockIdx.x / p.ks % p.tiles, row0 = blockIdx.x / p.ks / p.tiles * p.row_tile;
  const int nrows = min(p.row_tile, p.rows - row0), cols = nrows * kCols;
  const int n_blocks = (p.cout + 15) / 16, n_sets = (n_blocks + RB - 1) / RB;
  // A tile's sets of RB blocks are cut into items: one set and one of kw parts of the CTA's share of the input channels.  Warp w
  // takes the items w, w + 16, ..., one after the other; each leaves its sum in shared memory.
  const int set0 = static_cast<int>(static_cast<long long>(n_sets) * tile / p.tiles), sets = static_cast<int>(static_cast<long long>(n_sets) * (tile + 1) / p.tiles) - set0;
  const int items = sets * p.kw;
  constexpr int kSteps = 2 / RB;  // records of a block that are one step
  const int ua = static_cast<int>(static_cast<long long>(p.n_units) * rank / p.ks), ub = static_cast<int>(static_cast<long long>(p.n_units) * (rank + 1) / p.ks);
  const int chunks = (ub - ua + p.chunk - 1) / p.chunk;

  // This warp's own ring of copies.  (What else was tried: records held in registers, four loads deep - a warp tells its loads apart
  // by six scoreboards and waits for all that share one; a copy of a whole record by one thread - some 90 instructions a record to
  // ask and to wait for, where two records copied by every lane take 24 each.)
  const unsigned xs = smem_u32(smem);
  const unsigned ring = xs + p.ring_at + warp * (kSlots * 2) * kRecord;
  // what is asked for next: `left` records of item a_item in chunk a_chunk, from `next` on
  const unsigned char* next = nullptr;
  size_t to_second = 0;
  int a_item = warp - kWarps, a_chunk = 0, left = 0;
  // records [first, last) of the CTA's share that item `item` has in chunk c: whole steps, but for the last of all
  auto range = [&](int item, int c, int& first, int& last) {
    const int part = item % p.kw, n = min(p.chunk, ub - ua - c * p.chunk), n_steps = (n + kSteps - 1) / kSteps;
    first = c * p.chunk + n_steps * part / p.kw * kSteps;
    last = c * p.chunk + min(n_steps * (part + 1) / p.kw * kSteps, n);
  };
  auto advance = [&] {  // to the next item that has records, if there is one
    while (left <= 0 && a_chunk < chunks) {
      a_item += kWarps;
      if (a_item >= items) {
        a_item = warp - kWarps;
        ++a_chunk;
        continue;
      }
      int first, last;
      range(a_item, a_chunk, first, last);
      left = last - first;
      const int block = (set0 + a_item / p.kw) * RB;
      next = p.wts + (static_cast<size_t>(block) * p.n_units + ua + first) * kRecord + lane * 16;
      if (RB == 2) to_second = block + 1 < n_blocks ? static_cast<size_t>(p.n_units) * kRecord : 0;  // (behind the last block: that one again)
    }
  };
  auto request = [&](unsigned slot) {
    if (left > 0) {
      const unsigned to = slot + lane * 16;
      copy16(to, next);
      copy16(to + 512, next + 512);
      if (RB == 2) {
        const unsigned char* other = next + to_second;
        const unsigned to2 = to + kRecord;
        copy16(to2, other);
        copy16(to2 + 512, other + 512);
        if (lane * 16 < kBehind) {
          copy16(to + 1024, next + 1024);
          copy16(to2 + 1024, other + 1024);
        }
      } else if (left > 1) {  // 2 x 1056 .. 1344 bytes
        copy16(to + 1024, next + 1024);
        copy16(to + 1536, next + 1536);
        if (lane * 16 < 2 * kBehind) copy16(to + 2048, next + 2048);
        if (512 < 2 * kBehind && 512 + lane * 16 < 2 * kBehind) copy16(to + 2560, next + 2560);
      } else if (lane * 16 < kBehind) {
        copy16(to + 1024, next + 1024);
      }
      next += kSteps * kRecord;
      left -= kSteps;
      if (left <= 0) advance();
    }
    copies_commit();
  };

  pdl_launch_dependents();
  advance();
  // What the first slots will hold is asked for while the kernel in front of this one ends: into L2 only, so that a blob that this
  // very kernel's predecessor wrote is read as it left it.
  if (lane == 0 && left > 0) {
    const unsigned bytes = min(left, kSlots * kSteps) * kRecord;
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(next), "r"(bytes) : "memory");
    if (RB == 2) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(next + to_second), "r"(bytes) : "memory");
  }
  pdl_wait();
#pragma unroll
  for (int j = 0; j < kSlots; ++j) request(ring + j * 2 * kRecord);

  float acc[RB][NT][4];
  const int pitch = p.chunk * kUnitK * 2 + 64;  // 64 modulo 128: the eight columns of a fragment lie in different banks
  // (lanes of columns that there are not read another's: a column of the product depends on its own column of x only)
  unsigned col_at[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) col_at[n] = min(n * 8 + g, cols - 1) * pitch;

  auto compute = [&](const uint4 (&w)[RB][2], const float2 (&f)[RB][HG], const unsigned (&zp)[RB][HG], unsigned at) {
    float part[RB][NT][4];
    // a chain of products on one sum waits for each of them: with one column tile, two chains a record at least
    constexpr int kChains = HG == 1 && NT == 1 ? 2 : HG;
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // 64 channels
      uint4 xb[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        xb[n][0] = lds128(at + col_at[n] + i * 128);
        xb[n][1] = lds128(at + col_at[n] + i * 128 + 64);
      }
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const unsigned word[4] = {w[b][i].x, w[b][i].y, w[b][i].z, w[b][i].w};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int q = 4 * i + s, h = q * HG / 8;  // 16 channels; their group
          const bool first = q * kChains % 8 == 0, last = (q + 1) * kChains % 8 == 0;
          const Zero z = ZP ? zero_of<BF>(p.q, zp[b][h] & 255u, zp[b][h] >> 8) : zero_of<BF>(p.q, 8u, 8u);
          unsigned a[4];
          expand<BF>(p.q, word[s], z, a);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint4& v = xb[n][s >> 1];
            const unsigned b0 = s & 1 ? v.z : v.x, b1 = s & 1 ? v.w : v.y;
            if (first) mma<BF, true>(part[b][n], a, b0, b1);
            else mma<BF, false>(part[b][n], a, b0, b1);
          }
          if (last) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              acc[b][n][0] = fmaf(f[b][h].x, part[b][n][0], acc[b][n][0]);
              acc[b][n][1] = fmaf(f[b][h].x, part[b][n][1], acc[b][n][1]);
              acc[b][n][2] = fmaf(f[b][h].y, part[b][n][2], acc[b][n][2]);
              acc[b][n][3] = fmaf(f[b][h].y, part[b][n][3], acc[b][n][3]);
            }
          }
        }
      }
    }
  };

  // sums of the items: [item][block][column][16 outputs]
  float* red = reinterpret_cast<float*>(smem + p.red_at);
  unsigned from = ring;
  for (int c = 0; c < chunks; ++c) {
    if (c) __syncthreads();  // every warp is done with the chunk before
    stage_x<XT, kGraph>(p, smem, pitch, row0, nrows, ua + c * p.chunk, min(p.chunk, ub - ua - c * p.chunk));
    __syncthreads();
    for (int item = warp; item < items; item += kWarps) {
      int first, last;
      range(item, c, first, last);
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[b][n][j] = 0.0f;
      unsigned at = xs + (first - c * p.chunk) * (kUnitK * 2) + t * 16;
      for (int i = first; i < last; i += kSteps) {
        copies_wait<kSlots - 1>();
        __syncwarp();  // every lane's copies have
        uint4 w[kSteps][RB][2];
        float2 f[kSteps][RB][HG];
        unsigned zp[kSteps][RB][HG];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int d = RB == 2 ? 0 : j, b = RB == 2 ? j : 0;
          const unsigned rec = from + j * kRecord;
          w[d][b][0] = lds128(rec + lane * 16);
          w[d][b][1] = lds128(rec + lane * 16 + kUnitWeights / 2);
#pragma unroll
          for (int h = 0; h < HG; ++h) {
            f[d][b][h] = load_scales<S32, BF>(rec + kUnitWeights + (h * 8 + g) * (S32 ? 8 : 4));
            if (ZP) zp[d][b][h] = lds16(rec + kZerosAt + (h * 8 + g) * 2);
          }
        }
        __syncwarp();  // every lane has what it needs of the slot
        request(from);
        from = from == ring + (kSlots - 1) * 2 * kRecord ? ring : from + 2 * kRecord;
        if (kSteps == 1 || i + 1 == last) {
          compute(w[0], f[0], zp[0], at);
        } else {
          compute(w[0], f[0], zp[0], at);
          compute(w[kSteps - 1], f[kSteps - 1], zp[kSteps - 1], at + kUnitK * 2);
        }
        at += kSteps * (kUnitK * 2);
      }
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int col = n * 8 + 2 * t + (j & 1);
            float* to = red + ((item * RB + b) * cols + col) * 16 + g + (j >> 1) * 8;
            if (col < cols) *to = c ? *to + acc[b][n][j] : acc[b][n][j];
          }
    }
  }

  // The items' sums are added in a fixed order; the CTAs of a cluster share the outputs out among themselves.
  if (p.ks > 1) cluster_sync();
  else __syncthreads();
  const int outs = sets * RB * 16, total = outs * nrows;
  for (int i = threadIdx.x + rank * kThreads; i < total; i += kThreads * p.ks) {
    const int r = i / outs, ol = i - r * outs, o = set0 * RB * 16 + ol;
    if (o >= p.cout) {
      // the channels that complete the last slice are zeros
      if (kGraph && p.y_slice && o < (p.cout + 3) / 4 * 4) static_cast<__half*>(p.y)[(o >> 2) * p.y_slice + (row0 + r) * 4ll + (o & 3)] = __float2half_rn(0.0f);
      continue;
    }
    const int bl = ol >> 4;
    float v = p.bias[o];
    for (int k = 0; k < p.ks; ++k) {
      const unsigned base = p.ks > 1 ? mapa_shared(xs + p.red_at, k) : 0u;
      for (int j = 0; j < p.kw; ++j) {
        const int at = (((bl / RB * p.kw + j) * RB + bl % RB) * cols + r * kCols) * 16 + (ol & 15);
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
    store_y<XT, kGraph>(p, row0 + r, o, v);
  }
  if (p.ks > 1) cluster_sync();  // nobody leaves while its shared memory is read
}

// ---------------------------------------------------------------- packing on the device (the host's linear_q4_pack, byte for byte)
struct PackParams {
  const unsigned char *q, *scales, *zeros;
  const float* bias;
  unsigned char* blob;
  long long pitch, n_groups;  // bytes of a row of q; groups of a row
  unsigned long long bias_at, power_at;
  int cin, cout, group, scale_dtype, n_units, parts, record, zeros_at, wide, top;
};

__device__ __forceinline__ float scale_at(const PackParams& p, long long i) {
  if (p.scale_dtype == GI_F32) return reinterpret_cast<const float*>(p.scales)[i];
  if (p.scale_dtype == GI_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.scales)[i]);
  return __half2float(reinterpret_cast<const __half*>(p.scales)[i]);
}

// a CTA a record: 64 threads its weights, the others what lies behind them
__global__ void __launch_bounds__(128) pack_records_kernel(const PackParams p) {
  const int block = blockIdx.x / p.n_units, u = blockIdx.x % p.n_units, tid = threadIdx.x;
  unsigned char* rec = p.blob + static_cast<size_t>(blockIdx.x) * p.record;
  if (tid < 64) {
    const int i = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    unsigned word[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const long long at = static_cast<long long>(u) * (kUnitK / 2) + i * 32 + (s >> 1) * 16 + t * 4 + (s & 1) * 2;
      unsigned v[2][2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int o = block * 16 + g + 8 * r;
#pragma unroll
        for (int k = 0; k < 2; ++k) v[r][k] = o < p.cout && at + k < p.pitch ? p.q[o * p.pitch + at + k] : 0u;
      }
      word[s] = (v[0][0] & 15u) | (v[1][0] & 15u) << 4 | (v[0][1] & 15u) << 8 | (v[1][1] & 15u) << 12 | (v[0][0] >> 4) << 16 | (v[1][0] >> 4) << 20 |
                (v[0][1] >> 4) << 24 | (v[1][1] >> 4) << 28;
    }
    *reinterpret_cast<uint4*>(rec + tid * 16) = make_uint4(word[0], word[1], word[2], word[3]);
    return;
  }
  for (int j = tid - 64; j < p.parts * 16; j += 64) {
    const int h = j >> 4, o = block * 16 + ((j & 15) >> 1) + 8 * (j & 1);
    const long long at = (static_cast<long long>(u) * kUnitK + h * (kUnitK / p.parts)) / p.group;
    const long long from = o * p.n_groups + min(at, p.n_groups - 1);
    const bool real = o < p.cout;
    if (p.wide) reinterpret_cast<float*>(rec + kUnitWeights)[j] = real ? scale_at(p, from) : 0.0f;
    else reinterpret_cast<unsigned short*>(rec + kUnitWeights)[j] = real ? reinterpret_cast<const unsigned short*>(p.scales)[from] : static_cast<unsigned short>(0);
    if (p.zeros) rec[p.zeros_at + j] = real ? p.zeros[from] & 15u : 0u;
  }
  for (int j = p.zeros_at + (p.zeros ? p.parts * 16 : 0) + tid - 64; j < p.record; j += 64) rec[j] = 0;
}

// a warp an output: its bias, and the power of two that brings its largest scale to 2^(top - 1) .. 2^top
__global__ void __launch_bounds__(128) pack_outputs_kernel(const PackParams p, int outputs) {
  const int o = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (o >= outputs) return;
  float largest = 0.0f;
  for (long long gr = lane; o < p.cout && gr < p.n_groups; gr += 32) {
    const float v = fabsf(scale_at(p, o * p.n_groups + gr));
    if (v <= 3.402823466e38f) largest = fmaxf(largest, v);
  }
  for (int k = 16; k; k >>= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, k));
  if (lane == 0) {
    float power = 1.0f;
    if (largest > 0.0f) {
      int e = 0;
      frexpf(largest, &e);
      power = ldexpf(1.0f, min(126, max(-126, p.top - e)));
    }
    reinterpret_cast<float*>(p.blob + p.power_at)[o] = power;
    reinterpret_cast<float*>(p.blob + p.bias_at)[o] = p.bias && o < p.cout ? p.bias[o] : 0.0f;
  }
}

template <int XT, int NT, int RB, bool S32>
cudaError_t launch_shape(const Params& p, int parts, bool zeros, unsigned grid, size_t smem, cudaStream_t stream) {
  void (*k)(const Params) = parts == 1   ? (zeros ? linear_q4_kernel<XT, NT, RB, 1, true, S32> : linear_q4_kernel<XT, NT, RB, 1, false, S32>)
                            : parts == 2 ? (zeros ? linear_q4_kernel<XT, NT, RB, 2, true, S32> : linear_q4_kernel<XT, NT, RB, 2, false, S32>)
                                         : (zeros ? linear_q4_kernel<XT, NT, RB, 4, true, S32> : linear_q4_kernel<XT, NT, RB, 4, false, S32>);
  static bool raised[3][2][kMaxDevices] = {};
  bool& done = raised[parts / 2][zeros][current_device_slot()];
  if (!done) {
    const cudaError_t err = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
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
  int nt, rb, tiles, kw, ks, row_tile;
};

// Which shape of the kernel runs a product: columns a CTA takes at once, tiles of outputs, CTAs (ks) that share a tile's sums and
// parts (kw) of a CTA's share of a sum.
Shape choose_shape(int rows, int cols_per_row, int n_blocks, int n_units, int sms) {
  Shape s{};
  s.row_tile = std::min(rows, cols_per_row == 1 ? 16 : 32 / cols_per_row);
  const int cols = s.row_tile * cols_per_row;
  s.nt = cols <= 8 ? 1 : cols <= 16 ? 2 : 4;
  s.rb = s.nt == 1 ? 1 : 2;
  const int n_sets = (n_blocks + s.rb - 1) / s.rb;
  // More than 8 columns: pairs of CTAs share x out among themselves, each stages half of its channels, whatever their number (16 rows
  // 8192 -> 8192 22.8 us, alone 28.5; 8 rows 4096 -> 12288 13.0 and 12.9).  Few outputs of many channels: while that leaves SMs idle, twice
  // as many CTAs share a sum if each then has 2048 channels of it or more - 512 of more than 8 columns (4 rows 16384 -> 512: 8 CTAs 7.5 us, 4 7.6, 1 35; 12 rows 1280 -> 1001: 2 4.5, 4 5.6;
  // one row 1280 -> 1001: 1 CTA 2.9, 2 3.5).
  const bool many = cols > 8;
  s.ks = many && n_units >= 2 ? 2 : 1;
  s.tiles = std::min(n_sets, sms / s.ks);
  while (s.ks < 8 && s.tiles * s.ks * 2 <= sms && n_units >= (many ? 8 : 32) * s.ks) s.ks *= 2;
  // items for most of the warps, of a step or more (16 rows 4096 -> 4096, 2 sets of outputs a CTA: 4 parts 9.8 us, 2 10.1, 1 12.7;
  // one row 8192 -> 28672, 12 sets: 4 31.2, 2 31.4, 1 32.2)
  s.kw = 1;
  auto sets = [&] { return (n_sets + s.tiles - 1) / s.tiles; };
  while (s.kw < (many ? 4 : 8) && sets() * s.kw < (many ? 8 : 14) && s.kw * s.ks * 2 <= n_units) s.kw *= 2;
  const int part = s.rb * cols * 16 * 4;  // bytes of an item's sum
  while (s.kw > 1 && sets() * s.kw * part > kSumBytes) s.kw /= 2;
  if (sets() * part > kSumBytes) {
    const int most = kSumBytes / part;
    s.tiles = (n_sets + most - 1) / most;
  }
  return s;
}

template <int XT, bool S32>
cudaError_t launch_type(const Params& p, const Shape& s, int parts, bool zeros, unsigned grid, size_t smem, cudaStream_t stream) {
  if (s.nt == 1) return launch_shape<XT, 1, 1, S32>(p, parts, zeros, grid, smem, stream);
  // (16 rows of a 16-bit type are two eights: more of them go to tcgen05)
  if constexpr (XT == GI_F32) {
    if (s.nt == 4) return launch_shape<XT, 4, 2, S32>(p, parts, zeros, grid, smem, stream);
  }
  return launch_shape<XT, 2, 2, S32>(p, parts, zeros, grid, smem, stream);
}

// a caller's scale in 32 bits: exact
float scale_at(const LinearQ4Weights& w, size_t i) {
  const uint8_t* p = static_cast<const uint8_t*>(w.scales) + i * (w.scale_dtype == GI_F32 ? 4 : 2);
  if (w.scale_dtype == GI_F32) {
    float f;
    std::memcpy(&f, p, 4);
    return f;
  }
  uint16_t v;
  std::memcpy(&v, p, 2);
  return w.scale_dtype == GI_F16 ? f16_to_f32(v) : bf16_to_f32(v);
}

}  // namespace

LinearQ4Layout linear_q4_layout(int cin, int cout, int group, int scale_dtype, bool zeros, int dtype) {
  LinearQ4Layout l;
  l.n_blocks = (cout + 15) / 16;
  l.n_units = (cin + kUnitK - 1) / kUnitK;
  l.parts = parts_of(group);
  l.zeros_at = zeros_at(l.parts, wide_scales(scale_dtype, dtype));
  l.record = record_bytes(l.parts, wide_scales(scale_dtype, dtype), zeros);
  l.bias = round_up_u64(static_cast<uint64_t>(l.n_blocks) * l.n_units * l.record, 256);
  l.power = l.bias + static_cast<uint64_t>(l.n_blocks) * 16 * sizeof(float);
  l.bytes = round_up_u64(l.power + static_cast<uint64_t>(l.n_blocks) * 16 * sizeof(float), 256);
  return l;
}

void linear_q4_pack(const LinearQ4Weights& w, const float* bias, uint8_t* blob) {
  const LinearQ4Layout l = linear_q4_layout(w.cin, w.cout, w.group, w.scale_dtype, w.zeros != nullptr, w.dtype);
  const int64_t pitch = (static_cast<int64_t>(w.cin) + 1) / 2;  // bytes of a row of the caller's
  const int64_t n_groups = (static_cast<int64_t>(w.cin) + w.group - 1) / w.group;
  const bool wide = wide_scales(w.scale_dtype, w.dtype);
  for (int b = 0; b < l.n_blocks; ++b)
    for (int u = 0; u < l.n_units; ++u) {
      // zero behind the last channel and the last output: x is staged as zeros there, such outputs are not stored
      uint8_t* rec = blob + (static_cast<size_t>(b) * l.n_units + u) * l.record;
      std::memset(rec + kUnitWeights, 0, l.record - kUnitWeights);
      uint32_t words[kUnitWeights / 4];
      for (int g = 0; g < 8; ++g) {
        uint8_t row[2][kUnitK / 2] = {};
        for (int i = 0; i < 2; ++i) {
          const int o = b * 16 + g + 8 * i;
          if (o >= w.cout) continue;
          const int64_t at = static_cast<int64_t>(u) * (kUnitK / 2), n = std::min<int64_t>(kUnitK / 2, pitch - at);
          std::memcpy(row[i], w.q + o * pitch + at, static_cast<size_t>(n));
          for (int h = 0; h < l.parts; ++h) {
            const int64_t gr = std::min<int64_t>((static_cast<int64_t>(u) * kUnitK + h * (kUnitK / l.parts)) / w.group, n_groups - 1);
            const size_t from = static_cast<size_t>(o) * n_groups + gr, to = h * 16 + g * 2 + i;
            if (wide) {
              const float f = scale_at(w, from);
              std::memcpy(rec + kUnitWeights + to * 4, &f, 4);
            } else {
              std::memcpy(rec + kUnitWeights + to * 2, static_cast<const uint8_t*>(w.scales) + from * 2, 2);
            }
            if (w.zeros) rec[l.zeros_at + to] = w.zeros[from] & 15u;
          }
        }
        for (int i = 0; i < 2; ++i)
          for (int t = 0; t < 4; ++t)
            for (int s = 0; s < 4; ++s) {
              const int at = i * 32 + (s >> 1) * 16 + t * 4 + (s & 1) * 2;  // byte of channel 64 i + 32 (s / 2) + 8 t + 4 (s % 2)
              const uint32_t a0 = row[0][at], a1 = row[0][at + 1], c0 = row[1][at], c1 = row[1][at + 1];
              words[(i * 32 + g * 4 + t) * 4 + s] = (a0 & 15u) | (c0 & 15u) << 4 | (a1 & 15u) << 8 | (c1 & 15u) << 12 | (a0 >> 4) << 16 |
                                                    (c0 >> 4) << 20 | (a1 >> 4) << 24 | (c1 >> 4) << 28;
            }
      }
      std::memcpy(rec, words, sizeof words);
    }
  const uint64_t end = static_cast<uint64_t>(l.n_blocks) * l.n_units * l.record;
  std::memset(blob + end, 0, l.bytes - end);
  if (bias) std::memcpy(blob + l.bias, bias, static_cast<size_t>(w.cout) * sizeof(float));
  // the power of two that brings an output's largest scale to 2^(top - 1) .. 2^top
  for (int o = 0; o < l.n_blocks * 16; ++o) {
    float largest = 0.0f, power = 1.0f;
    for (int64_t gr = 0; o < w.cout && gr < n_groups; ++gr) {
      const float v = std::fabs(scale_at(w, static_cast<size_t>(o) * n_groups + gr));
      if (std::isfinite(v)) largest = std::max(largest, v);
    }
    if (largest > 0.0f) {
      int e = 0;
      std::frexp(largest, &e);
      power = std::ldexp(1.0f, std::min(126, std::max(-126, power_top(w.dtype) - e)));
    }
    std::memcpy(blob + l.power + static_cast<size_t>(o) * 4, &power, 4);
  }
}

int launch_linear_q4_pack(const LinearQ4Weights& w, const float* bias, void* blob, void* stream) {
  const LinearQ4Layout l = linear_q4_layout(w.cin, w.cout, w.group, w.scale_dtype, w.zeros != nullptr, w.dtype);
  PackParams p{};
  p.q = w.q;
  p.scales = static_cast<const unsigned char*>(w.scales);
  p.zeros = w.zeros;
  p.bias = bias;
  p.blob = static_cast<unsigned char*>(blob);
  p.pitch = (static_cast<long long>(w.cin) + 1) / 2;
  p.n_groups = (static_cast<long long>(w.cin) + w.group - 1) / w.group;
  p.bias_at = l.bias;
  p.power_at = l.power;
  p.cin = w.cin;
  p.cout = w.cout;
  p.group = w.group;
  p.scale_dtype = w.scale_dtype;
  p.n_units = l.n_units;
  p.parts = l.parts;
  p.record = l.record;
  p.zeros_at = l.zeros_at;
  p.wide = wide_scales(w.scale_dtype, w.dtype);
  p.top = power_top(w.dtype);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const uint64_t end = static_cast<uint64_t>(l.n_blocks) * l.n_units * l.record;
  const cudaError_t err = cudaMemsetAsync(p.blob + end, 0, l.bytes - end, st);
  if (err != cudaSuccess) return static_cast<int>(err);
  const int outputs = l.n_blocks * 16;
  pack_records_kernel<<<static_cast<unsigned>(l.n_blocks) * l.n_units, 128, 0, st>>>(p);
  pack_outputs_kernel<<<static_cast<unsigned>(outputs + 3) / 4, 128, 0, st>>>(p, outputs);
  return static_cast<int>(cudaGetLastError());
}

int launch_linear_q4_op(const LaunchRec& r, const Ptrs& ptr, void* stream) {
  LinearQ4Call c;
  c.blob = ptr.wts;
  c.x = ptr.in0;
  c.res = ptr.res;
  c.y = ptr.out;
  const int plane = plane_pixels(r.H, r.W);
  c.rows = r.B * plane;
  c.cin = r.C;
  c.cout = r.Co;
  c.x_slice = c.res_slice = static_cast<long long>(c.rows) * 4;
  if (r.nhwc_out) {
    c.y_row = r.Co;
    c.plane = plane;
    c.real = r.H * r.W;
  } else {
    c.y_slice = c.x_slice;
  }
  c.group = r.q4_group;
  c.scale_dtype = r.q4_scale_dtype;
  c.zeros = r.q4_zeros != 0;
  c.ep = r.ep;
  return launch_linear_q4(c, stream);
}

int launch_linear_q4(const LinearQ4Call& c, void* stream) {
  if (c.rows <= 0) return 0;
  const LinearQ4Layout l = linear_q4_layout(c.cin, c.cout, c.group, c.scale_dtype, c.zeros, c.dtype);
  if (linear_q4_tc_wanted(c)) return launch_linear_q4_tc(c, l, stream);
  const int cols_per_row = c.dtype == GI_F32 ? 3 : 1;
  const Shape s = choose_shape(c.rows, cols_per_row, l.n_blocks, l.n_units, device_sm_count());
  const bool graph = c.x_slice || c.y_slice || c.plane || c.ep.has_res;
  if (graph && (c.dtype != GI_F16 || s.nt != 1)) return static_cast<int>(cudaErrorInvalidConfiguration);  // (a graph brings 8 rows of fp16 at most)
  Params p{};
  const unsigned char* blob = static_cast<const unsigned char*>(c.blob);
  p.wts = blob;
  p.q = masks_of(c.dtype);
  p.bias = reinterpret_cast<const float*>(blob + l.bias);
  p.x = c.x;
  p.res = c.res;
  p.y = c.y;
  p.x_row = c.x_row;
  p.x_slice = c.x_slice;
  p.y_row = c.y_row;
  p.y_slice = c.y_slice;
  p.res_slice = c.res_slice;
  p.rows = c.rows;
  p.cin = c.cin;
  p.cout = c.cout;
  p.n_units = l.n_units;
  p.kw = s.kw;
  p.ks = s.ks;
  p.row_tile = s.row_tile;
  const int elem = c.dtype == GI_F32 ? 4 : 2, cols = s.row_tile * cols_per_row;
  p.tiles = s.tiles;
  p.x_vec = c.x_slice == 0 && reinterpret_cast<uintptr_t>(c.x) % 16 == 0 && (c.rows == 1 || c.x_row * elem % 16 == 0);
  // shared memory: x (as much of it as there is room for), the rings of copies, the items' sums
  const int n_sets = (l.n_blocks + s.rb - 1) / s.rb, sets = (n_sets + s.tiles - 1) / s.tiles;
  const int rings = kWarps * kSlots * 2 * l.record, sums = sets * s.kw * s.rb * cols * 16 * 4;
  const int fit = ((kSmem - rings - sums - 64) / cols - 64) / (kUnitK * 2);  // (all are whole 64 bytes, the rings begin at 128)
  const int need = (l.n_units + s.ks - 1) / s.ks, step = 2 / s.rb;
  p.chunk = std::max(1, std::min(fit / step, (need + step - 1) / step)) * step;
  p.ring_at = (cols * (p.chunk * kUnitK * 2 + 64) + 127) / 128 * 128;
  p.red_at = p.ring_at + rings;
  p.act_pre = c.ep.act_pre;
  p.has_res = c.ep.has_res;
  p.act_post = c.ep.act_post;
  p.plane = c.plane;
  p.real = c.real;
  const size_t smem = static_cast<size_t>(p.red_at) + sums;
  const long long grid = static_cast<long long>(p.tiles) * s.ks * ((c.rows + s.row_tile - 1) / s.row_tile);
  if (grid > 0x7fffffffll || smem > static_cast<size_t>(kSmem)) return static_cast<int>(cudaErrorInvalidConfiguration);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const unsigned n = static_cast<unsigned>(grid);
  const int parts = parts_of(c.group);
  cudaError_t err;
  if (wide_scales(c.scale_dtype, c.dtype)) {
    err = c.dtype == GI_F16    ? launch_type<GI_F16, true>(p, s, parts, c.zeros, n, smem, st)
          : c.dtype == GI_BF16 ? launch_type<GI_BF16, true>(p, s, parts, c.zeros, n, smem, st)
                               : launch_type<GI_F32, true>(p, s, parts, c.zeros, n, smem, st);
  } else {
    err = c.dtype == GI_F16    ? launch_type<GI_F16, false>(p, s, parts, c.zeros, n, smem, st)
          : c.dtype == GI_BF16 ? launch_type<GI_BF16, false>(p, s, parts, c.zeros, n, smem, st)
                               : launch_type<GI_F32, false>(p, s, parts, c.zeros, n, smem, st);
  }
  return static_cast<int>(err);
}

}  // namespace gi
