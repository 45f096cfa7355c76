// Fully connected layer with 4-bit weights for many rows of x, on tcgen05: y = act(x w^T + bias) (linear_q4.cu has the few rows and
// the weights' layout).
//
// Beyond some 16 rows the warp-level matrix instruction takes longer than the weights' bytes (8 cycles for 16 outputs x 8 rows x 16
// channels).  Here a CTA computes 128 outputs x up to 256 rows: the weights are the A operand - sixteen warps, two for each block of 16
// outputs, expand the records that their own rings of copies bring, scale them and store them to shared memory in the swizzled
// layout (rows of 64 channels = 128 bytes, 16-byte units exchanged by the row's number) - and the rows of x the B operand, copied by
// one thread as tiles of the same layout (rows that are not in whole 16-byte units are loaded by the expanding warps instead).  One thread
// issues the products, 128 x N x 16 each; the sums stay in tensor memory until the last channel.  Expanding a record of 16 x 128 weights is
// shared by all rows of the tile.  Where outputs are few, the CTAs of a cluster share the input channels and add their sums up through
// distributed shared memory, in a fixed order.
//
// Precision: scale * (q - zero) enters as the sum of two numbers of x's type, the nearest one and what that leaves, each with a product and
// a sum of its own (where the first sum is no number, the second does not count: what is left may be 0 or of the other sign).  For scales
// in 16 bits (times 4 bits of q - zero) the two are all of it; of a scale in 32 bits, which enters in two parts as well, at least 14 digits
// are left in bf16 (16 were the fewest of 200 000), 20 in fp16 (22).  fp16 lacks range: a power of two for each output brings its largest
// scale to 2^11 .. 2^12, where 15 times it is still a number; what lies below the smallest step there is 2^-31 of that scale at most.
// Weights rounded once would take 24.8 instead of 31.7 us for 32 rows and 35 instead of 51 for 256.  q - zero alone, exact, needs sums of
// its own for each group, which the sixteen warps have to read out of tensor memory, scale and add up: 35 us for 32 rows, 78 for 256, with
// groups of 32 50 and 113.
//
// Measured (B200, 4096 -> 12288): 256 rows 51 us, 1024 rows 147 - two products for each weight, 1.0 and 1.4 PFLOP/s of them, the
// former on 96 of the 148 SMs - 32 rows 31.7 us, bound by the expansion, and 256 rows 4096 -> 4096 23 us with 4 CTAs to a sum.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "kernels.h"
#include "pdl.cuh"
#include "q4_record.cuh"
#include "sm100_ptx.cuh"
#include "tma_host.h"

namespace gi {
namespace {

using namespace ptx;
using namespace q4;

constexpr int kBlocks = 8;                     // blocks of 16 outputs of a CTA
constexpr int kWorkers = 2 * kBlocks;          // warps that expand weights - a block's two take the halves of its records - and store the results
constexpr int kCopyWarp = kWorkers, kMmaWarp = kWorkers + 1;
constexpr int kThreads = (kWorkers + 2) * 32;
constexpr int kOuts = 128, kStageK = 64;       // outputs of a CTA, channels of a stage
constexpr int kABytes = kOuts * kStageK * 2;
constexpr int kMaxStages = 4, kRing = 3;       // records that a worker has in flight
constexpr int kHeader = 1024;
constexpr unsigned kWaitNs = 1000000000u;
constexpr int kSmem = 227 * 1024;
constexpr unsigned kErrLoad = 1u, kErrMma = 2u, kErrWork = 4u, kErrDrain = 8u;

struct Params {
  const unsigned char* wts;
  const float *bias, *power;
  const unsigned short* x;   // gathered rows only
  void* y;
  long long x_row, y_row;
  int rows, cin, cout, n_blocks, n_units;
  int m_tiles, n, ks;        // tiles of outputs; rows of a tile; CTAs that share a sum
  int stages, tmem_cols;
  int act, words;            // words: rows of x in whole 32-bit words
  Masks q;
};

struct Header {
  unsigned long long full_a[kMaxStages], full_b[kMaxStages], empty[kMaxStages], done;
  unsigned tmem, abort;
};

__device__ unsigned g_q4_tc_error = 0;

// operand of rows of 128 bytes, 8 of them 1024 bytes, swizzled
__device__ __forceinline__ unsigned long long desc_of(unsigned addr) {
  return static_cast<unsigned long long>((addr & 0x3ffffu) >> 4) | 1ull << 16 | static_cast<unsigned long long>(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

__device__ __forceinline__ float act_nan(float v, int act) {
  if (act != GI_ACT_NONE && v < 0.0f) v = 0.0f;
  if (act == GI_ACT_RELU6 && v > 6.0f) v = 6.0f;
  return v;
}

// a scale of a row, doubled up in two 16-bit halves: s, and what s leaves of it
template <bool BF>
__device__ __forceinline__ void halves(float v, unsigned& s, unsigned& rest) {
  if (BF) {
    const __nv_bfloat16 h = __float2bfloat16_rn(v);
    const __nv_bfloat162 a = __bfloat162bfloat162(h), b = __float2bfloat162_rn(v - __bfloat162float(h));
    s = *reinterpret_cast<const unsigned*>(&a);
    rest = *reinterpret_cast<const unsigned*>(&b);
  } else {
    const __half h = __float2half_rn(v);
    const __half2 a = __half2half2(h), b = __float2half2_rn(v - __half2float(h));
    s = *reinterpret_cast<const unsigned*>(&a);
    rest = *reinterpret_cast<const unsigned*>(&b);
  }
}
template <bool BF>
__device__ __forceinline__ unsigned mul(unsigned a, unsigned b) {
  if (BF) {
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const unsigned*>(&r);
  }
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const unsigned*>(&r);
}
template <bool BF>
__device__ __forceinline__ unsigned fma(unsigned a, unsigned b, unsigned c) {
  if (BF) {
    const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b), *reinterpret_cast<const __nv_bfloat162*>(&c));
    return *reinterpret_cast<const unsigned*>(&r);
  }
  const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b), *reinterpret_cast<const __half2*>(&c));
  return *reinterpret_cast<const unsigned*>(&r);
}

// a b - c
template <bool BF>
__device__ __forceinline__ unsigned fms(unsigned a, unsigned b, unsigned c) {
  if (BF) {
    const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b), __hneg2(*reinterpret_cast<const __nv_bfloat162*>(&c)));
    return *reinterpret_cast<const unsigned*>(&r);
  }
  const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b), __hneg2(*reinterpret_cast<const __half2*>(&c)));
  return *reinterpret_cast<const unsigned*>(&r);
}

template <bool BF>
__device__ __forceinline__ void store_y(const Params& p, int r, int o, float v) {
  v = act_nan(v, p.act);
  if (BF) static_cast<__nv_bfloat16*>(p.y)[r * p.y_row + o] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p.y)[r * p.y_row + o] = __float2half_rn(v);
}

// Eight channels k .. k + 7 of row r of x, zero behind the last one and behind the last row.
__device__ __forceinline__ uint4 gather8(const Params& p, int r, int k) {
  if (r >= p.rows) return make_uint4(0u, 0u, 0u, 0u);
  const unsigned short* x = p.x + r * p.x_row + k;
  unsigned v[8];
  if (p.words) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = k + 2 * i < p.cin ? reinterpret_cast<const unsigned*>(x)[i] : 0u;
    return make_uint4(v[0], v[1], v[2], v[3]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = k + i < p.cin ? x[i] : 0u;
  return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

// GATHER: rows of x that a tiled copy cannot read (not in whole 16-byte units) are loaded by the warps that expand the weights.
template <bool BF, int HG, bool ZP, bool S32, bool GATHER>
__global__ void __launch_bounds__(kThreads, 1) linear_q4_tc_kernel(const __grid_constant__ CUtensorMap map, const Params p) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  constexpr int kZerosAt = zeros_at(HG, S32), kRecord = record_bytes(HG, S32, ZP), kBehind = kRecord - kUnitWeights;
  constexpr int kSlot = 512 + kBehind;  // half a record's weights, and what lies behind them
  Header* hdr = reinterpret_cast<Header*>(smem_raw);
  volatile unsigned* abort_flag = &hdr->abort;
  const unsigned base = smem_u32(smem_raw), st0 = base + kHeader;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x % p.ks, mt = blockIdx.x / p.ks % p.m_tiles, row0 = blockIdx.x / p.ks / p.m_tiles * p.n;
  const int ua = static_cast<int>(static_cast<long long>(p.n_units) * rank / p.ks), ub = static_cast<int>(static_cast<long long>(p.n_units) * (rank + 1) / p.ks);
  const int n_st = 2 * (ub - ua), b_bytes = p.n * kStageK * 2, stage_bytes = 2 * kABytes + b_bytes;  // (a stage: weights, what they leave, rows)
  const unsigned full_a = smem_u32(hdr->full_a), full_b = smem_u32(hdr->full_b), empty = smem_u32(hdr->empty), done = smem_u32(&hdr->done);

  if (threadIdx.x == 0) {
    if (!GATHER) prefetch_tensormap(&map);
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(full_a + i * 8, kBlocks);
      mbar_init(full_b + i * 8, 1);
      mbar_init(empty + i * 8, 1);
    }
    mbar_init(done, 1);
    hdr->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(&hdr->tmem), p.tmem_cols);
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  // only now: a CTA of the next kernel that took this SM's tensor memory first would wait for this kernel's end, and this CTA for it
  pdl_launch_dependents();
  const unsigned tmem = hdr->tmem;
  int asked = 0;  // copies of x asked for (the copying thread)

  if (warp < kWorkers) {
    const int half = warp / kBlocks, bl = warp % kBlocks;  // of a record; of the CTA's blocks
    const int block = min(mt * kBlocks + bl, p.n_blocks - 1), g = lane >> 2, t = lane & 3, odd = g & 1;
    const unsigned ring = st0 + p.stages * stage_bytes + warp * (kRing * kSlot);
    const unsigned char* next = p.wts + (static_cast<size_t>(block) * p.n_units + ua) * kRecord;
    if (lane == 0 && half == 0) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(next), "r"(min(kRing, ub - ua) * kRecord) : "memory");
    next += lane * 16;
    pdl_wait();
    const float power_lo = p.power[block * 16 + g], power_hi = p.power[block * 16 + g + 8];
    auto request = [&](unsigned slot) {
      copy16(slot + lane * 16, next + half * 512);
      if (lane * 16 < kBehind) copy16(slot + 512 + lane * 16, next + kUnitWeights);
      next += kRecord;
    };
#pragma unroll
    for (int j = 0; j < kRing; ++j) {
      if (j < ub - ua) request(ring + j * kSlot);
      copies_commit();
    }
    unsigned from = ring;
    int stage = half, phase = 1;  // every second stage (the first round finds them empty)
    for (int u = ua; u < ub; ++u) {
      copies_wait<kRing - 1>();
      __syncwarp();
      const uint4 w = lds128(from + lane * 16);
      // Rows of odd numbers begin with their second 32 channels: the two rows that a quarter of a warp stores at a time then lie in
      // different banks.
      const unsigned word[4] = {odd ? w.z : w.x, odd ? w.w : w.y, odd ? w.x : w.z, odd ? w.y : w.w};
      float2 f[2];
      unsigned zp[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // 32 channels: one group
        const int part = HG == 4 ? 2 * half + (h ^ odd) : HG == 2 ? half : 0;
        f[h] = load_scales<S32, BF>(from + 512 + (part * 8 + g) * (S32 ? 8 : 4));
        if (ZP) zp[h] = lds16(from + 512 + kZerosAt - kUnitWeights + (part * 8 + g) * 2);
      }
      __syncwarp();
      if (u + kRing < ub) request(from);
      copies_commit();
      from = from == ring + (kRing - 1) * kSlot ? ring : from + kSlot;
      // (the first 32 KB of the rows, half a tile of 256, are asked for ahead of the expansion)
      const int k0 = u * kUnitK + half * kStageK, chunk = bl * 32 + lane;  // 16-byte units of the tile: 8 a row, 256 by these warps at a time
      uint4 xv[4];
      if (GATHER) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j * 32 < p.n) xv[j] = gather8(p, row0 + j * 32 + chunk / 8, k0 + chunk % 8 * 8);
      }
      uint4 out[2][2][2];  // the weights; what they leave
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Zero z = ZP ? zero_of<BF>(p.q, zp[h] & 255u, zp[h] >> 8) : zero_of<BF>(p.q, 8u, 8u);
        unsigned s0, s1, r0, r1, a[2][4], left[2][4];
        halves<BF>(f[h].x * power_lo, s0, r0);
        halves<BF>(f[h].y * power_hi, s1, r1);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          expand<BF>(p.q, word[2 * h + s], z, a[s]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const unsigned v = a[s][e], sc = e & 1 ? s1 : s0, rest = e & 1 ? r1 : r0;
            a[s][e] = S32 ? fma<BF>(v, sc, mul<BF>(v, rest)) : mul<BF>(v, sc);
            left[s][e] = fms<BF>(v, sc, a[s][e]);  // exact
            if (S32) left[s][e] = fma<BF>(v, rest, left[s][e]);
          }
        }
        out[0][h][0] = make_uint4(a[0][0], a[0][2], a[1][0], a[1][2]);
        out[0][h][1] = make_uint4(a[0][1], a[0][3], a[1][1], a[1][3]);
        out[1][h][0] = make_uint4(left[0][0], left[0][2], left[1][0], left[1][2]);
        out[1][h][1] = make_uint4(left[0][1], left[0][3], left[1][1], left[1][3]);
      }
      if (!mbar_wait_warp(empty + stage * 8, phase, abort_flag, kWaitNs, &g_q4_tc_error, kErrWork)) break;
      const unsigned row = st0 + stage * stage_bytes + (bl * 16 + g) * 128;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const unsigned at = static_cast<unsigned>((4 * (h ^ odd) + t) ^ g) << 4;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          sts128(row + i * kABytes + at, out[i][h][0].x, out[i][h][0].y, out[i][h][0].z, out[i][h][0].w);
          sts128(row + i * kABytes + 8 * 128 + at, out[i][h][1].x, out[i][h][1].y, out[i][h][1].z, out[i][h][1].w);
        }
      }
      if (GATHER) {
        const unsigned b = st0 + stage * stage_bytes + 2 * kABytes;
        for (int j0 = 0; j0 < p.n; j0 += 128) {
          if (j0) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (j0 + j * 32 < p.n) xv[j] = gather8(p, row0 + j0 + j * 32 + chunk / 8, k0 + chunk % 8 * 8);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int r = j0 + j * 32 + chunk / 8;
            if (r < p.n) sts128(b + r * 128 + static_cast<unsigned>((chunk ^ r) & 7) * 16, xv[j].x, xv[j].y, xv[j].z, xv[j].w);
          }
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // visible to the tensor core
      __syncwarp();
      if (lane == 0) mbar_arrive(full_a + stage * 8);
      stage += 2;
      if (stage >= p.stages) stage -= p.stages, phase ^= 1;
    }
    copies_wait<0>();
  } else if (warp == kCopyWarp) {
    if (!GATHER && lane == 0) {
      pdl_wait();
      int stage = 0, phase = 1;
      for (; asked < n_st; ++asked) {
        if (!mbar_wait_parked(empty + stage * 8, phase, abort_flag, kWaitNs, &g_q4_tc_error, kErrLoad)) break;
        mbar_expect_tx(full_b + stage * 8, b_bytes);
        tma_load_2d(st0 + stage * stage_bytes + 2 * kABytes, &map, ua * kUnitK + asked * kStageK, row0, full_b + stage * 8);
        if (++stage == p.stages) stage = 0, phase ^= 1;
      }
    }
    __syncwarp();
  } else {
    const bool issuer = elect_one();
    const unsigned idesc = (1u << 4) | (BF ? (1u << 7) | (1u << 10) : 0u) | (static_cast<unsigned>(p.n >> 3) << 17) | ((kOuts >> 4) << 24);
    int stage = 0, phase = 0;
    for (int it = 0; it < n_st; ++it) {
      if ((!GATHER && !mbar_wait_warp(full_b + stage * 8, phase, abort_flag, kWaitNs, &g_q4_tc_error, kErrMma)) ||
          !mbar_wait_warp(full_a + stage * 8, phase, abort_flag, kWaitNs, &g_q4_tc_error, kErrMma))
        break;
      tc_fence_after();
      if (issuer) {
        const unsigned at = st0 + stage * stage_bytes;
        const unsigned long long a = desc_of(at), left = desc_of(at + kABytes), b = desc_of(at + 2 * kABytes);
#pragma unroll
        for (int k = 0; k < kStageK / 16; ++k) {
          umma_f16(tmem, a + k * 2, b + k * 2, idesc, it > 0 || k > 0 ? 1u : 0u);
          umma_f16(tmem + p.n, left + k * 2, b + k * 2, idesc, it > 0 || k > 0 ? 1u : 0u);
        }
        umma_commit(empty + stage * 8);
      }
      __syncwarp();
      if (++stage == p.stages) stage = 0, phase ^= 1;
    }
    if (issuer) umma_commit(done);  // (also where it gave up: nothing is freed while products are in flight)
    __syncwarp();
  }

  bool good = true;
  if (warp < kWorkers || warp == kMmaWarp) good = mbar_wait_warp(done, 0, abort_flag, kWaitNs, &g_q4_tc_error, warp == kMmaWarp ? kErrDrain : kErrWork);
  if (warp == kMmaWarp && !good) {
    unsigned none = 0;
    mbar_wait_warp(done, 0, &none, kWaitNs, &g_q4_tc_error, kErrDrain);
  }
  tc_fence_after();
  const bool give_up = __syncthreads_or(static_cast<int>(*abort_flag));
  if (give_up) {
    // the copies in flight land before the CTA leaves (bounded as well), nothing is stored
    if (warp == kCopyWarp && lane == 0)
      for (int j = max(0, asked - p.stages); j < asked; ++j) {
        unsigned none = 0;
        mbar_wait(full_b + j % p.stages * 8, (j / p.stages) & 1, &none, kWaitNs, &g_q4_tc_error, kErrDrain);
      }
  } else if (warp < kWorkers) {
    // a thread holds an output, 16 rows at a time
    const int ol = (warp & 3) * 32 + lane, o = mt * kOuts + ol;
    const bool real = o < p.cout;
    const float inverse = real ? 1.0f / p.power[o] : 0.0f, bias = real ? p.bias[o] : 0.0f;
    float* sums = reinterpret_cast<float*>(smem_raw + kHeader);  // [row][output]: the stages' place
    for (int c = (warp >> 2) * 16; c < p.n; c += kWorkers / 4 * 16) {
      unsigned v[16], left[16];
      tmem_ld16(tmem + (static_cast<unsigned>((warp & 3) * 32) << 16) + c, v);
      tmem_ld16(tmem + (static_cast<unsigned>((warp & 3) * 32) << 16) + p.n + c, left);
      tmem_ld_wait16(v);
      tmem_ld_wait16(left);
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        // (an infinity in x times what is left of a weight, which may be 0 or of the other sign, is not to count)
        if ((v[j] & 0x7f800000u) != 0x7f800000u) v[j] = __float_as_uint(__uint_as_float(v[j]) + __uint_as_float(left[j]));
        if (p.ks > 1) sums[(c + j) * kOuts + ol] = __uint_as_float(v[j]);
        else if (real && row0 + c + j < p.rows) store_y<BF>(p, row0 + c + j, o, fmaf(__uint_as_float(v[j]), inverse, bias));
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, p.tmem_cols);
  }
  if (p.ks > 1) {
    cluster_sync();
    if (!give_up) {
      const unsigned sums = st0;
      const int total = min(p.n, p.rows - row0) * kOuts;
      for (int i = (threadIdx.x + rank * kThreads) * 4; i < total; i += kThreads * p.ks * 4) {
        const int o = mt * kOuts + (i & (kOuts - 1)), row = row0 + i / kOuts;
        float4 part[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k < p.ks) {
            const unsigned from = mapa_shared(sums + i * 4, k);
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(part[k].x), "=f"(part[k].y), "=f"(part[k].z), "=f"(part[k].w)
                         : "r"(from)
                         : "memory");
          }
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k < p.ks) {
            v[0] += part[k].x;
            v[1] += part[k].y;
            v[2] += part[k].z;
            v[3] += part[k].w;
          }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (o + j < p.cout) store_y<BF>(p, row, o + j, fmaf(v[j], 1.0f / p.power[o + j], p.bias[o + j]));
      }
    }
    cluster_sync();  // nobody leaves while its shared memory is read
  }
}

template <bool BF, bool S32, bool G>
void (*kernel_of(int parts, bool zeros))(const CUtensorMap, const Params) {
  return parts == 1   ? (zeros ? linear_q4_tc_kernel<BF, 1, true, S32, G> : linear_q4_tc_kernel<BF, 1, false, S32, G>)
         : parts == 2 ? (zeros ? linear_q4_tc_kernel<BF, 2, true, S32, G> : linear_q4_tc_kernel<BF, 2, false, S32, G>)
                      : (zeros ? linear_q4_tc_kernel<BF, 4, true, S32, G> : linear_q4_tc_kernel<BF, 4, false, S32, G>);
}
template <bool G>
void (*kernel_of(bool bf, bool wide, int parts, bool zeros))(const CUtensorMap, const Params) {
  return bf ? (wide ? kernel_of<true, true, G>(parts, zeros) : kernel_of<true, false, G>(parts, zeros))
            : (wide ? kernel_of<false, true, G>(parts, zeros) : kernel_of<false, false, G>(parts, zeros));
}

}  // namespace

bool linear_q4_tc_wanted(const LinearQ4Call& c) {
  return c.rows > 16 && c.dtype != GI_F32 && !c.x_slice && !c.y_slice && !c.plane && !c.ep.has_res;
}

int launch_linear_q4_tc(const LinearQ4Call& c, const LinearQ4Layout& l, void* stream) {
  Params p{};
  const unsigned char* blob = static_cast<const unsigned char*>(c.blob);
  p.wts = blob;
  p.bias = reinterpret_cast<const float*>(blob + l.bias);
  p.power = reinterpret_cast<const float*>(blob + l.power);
  p.y = c.y;
  p.y_row = c.y_row;
  p.x = static_cast<const unsigned short*>(c.x);
  p.x_row = c.x_row;
  p.rows = c.rows;
  p.cin = c.cin;
  p.cout = c.cout;
  p.words = reinterpret_cast<uintptr_t>(c.x) % 4 == 0 && c.x_row % 2 == 0 && c.cin % 2 == 0;
  // rows in whole 16-byte units are what a tiled copy can read
  const bool gather = reinterpret_cast<uintptr_t>(c.x) % 16 != 0 || c.x_row % 8 != 0;
  p.n_blocks = l.n_blocks;
  p.n_units = l.n_units;
  p.act = c.ep.act_pre;
  p.q = masks_of(c.dtype);
  p.m_tiles = (l.n_blocks + kBlocks - 1) / kBlocks;
  // Tiles of up to 256 rows, which expand the weights once; CTAs that share a sum, as many as fill the GPU, each with 512 channels or
  // more; where even that leaves SMs idle, smaller tiles of rows (256 rows 1280 -> 1001 17 us with 16 CTAs).
  const int sms = device_sm_count();
  long long row_tiles = (static_cast<long long>(c.rows) + 255) / 256;
  p.ks = 1;
  while (p.ks < 8 && p.m_tiles * row_tiles * p.ks * 2 <= sms && p.n_units >= 8 * p.ks) p.ks *= 2;
  while (p.m_tiles * row_tiles * p.ks * 2 <= sms && c.rows > 32 * row_tiles) row_tiles *= 2;
  p.n = static_cast<int>((c.rows + row_tiles - 1) / row_tiles + 15) / 16 * 16;
  row_tiles = (static_cast<long long>(c.rows) + p.n - 1) / p.n;
  p.tmem_cols = 32;
  while (p.tmem_cols < 2 * p.n) p.tmem_cols *= 2;
  const int rings = kWorkers * kRing * (l.record - kUnitWeights / 2), stage = 2 * kABytes + p.n * kStageK * 2;
  p.stages = std::min(kMaxStages, (kSmem - kHeader - rings) / stage);
  const size_t smem = kHeader + std::max<size_t>(static_cast<size_t>(p.stages) * stage + rings, p.ks > 1 ? static_cast<size_t>(p.n) * kOuts * 4 : 0);
  const long long grid = p.m_tiles * row_tiles * p.ks;
  if (grid > 0x7fffffffll || p.stages < 2 || smem > static_cast<size_t>(kSmem)) return static_cast<int>(cudaErrorInvalidConfiguration);

  CUtensorMap map{};
  EncodeTiledFn enc = tensor_map_encoder();
  if (!gather && !enc) return static_cast<int>(cudaErrorNotSupported);
  const cuuint64_t dim[2] = {static_cast<cuuint64_t>(c.cin), static_cast<cuuint64_t>(c.rows)};
  const cuuint64_t pitch[1] = {static_cast<cuuint64_t>(c.x_row) * 2};
  const cuuint32_t box[2] = {kStageK, static_cast<cuuint32_t>(p.n)};
  const cuuint32_t one[2] = {1, 1};
  if (!gather && enc(&map, c.dtype == GI_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(c.x), dim, pitch, box, one,
          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return static_cast<int>(cudaErrorInvalidValue);

  const int parts = parts_of(c.group);
  const bool wide = wide_scales(c.scale_dtype, c.dtype), bf = c.dtype == GI_BF16;
  void (*k)(const CUtensorMap, const Params) = gather ? kernel_of<true>(bf, wide, parts, c.zeros) : kernel_of<false>(bf, wide, parts, c.zeros);
  static bool raised[2][2][2][3][2][kMaxDevices] = {};
  bool& ready = raised[gather][bf][wide][parts / 2][c.zeros][current_device_slot()];
  if (!ready) {
    const cudaError_t err = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (err != cudaSuccess) return static_cast<int>(err);
    ready = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(p.ks);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.ks > 1 ? 2 : 1;
  return static_cast<int>(cudaLaunchKernelEx(&cfg, k, map, p));
}

unsigned int linear_q4_tc_error_word(int* cuda_err) {
  unsigned int v = 0;
  const cudaError_t e = cudaMemcpyFromSymbol(&v, g_q4_tc_error, sizeof v);
  if (cuda_err) *cuda_err = static_cast<int>(e);
  return v;
}

}  // namespace gi
