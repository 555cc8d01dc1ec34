// Rotary positions with one or several axes, and the page append that rotates on the way, for gfx950.
//
// Mathematics: pair i of a head (dims i and i + rot/2, or 2 i and 2 i + 1) turns by
// angle = position * inv_freq[i].  The angle is formed in turns in 64 bits,
// position * (inv_freq / 2 pi), and only its distance from the nearest whole turn is rounded to
// fp32 (2^-26 of a turn), for the hardware's sine and cosine, which take turns.
//
// A wave takes one row (token) and 8 kHeads of its heads (a workgroup four rows; workgroups of the same rows
// follow one another); lane l holds unit l % 8 of head l / 8, the 16 elements of 8 pairs in two 16-byte
// chunks, so that a lane's 8 sines and cosines serve all its heads and rows of a head are read and
// written whole.  Units past the rotated dims, and V's, are copied.  Nothing is shared between waves: no LDS, no barrier.
// Bound by the memory for many rows: 35107 rows of 32 + 8 + 8 heads, 863 MB, 160 us, 5.4 TB/s (171 with one head a
// lane; 217 with one head a lane and the groups of a row far apart); by the chain of loads for few: one row 2.9 us, 512
// rows 4.6 us (4.8 with two heads a lane), in a graph, one call after another.
#include "launch.h"
#include "s2l.h"
#include "s2l_device.h"

namespace s2l {

namespace {

// 16 and 8 bytes at any element's address (the hardware takes unaligned vectors).
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

struct RowPlace {
  int32_t req, pos;   // the request that row `row` belongs to, and its position there
};

// The request of a row and the row's position in it: the largest r with cu[r] <= row.  Each step looks at
// up to 64 offsets at once, one a lane; up to 64 requests take one round of loads.  Wave-uniform.
__device__ inline RowPlace place_row(const int32_t* __restrict__ prefix_lens, const int32_t* __restrict__ cu,
                                     int32_t num_reqs, int32_t row) {
  const int lane = threadIdx.x & 63;
  int32_t lo = 0, n = num_reqs;   // the request is one of lo .. lo + n - 1
  while (n > 64) {
    const int32_t step = (n + 63) / 64;
    const int32_t k = (lane + 1) * step;
    const bool below = k < n && cu[lo + k] <= row;
    const int32_t c = __popcll(__ballot(below));
    lo += c * step;
    n = n - c * step < step ? n - c * step : step;
  }
  const int32_t r = lo + (lane < n ? lane : n - 1);
  const int32_t begin = cu[r], p = prefix_lens[r];
  const int32_t c = __popcll(__ballot(lane < n && begin <= row)) - 1;
  RowPlace w;
  w.req = __builtin_amdgcn_readfirstlane(lo + c);
  w.pos = __builtin_amdgcn_readfirstlane(__shfl(p - begin, c, 64)) + row;
  return w;
}

__device__ inline u32x4 pack8(const float* y) {
  return u32x4{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
}
__device__ inline void unpack8(const u32x4& x, float* y) {
#pragma unroll
  for (int i = 0; i < 4; ++i) y[2 * i] = bf16lo(x[i]), y[2 * i + 1] = bf16hi(x[i]);
}
// (a, b) turned.  Products and sums are written out as the fused operations that they are: left to the compiler, the forms
// of the kernel could round differently, and pages must be those of the separate calls bit for bit.
__device__ inline void turn(float a, float b, float cs, float sn, float* ya, float* yb) {
  *ya = __builtin_fmaf(a, cs, -(b * sn));
  *yb = __builtin_fmaf(b, cs, a * sn);
}
// As the append without rotation: code = e4m3(fp32(x) * fp32(1 / scale)).
__device__ inline u32x2 encode8(const u32x4& x, float inv) {
  return u32x2{f32x4_to_fp8x4(bf16lo(x[0]) * inv, bf16hi(x[0]) * inv, bf16lo(x[1]) * inv, bf16hi(x[1]) * inv),
               f32x4_to_fp8x4(bf16lo(x[2]) * inv, bf16hi(x[2]) * inv, bf16lo(x[3]) * inv, bf16hi(x[3]) * inv)};
}

template <bool kAdjacent, bool kAppend, bool kFp8, int kHeads>
__global__ __launch_bounds__(256) void rope_kernel(RopeLaunch a) {
  const int lane = threadIdx.x & 63, unit = lane & 7;
  const int heads = a.hq + a.hkv * (kAppend ? 2 : 1);
  const uint32_t groups = (heads + 8 * kHeads - 1) / (8 * kHeads);
  const int first = (int)(blockIdx.x % groups) * 8 * kHeads;   // the wave's first head
  const int64_t row = (int64_t)(blockIdx.x / groups) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.total_rows) return;
  const int head0 = first + (lane >> 3);
  const int half = a.rot_dim / 2;
  const bool turns = unit < a.rot_dim / 16 && (!kAppend || first < a.hq + a.hkv);
  const bool pairs_apart = !kAdjacent && unit < a.rot_dim / 16;
  const int oa = pairs_apart ? 8 * unit : 16 * unit, ob = pairs_apart ? oa + half : oa + 8;

  RowPlace at{0, 0};
  if (kAppend || a.positions == nullptr) {
    if (row >= a.cu_chunk[a.num_reqs]) return;   // the device lengths hold less than the host copies: no row's page
    at = place_row(a.prefix_lens, a.cu_chunk, a.num_reqs, (int32_t)row);
  }

  u32x4 xa[kHeads], xb[kHeads];
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    const int h = head0 + 8 * j;
    if (h >= heads) continue;
    const uint16_t* src = h < a.hq ? a.q + row * a.q_stride + h * 128
                          : h < a.hq + a.hkv ? a.k + row * a.k_stride + (h - a.hq) * 128
                                             : a.v + row * a.v_stride + (h - a.hq - a.hkv) * 128;
    xa[j] = *reinterpret_cast<const u32x4_any*>(src + oa);
    xb[j] = *reinterpret_cast<const u32x4_any*>(src + ob);
  }

  float cs[8], sn[8];
  if (turns) {
    double pos[S2L_ROPE_MAX_AXES];
#pragma unroll
    for (int i = 0; i < S2L_ROPE_MAX_AXES; ++i)
      pos[i] = (double)(a.positions == nullptr ? at.pos : a.positions[(i < a.num_axes ? i : 0) * a.pos_stride + row]);
    const f32x4 f0 = *reinterpret_cast<const f32x4_any*>(a.inv_freq + 8 * unit);
    const f32x4 f1 = *reinterpret_cast<const f32x4_any*>(a.inv_freq + 8 * unit + 4);
    const uint32_t axes = (uint32_t)(a.pair_axes[unit >> 2] >> (16 * (unit & 3)));   // two bits a pair
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t axis = axes >> (2 * i) & 3;
      const double p = axis & 2 ? (axis & 1 ? pos[3] : pos[2]) : (axis & 1 ? pos[1] : pos[0]);
      const double f = (double)(i < 4 ? f0[i & 3] : f1[i & 3]) * 0.15915494309189535;
      const float angle = (float)__builtin_fma(p, f, -__builtin_rint(p * f));
      cs[i] = a.scale * __builtin_amdgcn_cosf(angle);
      sn[i] = a.scale * __builtin_amdgcn_sinf(angle);
    }
  }

  int64_t slot_row = 0;   // (page * Hkv) * 16 + slot: the row's place in the pools, head 0
  if (kAppend) {
    const int64_t page = a.block_tables[(int64_t)at.req * a.max_pages + (at.pos >> 4)];
    slot_row = page * a.hkv * 16 + (at.pos & 15);
  }
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    const int h = head0 + 8 * j;
    if (h >= heads) continue;
    if (turns && (!kAppend || h < a.hq + a.hkv)) {
      float x[8], y[8];
      unpack8(xa[j], x);
      unpack8(xb[j], y);
      float u[8], w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (!kAdjacent) turn(x[i], y[i], cs[i], sn[i], &u[i], &w[i]);
        else if (i < 4) turn(x[2 * i], x[2 * i + 1], cs[i], sn[i], &u[2 * i], &u[2 * i + 1]);
        else turn(y[2 * i - 8], y[2 * i - 7], cs[i], sn[i], &w[2 * i - 8], &w[2 * i - 7]);
      }
      xa[j] = pack8(u);
      xb[j] = pack8(w);
    }
    if (h < a.hq) {
      uint16_t* dst = a.q_out + row * a.q_out_stride + h * 128;
      *reinterpret_cast<u32x4_any*>(dst + oa) = xa[j];
      *reinterpret_cast<u32x4_any*>(dst + ob) = xb[j];
    } else if constexpr (!kAppend) {
      uint16_t* dst = a.k_out + row * a.k_out_stride + (h - a.hq) * 128;
      *reinterpret_cast<u32x4_any*>(dst + oa) = xa[j];
      *reinterpret_cast<u32x4_any*>(dst + ob) = xb[j];
    } else {
      const bool is_v = h >= a.hq + a.hkv;
      const int g = h - a.hq - (is_v ? a.hkv : 0);
      const int64_t dst = (slot_row + g * 16) * 128;
      void* pool = is_v ? a.v_pool : a.k_pool;
      if constexpr (kFp8) {
        const float inv = __fdiv_rn(1.0f, (is_v ? a.v_scale : a.k_scale)[g]);
        *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(pool) + dst + oa) = encode8(xa[j], inv);
        *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(pool) + dst + ob) = encode8(xb[j], inv);
      } else {
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(pool) + dst + oa) = xa[j];
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(pool) + dst + ob) = xb[j];
      }
    }
  }
}

// Two heads a lane share its sines and cosines and halve the waves; as long as waves are few (6 a SIMD), more of them
// hide more.  One head a lane and two, us in a graph: 32 + 8 + 8 heads, 512 rows 4.6 and 4.8, 1024 (6144 waves) 7.9 and
// 7.9, 1365 (8190) 9.6 and 8.9, 4096 24.0 and 21.8; 64 + 8 + 8 into e4m3 pages, 600 (6000) 8.3 and 8.1, 1000 11.4 and
// 10.1; 32 + 32 without pages, 768 (6144) 8.4 and 8.4, 1024 10.1 and 10.1.
template <bool kAdjacent, bool kAppend, bool kFp8>
void launch(const RopeLaunch& a, hipStream_t stream) {
  constexpr int64_t kFewWaves = 6144;
  const int heads = a.hq + a.hkv * (kAppend ? 2 : 1);
  const int64_t four_rows = ((int64_t)a.total_rows + 3) / 4, groups = (heads + 7) / 8;
  if (a.total_rows * groups <= kFewWaves)
    rope_kernel<kAdjacent, kAppend, kFp8, 1><<<dim3((uint32_t)(four_rows * groups)), 256, 0, stream>>>(a);
  else
    rope_kernel<kAdjacent, kAppend, kFp8, 2><<<dim3((uint32_t)(four_rows * ((groups + 1) / 2))), 256, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_rope(const RopeLaunch& a, hipStream_t stream) {
  if (a.total_rows == 0 || a.hq + a.hkv == 0) return hipSuccess;
  if (a.k_pool == nullptr) {
    if (a.adjacent) launch<true, false, false>(a, stream);
    else launch<false, false, false>(a, stream);
  } else if (a.fp8) {
    if (a.adjacent) launch<true, true, true>(a, stream);
    else launch<false, true, true>(a, stream);
  } else {
    if (a.adjacent) launch<true, true, false>(a, stream);
    else launch<false, true, false>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace s2l
