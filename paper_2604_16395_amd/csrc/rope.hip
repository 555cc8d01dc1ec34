// Rotary positions with one or several axes, and the page append that rotates on the way, for gfx950.
//
// Mathematics: pair i of a head (dims i and i + rot/2, or 2 i and 2 i + 1) turns by
// angle = position * inv_freq[i].  The angle is formed in turns in 64 bits,
// position * (inv_freq / 2 pi), and only its distance from the nearest whole turn is rounded to
// fp32 (2^-26 of a turn), for the hardware's sine and cosine, which take turns.
//
// Norms (kNorm): a head's squares are summed over its eight lanes before the rotation, fp32 until the one rounding at
// the end.  One row 2.95 us, 35107 rows of 32 + 8 + 8 heads 163 us, as fast as a copy moves their 863 MB; 2342 rows of
// 32 + 32 without pages 18 us (77 MB, which the last-level cache holds), bound by the arithmetic and, as all waves
// are resident at once, by loading, computing and storing one after another.  Into MXFP4 pages one row 3.05 us, 35107 rows
// 148 us (757 MB), without norms 2.5 and 138; into e4m3 pages 3.1 and 149, 2.6 and 144.
//
// A wave takes one row (token) and 8 kHeads of its heads (a workgroup four rows; workgroups of the same rows
// follow one another); lane l holds unit l % 8 of head l / 8, the 16 elements of 8 pairs in two 16-byte
// chunks, so that a lane's 8 sines and cosines serve all its heads and rows of a head are read and
// written whole.  Units past the rotated dims, and V's, are copied.  Nothing is shared between waves: no barrier.
// Bound by the memory for many rows: 35107 rows of 32 + 8 + 8 heads, 863 MB, 160 us, 5.4 TB/s (171 with one head a
// lane; 217 with one head a lane and the groups of a row far apart); by the chain of loads for few: one row 2.9 us, 512
// rows 4.3 us, in a graph, one call after another.
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

// A head's norm: its 16 elements a lane times 1 / sqrt(mean square + eps) and the weights, fp32.  The sum runs over
// the head's eight lanes in a fixed order.
__device__ inline void norm16(float* x, float* y, const float* wx, const float* wy, float eps) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x[i], x[i], s);
#pragma unroll
  for (int i = 0; i < 8; ++i) s = __builtin_fmaf(y[i], y[i], s);
  s += u2f(lane_xor1(f2u(s)));
  s += u2f(lane_xor2(f2u(s)));
  s += u2f(lane_of_other_four(f2u(s)));
  const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(s, 1.0f / 128.0f, eps));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] * r * wx[i], y[i] = y[i] * r * wy[i];
}
// Eight of a head's weights from dim `d` on, with the offset.
__device__ inline void load_weights(const void* weight, bool fp32, int d, float offset, float* w) {
  if (weight == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
    return;
  }
  if (fp32) {
    const f32x4_any* p = reinterpret_cast<const f32x4_any*>(static_cast<const float*>(weight) + d);
    const f32x4 a = p[0], b = p[1];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (i < 4 ? a[i & 3] : b[i & 3]) + offset;
  } else {
    unpack8(*reinterpret_cast<const u32x4_any*>(static_cast<const uint16_t*>(weight) + d), w);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] += offset;
  }
}

template <bool kAdjacent, bool kAppend, PageKind kKind, bool kNorm, int kHeads>
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

  // the weights of the wave's first head, which are those of all its heads but where queries end within them
  float wa[8], wb[8];
  const int last = min(first + 8 * kHeads, a.hq + a.hkv) - 1;   // the wave's last head that is normed
  const bool mixed = kNorm && kHeads > 1 && first < a.hq && last >= a.hq;
  auto weights_of = [&](int h) {
    const void* weight = h < a.hq ? a.q_weight : a.k_weight;
    load_weights(weight, a.norm_fp32, oa, a.offset, wa);
    load_weights(weight, a.norm_fp32, ob, a.offset, wb);
  };
  if constexpr (kNorm) {
    if (first <= last) weights_of(head0);
  }

  // lane i takes pair i's sine and cosine, and hands them to the lanes that turn by it through the wave's part of LDS.
  // Against each lane's own 8 pairs, their sums in doubles eight times over, us: one row 2.95 and 3.18 (32 + 8 + 8 heads, normed),
  // 512 rows 4.3 and 5.3, 1024 normed 8.2 and 9.2, 4096 23.7 and 24.6; 35107 the same.
  __shared__ __attribute__((aligned(16))) float turn_by[4][2][64];
  float cs[8], sn[8];
  if (!kAppend || first < a.hq + a.hkv) {
    const int pair = lane < half ? lane : 0;
    const uint32_t axis = (uint32_t)(a.pair_axes[pair >> 5] >> (2 * (pair & 31))) & 3;   // two bits a pair
    const double p = (double)(a.positions == nullptr ? at.pos : a.positions[axis * a.pos_stride + row]);
    const double f = (double)a.inv_freq[pair] * 0.15915494309189535;
    const float angle = (float)__builtin_fma(p, f, -__builtin_rint(p * f));
    float* by = turn_by[threadIdx.x >> 6][0];
    by[lane] = a.scale * __builtin_amdgcn_cosf(angle);
    by[64 + lane] = a.scale * __builtin_amdgcn_sinf(angle);
    __builtin_amdgcn_wave_barrier();   // a wave's accesses to LDS keep their order
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const f32x4 c4 = *reinterpret_cast<const f32x4*>(by + 8 * unit + i), s4 = *reinterpret_cast<const f32x4*>(by + 64 + 8 * unit + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) cs[i + k] = c4[k], sn[i + k] = s4[k];
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
    const bool rotates = turns && (!kAppend || h < a.hq + a.hkv);
    if (rotates || (kNorm && h < a.hq + a.hkv)) {
      float x[8], y[8];
      unpack8(xa[j], x);
      unpack8(xb[j], y);
      if constexpr (kNorm) {
        if (j > 0 && mixed) weights_of(h);
        norm16(x, y, wa, wb, a.eps);
      }
      if (!kNorm || rotates) {
        float u[8], w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (!kAdjacent) turn(x[i], y[i], cs[i], sn[i], &u[i], &w[i]);
          else if (i < 4) turn(x[2 * i], x[2 * i + 1], cs[i], sn[i], &u[2 * i], &u[2 * i + 1]);
          else turn(y[2 * i - 8], y[2 * i - 7], cs[i], sn[i], &w[2 * i - 8], &w[2 * i - 7]);
        }
        xa[j] = pack8(u);
        xb[j] = pack8(w);
      } else {
        xa[j] = pack8(x);
        xb[j] = pack8(y);
      }
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
      if constexpr (kKind == kMxfp4Pages) {
        // the head's 16 chunks of eight dims lie over its eight lanes as they were paired: each block's
        // largest magnitude from its four, by a 16-bit field a block
        uint32_t m[2] = {0, 0};
        const uint32_t ma = max_magnitude(xa[j]), mb = max_magnitude(xb[j]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t fa = oa >> 6 == i ? ma << ((oa >> 1) & 16) : 0, fb = ob >> 6 == i ? mb << ((ob >> 1) & 16) : 0;
          m[i] = max_u16x2(fa, fb);
          m[i] = max_u16x2(m[i], lane_xor1(m[i]));
          m[i] = max_u16x2(m[i], lane_xor2(m[i]));
          m[i] = max_u16x2(m[i], lane_of_other_four(m[i]));
        }
        uint32_t bytes = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) bytes |= mx_scale_byte(m[i >> 1] >> (16 * (i & 1)) & 0xFFFFu) << (8 * i);
        const int slot = (int)(slot_row & 15);
        uint8_t* run = static_cast<uint8_t*>(pool) + ((slot_row >> 4) + g) * kMxRunBytes;
        uint8_t* codes = run + slot * kMxCodeBytes;
        *reinterpret_cast<uint32_t*>(codes + oa / 2) = mx_encode8(xa[j], bytes >> (oa / kMxBlock * 8) & 255u);
        *reinterpret_cast<uint32_t*>(codes + ob / 2) = mx_encode8(xb[j], bytes >> (ob / kMxBlock * 8) & 255u);
        if (unit == 0) *reinterpret_cast<uint32_t*>(run + kMxScalesAt + slot * kMxScaleBytes) = bytes;
      } else if constexpr (kKind == kE4m3Pages) {
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

// Two heads a lane halve the waves and what each does beside its heads; as long as waves are few (6 a SIMD), more of them
// hide more.  One head a lane and two, us in a graph, 32 + 8 + 8 heads: 512 rows 4.3 and 4.6, 1024 (6144 waves) 7.3 and 7.7,
// 1365 (8190) 8.8 and 8.7, 2048 10.9 and 10.5, 4096 21.8 and 22.8, 8192 40.5 and 41.0.
// With norms, four heads a lane for rows of more than 32 heads without pages, and for rows appended whose heads are 7, 11 or
// 15 groups of eight.  Time of four over that of two, mean of 1000 to 20000 rows: without pages 4 groups 1.04, 7 0.95, 8 0.96 and 1.00, 10 and 11 0.98, 12 to 16 0.99 to 1.01 (2342 rows of 32 + 32 heads 15.1 us
// and 17.1); into bf16, e4m3 and MXFP4 pages 4 groups 1.09, 1.08, 1.08, 7 0.98, 0.91, 0.92, 8 1.03, 1.01, 1.01, 10 1.01, 1.00, 1.00,
// 11 1.00, 0.96, 0.96, 12 1.02, 1.00, 1.00, 13 1.16, 1.21, 1.20, 14 1.03, 1.01, 1.01, 15 1.00, 0.91, 0.93, 16 1.02, 1.02, 1.02.
// 35107 rows of 32 + 8 + 8 into bf16 pages with two, three and four: 163.0, 164.2, 173.6 us.
template <bool kAdjacent, bool kAppend, PageKind kKind, bool kNorm>
void launch(const RopeLaunch& a, hipStream_t stream) {
  constexpr int64_t kFewWaves = 6144;
  const int heads = a.hq + a.hkv * (kAppend ? 2 : 1);
  const int64_t four_rows = ((int64_t)a.total_rows + 3) / 4, groups = (heads + 7) / 8;
  auto run = [&](auto heads_a_lane) {
    constexpr int kHeads = decltype(heads_a_lane)::value;
    rope_kernel<kAdjacent, kAppend, kKind, kNorm, kHeads>
        <<<dim3((uint32_t)(four_rows * ((groups + kHeads - 1) / kHeads))), 256, 0, stream>>>(a);
  };
  const int64_t waves = (groups + 3) / 4, a_lane = (groups + waves - 1) / waves;   // of a row: at most four heads a lane, evenly
  const bool four = kNorm && groups > 4 && (kAppend ? groups % 4 == 3 : a_lane == 4);
  if (a.total_rows * groups <= kFewWaves || (kNorm && a_lane == 1)) run(std::integral_constant<int, 1>{});
  else if (four) run(std::integral_constant<int, kNorm ? 4 : 2>{});
  else run(std::integral_constant<int, 2>{});
}

template <bool kAppend, PageKind kKind>
void launch_kind(const RopeLaunch& a, hipStream_t stream) {
  if (a.norm) {
    if (a.adjacent) launch<true, kAppend, kKind, true>(a, stream);
    else launch<false, kAppend, kKind, true>(a, stream);
  } else {
    if (a.adjacent) launch<true, kAppend, kKind, false>(a, stream);
    else launch<false, kAppend, kKind, false>(a, stream);
  }
}

}  // namespace

hipError_t launch_rope(const RopeLaunch& a, hipStream_t stream) {
  if (a.total_rows == 0 || a.hq + a.hkv == 0) return hipSuccess;
  if (a.k_pool == nullptr) launch_kind<false, kBf16Pages>(a, stream);
  else with_kind(a.kind, [&](auto kind) { launch_kind<true, decltype(kind)::value>(a, stream); });
  return hipGetLastError();
}

}  // namespace s2l
