// Linear attention with a decay for each head, for gfx950.
//
//   S <- l S + k_i v_i^T,   out_i = scale * q_i S      (S [128 k][128 v] in fp32, l = exp(log_decay))
//
// Recurrent form: a workgroup takes 32 columns of one (request, head) state.  Thread (kg, vq) keeps rows
// 4 kg .. + 3 and columns 4 vq .. + 3 of them in registers over the request's tokens, so the state is
// read and written once, whatever the chunk's length; a row's part of q S is summed over the eight row
// groups of a wave by lane swaps and over the four waves through LDS, 16 tokens at a time.
#include "launch.h"
#include "s2l_device.h"

namespace s2l {

namespace {

typedef u32x2 __attribute__((aligned(2))) u32x2_any;
constexpr int kState = 128 * 128;    // elements of one state
constexpr int kSliceCols = 32;       // columns of a recurrent workgroup
constexpr int kTokens = 16;          // tokens between two sums over the waves

// ln of the decay: at most 0, and finite, so that 0 tokens of it are a factor 1 (-1e4 forgets all: 0 in fp32).
__device__ inline double clean_log(float g) {
  return g > 0.f ? 0.0 : g < -1e4f ? -1e4 : (double)g;
}

__device__ inline f32x4 unpack4(const u32x2& x) { return f32x4{bf16lo(x[0]), bf16hi(x[0]), bf16lo(x[1]), bf16hi(x[1])}; }

__device__ inline f32x4 load4(const uint16_t* p) {
  const u32x2 x = *reinterpret_cast<const u32x2_any*>(p);
  return unpack4(x);
}

__global__ __launch_bounds__(256) void linear_recurrent_kernel(LinearLaunch a) {
  __shared__ float s_part[kTokens][4][kSliceCols];
  const int r = blockIdx.z, h = blockIdx.y, col0 = (int)blockIdx.x * kSliceCols;
  const int C = a.chunk_lens[r], si = a.slot_in[r], so = a.slot_out[r];
  const int64_t row0 = a.cu_chunk[r];
  const int g = h / (a.hq / a.hkv);
  const int vq = threadIdx.x & 7, kg = threadIdx.x >> 3, wave = threadIdx.x >> 6;
  const int64_t at = (int64_t)h * kState + (4 * kg) * 128 + col0 + 4 * vq;   // within a slot
  const int64_t slot = (int64_t)a.hq * kState;

  f32x4 s[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (si >= 0 && si < a.num_slots) s[j] = *reinterpret_cast<const f32x4*>(a.states + si * slot + at + j * 128);
    else s[j] = f32x4{} + (si == -1 ? 0.f : __builtin_nanf(""));
  }
  const float decay = (float)exp(clean_log(a.log_decay[h]));

  for (int t0 = 0; t0 < C; t0 += kTokens) {
    const int n = C - t0 < kTokens ? C - t0 : kTokens;
    for (int t = 0; t < n; ++t) {
      const int64_t row = row0 + t0 + t;
      const f32x4 k = load4(a.k + row * a.k_stride + g * 128 + 4 * kg);
      const f32x4 v = load4(a.v + row * a.v_stride + g * 128 + col0 + 4 * vq);
      const f32x4 q = load4(a.q + row * a.q_stride + h * 128 + 4 * kg);
      f32x4 o{};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s[j][c] = __builtin_fmaf(s[j][c], decay, k[j] * v[c]);
          o[c] = __builtin_fmaf(q[j], s[j][c], o[c]);
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        o[c] += __shfl_xor(o[c], 8, 64);
        o[c] += __shfl_xor(o[c], 16, 64);
        o[c] += __shfl_xor(o[c], 32, 64);
      }
      if ((threadIdx.x & 63) < 8) *reinterpret_cast<f32x4*>(&s_part[t][wave][4 * vq]) = o;
    }
    __syncthreads();
    for (int u = threadIdx.x; u < n * kSliceCols; u += 256) {
      const int t = u / kSliceCols, c = u % kSliceCols;
      const float o = s_part[t][0][c] + s_part[t][1][c] + s_part[t][2][c] + s_part[t][3][c];
      a.out[(row0 + t0 + t) * a.out_stride + h * 128 + col0 + c] = (uint16_t)pack_bf16x2(a.scale * o, 0.f);
    }
    __syncthreads();
  }
  if (so >= 0 && so < a.num_slots) {
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4*>(a.states + so * slot + at + j * 128) = s[j];
  }
}

}  // namespace

hipError_t launch_linear_attn(const LinearLaunch& a, hipStream_t stream) {
  if (a.num_reqs == 0) return hipSuccess;
  linear_recurrent_kernel<<<dim3(128 / kSliceCols, a.hq, a.num_reqs), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace s2l
