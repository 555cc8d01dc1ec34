// Linear attention with a decay for each head, for gfx950.
//
//   S <- l S + k_i v_i^T,   out_i = scale * q_i S      (S [128 k][128 v] in fp32, l = exp(log_decay))
//
// Requests of up to kLinearShortTokens new tokens take the recurrent form: a workgroup takes 32 columns of one
// (request, head) state.  Thread (kg, vq) keeps rows 4 kg .. + 3 and columns 4 vq .. + 3 of them in
// registers over the request's tokens, so the state is read and written once; a row's part of q S is
// summed over the eight row groups of a wave by lane swaps and over the four waves through LDS.  Bound by the
// states: 64 requests of a token, 32 heads, 270 MB, 49 us, 5.5 TB/s; one request 3.2 us, by its chain of loads.
// The launch has workgroups for every request, and those of long ones leave: a search for the short ones took
// 51.5 us there, 632 instead of 392 for 2048 requests of 8 heads; 64 chunks of 100 tokens and one token cost 2% more.
//
// Longer chunks take the blocked form, 32 tokens at a time: with n of them valid (zero rows behind),
//   out_i = scale (sum_{j <= i} l^(i-j) (q_i . k_j) v_j + l^(i+1) q_i S),
//   S'    = l^n S + sum_j k_j (l^(n-1-j) v_j)^T,
// all products on the bf16 MFMA.  A workgroup of four waves takes one head of one piece of a request; wave w owns
// columns 32 w .. + 31 of S (64 accumulators a lane) and of the output.  Waves share the Q, K and V tiles, and
// the block's scores, of which each forms a quarter (16 x 16), one block ahead.
//   * Scores come out transposed (A = K rows, B = Q rows): a lane holds one query and four keys, which it
//     writes as a part of that query's row; the rows are read back as an operand against V's columns, which the
//     transposing LDS read (ds_read_b64_tr_b16) hands out in the same order of keys.
//   * Accumulator row 16 s + 8 b + 4 half + a of a state tile holds key dim 16 s + 8 half + 4 b + a of it
//     (the K columns are read in that order), so that S^T is an operand against Q's rows as they lie.
//   * Factors that are no bf16 values are sums of bf16 terms.  For outputs, bf16 in the end, two terms do (scores,
//     S, and l^(n-1-j) v in the running S of a piece: off by 2^-16); for the state that the call returns three,
//     off by 2^-24.  One term in S would save 2% of a long prompt's time and make the error against 64 bits
//     1.4 times that of the final rounding alone.
// Two workgroups fit a CU (80 KiB of LDS, 256 registers a lane).  16 columns a wave and eight waves a workgroup took 1.25
// times as long: every wave reads all of K and Q from LDS.  Few whole chunks take 16 columns a wave all the same, and
// two workgroups a head (linear_narrow_kernel).
//
// A piece of a chunk needs the state before it.  Chunks that are cut take three launches: what each piece alone
// makes of its tokens, in its place of the workspace; their running sum under the decay; then the blocks,
// which read K and V a second time.  Bound by the memory: 32768 tokens of 32 heads, 1.08 GB, 372 to 388 us (127 to 142 for
// the pieces' own states, 12 for the sums, 240 to 310 for the blocks; 362 in all with the loads and stores alone).  Short
// chunks are bound by the blocks one after another and by the start of each launch (a unit's search 1 us, its states
// and first tiles 3): 32 heads, 64 tokens 7.9 us, 256 17.2, 512 29 to 30 either way, 2048 in pieces 47.
#include "launch.h"
#include "s2l_device.h"

namespace s2l {

namespace {

typedef u32x2 __attribute__((aligned(2))) u32x2_any;   // at any element's address (the hardware takes
typedef u32x4 __attribute__((aligned(2))) u32x4_any;   // unaligned vectors)
constexpr int kState = 128 * 128;    // elements of one state

// ln of the decay: at most 0, and finite, so that 0 tokens of it are a factor 1 (-1e4 forgets all: 0 in fp32).
__device__ inline double clean_log(float g) {
  return g > 0.f ? 0.0 : g < -1e4f ? -1e4 : (double)g;
}
// log2 of a decay in two fp32 terms, and powers of the decay: the whole part of the exponent is taken out before anything is
// rounded, so that a power is off by the rounding of its fraction (2^-25) and by exp2's (2^-23 at most) however large the
// exponent.  S is kept up to 2^kMostBehind behind and weights near 1 are products of such powers: with exponents rounded
// whole (2^-19 at 60) states after 2049 to 4205 tokens were off by up to 2.4e-6 of their norm, like this by 1.7e-7, for
// 0.4 to 0.9% of a call's time.
struct Decay {
  float hi, lo;
  __device__ explicit Decay(float log_decay) {
    const double l = clean_log(log_decay) * 1.4426950408889634;
    hi = (float)l;
    lo = (float)(l - (double)hi);
  }
  __device__ float exponent(int n) const { return __builtin_fmaf((float)n, hi, (float)n * lo); }
  __device__ float power(int n) const {
    const float m = (float)n, whole = fmaxf(__builtin_rintf(m * hi), -1000.f);   // 2^-1000 is 0 too, and an int
    return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(__builtin_fmaf(m, lo, __builtin_fmaf(m, hi, -whole))), (int)whole);
  }
};

// Piece `seg` of request `req`: what a workgroup works on.
struct Piece {
  int32_t req, seg, len;        // len: the request's tokens
  int32_t ws;                   // workspace index of the request's first piece
  int32_t row, slot_in, slot_out;   // of the request
};

// Inclusive sum over the lanes of a wave: within rows of 16 lanes, then across them (lanes that a step gives
// nothing add 0).
__device__ inline int32_t wave_scan(int32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // row_bcast:31 into rows 2 and 3
  return x;
}

// The idx-th of the batch's pieces of long requests (of all of them, or kCut: of those that are cut), 64 requests at a
// time, all that is known of them in one round of loads.  Pieces come longest first (by eighths of the longest): the
// longest then have a CU of their own while there are fewer than CUs, and do not begin last (11 requests of 17 to
// 2048 tokens, 32 heads: 199 us in the batch's order, 141 in this).
template <bool kCut>
__device__ inline Piece find_piece(const LinearLaunch& a, int32_t idx) {
  const int lane = threadIdx.x & 63;
  int32_t ws = 0;
  for (int32_t r0 = 0; r0 < a.num_reqs; r0 += 64) {
    const int32_t count = a.num_reqs - r0 < 64 ? a.num_reqs - r0 : 64;
    const int32_t r = r0 + (lane < count ? lane : 0);
    const int32_t row = a.cu_chunk[r], slot_in = a.slot_in[r], slot_out = a.slot_out[r], l = a.chunk_lens[r];
    const int32_t len = lane < count ? l : -1;
    const int32_t pieces = len > kLinearShortTokens ? (len + a.piece_tokens - 1) / a.piece_tokens : 0;
    const int32_t cut = pieces > 1 ? pieces : 0, entries = cut ? cut + 1 : 0;   // workspace entries
    const int32_t mine = kCut ? cut : pieces;
    int32_t before = 0, ws_before = 0;   // units that come before this lane's request's, and entries
    if (a.num_reqs > 1) {
      ws_before = wave_scan(entries) - entries;
      const int32_t size = len < a.piece_tokens ? len : a.piece_tokens;
      const int32_t eighth = min(7, (int32_t)((float)size * (8.f / (float)a.unit_tokens)));
      int32_t base = 0;
#pragma unroll
      for (int32_t c = 7; c >= 0; --c) {
        const int32_t sum = wave_scan(eighth == c ? mine : 0);
        if (eighth == c) before = base + sum - mine;
        base += __builtin_amdgcn_readlane(sum, 63);
      }
    }
    const uint64_t here = __ballot(idx >= before && idx < before + mine);
    if (here != 0) {
      const int32_t c = __builtin_ctzll(here);
      Piece p;
      p.req = r0 + c;
      p.len = __builtin_amdgcn_readlane(len, c);
      p.seg = idx - __builtin_amdgcn_readlane(before, c);
      p.ws = ws + __builtin_amdgcn_readlane(ws_before, c);
      p.row = __builtin_amdgcn_readlane(row, c);
      p.slot_in = __builtin_amdgcn_readlane(slot_in, c);
      p.slot_out = __builtin_amdgcn_readlane(slot_out, c);
      return p;
    }
    idx -= __builtin_amdgcn_readlane(wave_scan(mine), 63);
    ws += __builtin_amdgcn_readlane(wave_scan(entries), 63);
  }
  return Piece{-1, 0, 0, 0, 0, 0, 0};   // the device lengths hold less than the host copies: nothing to do
}

// ---- recurrent form ----

constexpr int kSliceCols = 32;       // columns of a recurrent workgroup

__device__ inline f32x4 unpack4(const u32x2& x) { return f32x4{bf16lo(x[0]), bf16hi(x[0]), bf16lo(x[1]), bf16hi(x[1])}; }

// The four slices of a state follow one another on one XCD (51.1 us without), five workgroups at a time on a CU: more of
// them spread over more pages of the memory (seven 50.4 us, 2048 requests of 8 heads 391 and with four 364), and fewer
// leave a rest (64 requests of 8 heads 13.2 us, with four 14.3).
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(5, 5))) void linear_recurrent_kernel(LinearLaunch a) {
  __shared__ float s_part[kLinearShortTokens][4][kSliceCols];
  const int r = blockIdx.y, h = (int)(blockIdx.x / 32) * 8 + (int)(blockIdx.x % 8), col0 = (int)(blockIdx.x / 8 % 4) * kSliceCols;
  if (h >= a.hq) return;
  const int C = a.chunk_lens[r], si = a.slot_in[r], so = a.slot_out[r];
  const int64_t row0 = a.cu_chunk[r];
  if (C > kLinearShortTokens) return;
  const int g = h / (a.hq / a.hkv);
  const int vq = threadIdx.x & 7, kg = threadIdx.x >> 3, wave = threadIdx.x >> 6;
  const int64_t at = (int64_t)h * kState + (4 * kg) * 128 + col0 + 4 * vq;   // within a slot
  const int64_t slot = (int64_t)a.hq * kState;

  f32x4 s[4];
  if (si >= 0 && si < a.num_slots) {
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = *reinterpret_cast<const f32x4*>(a.states + si * slot + at + j * 128);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = f32x4{} + (si == -1 ? 0.f : __builtin_nanf(""));
  }
  // four tokens' rows are loaded while the four before are worked on
  constexpr int kAhead = 4;
  const uint16_t* kp = a.k + row0 * a.k_stride + g * 128 + 4 * kg;
  const uint16_t* vp = a.v + row0 * a.v_stride + g * 128 + col0 + 4 * vq;
  const uint16_t* qp = a.q + row0 * a.q_stride + h * 128 + 4 * kg;
  u32x2 kn[kAhead] = {}, vn[kAhead] = {}, qn[kAhead] = {};
  auto load = [&](int t0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (t0 + i >= C) break;
      kn[i] = *reinterpret_cast<const u32x2_any*>(kp + (t0 + i) * a.k_stride);
      vn[i] = *reinterpret_cast<const u32x2_any*>(vp + (t0 + i) * a.v_stride);
      qn[i] = *reinterpret_cast<const u32x2_any*>(qp + (t0 + i) * a.q_stride);
    }
  };
  load(0);
  const float decay = (float)exp(clean_log(a.log_decay[h]));

  for (int t0 = 0; t0 < C; t0 += kAhead) {
    u32x2 kc[kAhead], vc[kAhead], qc[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) kc[i] = kn[i], vc[i] = vn[i], qc[i] = qn[i];
    if (t0 + kAhead < C) load(t0 + kAhead);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (t0 + i >= C) break;
      const f32x4 k = unpack4(kc[i]), v = unpack4(vc[i]), q = unpack4(qc[i]);
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
        o[c] += u2f(__builtin_amdgcn_update_dpp(0, f2u(o[c]), 0x128, 0xF, 0xF, false));   // row_ror:8
        o[c] = sum_of_four(o[c]);
      }
      if ((threadIdx.x & 63) < 8) *reinterpret_cast<f32x4*>(&s_part[t0 + i][wave][4 * vq]) = o;
    }
  }
  if (so >= 0 && so < a.num_slots) {
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4*>(a.states + so * slot + at + j * 128) = s[j];
  }
  __syncthreads();
  for (int u = threadIdx.x; u < C * kSliceCols; u += 256) {
    const int t = u / kSliceCols, c = u % kSliceCols;
    const float o = s_part[t][0][c] + s_part[t][1][c] + s_part[t][2][c] + s_part[t][3][c];
    a.out[(row0 + t) * a.out_stride + h * 128 + col0 + c] = (uint16_t)pack_bf16x2(a.scale * o, 0.f);
  }
}

// ---- blocked form ----

constexpr int kB = kLinearBlockTokens;
static_assert(kB == 32, "a block is one MFMA tile of tokens");
constexpr int kRow = 256;                // bytes of a row of a tile in LDS
constexpr int kTile = kB * kRow;
// Rows lie with their 16-byte chunks permuted, chunk c of row r at c ^ perm(r): 16 consecutive rows put one
// chunk on 16 places (reads of one chunk of many rows), four consecutive rows put four chunks into four
// different quarters (transposing reads of four rows by four chunks).
__device__ inline int perm(int row) { return (row & 3) << 2 | ((row >> 2) & 3); }

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

// Columns of 4 + 4 rows of a tile (the rows 8 apart), as an operand: addresses of the two reads.
__device__ inline bf16x8 read_columns(const uint8_t* x, const uint8_t* y) {
  const v4i16 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)x);
  const v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)y);
  const u32x2 a = __builtin_bit_cast(u32x2, u), b = __builtin_bit_cast(u32x2, v);
  return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
}
__device__ inline bf16x8 read_row(const uint8_t* p) { return *reinterpret_cast<const bf16x8*>(p); }

__device__ inline bf16x8 read_halves(const uint8_t* x, const uint8_t* y) {
  const u32x2 a = *reinterpret_cast<const u32x2*>(x), b = *reinterpret_cast<const u32x2*>(y);
  return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
}

__device__ inline f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mfma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// (lo, hi) less the bf16 pair w: one v_dot2_f32_bf16 each instead of unpacking and subtracting.  Exact,
// as w is their rounding.  (By value: a bit cast of a vector's element itself takes the vector's first.)
// (-1, 0) is kept in a register: written as the inline constant -1.0 it came out as (0, -1).
__device__ inline void take_off(uint32_t w, float& lo, float& hi) {
  uint32_t first = 0x0000BF80u;
  __asm__("" : "+s"(first));
  const bf16x2 p = __builtin_bit_cast(bf16x2, w);
  lo = __builtin_amdgcn_fdot2_f32_bf16(p, __builtin_bit_cast(bf16x2, first), lo, false);
  hi = __builtin_amdgcn_fdot2_f32_bf16(p, __builtin_bit_cast(bf16x2, 0xBF800000u), hi, false);
}

// x as a sum of kTerms bf16 vectors, each the rounding of what the ones before leave.
template <int kTerms>
struct Terms {
  bf16x8 t[kTerms];
};
template <int kTerms>
__device__ inline Terms<kTerms> split(float* x) {
  Terms<kTerms> r;
#pragma unroll
  for (int i = 0; i < kTerms; ++i) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
      take_off(w[j], x[2 * j], x[2 * j + 1]);   // unused after the last: gone
    }
    r.t[i] = __builtin_bit_cast(bf16x8, w);
  }
  return r;
}

// acc where both bf16 of w are finite (0 times them is 0), else NaN.
__device__ inline float probe_bf16x2(uint32_t w, float acc) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), bf16x2{}, acc, false);
}

// The block's tile is there: at most kNewer vector-memory operations of this wave are younger than its
// copies, and every wave has read what it wanted of the tile that is overwritten next.
template <int kNewer>
__device__ inline void tile_barrier() {
  __asm__ volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kNewer) : "memory");
}
// What the workgroup's waves wrote to LDS is there.
__device__ inline void lds_barrier() { __asm__ volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// kOutputs: the blocks of all pieces, with outputs; of requests that are not cut, the state after them too.
// Otherwise what each piece of a cut request alone makes of its tokens (piece 0: of the request's state
// too), and a copy of the request's state.
// kDirect: tiles are copied straight into LDS, kStages - 1 blocks ahead; rows at addresses or strides that
// those copies do not take go through registers, one block ahead.
constexpr float kMostBehind = 60.f;
constexpr int kScores = kB * 2 * kB;     // bytes of a block's scores in one term: rows of a query's 32 bf16
template <bool kOutputs, bool kDirect>
__global__ __launch_bounds__(256, 2) void linear_block_kernel(LinearLaunch a) {
  constexpr int kTiles = kOutputs ? 3 : 2;             // K, V, Q
  constexpr int kStages = kOutputs ? 3 : kDirect ? 4 : 2;
  constexpr int kStage = kTiles * kTile, kRing = kStages * kStage;
  constexpr int kCopies = 2 * kTiles, kStores = 2;   // a wave's, for a block
  __shared__ __attribute__((aligned(1024))) uint8_t s_ring[kRing];
  __shared__ __attribute__((aligned(1024))) uint8_t s_score[kOutputs ? 4 * kScores : 16];   // two blocks' two terms
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, n = lane & 31;
  const int group = a.hq / a.hkv;
  // workgroups of one key head's queries follow one another on one XCD, which then reads K and V once
  const int unit = (int)(blockIdx.x / (8 * group)) * 8 + (int)(blockIdx.x % 8);
  const int h0 = (int)(blockIdx.x / 8) % group;
  if (unit >= a.num_units * a.hkv) return;
  const int g = unit % a.hkv, h = g * group + h0;
  const float log_decay = a.log_decay[h];
  Piece p = find_piece<!kOutputs>(a, unit / a.hkv);
  if (p.req < 0) return;
  p.seg = __builtin_amdgcn_readfirstlane(p.seg);
  p.len = __builtin_amdgcn_readfirstlane(p.len);
  p.ws = __builtin_amdgcn_readfirstlane(p.ws);
  p.row = __builtin_amdgcn_readfirstlane(p.row);
  const int pieces = (p.len + a.piece_tokens - 1) / a.piece_tokens;
  const bool cut = pieces > 1;
  const int first = p.seg * a.piece_tokens, len = min(a.piece_tokens, p.len - first);
  if (cut && p.ws + pieces >= a.ws_states) return;   // as above: more than the host copies hold
  const int64_t row0 = (int64_t)p.row + first;
  const int si = __builtin_amdgcn_readfirstlane(p.slot_in), so = __builtin_amdgcn_readfirstlane(p.slot_out);
  const int64_t slot = (int64_t)a.hq * kState;
  float* const ws = a.ws + ((int64_t)p.ws + p.seg) * slot + (int64_t)h * kState;
  const int blocks = (len + kB - 1) / kB;

  // this wave's rows 8 wave + 4 d + (lane / 16) of each tile, 16 bytes a lane
  const int srow = 8 * wave + (lane >> 4), place = lane & 15;
  const uint16_t* src[3] = {a.k + row0 * a.k_stride + g * 128, a.v + row0 * a.v_stride + g * 128,
                            kOutputs ? a.q + row0 * a.q_stride + h * 128 : nullptr};
  const int64_t stride[3] = {a.k_stride, a.v_stride, a.q_stride};
  const uint32_t ring0 = (uint32_t)(uintptr_t)(lds_void*)s_ring;
  uint32_t off[kTiles][2];
  u32x4 st[kTiles][2];
  // A piece's own state takes its blocks from the last to the first: the launch leaves the first ones in the
  // memory-side cache, where the outputs' launch begins.
  auto nth = [&](int b) { return kOutputs ? b : blocks - 1 - b; };
  auto copy = [&](int b, int at) {      // straight into LDS; rows past the piece read as zero
    const int block = nth(b), rows = min(kB, len - block * kB);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const i32x4 rs = sgpr_rsrc(src[t] + (int64_t)block * kB * stride[t], (rows - 1) * (int32_t)stride[t] * 2 + kRow);
#pragma unroll
      for (int d = 0; d < 2; ++d)
        lds_dma_b128(rs, off[t][d], __builtin_amdgcn_readfirstlane(ring0 + at + t * kTile + (8 * wave + 4 * d) * kRow));
    }
  };
  auto load = [&](int b) {
    const int block = nth(b);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int64_t row = (int64_t)block * kB + srow + 4 * d;
        st[t][d] = u32x4{};
        if (row < len) st[t][d] = *reinterpret_cast<const u32x4_any*>(src[t] + row * stride[t] + 8 * place);
      }
  };
  auto store = [&](int at) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int row = srow + 4 * d;
        *reinterpret_cast<u32x4*>(s_ring + at + t * kTile + row * kRow + ((place ^ perm(row)) << 4)) = st[t][d];
      }
  };
  if constexpr (kDirect) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int row = srow + 4 * d;
        off[t][d] = (uint32_t)row * (uint32_t)stride[t] * 2 + ((place ^ perm(row)) << 4);
      }
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
      if (s < blocks) copy(s, s * kStage);
  } else {
    load(0);
  }

  // state: register (m, i) is key dim 32 m + dim(i), column 32 wave + n
  auto dim = [&](int i) { return 16 * (i >> 3) + 8 * half + 4 * ((i >> 2) & 1) + (i & 3); };
  f32x16 S[4];
  const Decay decay(log_decay);
  const bool own_state = kOutputs ? !cut : p.seg == 0;   // the request's, not the workspace's or none
  const float* from = own_state ? (si >= 0 && si < a.num_slots ? a.states + si * slot + (int64_t)h * kState : nullptr)
                      : kOutputs ? ws : nullptr;
  const float none = !own_state || si == -1 ? 0.f : __builtin_nanf("");
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int i = 0; i < 16; ++i) S[m][i] = from ? from[(32 * m + dim(i)) * 128 + 32 * wave + n] : none;

  // Operand addresses within a stage; chunk bits are apart from the rest, so other chunks are an exclusive or away.
  const int rows = n * kRow + ((half ^ perm(n)) << 4);   // row n, dims 16 s + 8 half .. + 7: ^ s << 5
  const int j = lane & 15, b4 = (lane >> 4) & 1, trow = 8 * half + (j >> 2);
  int kcol[2], vcol[2];       // rows + 0, + 4 of 8 half; state tile m: ^ m << 6
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int row = trow + 4 * y;
    kcol[y] = row * kRow + (((2 * b4 + (j & 1)) ^ perm(row)) << 4) + 8 * ((j >> 1) & 1);
    vcol[y] = kTile + row * kRow + (((4 * wave + 2 * b4 + ((j >> 1) & 1)) ^ perm(row)) << 4) + 8 * (j & 1);
  }
  // scores: this wave's 16 queries by 16 keys, lane (j, quarter) dims 32 s + 8 quarter .. + 7 of row j: ^ s << 6;
  // the results are keys key0 .. + 3 of query0.  A query's row lies with its 16-byte chunks permuted by query / 4, so
  // that 16 queries put one chunk on all banks.
  const int quarter = lane >> 4, query0 = 16 * (wave >> 1) + j, key0 = 16 * (wave & 1) + 4 * quarter;
  const int krow = (16 * (wave & 1) + j) * kRow + ((quarter ^ perm(j)) << 4);
  const int qrow = 2 * kTile + query0 * kRow + ((quarter ^ perm(j)) << 4);
  const int score_to = query0 * 2 * kB + (((key0 >> 3) ^ ((query0 >> 2) & 3)) << 4) + 8 * (quarter & 1);
  int score_from[2];          // keys 16 k2 + 8 half .. + 7 of query n
#pragma unroll
  for (int k2 = 0; k2 < 2; ++k2) score_from[k2] = n * 2 * kB + (((2 * k2 + half) ^ ((n >> 2) & 3)) << 4);

  auto key_of = [&](int i) { return 16 * (i >> 3) + 8 * half + (i & 7); };   // of a column operand's element
  float within[4], fade[16];   // scale l^(query - key), 0 for later keys; l^(kB-1-key)
  if constexpr (kOutputs) {
#pragma unroll
    for (int i = 0; i < 4; ++i) within[i] = query0 >= key0 + i ? a.scale * decay.power(query0 - key0 - i) : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) fade[i] = decay.power(kB - 1 - key_of(i));
  const float since = a.scale * decay.power(n + 1);

  if (!kOutputs && p.seg == 0) {   // the state before piece 0 stays: the request may advance in place
    const float f = decay.power(len);
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        ws[(32 * m + dim(i)) * 128 + 32 * wave + n] = S[m][i];
        S[m][i] *= f;
      }
  }

  if constexpr (!kDirect) {
    store(0);
    if (1 < blocks) load(1);
    if (kOutputs && 1 < blocks) {
      store(kStage);
      if (2 < blocks) load(2);
    }
  }
  // This wave's quarter of a block's scores, in two terms.
  auto scores = [&](int stage, int parity) {
    f32x4 sc{};
#pragma unroll
    for (int s = 0; s < 4; ++s)
      sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(read_row(s_ring + ((stage + krow) ^ s << 6)), read_row(s_ring + ((stage + qrow) ^ s << 6)), sc, 0, 0, 0);
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = query0 >= key0 + i ? sc[i] * within[i] : 0.f;
    uint8_t* const to = s_score + 2 * kScores * parity + score_to;
    const uint32_t w0 = pack_bf16x2(y[0], y[1]), w1 = pack_bf16x2(y[2], y[3]);
    *reinterpret_cast<u32x2*>(to) = u32x2{w0, w1};
    take_off(w0, y[0], y[1]);
    take_off(w1, y[2], y[3]);
    *reinterpret_cast<u32x2*>(to + kScores) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
  };
  if constexpr (kOutputs) {
    if (kDirect && blocks > 1) tile_barrier<kCopies>();
    else if (kDirect) tile_barrier<0>();
    else lds_barrier();
    scores(0, 0);
  }
  int behind = 0;      // tokens that S has yet to fade by: the state is l^behind S
  float late = 1.f;    // l^behind
  int at = 0;          // the block's stage
  for (int b = 0; b < blocks; ++b) {
    // With outputs the next block's tile has to be there too, for its scores.
    if constexpr (!kDirect) lds_barrier();
    else if constexpr (kOutputs) {
      if (b == 0) tile_barrier<0>();
      else if (b + 1 < blocks) tile_barrier<kStores>();
      else lds_barrier();
    } else {
      if (b + kStages - 2 >= blocks) tile_barrier<0>();
      else tile_barrier<(kStages - 2) * kCopies>();
    }
    if constexpr (kDirect) {
      // the stage before this one's is read out
      if (b + kStages - 1 < blocks) copy(b + kStages - 1, at == 0 ? kRing - kStage : at - kStage);
      __asm__ volatile("" ::: "memory");   // the block's stores are younger than the copies
    }
    const int valid = min(kB, len - nth(b) * kB);
    const uint8_t* const tile = s_ring;
    const bf16x8 vc[2] = {read_columns(tile + at + vcol[0], tile + at + vcol[1]),
                          read_columns(tile + at + vcol[0] + 16 * kRow, tile + at + vcol[1] + 16 * kRow)};
    u32x4 vw[2] = {__builtin_bit_cast(u32x4, vc[0]), __builtin_bit_cast(u32x4, vc[1])};

    // What joins the state.  Without outputs each block fades to the piece's end at once.  With them S fades only
    // when it is behind by a factor of more than 2^kMostBehind (or at the end), and what joins it is blown up
    // by as much.
    const int after = behind + valid;
    const bool fades = kOutputs && (b + 1 == blocks || -decay.exponent(after) > kMostBehind);
    const float by = kOutputs ? decay.power(after) : 1.f;
    float f[16];
    if (valid == kB) {
      const float join = decay.power(kOutputs ? (fades ? 0 : -after) : len - (nth(b) + 1) * kB);
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = fade[i] * join;
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = decay.power(max(valid - 1 - key_of(i), 0));
    }

    bool bad = false;
    int bad_row = kB;    // the first such row of column n
    if constexpr (kOutputs) {
      // A value of v that is not finite is no matter of the rows before it: 0 in their sums, and NaN put
      // into the rows from its own on.  (0 times it is NaN, 0 times any other 0.)
      float probe = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) probe = probe_bf16x2(vw[i >> 2][i & 3], probe);
      bad = __ballot(probe != probe) != 0;
      if (bad) {
        int from_row = kB;
#pragma unroll
        for (int i = 15; i >= 0; --i) {
          const uint32_t w = vw[i >> 3][(i >> 1) & 3];
          const uint32_t bits = i & 1 ? w >> 16 : w & 0xFFFFu;
          if ((bits & 0x7F80u) == 0x7F80u) {
            from_row = min(from_row, key_of(i));
            vw[i >> 3][(i >> 1) & 3] = w & (i & 1 ? 0x0000FFFFu : 0xFFFF0000u);
          }
        }
        bad_row = min(from_row, __shfl_xor(from_row, 32, 64));
      }
      // the next block's scores (of a block that there is not: of what lies there, and not used)
      scores(at + kStage == kRing ? 0 : at + kStage, (b + 1) & 1);
    }

    constexpr int kTerms = kOutputs ? 2 : 3;   // for outputs, in bf16 in the end, two will do
    float x[2][8];
    Terms<kTerms> vx[2];
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      const u32x4 w = __builtin_bit_cast(u32x4, vc[k2]);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[k2][i] = (i & 1 ? bf16hi(w[i >> 1]) : bf16lo(w[i >> 1])) * f[8 * k2 + i];
      vx[k2] = split<kTerms>(x[k2]);
    }
    f32x16 o{};
    if constexpr (kOutputs) {
      const int row = at + rows;
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const bf16x8 q = read_row(tile + 2 * kTile + (row ^ s << 5));
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = S[s >> 1][8 * (s & 1) + i];
        const Terms<2> sx = split<2>(z);
        o = mfma(sx.t[1], q, o);
        o = mfma(sx.t[0], q, o);
      }
      if (fades) {
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int i = 0; i < 16; ++i) S[m][i] *= by;
      }
    }
    auto join_state = [&](const bf16x8* terms0, const bf16x8* terms1, int count) {
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const bf16x8 kk = read_columns(tile + ((at + kcol[0]) ^ m << 6) + 16 * k2 * kRow, tile + ((at + kcol[1]) ^ m << 6) + 16 * k2 * kRow);
#pragma unroll
          for (int i = count - 1; i >= 0; --i) S[m] = mfma(kk, (k2 ? terms1 : terms0)[i], S[m]);
        }
    };
    join_state(vx[0].t, vx[1].t, kTerms);
    if constexpr (kOutputs) {
      const float reach = since * late;
#pragma unroll
      for (int i = 0; i < 16; ++i) o[i] *= reach;
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        const uint8_t* sr = s_score + 2 * kScores * (b & 1) + score_from[k2];
        const bf16x8 vv = __builtin_bit_cast(bf16x8, vw[k2]);
        o = mfma(vv, read_row(sr + kScores), o);
        o = mfma(vv, read_row(sr), o);
      }
      if (bad) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (n >= __shfl(bad_row, 8 * (i >> 2) + 4 * half + (i & 3), 64)) o[i] = __builtin_nanf("");
      }
      // lane (n, half) holds columns 8 c + 4 half + 0 .. 3 of row n: exchanged to eight in a row
      uint16_t* dst = a.out + (row0 + b * kB + n) * a.out_stride + h * 128 + 32 * wave + 8 * half;
      u32x4 y[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const u32x2 u = swap_halves(pack_bf16x2(o[8 * c], o[8 * c + 1]), pack_bf16x2(o[8 * c + 4], o[8 * c + 5]));
        const u32x2 w = swap_halves(pack_bf16x2(o[8 * c + 2], o[8 * c + 3]), pack_bf16x2(o[8 * c + 6], o[8 * c + 7]));
        y[c] = u32x4{u[0], w[0], u[1], w[1]};
      }
      if (valid == kB) {       // kStores stores, which the next tile_barriers count on
        *reinterpret_cast<u32x4_any*>(dst) = y[0];
        *reinterpret_cast<u32x4_any*>(dst + 16) = y[1];
      } else if (n < valid) {
        *reinterpret_cast<u32x4_any*>(dst) = y[0];
        *reinterpret_cast<u32x4_any*>(dst + 16) = y[1];
      }
      if (!cut) {              // this state is what the call returns: the third term too
        Terms<1> rest[2] = {split<1>(x[0]), split<1>(x[1])};
        join_state(rest[0].t, rest[1].t, 1);
      }
    }
    behind = fades ? 0 : after;
    late = fades ? 1.f : by;
    at = at + kStage == kRing ? 0 : at + kStage;
    if constexpr (!kDirect) {
      constexpr int kAhead = kOutputs ? 2 : 1;
      if (b + kAhead < blocks) {
        store(kOutputs ? (at + kStage == kRing ? 0 : at + kStage) : at);
        if (b + kAhead + 1 < blocks) load(b + kAhead + 1);
      }
    }
  }

  float* to = !kOutputs ? ws + slot : !cut && so >= 0 && so < a.num_slots ? a.states + so * slot + (int64_t)h * kState : nullptr;
  if (to) {
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) to[(32 * m + dim(i)) * 128 + 32 * wave + n] = S[m][i];
  }
}

// The blocked form of whole chunks with half of a head's columns a workgroup, 16 a wave.  Where there are few
// workgroups, the blocks one after another are the time, and a wave has half as much to do in each: 1.5 us a block
// instead of 2.0 (32 heads, 64 to 512 tokens; 0.2 more with the operands read where they are used).  Where there are many,
// reading K and Q for half as many columns costs 1.12 to 1.15 times as much (16 requests of 512 and 1024 tokens).
// Other than above, products are 16 x 16 x 32 and state register (t, i) is key dim 16 t + 4 quarter + i of column
// n: two of its quads are an operand's eight key dims, and Q's rows are read in the same halves.
template <bool kDirect>
__global__ __launch_bounds__(256, 2) void linear_narrow_kernel(LinearLaunch a) {
  constexpr int kTiles = 3, kStages = 3, kStage = kTiles * kTile, kRing = kStages * kStage;
  constexpr int kCopies = 2 * kTiles, kStores = 2;   // a wave's, for a block
  __shared__ __attribute__((aligned(1024))) uint8_t s_ring[kRing];
  __shared__ __attribute__((aligned(1024))) uint8_t s_score[4 * kScores];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, quarter = lane >> 4;
  const int group = a.hq / a.hkv;
  // the workgroups of one key head's queries follow one another on one XCD, which then reads K and V once
  const int unit = (int)(blockIdx.x / (16 * group)) * 8 + (int)(blockIdx.x % 8);
  const int h0 = (int)(blockIdx.x / 8) % (2 * group);
  if (unit >= a.num_units * a.hkv) return;
  const int g = unit % a.hkv, h = g * group + (h0 >> 1), col0 = 64 * (h0 & 1) + 16 * wave;
  const float log_decay = a.log_decay[h];
  Piece p = find_piece<false>(a, unit / a.hkv);
  if (p.req < 0) return;
  const int len = __builtin_amdgcn_readfirstlane(p.len), blocks = (len + kB - 1) / kB;
  const int64_t row0 = __builtin_amdgcn_readfirstlane(p.row);
  const int si = __builtin_amdgcn_readfirstlane(p.slot_in), so = __builtin_amdgcn_readfirstlane(p.slot_out);
  const int64_t slot = (int64_t)a.hq * kState;

  // this wave's rows 8 wave + 4 d + (lane / 16) of each tile, 16 bytes a lane
  const int srow = 8 * wave + quarter;
  const uint16_t* src[3] = {a.k + row0 * a.k_stride + g * 128, a.v + row0 * a.v_stride + g * 128, a.q + row0 * a.q_stride + h * 128};
  const int64_t stride[3] = {a.k_stride, a.v_stride, a.q_stride};
  const uint32_t ring0 = (uint32_t)(uintptr_t)(lds_void*)s_ring;
  uint32_t off[kTiles][2];
  u32x4 st[kTiles][2];
  auto copy = [&](int block, int at) {      // straight into LDS; rows past the chunk read as zero
    const int rows = min(kB, len - block * kB);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const i32x4 rs = sgpr_rsrc(src[t] + (int64_t)block * kB * stride[t], (rows - 1) * (int32_t)stride[t] * 2 + kRow);
#pragma unroll
      for (int d = 0; d < 2; ++d)
        lds_dma_b128(rs, off[t][d], __builtin_amdgcn_readfirstlane(ring0 + at + t * kTile + (8 * wave + 4 * d) * kRow));
    }
  };
  auto load = [&](int block) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int64_t row = (int64_t)block * kB + srow + 4 * d;
        st[t][d] = u32x4{};
        if (row < len) st[t][d] = *reinterpret_cast<const u32x4_any*>(src[t] + row * stride[t] + 8 * n);
      }
  };
  auto store = [&](int at) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int row = srow + 4 * d;
        *reinterpret_cast<u32x4*>(s_ring + at + t * kTile + row * kRow + ((n ^ perm(row)) << 4)) = st[t][d];
      }
  };
  if constexpr (kDirect) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int row = srow + 4 * d;
        off[t][d] = (uint32_t)row * (uint32_t)stride[t] * 2 + ((n ^ perm(row)) << 4);
      }
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
      if (s < blocks) copy(s, s * kStage);
  } else {
    load(0);
  }

  const Decay decay(log_decay);
  const int state0 = 4 * quarter * 128 + col0 + n;
  f32x4 S[8];
  const float* from = si >= 0 && si < a.num_slots ? a.states + si * slot + (int64_t)h * kState : nullptr;
  const float none = si == -1 ? 0.f : __builtin_nanf("");
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) S[t][i] = from ? from[state0 + (16 * t + i) * 128] : none;

  // Operand addresses within a stage; chunk bits are apart from the rest, so other chunks are an exclusive or away.
  // Scores: dims 32 s + 8 quarter .. + 7 of a row, ^ s << 6.  Against the state: dims 32 s + 4 quarter .. + 3, and 16
  // on (^ 32), of row n, ^ s << 6.  Columns: lane n of a quarter addresses columns 4 (n % 4) .. + 3 of row
  // 8 quarter + n / 4, and of the fourth on; key dims 16 t .. + 15: ^ t << 5.
  int row8[2];   // of query n, of query n + 16
  row8[0] = 2 * kTile + n * kRow + (((quarter >> 1) ^ perm(n)) << 4) + 8 * (quarter & 1);
  row8[1] = row8[0] + 16 * kRow;
  // Hidden from the compiler: two 8-byte reads a fixed distance apart become one instruction, which takes 16 lanes at a
  // time, whose reads lie on half of the banks (17% of the cycles were conflicts; now 8%).
  __asm__("" : "+v"(row8[1]));
  int kcol[2], vcol[2];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int row = 8 * quarter + 4 * y + (n >> 2), chunk = (n >> 1) & 1;
    kcol[y] = row * kRow + ((chunk ^ perm(row)) << 4) + 8 * (n & 1);
    vcol[y] = kTile + row * kRow + (((col0 / 8 + chunk) ^ perm(row)) << 4) + 8 * (n & 1);
  }
  // this wave's 16 queries by 16 keys; results are keys key0 .. + 3 of query0
  const int query0 = 16 * (wave >> 1) + n, key0 = 16 * (wave & 1) + 4 * quarter;
  const int krow = (16 * (wave & 1) + n) * kRow + ((quarter ^ perm(n)) << 4);
  const int qrow = 2 * kTile + query0 * kRow + ((quarter ^ perm(n)) << 4);
  const int score_to = query0 * 2 * kB + (((key0 >> 3) ^ ((query0 >> 2) & 3)) << 4) + 8 * (quarter & 1);
  const int score_from = n * 2 * kB + ((quarter ^ ((n >> 2) & 3)) << 4);   // keys 8 quarter .. + 7 of queries n, n + 16

  float within[4], fade[8];   // scale l^(query - key), 0 for later keys; l^(kB-1-key) of key 8 quarter + i
#pragma unroll
  for (int i = 0; i < 4; ++i) within[i] = query0 >= key0 + i ? a.scale * decay.power(query0 - key0 - i) : 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) fade[i] = decay.power(kB - 1 - 8 * quarter - i);
  const float since[2] = {a.scale * decay.power(n + 1), a.scale * decay.power(n + 17)};

  if constexpr (!kDirect) {
    store(0);
    if (1 < blocks) {
      load(1);
      store(kStage);
      if (2 < blocks) load(2);
    }
  }
  bf16x8 sk[4], sq[4];
  auto read_scores = [&](int stage) {
#pragma unroll
    for (int s = 0; s < 4; ++s) sk[s] = read_row(s_ring + ((stage + krow) ^ s << 6)), sq[s] = read_row(s_ring + ((stage + qrow) ^ s << 6));
  };
  auto scores = [&](int parity) {
    f32x4 sc{};
#pragma unroll
    for (int s = 0; s < 4; ++s) sc = mfma16(sk[s], sq[s], sc);
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = query0 >= key0 + i ? sc[i] * within[i] : 0.f;
    uint8_t* const to = s_score + 2 * kScores * parity + score_to;
    const uint32_t w0 = pack_bf16x2(y[0], y[1]), w1 = pack_bf16x2(y[2], y[3]);
    *reinterpret_cast<u32x2*>(to) = u32x2{w0, w1};
    take_off(w0, y[0], y[1]);
    take_off(w1, y[2], y[3]);
    *reinterpret_cast<u32x2*>(to + kScores) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
  };
  if (kDirect && blocks > 1) tile_barrier<kCopies>();
  else if (kDirect) tile_barrier<0>();
  else lds_barrier();
  read_scores(0);
  scores(0);

  int behind = 0;      // tokens that S has yet to fade by: the state is l^behind S
  float late = 1.f;    // l^behind
  int at = 0;          // the block's stage
  for (int b = 0; b < blocks; ++b) {
    // the next block's tile has to be there too, for its scores
    if constexpr (!kDirect) lds_barrier();
    else if (b == 0) tile_barrier<0>();
    else if (b + 1 < blocks) tile_barrier<kStores>();
    else lds_barrier();
    const int next = at + kStage == kRing ? 0 : at + kStage;
    if constexpr (kDirect) {
      // the stage before this one's is read out
      if (b + 2 < blocks) copy(b + 2, at == 0 ? kRing - kStage : at - kStage);
      __asm__ volatile("" ::: "memory");   // the block's stores are younger than the copies
    }
    const int valid = min(kB, len - b * kB);
    // all of the block's operands are read ahead of what waits for them
    const bf16x8 vc = read_columns(s_ring + at + vcol[0], s_ring + at + vcol[1]);
    read_scores(next);
    bf16x8 qh[4][2];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        qh[s][u] = read_halves(s_ring + ((at + row8[u]) ^ s << 6), s_ring + ((at + row8[u]) ^ (s << 6 | 32)));
    __builtin_amdgcn_sched_barrier(0);
    u32x4 vw = __builtin_bit_cast(u32x4, vc);

    // values of v that are not finite: as above
    float probe = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) probe = probe_bf16x2(vw[i], probe);
    const bool bad = __ballot(probe != probe) != 0;
    int bad_row = kB;    // the first such row of column n
    if (bad) {
      int from_row = kB;
#pragma unroll
      for (int i = 7; i >= 0; --i) {
        const uint32_t w = vw[i >> 1], bits = i & 1 ? w >> 16 : w & 0xFFFFu;
        if ((bits & 0x7F80u) == 0x7F80u) {
          from_row = 8 * quarter + i;
          vw[i >> 1] = w & (i & 1 ? 0x0000FFFFu : 0xFFFF0000u);
        }
      }
      from_row = min(from_row, __shfl_xor(from_row, 16, 64));
      bad_row = min(from_row, __shfl_xor(from_row, 32, 64));
    }

    const int after = behind + valid;
    const bool fades = b + 1 == blocks || -decay.exponent(after) > kMostBehind;
    const float by = decay.power(after);
    float f[8];
    if (valid == kB) {
      const float join = decay.power(fades ? 0 : -after);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = fade[i] * join;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = decay.power(max(valid - 1 - 8 * quarter - i, 0));
    }

    // the next block's scores (of a block that there is not: of what lies there, and not used)
    scores((b + 1) & 1);
    bf16x8 kk[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) kk[t] = read_columns(s_ring + ((at + kcol[0]) ^ t << 5), s_ring + ((at + kcol[1]) ^ t << 5));
    __builtin_amdgcn_sched_barrier(0);
    float x[8];
    {
      const u32x4 w = __builtin_bit_cast(u32x4, vc);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (i & 1 ? bf16hi(w[i >> 1]) : bf16lo(w[i >> 1])) * f[i];
    }
    const Terms<3> vx = split<3>(x);

    f32x4 o[2] = {};
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      float z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = S[2 * s + (i >> 2)][i & 3];
      const Terms<2> sx = split<2>(z);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        o[u] = mfma16(sx.t[1], qh[s][u], o[u]);
        o[u] = mfma16(sx.t[0], qh[s][u], o[u]);
      }
    }
    if (fades) {
#pragma unroll
      for (int t = 0; t < 8; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) S[t][i] *= by;
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) {
#pragma unroll
      for (int i = 2; i >= 0; --i) S[t] = mfma16(kk[t], vx.t[i], S[t]);
    }
    const bf16x8 vv = __builtin_bit_cast(bf16x8, vw);
    uint16_t* dst = a.out + (row0 + b * kB + n) * a.out_stride + h * 128 + col0 + 4 * quarter;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float reach = since[u] * late;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[u][i] *= reach;
      const uint8_t* sr = s_score + 2 * kScores * (b & 1) + score_from + 16 * u * 2 * kB;
      o[u] = mfma16(vv, read_row(sr + kScores), o[u]);
      o[u] = mfma16(vv, read_row(sr), o[u]);
    }
    if (bad) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * u + n >= __shfl(bad_row, 4 * quarter + i, 64)) o[u][i] = __builtin_nanf("");
    }
    const u32x2 y[2] = {{pack_bf16x2(o[0][0], o[0][1]), pack_bf16x2(o[0][2], o[0][3])},
                        {pack_bf16x2(o[1][0], o[1][1]), pack_bf16x2(o[1][2], o[1][3])}};
    if (valid == kB) {       // kStores stores, which the next tile_barriers count on
      *reinterpret_cast<u32x2_any*>(dst) = y[0];
      *reinterpret_cast<u32x2_any*>(dst + 16 * a.out_stride) = y[1];
    } else {
      if (n < valid) *reinterpret_cast<u32x2_any*>(dst) = y[0];
      if (n + 16 < valid) *reinterpret_cast<u32x2_any*>(dst + 16 * a.out_stride) = y[1];
    }
    behind = fades ? 0 : after;
    late = fades ? 1.f : by;
    at = next;
    if constexpr (!kDirect) {
      if (b + 2 < blocks) {
        store(next + kStage == kRing ? 0 : next + kStage);
        if (b + 3 < blocks) load(b + 3);
      }
    }
  }

  if (so >= 0 && so < a.num_slots) {
    float* to = a.states + so * slot + (int64_t)h * kState;
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) to[state0 + (16 * t + i) * 128] = S[t][i];
  }
}

// The states between the pieces of cut requests: workspace entry s + 1 of a request holds what piece s
// alone makes of its tokens (piece 0: of the request's state too), and gets the sum with the entry before it, faded
// by piece s; the last one goes to the request's slot.  A thread takes four elements of one head's
// states through all pieces.
__global__ __launch_bounds__(256) void linear_carry_kernel(LinearLaunch a) {
  const int h = blockIdx.y;
  const int lane = threadIdx.x & 63;
  // the blockIdx.z-th cut request
  int32_t idx = blockIdx.z, ws = 0, pieces = 0, req = 0, len = 0;
  for (int32_t r0 = 0; r0 < a.num_reqs; r0 += 64) {
    const int32_t l = r0 + lane < a.num_reqs ? a.chunk_lens[r0 + lane] : -1;
    const int32_t cut = l > kLinearShortTokens && l > a.piece_tokens ? (l + a.piece_tokens - 1) / a.piece_tokens : 0;
    const int32_t entries = cut ? cut + 1 : 0;
    const uint64_t is = __ballot(cut > 0);
    const int32_t total = __popcll(is), sum = wave_scan(entries);
    if (idx < total) {
      const uint64_t here = __ballot(cut > 0 && __popcll(is & (((uint64_t)1 << lane) - 1)) == idx);
      const int32_t c = __builtin_ctzll(here);
      pieces = __builtin_amdgcn_readlane(cut, c);
      len = __builtin_amdgcn_readlane(l, c);
      ws += __builtin_amdgcn_readlane(sum, c) - pieces - 1;
      req = r0 + c;
      break;
    }
    idx -= total;
    ws += __builtin_amdgcn_readlane(sum, 63);
  }
  if (pieces == 0 || ws + pieces >= a.ws_states) return;
  const int so = a.slot_out[req];
  const int64_t slot = (int64_t)a.hq * kState, at = (int64_t)h * kState / 4 + blockIdx.x * 256 + threadIdx.x;
  f32x4* p = reinterpret_cast<f32x4*>(a.ws + ws * slot) + at;
  f32x4 sum = p[slot / 4];
  const double log_decay = clean_log(a.log_decay[h]);
  const float fade = (float)exp(log_decay * a.piece_tokens), fade_last = (float)exp(log_decay * (len - (pieces - 1) * a.piece_tokens));
  constexpr int kAhead = 8;   // loads do not wait for one another
  for (int s0 = 2; s0 <= pieces; s0 += kAhead) {
    f32x4 x[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (s0 + i <= pieces) x[i] = p[(s0 + i) * (slot / 4)];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (s0 + i > pieces) break;
#pragma unroll
      for (int c = 0; c < 4; ++c) sum[c] = __builtin_fmaf(sum[c], s0 + i < pieces ? fade : fade_last, x[i][c]);
      if (s0 + i < pieces) p[(s0 + i) * (slot / 4)] = sum;
    }
  }
  if (so >= 0 && so < a.num_slots) reinterpret_cast<f32x4*>(a.states + so * slot)[at] = sum;
}

}  // namespace

hipError_t launch_linear_attn(const LinearLaunch& launch, const LinearPlan& plan, hipStream_t stream) {
  LinearLaunch a = launch;
  a.piece_tokens = plan.piece_tokens;
  a.ws_states = plan.ws_states;
  a.unit_tokens = plan.unit_tokens;
  const int group = a.hq / a.hkv;
  auto blocks = [&](int64_t units) { return dim3((uint32_t)((units * a.hkv + 7) / 8 * 8 * group)); };
  // what a copy straight into LDS takes: 16-byte steps, a row's end before the next one's start, 32-bit offsets
  auto direct = [](const uint16_t* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0 && stride >= 128 && stride <= (1 << 24);
  };
  const bool kv = direct(a.k, a.k_stride) && direct(a.v, a.v_stride), qkv = kv && direct(a.q, a.q_stride);
  if (plan.cut_reqs > 0) {
    a.num_units = plan.ws_states - plan.cut_reqs;   // their pieces
    if (kv) linear_block_kernel<false, true><<<blocks(a.num_units), 256, 0, stream>>>(a);
    else linear_block_kernel<false, false><<<blocks(a.num_units), 256, 0, stream>>>(a);
    linear_carry_kernel<<<dim3(kState / 1024, a.hq, plan.cut_reqs), 256, 0, stream>>>(a);
  }
  if (plan.pieces > 0 && plan.narrow) {
    a.num_units = plan.pieces;
    const dim3 grid((uint32_t)(((int64_t)a.num_units * a.hkv + 7) / 8 * 16 * group));
    if (qkv) linear_narrow_kernel<true><<<grid, 256, 0, stream>>>(a);
    else linear_narrow_kernel<false><<<grid, 256, 0, stream>>>(a);
  } else if (plan.pieces > 0) {
    a.num_units = plan.pieces;
    if (qkv) linear_block_kernel<true, true><<<blocks(a.num_units), 256, 0, stream>>>(a);
    else linear_block_kernel<true, false><<<blocks(a.num_units), 256, 0, stream>>>(a);
  }
  if (plan.short_reqs > 0)
    linear_recurrent_kernel<<<dim3(32 * ((a.hq + 7) / 8), a.num_reqs), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace s2l
