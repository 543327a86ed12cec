// Device helpers that the kernels share: packing and reductions, the rotary
// tables, and the rows of an append launch with their norm and rotation.
#pragma once

#include <hip/hip_runtime.h>

#include "ws_kernels.hpp"

namespace ws {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kNegInf = -__builtin_inff();
// Largest logit bound (log2 units) used as a fixed softmax shift.
constexpr float kShiftBoundMax = 40.0f;
// Above it the video kernel's shift is a running maximum, raised when a logit
// exceeds it by more than this (so p <= 2^8).
constexpr float kRaiseAbove = 8.0f;

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Two fp32 -> packed bf16 pair, round to nearest even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  bf16x2 r = __builtin_convertvector((f32x2){lo, hi}, bf16x2);
  return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// max and sum over lanes l, l ^ 16 (kLane = 16) or l, l ^ 32 (v_permlane*_swap:
// no LDS round trip)
template <int kLane>
__device__ __forceinline__ float pair_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = kLane == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false)
                             : __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int kLane>
__device__ __forceinline__ float pair_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = kLane == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false)
                             : __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// max over the wave (rotations within a row of 16, then the swaps)
template <int kRor>
__device__ __forceinline__ float ror_max(float v) {
  const int u = __float_as_int(v);
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(u, u, 0x120 + kRor, 0xf, 0xf, false)));
}
__device__ __forceinline__ float wave_max(float v) {
  return pair_max<32>(pair_max<16>(ror_max<1>(ror_max<2>(ror_max<4>(ror_max<8>(v))))));
}
// sum over the 16 lanes of a row, in every lane
template <int kRor>
__device__ __forceinline__ float ror_add(float v) {
  const int u = __float_as_int(v);
  return v + __int_as_float(__builtin_amdgcn_update_dpp(u, u, 0x120 + kRor, 0xf, 0xf, false));
}
__device__ __forceinline__ float row_sum(float v) { return ror_add<1>(ror_add<2>(ror_add<4>(ror_add<8>(v)))); }
// |x|^2 of the lane's words, in fp32 products and sums
__device__ __forceinline__ float norm2_fma(u32x4 w) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = bf16_lo(w[i]), hi = bf16_hi(w[i]);
    s = fmaf(lo, lo, s);
    s = fmaf(hi, hi, s);
  }
  return s;
}
// the same by the dot product instruction, added to acc: for bounds only (its
// rounding and subnormals are the instruction's own)
__device__ __forceinline__ float norm2_words(u32x4 w, float acc) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = w[i];
    acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), __builtin_bit_cast(bf16x2, x), acc, false);
  }
  return acc;
}

// (cos, sin) of rotary pair p (0..63) for a token at position pos (t, h, w).
__device__ __forceinline__ float2 rope_cs(const RopeTables& r, int p, int pt, int ph, int pw) {
  const int p0 = r.pairs[0], p01 = r.pairs[0] + r.pairs[1];
  if (p < p0) return r.tab[0][pt * r.pairs[0] + p];
  if (p < p01) return r.tab[1][ph * r.pairs[1] + (p - p0)];
  return r.tab[2][pw * r.pairs[2] + (p - p01)];
}

// Clamps a token's (t, h, w) into the table; flags a clamp.
__device__ __forceinline__ void clamp_pos(const RopeTables& r, int t, int h, int w, uint32_t* flags,
                                          int& pt, int& ph, int& pw) {
  const int ct = min(max(t, 0), r.max_pos[0] - 1);
  const int ch = min(max(h, 0), r.max_pos[1] - 1);
  const int cw = min(max(w, 0), r.max_pos[2] - 1);
  if ((ct != t) | (ch != h) | (cw != w)) atomicOr(flags, kFlagPositionClamped);
  pt = ct;
  ph = ch;
  pw = cw;
}

// Loads a token's (t, h, w), clamped into the table; flags a clamp.
__device__ __forceinline__ void load_pos(const RopeTables& r, const int32_t* positions, int tok,
                                         uint32_t* flags, int& pt, int& ph, int& pw) {
  clamp_pos(r, positions[3 * tok + 0], positions[3 * tok + 1], positions[3 * tok + 2], flags, pt, ph, pw);
}

// Read-only for a whole launch: accessed through the constant address space
// so that uniform reads become scalar loads.
typedef const __attribute__((address_space(4))) int2* const_page_list;

typedef const __attribute__((address_space(4))) AppendSeg* const_append_seg;
typedef const __attribute__((address_space(4))) AppendArgs* const_append_args;

// The append launch's arguments, read in place from the kernel argument
// segment (the kernel's only argument is the AppendArgs): with run-time
// indexes into the by-value argument the compiler copies all of it to
// private memory.
__device__ __forceinline__ const_append_args append_args() {
  return (const_append_args)__builtin_amdgcn_kernarg_segment_ptr();
}

// Four rotary pairs (4 c .. 4 c + 3) of a token: their (cos, sin).  A pair's
// band is a select on its index, not a branch, so that the loads of several
// tokens are in flight together.
__device__ __forceinline__ void rope_pairs(const RopeTables& r, int c, const int (&pos)[3], float2 (&cs)[4]) {
  const int p0 = r.pairs[0], p01 = p0 + r.pairs[1];
  const float2* row[3] = {r.tab[0] + static_cast<int64_t>(pos[0]) * r.pairs[0],
                          r.tab[1] + static_cast<int64_t>(pos[1]) * r.pairs[1] - p0,
                          r.tab[2] + static_cast<int64_t>(pos[2]) * r.pairs[2] - p01};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int p = 4 * c + i;
    cs[i] = (p < p0 ? row[0] : p < p01 ? row[1] : row[2])[p];
  }
}

// RMS norm, gamma and rotation of one row's eight dims (x, dims 8 c .. of the 16
// lanes of the row), times scale, rounded once to bf16.
__device__ __forceinline__ u32x4 norm_rope_row(u32x4 x, const float (&g)[8], float eps, const float2 (&cs)[4],
                                               float scale) {
  const float inv = rsqrtf(row_sum(norm2_fma(x)) * (1.0f / kHeadDim) + eps);
  u32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float y0 = bf16_lo(x[i]) * inv * g[2 * i];
    const float y1 = bf16_hi(x[i]) * inv * g[2 * i + 1];
    y[i] = pack_bf16((y0 * cs[i].x - y1 * cs[i].y) * scale, (y0 * cs[i].y + y1 * cs[i].x) * scale);
  }
  return y;
}
// The same in fp32, for rows that are stored in 8 bits.
__device__ __forceinline__ void norm_rope_vals(u32x4 x, const float (&g)[8], float eps, const float2 (&cs)[4],
                                               float (&y)[8]) {
  const float inv = rsqrtf(row_sum(norm2_fma(x)) * (1.0f / kHeadDim) + eps);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float y0 = bf16_lo(x[i]) * inv * g[2 * i];
    const float y1 = bf16_hi(x[i]) * inv * g[2 * i + 1];
    y[2 * i] = y0 * cs[i].x - y1 * cs[i].y;
    y[2 * i + 1] = y0 * cs[i].y + y1 * cs[i].x;
  }
}

// A segment's rows of one tile as the append's arithmetic takes them: 16 lanes
// per token row (lane c: dims 8 c ..), rows rr, rr + 16, rr + 32, rr + 48.
struct AppendRows {
  u32x4 x[4];
  int pos[4][3];
};
__device__ __forceinline__ void load_rows(const_append_seg sg, int tok0, int head, bool norm_rope, int c, int rr,
                                          AppendRows& r) {
  const uint16_t* src = sg->k;
  const int64_t tok_stride = sg->tok_stride;
  const int n_tokens = sg->n_tokens;
  const int32_t* positions = sg->positions;
  src += head * sg->head_stride + 8 * c;
  if (norm_rope) {
#pragma unroll
    for (int pass = 0; pass < 4; ++pass) {
      const int tok = min(tok0 + pass * 16 + rr, n_tokens - 1);
#pragma unroll
      for (int b = 0; b < 3; ++b) r.pos[pass][b] = positions[3 * tok + b];
    }
  }
#pragma unroll
  for (int pass = 0; pass < 4; ++pass) {
    const int tok = tok0 + pass * 16 + rr;
    r.x[pass] = tok < n_tokens ? *reinterpret_cast<const u32x4*>(src + tok * tok_stride) : (u32x4){0u, 0u, 0u, 0u};
  }
}
__device__ __forceinline__ void load_gamma(const_append_seg sg, int c, float (&g)[8]) {
  const float* gamma = sg->gamma;
  const float4 g0 = *reinterpret_cast<const float4*>(gamma + 8 * c);
  const float4 g1 = *reinterpret_cast<const float4*>(gamma + 8 * c + 4);
  g[0] = g0.x; g[1] = g0.y; g[2] = g0.z; g[3] = g0.w;
  g[4] = g1.x; g[5] = g1.y; g[6] = g1.z; g[7] = g1.w;
}
// store(pass, slot, words) for the tile's 64 rows: normed, rotated and scaled
// (two rows' table entries in flight at a time, which keeps the registers to
// six blocks per CU), or scaled only.
template <class F>
__device__ __forceinline__ void rotate_rows(const RopeTables& rope, uint32_t* flags, const_append_seg sg, int tok0,
                                            float scale, int c, int rr, AppendRows& r, F&& store) {
  float g[8];
  load_gamma(sg, c, g);
  const float eps = sg->eps;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    float2 cs[2][4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      // (a row past the end holds the last token's positions)
      int (&p)[3] = r.pos[2 * half + k];
      int q[3];
      clamp_pos(rope, p[0], p[1], p[2], flags, q[0], q[1], q[2]);
      rope_pairs(rope, c, q, cs[k]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int pass = 2 * half + k, slot = pass * 16 + rr;
      store(pass, slot, norm_rope_row(r.x[pass], g, eps, cs[k], scale));
    }
  }
}

// Query preparation, one block of an append launch: tokens 64 chunk ..
// 64 chunk + 63 of query set si, one head, 16 threads per token row as in
// the key path below.  Q'' = RoPE(RMSNorm(Q) * gamma, positions) * scale *
// log2(e) (mode 3) or Q * scale * log2(e) (mode 2), in fp32, rounded once to
// bf16: the attention kernels' own query prologue, done once per step
// instead of once per workgroup that reads the queries.
__device__ __forceinline__ void prepare_queries(const RopeTables& rope, uint32_t* flags, const_append_seg sg,
                                                int chunk, int head) {
  const int n_tokens = sg->n_tokens;
  const bool norm_rope = (sg->mode & 1) != 0;
  const float scale = sg->scale_log2;
  const int t = threadIdx.x, c = t & 15, rr = t >> 4;
  const int tok0 = chunk * kPageTokens;
  AppendRows r;
  load_rows(sg, tok0, head, norm_rope, c, rr, r);
  uint16_t* const dst = sg->q_out + head * sg->out_head_stride + 8 * c;
  const int64_t out_tok_stride = sg->out_tok_stride;
  auto put = [&](int, int slot, u32x4 y) {
    const int tok = tok0 + slot;
    if (tok < n_tokens) *reinterpret_cast<u32x4*>(dst + tok * out_tok_stride) = y;
  };
  if (norm_rope) {
    rotate_rows(rope, flags, sg, tok0, scale, c, rr, r, put);
  } else {
#pragma unroll
    for (int pass = 0; pass < 4; ++pass) {
      u32x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = pack_bf16(bf16_lo(r.x[pass][i]) * scale, bf16_hi(r.x[pass][i]) * scale);
      put(pass, pass * 16 + rr, y);
    }
  }
}

}  // namespace
}  // namespace ws
