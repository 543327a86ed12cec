// gfx950 (MI355X, CDNA4) kernels of the 8-bit pools and of token windows.
//
//  kv_append_q     writes a segment's K/V into 8-bit cache pages: keys normed,
//                  rotated and quantised on the way, values quantised and
//                  transposed, one scale per (page, head) tile and pool.
//  kv_gather       reads segments back as bf16 rows in token order.
//  few_attn        attention of few rows over 8-bit pages, or under a token
//                  window over pages of any format: split-KV, operands straight
//                  from global memory to registers.
#include <hip/hip_ext.h>

#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "quant_device.hpp"
#include "ws_kernels.hpp"

namespace ws {
namespace {

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
constexpr uint32_t kInfBits = 0x7f800000u;
// Magnitudes from here on are not stored: infinities and NaN, and for int8 2^118
// and more, for which 1152 times the scale (QuantScale) would not be finite.
template <int kFmt>
constexpr uint32_t kTooLarge = kFmt == kFmtInt8 ? 0x7a800000u : kInfBits;

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// largest of the wave's values, in every lane
template <int kRor>
__device__ __forceinline__ uint32_t ror_umax(uint32_t v) {
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(v, v, 0x120 + kRor, 0xf, 0xf, false)));
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
  v = ror_umax<1>(ror_umax<2>(ror_umax<4>(ror_umax<8>(v))));
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(r[0], r[1]);
  const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(s[0], s[1]);
}

// The scale of a tile whose largest magnitude has the bits a, and its inverse.
template <int kFmt>
__device__ __forceinline__ void tile_scale(uint32_t a, float& s, float& inv) {
  if constexpr (kFmt == kFmtInt8) {
    const uint32_t q = (__float_as_uint(__uint_as_float(a) / 127.0f) + 255u) & ~255u;
    s = __uint_as_float(max(q, 0x00800000u));
    inv = 1.0f / s;
  } else {
    // a = m 2^x with m in [0.5, 1), 448 = 0.875 2^9
    const int e = max(static_cast<int>(a >> 23) - 135 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0), -126);
    s = __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
    inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  }
}

// Eight values to codes (two words), and |x|^2 of them (int8) or of what the codes
// stand for (e4m3, in scales).
//
// int8: x inv + 1.5 2^23 + 128, rounded once, has code + 128 in its low byte.  Only
// inv is off (2^-25), by at most 127 2^-25 < 2^-18 in the quotient; a bf16 value's
// quotient by a scale of 16 bits is at least 2^-17 from the middle of two integers
// where it is not in it (then s is a power of two and inv exact), so the code is the
// nearest one.
template <int kFmt>
__device__ __forceinline__ u32x2 quantise8(const float (&x)[8], float inv, float& norm2) {
  u32x2 w;
  norm2 = 0.f;
  if constexpr (kFmt == kFmtInt8) {
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      norm2 = fmaf(x[i], x[i], norm2);
      c[i] = __float_as_uint(fmaf(x[i], inv, 12583040.0f));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t lo = __builtin_amdgcn_perm(c[4 * i + 1], c[4 * i], 0x0c0c0400u);
      const uint32_t hi = __builtin_amdgcn_perm(c[4 * i + 3], c[4 * i + 2], 0x0c0c0400u);
      w[i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, 0, false);
      r = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, r, true);
      const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(r, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(r, true);
      norm2 = fmaf(a[0], a[0], fmaf(a[1], a[1], fmaf(b[0], b[0], fmaf(b[1], b[1], norm2))));
      w[i] = static_cast<uint32_t>(r);
    }
  }
  return w;
}

// 4 x 4 bytes transposed: byte j of w[r] becomes byte r of out[j].
__device__ __forceinline__ void transpose4(const uint32_t (&w)[4], uint32_t (&out)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  out[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// ------------------------------------------------------------------------- //
// kv_append_q: one (item, head) tile, as kv_append.  The tile's largest
// magnitudes need all of its rows before the first code is made, so the rows
// stay in registers (fp32 keys: one rounding, to the code), and K and V share the
// block-wide reduction.  V is quantised first and transposed through LDS as
// bytes: rows of 128 d, the 4-byte word d / 4 of row r at position
// (d / 4) ^ 4 (r / 8).
// Bound by memory (4 bytes read and 2 written a pair of elements) and by the chain of
// row, rotation, block maximum, code.  8 units of 917 tokens, 40 heads, int8: 55 us,
// 4.1 TB/s; a step of 1180 tokens, e4m3: 12.9 us, 2.8 TB/s.  A tile a block iteration,
// four blocks a CU (three to six measure alike).
// ------------------------------------------------------------------------- //
struct AppendLds {
  uint32_t v[kPageTokens][kHeadDim / 4];
  uint32_t top[2][2][4];  // [round][pool][wave]
  float norm2[4];
};

template <int kFmt>
__device__ __forceinline__ void append_tile_q(const const_append_args A, int item, int head, AppendLds& lds) {
  const const_append_seg sg = A->seg + A->blk_seg[item];
  RopeTables rope;
#pragma unroll
  for (int b = 0; b < 3; ++b) {
    rope.tab[b] = A->rope.tab[b];
    rope.max_pos[b] = A->rope.max_pos[b];
    rope.pairs[b] = A->rope.pairs[b];
  }
  uint32_t* const flags = A->flags;
  if (sg->mode & kAppendQuery) {
    prepare_queries(rope, flags, sg, A->blk_page[item], head);
    return;
  }
  const int num_heads = A->num_heads;
  const int64_t tile = static_cast<int64_t>(A->pages[item]) * num_heads + head;
  const int64_t tok_stride = sg->tok_stride;
  const int n_tokens = sg->n_tokens;
  const bool norm_rope = sg->mode == 1;
  const int tok0 = A->blk_page[item] * kPageTokens;
  const int t = threadIdx.x, c = t & 15, rr = t >> 4, wave = t >> 6;

  AppendRows r;
  load_rows(sg, tok0, head, norm_rope, c, rr, r);
  const uint16_t* const src_v = sg->v + head * sg->head_stride + 8 * c;
  u32x4 vx[4];
#pragma unroll
  for (int pass = 0; pass < 4; ++pass) {
    const int tok = tok0 + pass * 16 + rr;
    vx[pass] = tok < n_tokens ? *reinterpret_cast<const u32x4*>(src_v + tok * tok_stride) : (u32x4){0u, 0u, 0u, 0u};
  }

  float k[4][8];
  if (norm_rope) {
    float g[8];
    load_gamma(sg, c, g);
    const float eps = sg->eps;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float2 cs[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        int (&p)[3] = r.pos[2 * half + n];
        int q[3];
        clamp_pos(rope, p[0], p[1], p[2], flags, q[0], q[1], q[2]);
        rope_pairs(rope, c, q, cs[n]);
      }
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int pass = 2 * half + n;
        norm_rope_vals(r.x[pass], g, eps, cs[n], k[pass]);
        const bool in = tok0 + pass * 16 + rr < n_tokens;  // empty slots hold zeros whatever gamma and eps are
#pragma unroll
        for (int i = 0; i < 8; ++i) k[pass][i] = in ? k[pass][i] : 0.f;
      }
    }
  } else {
#pragma unroll
    for (int pass = 0; pass < 4; ++pass)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        k[pass][2 * i] = bf16_lo(r.x[pass][i]);
        k[pass][2 * i + 1] = bf16_hi(r.x[pass][i]);
      }
  }

  // largest magnitudes of the tile (as bits: infinities and NaN come out on top)
  uint32_t top[2];
  auto reduce = [&](int round) {
    uint32_t mk = 0;
    u16x2 pairs = {0, 0};
#pragma unroll
    for (int pass = 0; pass < 4; ++pass)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mk = max(mk, max(abs_bits(k[pass][2 * i]), abs_bits(k[pass][2 * i + 1])));
        pairs = __builtin_elementwise_max(pairs, __builtin_bit_cast(u16x2, vx[pass][i] & 0x7fff7fffu));
      }
    mk = wave_umax(mk);
    const uint32_t mv = wave_umax(static_cast<uint32_t>(max(pairs[0], pairs[1])) << 16);
    if ((t & 63) == 0) {
      lds.top[round][0][wave] = mk;
      lds.top[round][1][wave] = mv;
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 2; ++n)
      top[n] = max(max(lds.top[round][n][0], lds.top[round][n][1]), max(lds.top[round][n][2], lds.top[round][n][3]));
  };
  reduce(0);
  constexpr uint32_t too_large = kTooLarge<kFmt>;
  if (max(top[0], top[1]) >= too_large) {  // (the same in every thread)
    if (t == 0) atomicOr(flags, kFlagNotStored);
#pragma unroll
    for (int pass = 0; pass < 4; ++pass)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (abs_bits(k[pass][2 * i]) >= too_large) k[pass][2 * i] = 0.f;
        if (abs_bits(k[pass][2 * i + 1]) >= too_large) k[pass][2 * i + 1] = 0.f;
        if ((vx[pass][i] & 0x7fffffffu) >= too_large) vx[pass][i] &= 0xffffu;
        if (((vx[pass][i] << 16) & 0x7fffffffu) >= too_large) vx[pass][i] &= 0xffff0000u;
      }
    reduce(1);
  }
  float ks, kinv, vs, vinv;
  tile_scale<kFmt>(top[0], ks, kinv);
  tile_scale<kFmt>(top[1], vs, vinv);

  uint8_t* const kdst = reinterpret_cast<uint8_t*>(A->kpool) + tile * kPageHeadElems;
  uint8_t* const vdst = reinterpret_cast<uint8_t*>(A->vpool) + tile * kPageHeadElems;
  float norm2 = 0.f;
#pragma unroll
  for (int pass = 0; pass < 4; ++pass) {
    const int row = pass * 16 + rr;
    float v[8], n2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16_lo(vx[pass][i]);
      v[2 * i + 1] = bf16_hi(vx[pass][i]);
    }
    float unused;
    const u32x2 vw = quantise8<kFmt>(v, vinv, unused);
    *reinterpret_cast<u32x2*>(&lds.v[row][(2 * c) ^ (4 * (row >> 3))]) = vw;
    const u32x2 kw = quantise8<kFmt>(k[pass], kinv, n2);
    *reinterpret_cast<u32x2*>(kdst + k8_tile_index(row, 8 * c)) = kw;
    norm2 = fmaxf(norm2, row_sum(n2));
  }
  norm2 = pair_max<32>(pair_max<16>(norm2));
  if ((t & 63) == 0) lds.norm2[wave] = norm2;
  __syncthreads();
  // thread: d quad dq (four rows of V^T), slots 8 oct .. 8 oct + 7
  const int oct = t & 7, dq = t >> 3;
  uint32_t w0[4], w1[4], o0[4], o1[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w0[i] = lds.v[8 * oct + i][dq ^ (4 * oct)];
    w1[i] = lds.v[8 * oct + 4 + i][dq ^ (4 * oct)];
  }
  transpose4(w0, o0);
  transpose4(w1, o1);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *reinterpret_cast<u32x2*>(vdst + v8_tile_index(8 * oct, 4 * dq + j)) = (u32x2){o0[j], o1[j]};
  if (t == 0) {
    A->kscale[tile] = ks;
    A->vscale[tile] = vs;
    // a bound on the norm of the operands the attention makes of them.  int8: each of
    // 128 codes is off by half a scale at most, and code times scale rounded to bf16
    // (up by at most 2^-8); e4m3: exact
    const float top2 = fmaxf(fmaxf(lds.norm2[0], lds.norm2[1]), fmaxf(lds.norm2[2], lds.norm2[3]));
    const float norm = kFmt == kFmtInt8 ? 1.004f * (sqrtf(top2) + 5.66f * ks) : sqrtf(top2) * ks;
    A->knorm2[tile] = norm * norm;
  }
}

template <int kFmt>
__global__ __launch_bounds__(256) void kv_append_q_kernel(const AppendArgs args) {
  (void)args;  // read in place, through append_args()
  __shared__ __attribute__((aligned(16))) AppendLds lds;
  const const_append_args A = append_args();
  const int heads = A->num_heads;
  const int n_tiles = A->n_blocks * heads;
  for (int tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
    append_tile_q<kFmt>(A, tile / heads, tile % heads, lds);
    __syncthreads();  // the LDS is rewritten by the next tile
  }
}

// ------------------------------------------------------------------------- //
// kv_gather: a (page, head) tile back to bf16 rows.  256 threads; V goes through
// LDS (words of 4 slots, or pairs of slots, of a dim) to come out in rows.  Bound by
// memory: 107 pages of 40 heads in 33 us, 6.4 TB/s (much of it from the caches).
// ------------------------------------------------------------------------- //
typedef const __attribute__((address_space(4))) GatherArgs* const_gather_args;

template <int kFmt>
__device__ __forceinline__ void gather_tile(const const_gather_args A, int item, int head, uint32_t* lds) {
  const auto* sg = A->seg + A->blk_seg[item];
  const int tok0 = A->blk_page[item] * kPageTokens;
  const int valid = min(sg->n_tokens - tok0, kPageTokens);
  const int64_t tok_stride = sg->tok_stride;
  uint16_t* const ko = sg->k ? sg->k + tok0 * tok_stride + head * sg->head_stride : nullptr;
  uint16_t* const vo = sg->v ? sg->v + tok0 * tok_stride + head * sg->head_stride : nullptr;
  const int64_t tile = static_cast<int64_t>(A->pages[item]) * A->num_heads + head;
  const int t = threadIdx.x;
  if constexpr (kFmt == kFmtBf16) {
    const uint16_t* const ks = A->kpool + tile * kPageHeadElems;
    const uint16_t* const vs = A->vpool + tile * kPageHeadElems;
    const int c = t & 15, rr = t >> 4;
    if (ko) {
#pragma unroll
      for (int pass = 0; pass < 4; ++pass) {
        const int slot = pass * 16 + rr;
        if (slot < valid)
          *reinterpret_cast<u32x4*>(ko + slot * tok_stride + 8 * c) =
              *reinterpret_cast<const u32x4*>(ks + k_tile_index(slot, 8 * c));
      }
    }
    if (vo) {
      uint16_t* const vt = reinterpret_cast<uint16_t*>(lds);  // [64 slots][136]
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = t + 256 * i, d = (p >> 2) & 127, s0 = 32 * (p >> 9) + 8 * (p & 3);
        const u32x4 w = *reinterpret_cast<const u32x4*>(vs + v_tile_index(s0, d));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          vt[(s0 + 2 * j) * 136 + d] = static_cast<uint16_t>(w[j]);
          vt[(s0 + 2 * j + 1) * 136 + d] = static_cast<uint16_t>(w[j] >> 16);
        }
      }
      __syncthreads();
#pragma unroll
      for (int pass = 0; pass < 4; ++pass) {
        const int slot = pass * 16 + rr;
        if (slot < valid)
          *reinterpret_cast<u32x4*>(vo + slot * tok_stride + 8 * c) =
              *reinterpret_cast<const u32x4*>(vt + slot * 136 + 8 * c);
      }
    }
  } else {
    const uint8_t* const ks = reinterpret_cast<const uint8_t*>(A->kpool) + tile * kPageHeadElems;
    const uint8_t* const vs = reinterpret_cast<const uint8_t*>(A->vpool) + tile * kPageHeadElems;
    if (ko) {
      const QuantScale q = quant_scale<kFmt>(A->kscale[tile]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // piece: 16 dims of a key
        const int slot = (t >> 2) & 63, d = 64 * i + 16 * (t & 3);
        const u32x4 w = *reinterpret_cast<const u32x4*>(ks + k8_tile_index(slot, d));
        if (slot < valid) {
          u32x4* const dst = reinterpret_cast<u32x4*>(ko + slot * tok_stride + d);
          dst[0] = codes8<kFmt>(w[0], w[1], q);
          dst[1] = codes8<kFmt>(w[2], w[3], q);
        }
      }
    }
    if (vo) {
      const QuantScale q = quant_scale<kFmt>(A->vscale[tile]);
      constexpr int kRow = 17;  // words of a dim's 64 slots, and one against bank conflicts
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // piece: 16 slots of a dim
        const int p = t + 256 * i, d = p >> 2, kq = p & 3;
        const u32x4 w = *reinterpret_cast<const u32x4*>(vs + v8_tile_index(16 * kq, d));
#pragma unroll
        for (int j = 0; j < 4; ++j) lds[d * kRow + 4 * kq + j] = w[j];
      }
      __syncthreads();
      const int dg = t & 15, sq = t >> 4;  // dims 8 dg .., slots 4 sq ..
      uint32_t w0[4], w1[4], o0[4], o1[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w0[j] = lds[(8 * dg + j) * kRow + sq];
        w1[j] = lds[(8 * dg + 4 + j) * kRow + sq];
      }
      transpose4(w0, o0);
      transpose4(w1, o1);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int slot = 4 * sq + j;
        if (slot < valid) *reinterpret_cast<u32x4*>(vo + slot * tok_stride + 8 * dg) = codes8<kFmt>(o0[j], o1[j], q);
      }
    }
  }
}

template <int kFmt>
__global__ __launch_bounds__(256) void kv_gather_kernel(const GatherArgs args) {
  (void)args;  // read in place
  __shared__ __attribute__((aligned(16))) uint32_t lds[kFmt == kFmtBf16 ? 64 * 136 / 2 : 128 * 17];
  const const_gather_args A = (const_gather_args)__builtin_amdgcn_kernarg_segment_ptr();
  const int heads = A->num_heads;
  const int n_tiles = A->n_blocks * heads;
  for (int tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
    gather_tile<kFmt>(A, tile / heads, tile % heads, lds);
    __syncthreads();
  }
}

// ------------------------------------------------------------------------- //
// few_attn: the structure of audio_attn (a workgroup of 4 waves takes one (head,
// 16-query tile, key range); wave w streams pages w, w + 4, ... on its own and the
// waves merge through LDS), for 8-bit pages and token windows.
//
// With lane l = 16 g + i, per page S^T = K Q''^T and O^T += V^T P^T by
// v_mfma_f32_16x16x32_bf16.  Row m of key tile t holds key key_of(t, m), so that
// accumulator registers r of tiles 2c and 2c + 1 in lane group g are eight
// consecutive keys, the B operand of chunk c:
//   bf16   key_of = 32 (t/2) + 8 (m/4) + 4 (t%2) + m%4   (16 bytes are 8 values)
//   8 bit  key_of = 16 (m/4) + 4 t + m%4: both chunks' keys of a lane group are 16
//          consecutive ones, one 16-byte load of V^T; and the dims of the k-step
//          pair 2u, 2u + 1 in lane group g are 64 u + 16 g + 0..15, one of K.
// Bound by memory over long ranges: 4 rows, 40 heads, 8.7k keys of e4m3 in 20 us, 4.4
// TB/s, and 4 us of merge.  Over pages of few tokens by their count, a page being a
// chain of load, product, softmax, product whatever it holds: 132 pages of 4 tokens,
// 40 heads, 16 us.
// ------------------------------------------------------------------------- //
template <int kFmt>
__device__ __forceinline__ int key_of(int t, int m) {
  return kFmt == kFmtBf16 ? 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3) : 16 * (m >> 2) + 4 * t + (m & 3);
}
// first of the eight dims of k-step s in lane group g
template <int kFmt>
__device__ __forceinline__ int dims_of(int s, int g) {
  return kFmt == kFmtBf16 ? 32 * s + 8 * g : 64 * (s >> 1) + 16 * g + 8 * (s & 1);
}

template <int kFmt>
struct FewPage {
  static constexpr int kLoads = kFmt == kFmtBf16 ? 16 : 8;
  u32x4 k[kLoads], v[kLoads];
};

// Tiles are read through buffer descriptors: a lane whose row or columns lie past
// n_valid asks past the end and gets zeros without a memory access.  (Redirected to
// a block of zeros, such lanes of all CUs meet at its few lines: 2.6 us a page of 4
// tokens, where a full page takes 1.3.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const uint16_t* pool, int64_t tile, int bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(pool) + static_cast<uint64_t>(tile) * bytes;
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(at), 0, bytes, 0x00020000);
}
constexpr int kPastEnd = 1 << 30;
template <int kFmt>
constexpr int kTileBytes = kFmt == kFmtBf16 ? 2 * kPageHeadElems : kPageHeadElems;
__device__ __forceinline__ u32x4 buffer16(__amdgpu_buffer_rsrc_t r, int lane_off, int off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_off, off, 0));
}
template <int kFmt>
__device__ __forceinline__ void few_load_k(u32x4 (&k)[FewPage<kFmt>::kLoads], const uint16_t* pool, int64_t tile,
                                           int n_valid, int g, int i) {
  const auto r = tile_rsrc(pool, tile, kTileBytes<kFmt>);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int key = key_of<kFmt>(t, i);
    if constexpr (kFmt == kFmtBf16) {
      const int off = key < n_valid ? 2 * k_tile_index(key, 8 * g) : kPastEnd;
#pragma unroll
      for (int s = 0; s < 4; ++s) k[4 * t + s] = buffer16(r, off, 2 * k_tile_index(0, 32) * s);
    } else {
      const int off = key < n_valid ? k8_tile_index(key, 16 * g) : kPastEnd;
#pragma unroll
      for (int u = 0; u < 2; ++u) k[2 * t + u] = buffer16(r, off, k8_tile_index(0, 64) * u);
    }
  }
}
template <int kFmt>
__device__ __forceinline__ void few_load_v(u32x4 (&v)[FewPage<kFmt>::kLoads], const uint16_t* pool, int64_t tile,
                                           int n_valid, int g, int i) {
  const auto r = tile_rsrc(pool, tile, kTileBytes<kFmt>);
  if constexpr (kFmt == kFmtBf16) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int off = 32 * c + 8 * g < n_valid ? 2 * v_tile_index(32 * c + 8 * g, i) : kPastEnd;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) v[2 * dt + c] = buffer16(r, off, 2 * v_tile_index(0, 16) * dt);
    }
  } else {
    const int off = 16 * g < n_valid ? v8_tile_index(16 * g, i) : kPastEnd;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) v[dt] = buffer16(r, off, v8_tile_index(0, 16) * dt);
  }
}
__device__ __forceinline__ bf16x8 operand(u32x4 w) { return __builtin_bit_cast(bf16x8, w); }
template <int kFmt>
__device__ __forceinline__ bf16x8 k_operand(const u32x4 (&k)[FewPage<kFmt>::kLoads], int t, int s, const QuantScale& q) {
  if constexpr (kFmt == kFmtBf16) return operand(k[4 * t + s]);
  else return operand(codes8<kFmt>(k[2 * t + (s >> 1)][2 * (s & 1)], k[2 * t + (s >> 1)][2 * (s & 1) + 1], q));
}
template <int kFmt>
__device__ __forceinline__ bf16x8 v_operand(const u32x4 (&v)[FewPage<kFmt>::kLoads], int dt, int c, const QuantScale& q) {
  if constexpr (kFmt == kFmtBf16) return operand(v[2 * dt + c]);
  else return operand(codes8<kFmt>(v[dt][2 * c], v[dt][2 * c + 1], q));
}

// The call's page list: in device memory, or in the kernel arguments (the
// kernel's only argument is the AttnArgs).
__device__ __forceinline__ const_page_list call_pages(const AttnArgs& a) {
  if (a.pages) return (const_page_list)a.pages;
  const __attribute__((address_space(4))) char* seg =
      (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
  return (const_page_list)(seg + offsetof(AttnArgs, inline_pages));
}

typedef const __attribute__((address_space(4))) float* const_floats;

template <int kFmt>
__global__ __launch_bounds__(256, 2) void few_attn_kernel(const AttnArgs a) {
  __shared__ float sm_o[4][kHeadDim][16];  // per wave O^T, merged at the end
  __shared__ float sm_ml[4][2][16];        // per wave (m, l) per query
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, i16 = lane & 15;
  const int bid = blockIdx.x;
  const int split = bid % a.n_splits;
  const int rest = bid / a.n_splits;
  const int qtile = rest % a.n_qtiles;
  const int head = rest / a.n_qtiles;
  const int p_begin = split * a.pages_per_split + wave;
  const int p_end = min(a.n_pages, (split + 1) * a.pages_per_split);
  const const_page_list pages = call_pages(a);
  const bool window = a.win.on != 0;

  // (the scales come with a page's entry, a page ahead of their use)
  struct Entry {
    int valid, start;
    int64_t tile;
    float ks, vs;
  };
  const const_floats kscale = (const_floats)a.kscale, vscale = (const_floats)a.vscale;
  auto entry = [&](int p) {
    if (p >= p_end) return Entry{0, 0, 0, 1.f, 1.f};  // past the last page: zeros
    const int x = pages[p].x;
    const uint32_t y = static_cast<uint32_t>(pages[p].y);
    Entry e{static_cast<int>(y & 127u), static_cast<int>(y >> 7), static_cast<int64_t>(x) * a.num_heads + head, 1.f, 1.f};
    if (kFmt != kFmtBf16) {
      e.ks = kscale[e.tile];
      e.vs = vscale[e.tile];
    }
    return e;
  };

  // the wave's first page is requested before the query prologue
  FewPage<kFmt> pg;
  Entry cur = entry(p_begin);
  few_load_k<kFmt>(pg.k, a.kpool, cur.tile, cur.valid, g, i16);
  few_load_v<kFmt>(pg.v, a.vpool, cur.tile, cur.valid, g, i16);

  // lane holds Q''[q][dims_of(s, g) ..], with the softmax scale and log2(e) in it
  const int q = qtile * kAudioQTile + i16;
  const bool q_ok = q < a.n_q;
  const uint16_t* qp = a.q + q * a.q_tok_stride + head * a.q_head_stride;
  u32x4 qraw[4];
  bf16x8 qreg[4];
#pragma unroll
  for (int s = 0; s < 4; ++s)
    qraw[s] = q_ok ? *reinterpret_cast<const u32x4*>(qp + dims_of<kFmt>(s, g)) : (u32x4){0u, 0u, 0u, 0u};
  if (a.mode == 1) {
    int pt = 0, ph = 0, pw = 0;
    if (q_ok) load_pos(a.rope, a.positions, q, a.flags, pt, ph, pw);
    float ss = 0.f;
#pragma unroll
    for (int s = 0; s < 4; ++s) ss += norm2_fma(qraw[s]);
    ss = pair_sum<32>(pair_sum<16>(ss));
    const float inv = rsqrtf(ss * (1.0f / kHeadDim) + a.eps);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int d0 = dims_of<kFmt>(s, g);
      const float4 g0 = *reinterpret_cast<const float4*>(a.gamma + d0);
      const float4 g1 = *reinterpret_cast<const float4*>(a.gamma + d0 + 4);
      const float gg[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
      u32x4 w;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float y0 = bf16_lo(qraw[s][k]) * inv * gg[2 * k];
        const float y1 = bf16_hi(qraw[s][k]) * inv * gg[2 * k + 1];
        const float2 cs = rope_cs(a.rope, (d0 >> 1) + k, pt, ph, pw);
        w[k] = pack_bf16((y0 * cs.x - y1 * cs.y) * a.scale_log2, (y0 * cs.y + y1 * cs.x) * a.scale_log2);
      }
      qreg[s] = operand(q_ok ? w : (u32x4){0u, 0u, 0u, 0u});
    }
  } else {
    const float sc = a.mode == 2 ? 1.0f : a.scale_log2;  // prepared: Q'' as given (x 1 is exact)
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      u32x4 w;
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = pack_bf16(bf16_lo(qraw[s][k]) * sc, bf16_hi(qraw[s][k]) * sc);
      qreg[s] = operand(w);
    }
  }

  // Softmax shift, as in the audio kernel: the logit bound |Q''_q| max |k| over the
  // wave's pages when it is small enough for all 16 queries, else a running maximum.
  float kn2 = 0.f;
  for (int p = p_begin + 4 * lane; p < p_end; p += 256)
    kn2 = fmaxf(kn2, a.knorm2[static_cast<int64_t>(pages[p].x) * a.num_heads + head]);
  kn2 = fminf(wave_max(kn2), 3.0e38f);
  float qn2 = 0.f;
#pragma unroll
  for (int s = 0; s < 4; ++s) qn2 += norm2_fma(__builtin_bit_cast(u32x4, qreg[s]));
  const float bound = sqrtf(pair_sum<32>(pair_sum<16>(qn2)) * kn2);
  const bool fixed_shift = a.fixed_shift != 0 && __all(bound <= kShiftBoundMax);
  float m_run = fixed_shift ? bound : kNegInf, l_run = 0.f;

  // a page all of whose keys every row of the tile sees needs no mask
  const int t_first = a.win.t0 + qtile * kAudioQTile;
  const int t_last = a.win.t0 + min(qtile * kAudioQTile + kAudioQTile, a.n_q) - 1;
  const RowRange row = row_range(a.win, a.win.t0 + q);
  const int hi_all = row_range(a.win, t_first).hi, lo_all = row_range(a.win, t_last).lo;

  f32x4 o[8];
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) o[dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
  // one page: the first kChunks of the two 32-key chunks (8-bit pages of up to 8
  // tokens, such as a unit's audio, have keys in the first alone)
  auto attend = [&](auto chunks, int p) __attribute__((always_inline)) {
    constexpr int kChunks = decltype(chunks)::value;
    const QuantScale ks = quant_scale<kFmt>(cur.ks), vs = quant_scale<kFmt>(cur.vs);
    const Entry nxt = entry(p + 4);
    f32x4 sacc[2 * kChunks];
#pragma unroll
    for (int t = 0; t < 2 * kChunks; ++t) {
      sacc[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 4; ++s)
        sacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k_operand<kFmt>(pg.k, t, s, ks), qreg[s], sacc[t], 0, 0, 0);
    }
    few_load_k<kFmt>(pg.k, a.kpool, nxt.tile, nxt.valid, g, i16);
    const bool whole = cur.valid == kPageTokens &&
                       (!window || (cur.start + kPageTokens <= hi_all &&
                                    (cur.start >= lo_all || cur.start + kPageTokens <= a.win.sinks)));
    if (!whole) {
      const int hi = window ? min(cur.valid, row.hi - cur.start) : cur.valid;
      const int lo = window ? row.lo - cur.start : 0, sk = window ? a.win.sinks - cur.start : 0;
#pragma unroll
      for (int t = 0; t < 2 * kChunks; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int slot = key_of<kFmt>(t, 4 * g + r);
          if (!(slot < hi && (slot >= lo || slot < sk))) sacc[t][r] = kNegInf;
        }
    }
    if (!fixed_shift) {
      float mx = kNegInf;
#pragma unroll
      for (int t = 0; t < 2 * kChunks; ++t) mx = fmaxf(mx, fmaxf(fmaxf(sacc[t][0], sacc[t][1]), fmaxf(sacc[t][2], sacc[t][3])));
      mx = pair_max<32>(pair_max<16>(mx));
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_new == kNegInf ? 1.f : fast_exp2(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) o[dt] *= alpha;
    }
    const float m_use = m_run == kNegInf ? 0.f : m_run;
    u32x4 pw[kChunks];
    const bf16x2 ones = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4& sc = sacc[2 * c + h];
        const uint32_t w0 = pack_bf16(fast_exp2(sc[0] - m_use), fast_exp2(sc[1] - m_use));
        const uint32_t w1 = pack_bf16(fast_exp2(sc[2] - m_use), fast_exp2(sc[3] - m_use));
        pw[c][2 * h] = w0;
        pw[c][2 * h + 1] = w1;
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w0), ones, l_run, false);
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w1), ones, l_run, false);
      }
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_operand<kFmt>(pg.v, dt, c, vs), operand(pw[c]), o[dt], 0, 0, 0);
    few_load_v<kFmt>(pg.v, a.vpool, nxt.tile, nxt.valid, g, i16);
    cur = nxt;
  };
  for (int p = p_begin; p < p_end; p += 4) {
    if (kFmt != kFmtBf16 && cur.valid <= 8) attend(std::integral_constant<int, 1>{}, p);
    else attend(std::integral_constant<int, 2>{}, p);
  }

  // merge the four waves: lane holds O^T[16 dt + 4 g + r][q] of its keys
  float l_w = pair_sum<32>(pair_sum<16>(l_run));
#pragma unroll
  for (int dt = 0; dt < 8; ++dt)
#pragma unroll
    for (int r = 0; r < 4; ++r) sm_o[wave][16 * dt + 4 * g + r][i16] = o[dt][r];
  if (g == 0) {
    sm_ml[wave][0][i16] = m_run;
    sm_ml[wave][1][i16] = l_w;
  }
  if constexpr (kFmt == kFmtBf16) {
    uint32_t top = 0;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = max(top, abs_bits(o[dt][r]));
    if (__any(top >= kInfBits)) {
      window_rows_plain(a, head, qtile * kAudioQTile, kAudioQTile, p_begin, p_end, 4, lane,
                        [&](int p) { return make_int2(pages[p].x, pages[p].y); },
                        [&](int i, float m, float l, float o0, float o1) {
                          sm_o[wave][2 * lane][i] = o0;
                          sm_o[wave][2 * lane + 1][i] = o1;
                          if (lane == 0) {
                            sm_ml[wave][0][i] = m;
                            sm_ml[wave][1][i] = l;
                          }
                        });
    }
  }
  __syncthreads();
  // thread t: query t % 16, d = 8 (t / 16) .. + 8
  const int qi = tid & 15, d0 = 8 * (tid >> 4);
  float mw[4], big = kNegInf;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    mw[w] = sm_ml[w][0][qi];
    big = fmaxf(big, mw[w]);
  }
  float ew[4], l_tot = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    // (a wave without weight counts nothing, whatever its shift)
    ew[w] = big == kNegInf || sm_ml[w][1][qi] == 0.f ? 0.f : fast_exp2(mw[w] - big);
    l_tot += ew[w] * sm_ml[w][1][qi];
  }
  const int qq = qtile * kAudioQTile + qi;
  if (qq >= a.n_q) return;
  const float inv = l_tot > 0.f ? 1.0f / l_tot : 0.f;
  f32x4 out0, out1;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) v += ew[w] * sm_o[w][d0 + k][qi];
    if (k < 4) out0[k] = v * inv; else out1[k - 4] = v * inv;
  }
  if (a.audio_direct) {  // the only range: what the merge of one range gives (a row without weight: zeros)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      out0[k] = l_tot > 0.f ? out0[k] + 0.f : 0.f;
      out1[k] = l_tot > 0.f ? out1[k] + 0.f : 0.f;
    }
    *reinterpret_cast<u32x4*>(a.out + qq * a.out_tok_stride + head * a.out_head_stride + d0) =
        (u32x4){pack_bf16(out0[0], out0[1]), pack_bf16(out0[2], out0[3]), pack_bf16(out1[0], out1[1]),
                pack_bf16(out1[2], out1[3])};
    return;
  }
  const int64_t prow = (static_cast<int64_t>(split) * a.num_heads + head) * a.n_q + qq;
  float* po = a.part_o + prow * kHeadDim + d0;
  *reinterpret_cast<f32x4*>(po) = out0;
  *reinterpret_cast<f32x4*>(po + 4) = out1;
  if (tid < 16) a.part_lse[prow] = l_tot > 0.f ? big + __log2f(l_tot) : kNegInf;
}

template <class Kernel, class Args>
hipError_t launch(Kernel* kernel, int grid, const Args& a, hipStream_t stream, hipEvent_t start, hipEvent_t stop) {
  if (start || stop)
    hipExtLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, stream, start, stop, 0, a);
  else
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append_q(const AppendArgs& a, hipStream_t stream, hipEvent_t start, hipEvent_t stop) {
  const int grid = std::min(a.n_blocks * a.num_heads, std::max(1, a.grid_blocks));
  return launch(a.format == kFmtInt8 ? kv_append_q_kernel<kFmtInt8> : kv_append_q_kernel<kFmtE4m3>, grid, a, stream,
                start, stop);
}

hipError_t launch_kv_gather(const GatherArgs& a, hipStream_t stream, hipEvent_t start, hipEvent_t stop) {
  const auto kernel = a.format == kFmtBf16   ? kv_gather_kernel<kFmtBf16>
                      : a.format == kFmtInt8 ? kv_gather_kernel<kFmtInt8>
                                             : kv_gather_kernel<kFmtE4m3>;
  return launch(kernel, a.n_blocks * a.num_heads, a, stream, start, stop);
}

hipError_t launch_few_attention(const AttnArgs& a, hipStream_t stream, hipEvent_t start, hipEvent_t stop) {
  const auto kernel = a.format == kFmtBf16   ? few_attn_kernel<kFmtBf16>
                      : a.format == kFmtInt8 ? few_attn_kernel<kFmtInt8>
                                             : few_attn_kernel<kFmtE4m3>;
  return launch(kernel, a.num_heads * a.n_qtiles * a.n_splits, a, stream, start, stop);
}

}  // namespace ws
