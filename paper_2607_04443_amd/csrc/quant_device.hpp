// Device helpers of the 8-bit pools and of token windows: codes to matrix
// operands, rows' key ranges, and the plain evaluation of a window's rows.
#pragma once

#include "device_common.hpp"

namespace ws {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Two codes (the low or high half of a word) as packed bf16(code * scale).
//   e4m3: the conversion multiplies by the scale, a power of two: exact.
//   int8: bytes b = code + 128 behind 0x64: a half is 1024 + b; in fp32
//         (1024 + b) s - 1152 s = code s, exact because s has 16 significant
//         bits; then one rounding.  (A half per perm, a mixed fma each, one pack:
//         2 instructions a value; through v_cvt_f32_ubyte it is 2.5.)
struct QuantScale {
  float s, c;  // c = -1152 s (int8)
};
template <int kFmt>
__device__ __forceinline__ QuantScale quant_scale(float s) {
  return QuantScale{s, kFmt == kFmtInt8 ? -1152.0f * s : 0.f};
}
template <int kHalf>
__device__ __forceinline__ uint32_t spread_codes(uint32_t codes) {
  return __builtin_amdgcn_perm(0x64646464u, codes, kHalf ? 0x04030402u : 0x04010400u);
}
template <int kHalf>
__device__ __forceinline__ float spread_value(uint32_t p, const QuantScale& q) {
  return fmaf(static_cast<float>(__builtin_bit_cast(f16x2, p)[kHalf]), q.s, q.c);
}
template <int kFmt, int kHalf>
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t codes, const QuantScale& q) {
  if constexpr (kFmt == kFmtE4m3) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, q.s, kHalf == 1));
  } else {
    const uint32_t p = spread_codes<kHalf>(codes);
    return pack_bf16(spread_value<0>(p, q), spread_value<1>(p, q));
  }
}
// Eight codes (two words) as an MFMA operand.
template <int kFmt>
__device__ __forceinline__ u32x4 codes8(uint32_t w0, uint32_t w1, const QuantScale& q) {
  return (u32x4){codes_to_bf16<kFmt, 0>(w0, q), codes_to_bf16<kFmt, 1>(w0, q), codes_to_bf16<kFmt, 0>(w1, q),
                 codes_to_bf16<kFmt, 1>(w1, q)};
}

// The keys that the row at timeline index t sees: [lo, hi) and the first `sinks`
// below hi.  (t and the window are at most 2^30 in size: no overflow.)
struct RowRange {
  int lo, hi;
};
__device__ __forceinline__ RowRange row_range(const TokenWindow& w, int t) {
  return RowRange{t + 1 - w.window, min(t + w.ahead, w.n_keys)};
}
__device__ __forceinline__ bool row_sees(const TokenWindow& w, const RowRange& r, int j) {
  return j < r.hi && (j >= r.lo || j < w.sinks);
}

// ------------------------------------------------------------------------- //
// A row that does not see a key gives it weight 0, but a matrix product still
// multiplies that 0 with the key's value: an infinity or NaN there would reach
// rows that do not see it.  (An 8-bit cache holds finite values only.)  Where a
// window's result is not finite, the wave evaluates its rows again without
// matrix instructions, seen keys only: one row at a time, lane l holding dims
// 2 l and 2 l + 1 (rotary pair l).  Rows row0 .. row0 + n - 1 of the call over
// pages p_begin, p_begin + step, ... (< p_end) of the list; done(i, m, l, o0, o1)
// takes row i's running maximum (log2), sum and unnormalised pair.
// ------------------------------------------------------------------------- //
template <class Page, class Done>
__device__ __forceinline__ void window_rows_plain(const AttnArgs& a, int head, int row0, int n, int p_begin, int p_end,
                                                  int step, int lane, Page&& page_at, Done&& done) {
  for (int i = 0; i < n; ++i) {
    const int row = row0 + i;
    if (row >= a.n_q) break;
    const uint32_t w =
        *reinterpret_cast<const uint32_t*>(a.q + row * a.q_tok_stride + head * a.q_head_stride + 2 * lane);
    float q0 = bf16_lo(w), q1 = bf16_hi(w);
    if (a.mode == 1) {
      int pt, ph, pw;
      load_pos(a.rope, a.positions, row, a.flags, pt, ph, pw);
      const float ss = pair_sum<32>(pair_sum<16>(row_sum(fmaf(q0, q0, q1 * q1))));
      const float inv = rsqrtf(ss * (1.0f / kHeadDim) + a.eps);
      const float2 cs = rope_cs(a.rope, lane, pt, ph, pw);
      const float y0 = q0 * inv * a.gamma[2 * lane], y1 = q1 * inv * a.gamma[2 * lane + 1];
      q0 = (y0 * cs.x - y1 * cs.y) * a.scale_log2;
      q1 = (y0 * cs.y + y1 * cs.x) * a.scale_log2;
    } else if (a.mode == 0) {
      q0 *= a.scale_log2;
      q1 *= a.scale_log2;
    }
    const uint32_t qw = pack_bf16(q0, q1);
    q0 = bf16_lo(qw);
    q1 = bf16_hi(qw);
    const RowRange r = row_range(a.win, a.win.t0 + row);
    float m = kNegInf, l = 0.f, o0 = 0.f, o1 = 0.f;
    for (int p = p_begin; p < p_end; p += step) {
      const int2 e = page_at(p);
      const int valid = e.y & 127, start = static_cast<int>(static_cast<uint32_t>(e.y) >> 7);
      const int64_t tile = (static_cast<int64_t>(e.x) * a.num_heads + head) * kPageHeadElems;
      for (int slot = 0; slot < valid; ++slot) {
        if (!row_sees(a.win, r, start + slot)) continue;
        const uint32_t k = *reinterpret_cast<const uint32_t*>(a.kpool + tile + k_tile_index(slot, 2 * lane));
        const float s = pair_sum<32>(pair_sum<16>(row_sum(fmaf(q0, bf16_lo(k), q1 * bf16_hi(k)))));
        const float m_new = fmaxf(m, s);
        if (m_new == kNegInf) continue;
        const float keep = fast_exp2(m - m_new), p_new = fast_exp2(s - m_new);
        const uint16_t* v = a.vpool + tile + v_tile_index(slot, 2 * lane);
        m = m_new;
        l = l * keep + p_new;
        o0 = o0 * keep + p_new * bf16_lo(v[0]);
        o1 = o1 * keep + p_new * bf16_lo(v[v_tile_index(0, 1)]);
      }
    }
    done(i, m, l, o0, o1);
  }
}

}  // namespace
}  // namespace ws
