// The video kernel's device code (kernels.hip: bf16 pages; paths.hip: 8-bit pages
// and token windows), and the audio kernel's parts that it shares for the rows
// that ride in it.
#pragma once

#include <cstddef>
#include <type_traits>
#include <utility>

#include "device_common.hpp"
#include "quant_device.hpp"
#include "ws_kernels.hpp"

namespace ws {
namespace {

// ------------------------------------------------------------------------- //
// unit_attn (video): query tiles of 256, 192 or 128 rows on 4 waves (one per
// SIMD) of 64, 48 or 32 queries, a last tile of at most 128 rows on waves of
// 32; 64-key pages through LDS.
//
// Per wave and page, with lane l = 16 g + i (i = query column of a 16-query
// subtile, g = lane group) and v_mfma_f32_16x16x32_bf16:
//   S^T[16 keys][16 q]  = K Q''^T    4 key tiles x 4 k-steps per subtile
//   O^T[16 d][16 q]    += V^T P^T    8 d tiles x 2 key chunks of 32
//   l[q]               += 1 P^T      2 key chunks (the row sums, on the matrix
//                                    pipe: over the same bf16 P as O)
// Row m = 4 g' + r of key tile t holds key 32 (t/2) + 8 g' + 4 (t%2) + r
// (audio_key below), so registers r of tiles 2c and 2c + 1 in lane group g are
// keys 32 c + 8 g + 0..7: directly the B operand of the P*V MFMA of chunk c.
//
// What bounds it: at the long windows the chip's power limit, then the matrix
// pipe.  The MFMA shape, the operand reuse and the row sums follow from that.
// Measured on the page loop alone (256 CUs, random operands, no page loads):
//   32x32x16 MFMAs, 8 waves x 32 rows               1.455 us per page
//   32x32x16 MFMAs, 4 waves x 64 rows               1.43  us
//   16x16x32 MFMAs, 8 waves x 32 rows               1.33-1.41 us
//   16x16x32 MFMAs, 4 waves x 64 rows, v_dot2 sums  1.30-1.40 us
//   16x16x32 MFMAs, 4 waves x 64 rows, MFMA sums    1.23-1.27 us
// (16x16x32 sustains 2170-2240 TFLOP/s on random register operands, 32x32x16
// 1950; 64 rows per wave halve the LDS operand reads; a row-sum MFMA costs
// less than the 16 v_dot2 it replaces.)
// ------------------------------------------------------------------------- //

// What a video kernel reads: pages of which format, and whether a token window may
// hide keys of a page from some rows.  Paths other than PlainPath take queries of
// any mode and no rider rows.
template <int kFormat, bool kWindow>
struct Path {
  static constexpr int kFmt = kFormat;
  static constexpr bool k8 = kFormat != kFmtBf16;
  static constexpr bool kWin = kWindow;
  static constexpr bool kPlain = kFormat == kFmtBf16 && !kWindow;
  static constexpr bool kPieces = kFormat == kFmtInt8;  // conversions an instruction at a time
  static constexpr bool kQ8 = kFormat == kFmtE4m3;  // S by 8-bit products (VideoState)
};
using PlainPath = Path<kFmtBf16, false>;
template <int>
struct Nothing {};

// f(Const<0>), ..., f(Const<N - 1>), unrolled by construction.
template <int N>
struct Const {
  static constexpr int value = N;
};
template <class F, int... Is>
__device__ __forceinline__ void static_for_seq(F&& f, std::integer_sequence<int, Is...>) {
  (f(Const<Is>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for_seq(f, std::make_integer_sequence<int, N>{});
}

// Row m (lane index i) of key tile t: the key it holds.
__device__ __forceinline__ int audio_key(int t, int m) {
  return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3);
}

// LDS stages of the video kernel (a ring of five pages, 160 KB: the previous
// page, whose V^T the pipelined schedule still reads, the current page, the
// next page, already complete so that its first operands can be read before
// the page barrier, and the two after it in flight), filled by direct
// global->LDS loads (global_load_lds_dwordx4: lane l of a wave writes 16
// bytes at base + 16 l).  A stage is a K tile, then a V tile:
//   K    [64 rows][16 chunks]: row 16 t + m holds key audio_key(t, m); its
//        logical chunk c (dims 8c..8c+7) sits at position c ^ m.
//   V^T  [128 d][8 chunks]: logical chunk c (keys 8c..8c+7) of row d sits at
//        position c ^ ((d >> 1) & 7).
// Either way the 16 lanes of a lane group read 16 distinct 16-byte bank groups.
constexpr int kStages = 5;
constexpr uint32_t kStageBytes = 2 * kPageHeadElems * 2;
constexpr uint32_t kStageV = kPageHeadElems * 2;  // offset of the V tile
__shared__ __attribute__((aligned(1024))) uint16_t g_stages[kStages * 2 * kPageHeadElems];

typedef int i32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// The call's visible page list: in device memory, or in the kernel
// arguments themselves (the kernel's only argument is the AttnArgs, at the
// start of the kernel argument segment; addressing it through the segment
// pointer keeps the compiler from copying the argument to private memory).
__device__ __forceinline__ const_page_list page_list(const AttnArgs& a) {
  if (a.pages) return (const_page_list)a.pages;
  const __attribute__((address_space(4))) char* seg =
      (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
  return (const_page_list)(seg + offsetof(AttnArgs, inline_pages));
}

// LDS byte offset of a pointer into a __shared__ object.
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)p));
}
// 16 bytes at an LDS byte offset.
__device__ __forceinline__ bf16x8 lds_read16(uint32_t off) {
  return as_bf16x8(*(const __attribute__((address_space(3))) u32x4*)off);
}

__device__ __forceinline__ void sched_fence() { __builtin_amdgcn_sched_barrier(0); }

// The video kernel's MFMAs.  The S tiles sit in vector registers (the softmax
// reads them; the build asks for that form of the MFMA builtins), O and l in
// accumulation registers, by inline asm: the compiler's own choice puts all
// of them in one bank, and every exponential or every O update then goes
// through a copy.  The compiler does not see the matrix pipe's latency behind
// the asm: O and l are read or written by other instructions only across
// mfma_drain(), and a P word or another vector operand is written at least
// two instructions ahead of the asm that reads it.
__device__ __forceinline__ void mfma_s(f32x4& d, bf16x8 a, bf16x8 b, const f32x4& c) {
  d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mfma_o(f32x4& d, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(d) : "v"(a), "v"(b));
}
// The first product into an accumulator (C = 0).
__device__ __forceinline__ void mfma_o_first(f32x4& d, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=a"(d) : "v"(a), "v"(b));
}
// An accumulator times a factor, in place: multiplied in plain code it would
// move to vector registers, and the page loop around the branch with it.
__device__ __forceinline__ void scale_acc(f32x4& d, float f) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float x = d[r], t;
    asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %1, %2\n\tv_accvgpr_write_b32 %0, %1"
                 : "+a"(x), "=&v"(t)
                 : "v"(f));
    d[r] = x;
  }
}
// S of a K tile's codes (a: 32 dims of a key per lane) and one term of the queries, on
// the scales 2^(k_exp - 127) and byte kTerm of q_exp.
template <int kTerm>
__device__ __forceinline__ void mfma_s8(f32x4& d, const i32x8& a, const i32x8& b, const f32x4& c, int k_exp, int q_exp) {
  d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, k_exp, kTerm, q_exp);
}
// A value the compiler cannot carry over from an earlier computation: the
// epilogue recomputes its addresses instead of keeping them live across the
// page loop.
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
// Waits until every MFMA issued so far has written its result (and, between a
// vector write and a following MFMA, until the write is visible to it).
__device__ __forceinline__ void mfma_drain() {
  sched_fence();
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
  sched_fence();
}

// What one page's iteration addresses, computed a little at a time during the
// iteration before it, so that the page boundary holds nothing but the
// barrier.
//
// 8-bit pages come through registers instead: the loads of the page three ahead
// go out as the codes of the page two ahead are turned to bf16 and written to its
// stage, part by part.
struct Ctx8 {
  uint32_t ks, vs;         // scales (bits) of the page two ahead (its codes are in the registers)
  uint32_t ks_load, vs_load;  // of the page three ahead
  uint32_t wk, wv;         // LDS offsets of this lane's writes of the page two ahead
  uint32_t vs1, k_exp;     // (e4m3) word of the page one ahead; exponent byte of the current page's K scale
};
template <class P>
struct PageCtx : std::conditional_t<P::k8, Ctx8, Nothing<0>> {
  uint32_t k[4];        // LDS offsets of this lane's operand reads: K, per k-step (key tile t: + 4096 t)
  uint32_t v;           // V^T chunk 0 (d tile dt: + 2048 dt)
  uint32_t vp;          // V^T chunk 1 of the page before
  const uint16_t* ldk;  // the loads to issue, of the page three ahead: K and V tile,
  const uint16_t* ldv;
  uint32_t lds;         // and their LDS offset
};

// A workgroup's share of one query tile's (head, page) units, lo .. lo + n - 1
// in head-major order: one continuous stream of pages through the LDS ring,
// whatever heads it crosses.  A unit's list entry is its tile index
// (page * H + head) and the page's valid tokens; each lane holds the entries
// of two units out of a window of 128, read with v_readlane, so that the page
// loop has no scalar load to wait for (scalar loads and LDS reads share a
// counter that only a full wait can order).
struct Stream8 {
  u32x4 raw[4];          // codes of the page two ahead: K dims 0-63 and 64-127, V dims 0-63 and 64-127
  uint32_t ks[2], vs[2]; // scales (bits) of the window's units (e4m3: both in vs, scale_word)
  const float* kscale;
  const float* vscale;
  uint32_t load[2];      // this lane's source byte offsets within a tile's halves
  uint32_t wk, wv;       // and its write offsets within a stage (first chunk)
};
struct StreamWin {
  int start[2];          // first timeline index of the window's units
  int head_pages, skip;  // the class's list: head_pages pages, then after `skip` others the rest
  int head0;             // head of stream index 0 (launches without classes)
  int hi_all, lo_all;    // keys [lo_all, hi_all) are seen by every row of the wave
  TokenWindow win;
};
template <class P>
struct VideoStream : std::conditional_t<P::k8, Stream8, Nothing<2>>, std::conditional_t<P::kWin, StreamWin, Nothing<3>> {
  const_page_list pages;
  FastDiv div_pages;
  int num_heads, n_pages, page0, lo, n;
  int lane;
  uint32_t ent[2];        // entries of units 64 k + lane of the window (tile index << 7 | valid tokens)
  int raw_head[2], raw_page[2], raw_valid[2];  // what ent is made of
  float kn2[2];           // key-norm maxima (squared) of the first window's units
  const uint16_t* kpool;
  const uint16_t* vpool;
  uint32_t dma_k, dma_v;  // this lane's source byte offsets within a tile (block 0)
  uint32_t k_read, v_read;  // this lane's operand read offsets within a stage (k-step 0, chunk 0)
  uint32_t lds0;          // LDS offset of the wave's first block in stage 0
  int at;                 // stream index of the current page
  uint32_t stage;         // its stage's LDS offset
  uint32_t valid;         // valid tokens of pages at .. at + 3, a byte each
  PageCtx<P> c;           // the current page's context
};

// (Past the end: the last unit's entry.  No lane-dependent branch here or
// anywhere else inside the page loops' regions: with one, the compiler
// serialises the uniform branches around it and keeps the accumulators of both
// sides.)
// Place in the page list of page `at` of the class's pages.
template <class P>
__device__ __forceinline__ int stream_place(const VideoStream<P>& s, int at) {
  if constexpr (P::kWin) at += at >= s.head_pages ? s.skip : 0;
  return s.page0 + at;
}
template <class P>
__device__ __forceinline__ uint32_t head_of(const VideoStream<P>& s, uint32_t head) {
  if constexpr (P::kWin) head += s.head0;
  return head;
}
// A list entry's valid tokens; with a window its first timeline index.
template <class P>
__device__ __forceinline__ uint32_t valid_of(int y) {
  return P::kWin ? static_cast<uint32_t>(y) & 127u : static_cast<uint32_t>(y);
}
__device__ __forceinline__ int start_of(int y) { return static_cast<int>(static_cast<uint32_t>(y) >> 7); }
// What hides slots of a page that starts at timeline index `start` from rows of the
// wave, kEdge* bits: a row's end (the page's own, or a row's last key), and a row's
// first key, in a page with sinks or without.  (Each a pass of its own over the S
// tiles, two or three instructions a value: all three conditions at once take five.)
constexpr int kEdgeHi = 1, kEdgeLo = 2, kEdgeSinks = 4;
template <class P>
__device__ __forceinline__ int page_edge(const VideoStream<P>& s, int start, int valid) {
  const int end = start + kPageTokens;
  const bool lo_hidden = (start < s.lo_all) & (end > s.win.sinks), hi_hidden = (valid < kPageTokens) | (end > s.hi_all);
  const int lo = lo_hidden ? (start < s.win.sinks ? kEdgeSinks : kEdgeLo) : 0, hi = hi_hidden ? kEdgeHi : 0;
  return lo | hi;
}
// The low 7 bits of a unit's entry: the page's valid tokens, and, with a window, 65
// for a full page with an edge (a shorter one has one): an edge is looked for once per
// unit, by the lane that holds it, and the page loop compares with 64.
template <class P>
__device__ __forceinline__ uint32_t entry_valid(const VideoStream<P>& s, int y) {
  uint32_t v = valid_of<P>(y);
  if constexpr (P::kWin) v = v == kPageTokens && page_edge(s, start_of(y), kPageTokens) != 0 ? kPageTokens + 1 : v;
  return v;
}
// e4m3: both scales of a page are powers of two; V's bits with K's exponent byte.
template <class P>
__device__ __forceinline__ uint32_t scale_word(const VideoStream<P>& s, uint32_t tile) {
  return __float_as_uint(s.vscale[tile]) | (__float_as_uint(s.kscale[tile]) >> 23);
}
template <class P>
__device__ __forceinline__ uint32_t stream_entry(const VideoStream<P>& s, int k, int* start = nullptr) {
  const uint32_t x = s.lo + min(k, s.n - 1), head = fast_div(x, s.div_pages);
  const int pi = stream_place(s, static_cast<int>(x - head * s.n_pages));
  const int y = s.pages[pi].y;
  if (start) *start = start_of(y);
  return ((s.pages[pi].x * s.num_heads + head_of(s, head)) << 7) | entry_valid(s, y);
}
// The first window: its list entries requested, then combined.
template <class P>
__device__ __forceinline__ void stream_request(VideoStream<P>& s) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t x = s.lo + min(64 * k + s.lane, s.n - 1), head = fast_div(x, s.div_pages);
    const int pi = stream_place(s, static_cast<int>(x - head * s.n_pages));
    s.raw_head[k] = head_of(s, head);
    s.raw_page[k] = s.pages[pi].x;
    s.raw_valid[k] = s.pages[pi].y;
  }
}
template <class P>
__device__ __forceinline__ void stream_combine(VideoStream<P>& s) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    s.ent[k] = ((s.raw_page[k] * s.num_heads + s.raw_head[k]) << 7) | entry_valid(s, s.raw_valid[k]);
    if constexpr (P::kWin) s.start[k] = start_of(s.raw_valid[k]);
  }
}
// A value of stream index k (uniform, inside the window), from the lanes' two.
template <class T>
__device__ __forceinline__ T peek_lanes(const T (&v)[2], int k) {
  const uint32_t w0 = __builtin_bit_cast(uint32_t, v[0]), w1 = __builtin_bit_cast(uint32_t, v[1]);
  const uint32_t e0 = __builtin_amdgcn_readlane(w0, k & 63), e1 = __builtin_amdgcn_readlane(w1, k & 63);
  return __builtin_bit_cast(T, (k & 64) ? e1 : e0);
}
// Entry of stream index k.
template <class P>
__device__ __forceinline__ uint32_t stream_peek(const VideoStream<P>& s, int k) {
  return peek_lanes(s.ent, k);
}
// Moves the window when the page to look up next, at + 4, enters a new half:
// it replaces the half that lies two behind.
template <class P>
__device__ __forceinline__ void stream_reach(VideoStream<P>& s) {
  const int k = s.at + 4;
  if ((k & 63) == 0 && k >= 128) {
    int start = 0;
    uint32_t e = stream_entry(s, k + s.lane, P::kWin ? &start : nullptr);
    asm volatile("" : "+v"(e));  // waited for here, not at every later use
    if constexpr (P::kWin) {
      asm volatile("" : "+v"(start));
      if (k & 64) s.start[1] = start; else s.start[0] = start;
    }
    if constexpr (P::kQ8) {
      uint32_t vs = scale_word(s, e >> 7);
      asm volatile("" : "+v"(vs));
      if (k & 64) s.vs[1] = vs; else s.vs[0] = vs;
    } else if constexpr (P::k8) {
      uint32_t ks = __float_as_uint(s.kscale[e >> 7]), vs = __float_as_uint(s.vscale[e >> 7]);
      asm volatile("" : "+v"(ks), "+v"(vs));
      if (k & 64) s.ks[1] = ks; else s.ks[0] = ks;
      if (k & 64) s.vs[1] = vs; else s.vs[0] = vs;
    }
    if (k & 64) s.ent[1] = e; else s.ent[0] = e;
  }
}
constexpr uint32_t kRingBytes = kStages * kStageBytes;
__device__ __forceinline__ uint32_t ring_add(uint32_t stage, uint32_t k) {
  const uint32_t x = stage + k * kStageBytes;
  return x >= kRingBytes ? x - kRingBytes : x;
}

// One direct load: each lane's 16 bytes at sbase + voff go to LDS at
// lds + kLdsAdd + 16 * lane.  Written as inline asm: with the compiler's own
// LDS-DMA intrinsic in flight, every later LDS read waits for lgkmcnt(0),
// which serializes the MFMA operand reads.  Completion is tracked by the
// explicit vmcnt waits below.  M0 is the asm's own: nothing the compiler
// emits in this kernel keeps a value in it.
template <uint32_t kLdsAdd>
__device__ __forceinline__ void dma16(const uint16_t* sbase, uint32_t voff, uint32_t lds) {
  // both are wave-uniform by construction; make that visible to the compiler
  // (readfirstlane returns int: widen through uint32_t, never sign-extend)
  lds = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(lds));
  const uint64_t b = reinterpret_cast<uint64_t>(sbase);
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(b >> 32)));
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(b)));
  sbase = reinterpret_cast<const uint16_t*>((static_cast<uint64_t>(hi) << 32) | lo);
  asm volatile(
      "s_add_u32 m0, %2, %3\n\t"
      "global_load_lds_dwordx4 %0, %1"
      :
      : "v"(voff), "s"(sbase), "s"(lds), "i"(kLdsAdd)
      : "memory", "scc");
}

// The direct loads of one page: 32 blocks of 1 KB, 8 per wave (block 4 i +
// wave of each tile, i = 0..3).  Block b of K is rows 4 b .. 4 b + 3, i.e.
// rows 4 wave .. of key tile i (keys 32 (i / 2) + 4 (i % 2) + 8 wave ..); block
// b of V^T is rows d = 8 b .. 8 b + 7.
constexpr int kDmaPerPage = 8;  // direct loads per wave and page
template <int kPart, class P>   // 0..3: K blocks, 4..7: V blocks
__device__ __forceinline__ void issue_load(const VideoStream<P>& s, const PageCtx<P>& c) {
  if constexpr (kPart < 4) {
    constexpr uint32_t src = 2u * k_tile_index(32 * (kPart >> 1) + 4 * (kPart & 1), 0);
    dma16<4096u * kPart>(c.ldk, s.dma_k + src, c.lds);
  } else {
    constexpr uint32_t src = 2u * v_tile_index(0, 32 * (kPart - 4));
    dma16<kStageV + 4096u * (kPart - 4)>(c.ldv, s.dma_v + src, c.lds);
  }
}
template <class P>
__device__ __forceinline__ void issue_page(const VideoStream<P>& s, const PageCtx<P>& c) {
  static_for<kDmaPerPage>([&](auto i) __attribute__((always_inline)) { issue_load<decltype(i)::value>(s, c); });
}
// The load part of a context: the page with entry e (8 bit: loaded to registers;
// else into ring stage `stage`).
constexpr uint32_t kCodeTileShift = 13;  // 8 KB of codes
template <class P>
__device__ __forceinline__ void set_load(const VideoStream<P>& s, uint32_t e, uint32_t stage, PageCtx<P>& c) {
  const uint64_t off = static_cast<uint64_t>(e >> 7) << (P::k8 ? kCodeTileShift : 14);  // 16 KB tiles
  c.ldk = reinterpret_cast<const uint16_t*>(reinterpret_cast<uint64_t>(s.kpool) + off);
  c.ldv = reinterpret_cast<const uint16_t*>(reinterpret_cast<uint64_t>(s.vpool) + off);
  c.lds = __builtin_amdgcn_readfirstlane(s.lds0 + stage);
}

// 8-bit pages.  A thread takes four 16-byte parts of a page (K: dims 64 i + 16 (t %
// 4) .. of key t / 4; V^T: keys 16 (t % 4) .. of dim 64 i + t / 4; t the thread),
// two 16-byte chunks of an LDS tile each.  One word of bf16 at a time: word n of 32
// is word n % 8 of part n / 8; a full chunk is written, a part whose codes are all
// used is loaded again (of the page three ahead).
typedef const __attribute__((address_space(1))) char* global_bytes;
template <int kPart, class P>
__device__ __forceinline__ void load_part(VideoStream<P>& s, const PageCtx<P>& c) {
  // (global: a flat load would count among the LDS accesses too)
  const global_bytes base = (global_bytes)(kPart < 2 ? c.ldk : c.ldv);
  s.raw[kPart] = *(const __attribute__((address_space(1))) u32x4*)(base + s.load[kPart & 1]);
}
// (The swizzles of K: chunk c of row m at position c ^ swap_low_bits(m).  e4m3: a part
// goes as it is, [64 rows][8 chunks], rows as above, chunk c (dims 16 c ..) at position
// c ^ codes_swizzle(m).)
__device__ __forceinline__ uint32_t swap_low_bits(uint32_t x) { return (x & ~3u) | ((x & 1) << 1) | ((x >> 1) & 1); }
__device__ __forceinline__ uint32_t codes_swizzle(uint32_t m) {
  return 4 * ((m >> 1) & 1) + 2 * (((m >> 2) ^ (m >> 3)) & 1) + ((m >> 2) & 1);
}
template <int kPart, bool kAgain, class P>
__device__ __forceinline__ void stage_codes(VideoStream<P>& s, const PageCtx<P>& c) {
  *(__attribute__((address_space(3))) u32x4*)(c.wk ^ (64u * kPart)) = s.raw[kPart];
  if constexpr (kAgain) load_part<kPart>(s, c);
}
template <int kWord, class P>
__device__ __forceinline__ void convert_word(const VideoStream<P>& s, const PageCtx<P>& c, u32x4& chunk) {
  constexpr int part = kWord >> 3;
  uint32_t scale = part < 2 ? c.ks : c.vs;
  if constexpr (P::kQ8) scale &= 0xff800000u;
  uint32_t w = codes_to_bf16<P::kFmt, kWord & 1>(s.raw[part][(kWord & 7) >> 1], quant_scale<P::kFmt>(__uint_as_float(scale)));
  asm volatile("" : "+v"(w));
  chunk[kWord & 3] = w;
}
// int8: the same an instruction at a time, in the order
//   spread word w, high value of w - 1 | pack w - 1, low value of w | ...
// which leaves an instruction between a mixed fma and what reads it (else a wait state):
// piece 2 w of 66 is the first pair, piece 2 w + 1 the second.
struct WordPieces {
  uint32_t u;
  float lo, hi;
};
template <int kPiece, class P>
__device__ __forceinline__ void convert_piece(VideoStream<P>& s, const PageCtx<P>& c, WordPieces& x, u32x4& chunk) {
  constexpr int word = kPiece >> 1, part = word >> 3, part_before = (word - 1) >> 3;
  const QuantScale qk = quant_scale<P::kFmt>(__uint_as_float(c.ks)), qv = quant_scale<P::kFmt>(__uint_as_float(c.vs));
  if constexpr ((kPiece & 1) == 0) {
    if constexpr (word > 0) x.hi = spread_value<1>(x.u, part_before < 2 ? qk : qv);
    if constexpr (word < 32) x.u = spread_codes<word & 1>(s.raw[part][(word & 7) >> 1]);
  } else {
    const float lo = x.lo;
    if constexpr (word < 32) x.lo = spread_value<0>(x.u, part < 2 ? qk : qv);
    if constexpr (word > 0) {
      uint32_t w = pack_bf16(lo, x.hi);
      asm volatile("" : "+v"(w));
      chunk[(word - 1) & 3] = w;
      if constexpr ((word & 3) == 0) write_chunk<(word >> 2) - 1>(c, chunk);
    }
  }
}
// What follows pieces kFrom .. kTo - 1 in their slot: their values stay in it, a part
// whose codes are all spread is loaded again.
template <int kFrom, int kTo, class P>
__device__ __forceinline__ void end_pieces(VideoStream<P>& s, const PageCtx<P>& c, WordPieces& x) {
  static_for<kTo - kFrom>([&](auto n) __attribute__((always_inline)) {
    constexpr int piece = kFrom + decltype(n)::value, word = piece >> 1;
    if constexpr ((piece & 1) == 0) {
      if constexpr (word > 0 && piece + 1 == kTo) asm volatile("" : "+v"(x.hi));
      if constexpr (word < 32 && piece + 1 == kTo) asm volatile("" : "+v"(x.u));
      if constexpr (word < 32 && (word & 7) == 7) load_part<(word >> 3)>(s, c);
    } else {
      if constexpr (word < 32 && piece + 1 == kTo) asm volatile("" : "+v"(x.lo));
    }
  });
}
template <int kChunk, class P>
__device__ __forceinline__ void write_chunk(const PageCtx<P>& c, const u32x4& chunk) {
  constexpr int part = kChunk >> 1, h = kChunk & 1;
  const uint32_t at = part < 2 ? (c.wk ^ (16u * h) ^ (128u * (part & 1))) : (c.wv ^ (16u * h)) + 8192u * (part & 1);
  *(__attribute__((address_space(3))) u32x4*)at = chunk;
}
template <int kWord, bool kAgain, class P>
__device__ __forceinline__ void stage_word(VideoStream<P>& s, const PageCtx<P>& c, u32x4& chunk) {
  convert_word<kWord>(s, c, chunk);
  if constexpr ((kWord & 3) == 3) write_chunk<(kWord >> 2)>(c, chunk);
  if constexpr (kAgain && (kWord & 7) == 7) load_part<(kWord >> 3)>(s, c);
}
template <bool kAgain, class P>
__device__ __forceinline__ void stage_page(VideoStream<P>& s, const PageCtx<P>& c) {
  u32x4 chunk;
  if constexpr (P::kQ8) {
    stage_codes<0, kAgain>(s, c);
    stage_codes<1, kAgain>(s, c);
  }
  static_for<P::kQ8 ? 16 : 32>([&](auto n) __attribute__((always_inline)) {
    stage_word<decltype(n)::value + (P::kQ8 ? 16 : 0), kAgain>(s, c, chunk);
  });
}
// Waits for the wave's LDS accesses, all or all but the operand reads that run ahead
// into the next page (three, e4m3 four).
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }
template <class P>
__device__ __forceinline__ void wait_lds_but_ahead() { __builtin_amdgcn_s_waitcnt(P::kQ8 ? 0xC47F : 0xC37F); }

// Waits for this wave's direct loads of every page but the one issued last
// (loads retire in order).  The barrier that follows then makes every wave's
// share visible.
__device__ __forceinline__ void wait_dma_all_but_last_page() {
  static_assert(kDmaPerPage == 8, "vmcnt encoding below");
  __builtin_amdgcn_s_waitcnt(0x0F78);  // vmcnt(8), expcnt(7), lgkmcnt(15)
}
__device__ __forceinline__ void wait_dma_all() { __builtin_amdgcn_s_waitcnt(0x0F70); }  // vmcnt(0)
// The page barrier alone: no wait for the LDS reads in flight, which belong
// to a page that stays.
__device__ __forceinline__ void page_barrier() {
  sched_fence();
  asm volatile("s_barrier" ::: "memory");
  sched_fence();
}

template <class T>
__device__ __forceinline__ void pin_s(T& x) { asm volatile("" : "+s"(x)); }
template <class T>
__device__ __forceinline__ void pin_v(T& x) { asm volatile("" : "+v"(x)); }

// The rest of a context: operand reads of the page in ring stage `stage`.
template <class P>
__device__ __forceinline__ void set_reads(const VideoStream<P>& s, uint32_t stage, PageCtx<P>& c) {
#pragma unroll
  for (int n = 0; n < 4; ++n) c.k[n] = (s.k_read + stage) ^ (64u * n);
  c.v = s.v_read + stage;
  c.vp = (s.v_read + ring_add(stage, kStages - 1)) ^ 64u;
}

// Starts the stream: key norms of its first window, the loads of its first
// three pages, and the context of its first page.  (Past a stream's end the
// last page is loaded once more, into a stage nothing reads.)
template <class P>
__device__ __forceinline__ void stream_start(const AttnArgs& a, VideoStream<P>& s) {
  stream_combine(s);
#pragma unroll
  for (int k = 0; k < 2; ++k) s.kn2[k] = a.knorm2[s.ent[k] >> 7];  // (past the end: the last unit's)
  if constexpr (P::k8) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if constexpr (P::kQ8) {
        s.vs[k] = scale_word(s, s.ent[k] >> 7);
      } else {
        s.ks[k] = __float_as_uint(s.kscale[s.ent[k] >> 7]);
        s.vs[k] = __float_as_uint(s.vscale[s.ent[k] >> 7]);
      }
    }
  }
  if (s.n == 0) return;
  s.valid = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t e = stream_peek(s, min(k, s.n - 1));
    s.valid |= (e & 127u) << (8 * k);
    set_load(s, e, k * kStageBytes, s.c);
    if constexpr (P::k8) {  // pages 0 and 1 to their stages, page 2 to the registers
      if constexpr (!P::kQ8) s.c.ks_load = peek_lanes(s.ks, min(k, s.n - 1));
      s.c.vs_load = peek_lanes(s.vs, min(k, s.n - 1));
      if (k < 3) {
        static_for<4>([&](auto i) __attribute__((always_inline)) { load_part<decltype(i)::value>(s, s.c); });
        if constexpr (P::kQ8) {
          s.c.k_exp = s.c.vs1;
          s.c.vs1 = s.c.vs;
        } else {
          s.c.ks = s.c.ks_load;
        }
        s.c.vs = s.c.vs_load;
        s.c.wk = s.wk + k * kStageBytes;
        s.c.wv = s.wv + k * kStageBytes;
        if (k < 2) stage_page<false>(s, s.c);
      }
    } else {
      if (k < 3) issue_page(s, s.c);
    }
  }
  set_reads(s, 0, s.c);
}

// e4m3 pages: S = K Q''^T is taken from the codes as they are, by
// v_mfma_scale_f32_16x16x128_f8f6f4 at twice the bf16 rate.  Q'' is split into two
// e4m3 terms of a row scale 2^f, q1 = e4m3(Q'' / 2^f) and q2 = e4m3((Q'' / 2^f - q1)
// 16): Q'' = (q1 + q2 / 16) 2^f to within 2^-8 of itself, as one more rounding to
// bf16 would be, or, where q2 is small, 2^-14 2^f (2^-21 of the row's largest).  The
// products' scale operands carry the page's K scale and the row's 2^f and 2^(f - 4), so
// S comes out as before.  (The 128 products of an instruction
// are added with about 17 bits below the largest: measured against 64 bits, 3e-5 of
// the sum of magnitudes at most on random codes of the whole range, exact on codes
// within 2^3 of each other.)  A page of 64 rows then takes 104 MFMAs of the same total
// length instead of 136, 24 operand reads instead of 32, and no conversion of K: 361
// instructions a page where one wave fills a SIMD (bf16 pages: 378), where converting K
// to bf16 as well took 445.
template <int kQT>
struct StateQ8 {
  i32x8 pair[2];     // operands in flight: K tiles ...
  u32x4 single[2];   // ... and, with the pairs' halves, V^T: slot = read % 6
  i32x8 q8[kQT][2];  // the row's two terms (accumulation registers)
  int q_exp[kQT];    // and their exponent bytes
};
// A wave's query rows: kQT subtiles of 16.
template <int kQT, class P>
struct VideoState : std::conditional_t<P::kQ8, StateQ8<kQT>, Nothing<4>> {
  f32x4 o[8][kQT];    // O^T[16 dt + 4 g + r][q]  (accumulation registers)
  f32x4 l[kQT];       // row sums, the same in every register and lane group
  f32x4 s_init[kQT];  // -m in every register: the S tiles start at the exp2 argument
  float m[kQT];       // softmax shift of row q
  bf16x8 q[kQT][4];   // Q''[q][32 s + 8 g .. + 8]
  // across pages
  f32x4 s3[kQT];      // S tile 3 of the previous page
  u32x4 p1[kQT];      // P words of its chunk 1 (tile 2's done)
  bf16x8 ring[4];     // operands in flight (slot = step % 4)
  // rows under a running maximum
  bool any_lazy;      // some row of the wave is one
  int t_row;          // (windows) timeline index of the lane's row of subtile 0
  bool any_unset;     // (windows) some such row has met no key it sees: m = kUnset
  uint32_t raised;    // subtiles whose O and l wait to be scaled (bit j) ...
  float scale[kQT];   // ... by this, row q
  u32x4 ones;         // bf16 ones (an opaque value: not rematerialised in front of an MFMA)
};
// The running maximum of a row that has met no key it sees; its S tiles start at 0.
constexpr float kUnset = 3.0e38f;
// Operand reads are issued this many steps ahead.  (Six, through eight
// registers, gives the narrower waves nothing: they are not latency-bound.)
constexpr int kRingAhead = 3;

// The queries live in accumulation registers (an MFMA reads its operands from
// either bank), which leaves the vector registers to the softmax.
template <int kQT, class P>
__device__ __forceinline__ void pin_queries(VideoState<kQT, P>& st) {
  if constexpr (P::kQ8) {
#pragma unroll
    for (int j = 0; j < kQT; ++j)
#pragma unroll
      for (int t = 0; t < 2; ++t) asm volatile("" : "+a"(st.q8[j][t]));
    return;
  }
#pragma unroll
  for (int j = 0; j < kQT; ++j)
#pragma unroll
    for (int t = 0; t < 4; ++t) asm volatile("" : "+a"(st.q[j][t]));
}

// Two adjacent exponentials to one word of P.
// The pins here and at the exponentials and S tiles keep them where they are
// scheduled: the compiler would sink them past the branches of a page tail.
__device__ __forceinline__ void put_word(u32x4& p, int word, float lo, float hi) {
  uint32_t w = pack_bf16(lo, hi);
  pin_v(w);
  p[word] = w;
}

// O and l of the rows raised at the last check, scaled to their new m.  No MFMA
// on them may be under way (the page loop: the last one was issued eight steps
// before).
template <int kQT, class P>
__device__ __forceinline__ void scale_raised(VideoState<kQT, P>& st) {
  if (st.raised == 0) return;
  sched_fence();
#pragma unroll
  for (int j = 0; j < kQT; ++j) {
    if (st.raised >> j & 1) {
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) scale_acc(st.o[dt][j], st.scale[j]);
      scale_acc(st.l[j], st.scale[j]);
    }
  }
  st.raised = 0;
  asm volatile("s_nop 7" ::: "memory");
  sched_fence();
}

// One page, software-pipelined across pages so that the softmax work is
// spread over the MFMA steps.  Iteration p (page p from the current stage,
// V^T of page p - 1 from the one before it): 32 steps of one LDS operand read
// (kRingAhead steps ahead, through a ring of four registers that runs on
// across the page barrier) and kQT MFMAs, one per subtile:
//   steps  0- 7  S tiles 0 and 1 of p       exponentials of tile 3 of p - 1
//   steps  8-15  P*V of p - 1, chunk 1      tile 0 of p (from step 10)
//   steps 16-23  S tiles 2 and 3 of p       tile 1 of p
//   steps 24-31  P*V of p, chunk 0          tile 2 of p (from step 26)
// The subtiles' exponentials run in streams of two subtiles, one exponential per
// stream and step (two in steps 10, 11, 26 and 27), each issued behind an MFMA
// of its own (an exponential takes 8 of the 16 cycles of an MFMA, a pack 4)
// and packed behind the next one, and each slot ends in a scheduling fence,
// so that the emitted order is the program order.  Every P word is complete
// before the P*V step that reads it.  Steps 0-7 also issue the direct loads
// of page p + 3 into the stage freed by page p - 2; at the end of the page
// each wave waits for its loads of page p + 2, so every load has two pages to
// land and the next page is complete a page before it is used.  One barrier
// per page.
// kFirst: a range's first page: no page p - 1.
//
// Rows under a running maximum (st.any_lazy; after the first page the kLazy
// form of the loop): the range's first 32 keys set a row's m to their maximum.
// From then on the largest S (a difference to m) of every chunk is taken in the
// steps that have no exponential (8 and 9, 24 and 25) and compared ahead of
// the chunk's exponentials; where it exceeds kRaiseAbove, the row takes it as
// its new m, and what O and l hold by then is scaled to it between the P*V of
// the chunk before and the chunk's own (after step 23, and after step 7 of the
// next page: their MFMAs are long done by then, and no P word is rounded
// twice).  Every choice is the row's own, so a row's result does not depend on
// the rows that share its wave, and a row under a fixed shift never exceeds it.
// A raised row's largest weight is exactly 1 instead of rounded like the others,
// which keeps the error of sharp attention down; a threshold of 4 gives more
// such rows and more raises (9% slower), one of 16 fewer (0.3% more error).
// Measured, 40 heads, 920 rows, 139 pages, us a step at query norm weights 1
// (no such row), 3, 4 and 7: 157, 190, 207, 223; without raises the loop takes
// 170.  (A shift fixed at 16 below the logit bound took 154 up to 4, but rounded
// the largest weight, and out of its reach, from 5 on, the range ran unpipelined
// under a running maximum: 344 to 455.)
//
// 8-bit pages: beside them the codes of page p + 2, in registers since the page before,
// are turned into its stage and those of page p + 3 requested.  int8: 128 instructions
// of conversion (WordPieces), in the slots without exponentials; they fill more than
// those have room for (517 instructions a page, 378 of bf16 pages), which costs the
// int8 kernel a fifth over bf16.  A word per step at its end took 5% longer.  e4m3: 16
// conversions of V^T in steps 8 and 9, the writes in the steps that read no operand.
// The operand reads that run ahead into the next page follow the last write, so a wait
// for all but those ends the page.
// Windows: what hides keys is a page's edge flag, the wave's own.  A row may meet
// its first visible key late: until then its m is unset and its S the bare logits.
template <int kQT, bool kFirst, bool kLazy, class P>
__device__ __forceinline__ void video_iter(VideoState<kQT, P>& st, VideoStream<P>& s) {
  const int n_valid = static_cast<int>(s.valid & 0xffu);
  const PageCtx<P> c = s.c;
  const bool tail = P::kWin ? n_valid != kPageTokens : n_valid < kPageTokens;
  PageCtx<P> nx;
  [[maybe_unused]] u32x4 chunk[P::kQ8 ? 4 : 1];
  [[maybe_unused]] WordPieces pieces;
  // (redefined every page, or the compiler widens them to pairs outside the loop and adds
  // the loads' scalar base to those)
  if constexpr (P::k8) asm volatile("" : "+v"(s.load[0]), "+v"(s.load[1]));
  pin_queries(st);
  pin_v(st.ones);
  page_barrier();
  // operand of step n
  auto oread = [&](auto nc) __attribute__((always_inline)) {
    constexpr int n = decltype(nc)::value;
    if constexpr (n >= 32) return lds_read16(nx.k[n - 32]);
    else if constexpr (n < 8) return lds_read16(c.k[n & 3] + 4096u * (n >> 2));
    else if constexpr (n < 16) return lds_read16(c.vp + 2048u * (n - 8));
    else if constexpr (n < 24) return lds_read16(c.k[n & 3] + 4096u * (2 + ((n - 16) >> 2)));
    else return lds_read16(c.v + 2048u * (n - 24));
  };
  // e4m3: read n of a page's 24 (K tiles 0 and 1 two each, V^T chunk 1 of the page
  // before eight, K tiles 2 and 3, V^T chunk 0; 24 to 27 are the next page's first), into
  // slot n % 6.  Steps 4-15 issue reads 4-15, steps 20-31 reads 16-27, each three steps or
  // more ahead of its use and behind the last use of the slot's former one; the steps
  // between them issue the writes.
  [[maybe_unused]] auto q8_read = [&](auto nc) __attribute__((always_inline)) {
    constexpr int n = decltype(nc)::value, slot = n % 6;
    if constexpr (P::kQ8) {
      uint32_t at;
      if constexpr (n >= 24) at = nx.k[n & 1] + 2048u * ((n - 24) >> 1);
      else if constexpr (n >= 16) at = c.v + 2048u * (n - 16);
      else if constexpr (n >= 12) at = c.k[n & 1] + 2048u * (2 + ((n - 12) >> 1));
      else if constexpr (n >= 4) at = c.vp + 2048u * (n - 4);
      else at = c.k[n & 1] + 2048u * (n >> 1);
      const u32x4 w = *(const __attribute__((address_space(3))) u32x4*)at;
      if constexpr (slot < 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) st.pair[slot >> 1][4 * (slot & 1) + i] = static_cast<int>(w[i]);
      } else {
        st.single[slot - 4] = w;
      }
    }
  };
  [[maybe_unused]] auto q8_operand = [&](auto nc) __attribute__((always_inline)) {
    constexpr int slot = decltype(nc)::value % 6;
    u32x4 w = {0u, 0u, 0u, 0u};
    if constexpr (P::kQ8) {
      if constexpr (slot < 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = static_cast<uint32_t>(st.pair[slot >> 1][4 * (slot & 1) + i]);
      } else {
        w = st.single[slot - 4];
      }
    }
    return as_bf16x8(w);
  };
  // operand of a P*V step
  auto pv_operand = [&](auto oc) __attribute__((always_inline)) {
    constexpr int o = decltype(oc)::value;
    if constexpr (P::kQ8) return q8_operand(Const<(o < 16 ? o - 4 : o - 8)>{});
    else return st.ring[o & 3];
  };
  if constexpr (kFirst) {
    if constexpr (P::kQ8) {
      static_for<4>(q8_read);
    } else {
      static_for<kRingAhead>([&](auto n) __attribute__((always_inline)) { st.ring[decltype(n)::value] = oread(n); });
    }
  }
  f32x4 sa[4][kQT];
  u32x4 p0[kQT], p1n[kQT];
  float cm[kQT], top;  // largest S of the lane's keys of a chunk, and of all subtiles
  // exponential x of a stream: tile x / 8, subtile (x / 4) % 2, register x % 4
  // (the last stream of an odd kQT has one subtile)
  constexpr int kStreams = (kQT + 1) / 2;
  float e[kStreams][32];

  auto exp_x = [&](auto kc_, auto xc) __attribute__((always_inline)) {
    constexpr int k = decltype(kc_)::value, x = decltype(xc)::value;
    constexpr int t = x >> 3, j = 2 * k + ((x >> 2) & 1), r = x & 3;
    if constexpr (j >= kQT) {
    } else if constexpr (t == 3) {
      if constexpr (!kFirst) { e[k][x] = fast_exp2(st.s3[j][r]); pin_v(e[k][x]); }
    } else {
      e[k][x] = fast_exp2(sa[t][j][r]);
      pin_v(e[k][x]);
    }
  };
  auto pack_x = [&](auto kc_, auto xc) __attribute__((always_inline)) {  // words of exponentials x, x + 1 (x even)
    constexpr int k = decltype(kc_)::value, x = decltype(xc)::value;
    constexpr int t = x >> 3, j = 2 * k + ((x >> 2) & 1), word = 2 * (t & 1) + ((x & 3) >> 1);
    if constexpr (j >= kQT) {
    } else if constexpr (t == 3) {
      if constexpr (!kFirst) put_word(st.p1[j], word, e[k][x], e[k][x + 1]);
    } else if constexpr (t == 2) {
      put_word(p1n[j], word, e[k][x], e[k][x + 1]);
    } else {
      put_word(p0[j], word, e[k][x], e[k][x + 1]);
    }
  };
  // the largest S of chunk a (tiles a, a + 1) in this lane
  auto take_max = [&](auto jc, auto ac) __attribute__((always_inline)) {
    constexpr int j = decltype(jc)::value, a = decltype(ac)::value;
    const f32x4 &x = sa[a][j], &y = sa[a + 1][j];
    cm[j] = fmaxf(fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), fmaxf(fmaxf(x[3], y[0]), y[1])), fmaxf(y[2], y[3]));
    pin_v(cm[j]);
  };
  auto take_top = [&](auto jc) __attribute__((always_inline)) {
    constexpr int j = decltype(jc)::value;
    top = j == 0 ? cm[0] : fmaxf(top, cm[j]);
    pin_v(top);
  };
  auto take_all = [&](auto ac) __attribute__((always_inline)) {
    static_for<kQT>([&](auto jc) __attribute__((always_inline)) {
      take_max(jc, ac);
      take_top(jc);
    });
  };
  // New maxima for the rows of a chunk that exceed theirs by too much.
  auto raise = [&](auto ac) __attribute__((always_inline)) {
    constexpr int a = decltype(ac)::value;
    st.raised = 0;
    if constexpr (P::kWin) {
      bool unset = false;
#pragma unroll
      for (int j = 0; j < kQT; ++j) {
        const float row = pair_max<32>(pair_max<16>(cm[j]));
        const bool first = st.m[j] == kUnset && row > -kUnset;  // (O and l are 0)
        const bool up_row = first || (st.m[j] != kUnset && row > kRaiseAbove);
        if (__any(up_row)) {
          const float up = up_row ? row : 0.f;
          st.raised |= 1u << j;
          st.scale[j] = first ? 1.f : fast_exp2(-up);
          st.m[j] = first ? row : st.m[j] == kUnset ? kUnset : st.m[j] + up;
          const float neg = st.m[j] == kUnset ? 0.f : -st.m[j];
          st.s_init[j] = (f32x4){neg, neg, neg, neg};
          sa[a][j] -= up;
          sa[a + 1][j] -= up;
        }
        unset = unset || st.m[j] == kUnset;
      }
      st.any_unset = __any(unset);
      return;
    }
#pragma unroll
    for (int j = 0; j < kQT; ++j) {
      const float row = pair_max<32>(pair_max<16>(cm[j]));
      if (__any(row > kRaiseAbove)) {
        const float up = row > kRaiseAbove ? row : 0.f;  // (0: nothing of the row changes)
        st.raised |= 1u << j;
        st.scale[j] = fast_exp2(-up);
        st.m[j] += up;
        const float neg = -st.m[j];
        st.s_init[j] = (f32x4){neg, neg, neg, neg};
        sa[a][j] -= up;
        sa[a + 1][j] -= up;
      }
    }
  };
  // a page tail's work on the chunk of tiles a and a + 1, and its maxima
  auto check_chunk = [&](auto ac) __attribute__((always_inline)) {
    constexpr int a = decltype(ac)::value;
    if (tail) {
      // logits of slots at or past n_valid become -inf, so they weigh exactly
      // 0 (a correction subtracted from the row sum afterwards would cancel
      // for rows whose logits all sit far below the shift)
      const int off = 8 * (opaque(s.lane) >> 4);
      [[maybe_unused]] int lim = n_valid - off;
      if constexpr (P::kWin) {
        // row by row: keys at or past hi, and from the sinks' end up to lo, are hidden
        const int start = peek_lanes(s.start, s.at), valid = min(n_valid, kPageTokens);
        const int edge = __builtin_amdgcn_readfirstlane(page_edge(s, start, valid));
        const int at = start + off;
        lim = valid - off;
        auto hide = [&](auto&& hidden) __attribute__((always_inline)) {
#pragma unroll
          for (int j = 0; j < kQT; ++j) {
            const RowRange rr = row_range(s.win, st.t_row + 16 * j);
#pragma unroll
            for (int t = a; t < a + 2; ++t)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                sa[t][j][r] = hidden(rr, 32 * (t >> 1) + 4 * (t & 1) + r) ? kNegInf : sa[t][j][r];
          }
        };
        if (edge & kEdgeHi)
          hide([&](const RowRange& rr, int slot) __attribute__((always_inline)) { return slot >= min(lim, rr.hi - at); });
        if (edge & kEdgeLo)
          hide([&](const RowRange& rr, int slot) __attribute__((always_inline)) { return slot < rr.lo - at; });
        if (edge & kEdgeSinks) {
          const int sk = s.win.sinks - at;
          hide([&](const RowRange& rr, int slot) __attribute__((always_inline)) { return slot >= sk && slot < rr.lo - at; });
        }
      } else {
#pragma unroll
        for (int t = a; t < a + 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < kQT; ++j)
              sa[t][j][r] = 32 * (t >> 1) + 4 * (t & 1) + r >= lim ? kNegInf : sa[t][j][r];
      }
      if constexpr (kLazy) take_all(ac);
    }
    if constexpr (kFirst) {
      if (st.any_lazy) {
        take_all(ac);
        if constexpr (P::kWin) {
          raise(ac);
        } else if constexpr (a == 0) {
#pragma unroll
          for (int j = 0; j < kQT; ++j) {
            // (a page's first chunk has a valid key; clamped all the same)
            const float row = fmaxf(pair_max<32>(pair_max<16>(cm[j])), -3.0e38f);
            const float up = st.m[j] < 0.f ? row : 0.f;  // (m < 0: not set yet)
            st.m[j] = st.m[j] < 0.f ? row : st.m[j];
            const float neg = -st.m[j];
            st.s_init[j] = (f32x4){neg, neg, neg, neg};
            sa[0][j] -= up;
            sa[1][j] -= up;
          }
        } else {
          raise(ac);
        }
      }
    } else if constexpr (kLazy) {
      bool look = __any(top > kRaiseAbove);
      if constexpr (P::kWin) look = look || st.any_unset;
      if (look) raise(ac);
    }
    sched_fence();
  };

  // the next page's context, one small piece per step
  int look = 0;
  uint32_t ent = 0, st_next = 0;
  // (at: the steps that take the pieces, by path.  8-bit paths keep them out of the
  // steps that conversions and 8-bit products fill; steps 32 + o are int8's second
  // place in step o)
  auto next_ctx = [&](auto oc) __attribute__((always_inline)) {
    constexpr int o = decltype(oc)::value;
    constexpr auto at = [](int plain, int e4m3, int int8) { return o == (P::kPieces ? int8 : P::kQ8 ? e4m3 : plain); };
    if constexpr (at(12, 12, 10)) { look = min(s.at + 4, s.n - 1); pin_s(look); }
    if constexpr (at(13, 13, 11)) { ent = __builtin_amdgcn_readlane(s.ent[0], look & 63); pin_s(ent); }
    if constexpr (at(14, 14, 32 + 26)) {
      const uint32_t e1 = __builtin_amdgcn_readlane(s.ent[1], look & 63);
      ent = (look & 64) ? e1 : ent;
      pin_s(ent);
    }
    if constexpr (at(15, 15, 26)) { st_next = ring_add(s.stage, 1); pin_s(st_next); }
    constexpr uint32_t tile_shift = P::k8 ? kCodeTileShift : 14;
    if constexpr (at(16, 30, 32 + 31)) {
      nx.ldk = reinterpret_cast<const uint16_t*>(reinterpret_cast<uint64_t>(s.kpool) + (static_cast<uint64_t>(ent >> 7) << tile_shift));
      pin_s(nx.ldk);
    }
    if constexpr (at(17, 31, 31)) {
      nx.ldv = reinterpret_cast<const uint16_t*>(reinterpret_cast<uint64_t>(s.vpool) + (static_cast<uint64_t>(ent >> 7) << tile_shift));
      pin_s(nx.ldv);
    }
    if constexpr (P::k8) {
      if constexpr (at(-1, 15, 26)) {
        if constexpr (P::kQ8) {
          nx.k_exp = c.vs1;
          nx.vs1 = c.vs;
        } else {
          nx.ks = c.ks_load;
        }
        nx.vs = c.vs_load;
      }
      if constexpr (at(-1, -1, 32 + 28)) { nx.ks_load = __builtin_amdgcn_readlane(s.ks[0], look & 63); pin_s(nx.ks_load); }
      if constexpr (at(-1, -1, 28)) {
        const uint32_t w1 = __builtin_amdgcn_readlane(s.ks[1], look & 63);
        nx.ks_load = (look & 64) ? w1 : nx.ks_load;
        pin_s(nx.ks_load);
      }
      if constexpr (at(-1, 28, 32 + 29)) { nx.vs_load = __builtin_amdgcn_readlane(s.vs[0], look & 63); pin_s(nx.vs_load); }
      if constexpr (at(-1, 29, 29)) {
        const uint32_t w1 = __builtin_amdgcn_readlane(s.vs[1], look & 63);
        nx.vs_load = (look & 64) ? w1 : nx.vs_load;
        pin_s(nx.vs_load);
      }
      if constexpr (at(-1, 24, 30)) { nx.wk = s.wk + ring_add(st_next, 2); pin_v(nx.wk); }
      if constexpr (at(-1, 25, 30)) { nx.wv = s.wv + ring_add(st_next, 2); pin_v(nx.wv); }
    } else {
      if constexpr (o == 18) { nx.lds = s.lds0 + ring_add(st_next, 3); pin_s(nx.lds); }
    }
    if constexpr (at(19, 24, 27)) { nx.k[0] = s.k_read + st_next; pin_v(nx.k[0]); }
    if constexpr (at(20, 25, 32 + 28)) { nx.k[1] = nx.k[0] ^ 64u; pin_v(nx.k[1]); }
    if constexpr (at(21, -1, 32 + 30)) { nx.k[2] = nx.k[0] ^ 128u; pin_v(nx.k[2]); }
    if constexpr (at(22, -1, 32 + 30)) { nx.k[3] = nx.k[0] ^ 192u; pin_v(nx.k[3]); }
    if constexpr (at(23, 30, 31)) { nx.v = s.v_read + st_next; pin_v(nx.v); }
    if constexpr (at(24, 14, 14)) { nx.vp = c.v ^ 64u; pin_v(nx.vp); }
    if constexpr (at(28, 31, 31)) { s.valid = __builtin_amdgcn_readfirstlane((s.valid >> 8) | ((ent & 127u) << 24)); }
  };
  static_for<32>([&](auto oc) __attribute__((always_inline)) {
    constexpr int o = decltype(oc)::value;
    static_for<kQT>([&](auto jc) __attribute__((always_inline)) {
      constexpr int j = decltype(jc)::value, k = j >> 1;
      constexpr bool even = (j & 1) == 0, last = j == kQT - 1;
      [[maybe_unused]] constexpr int last_odd = kQT == 4 ? 3 : kQT - 1;
      // ---- the MFMA ----
      constexpr bool s_step = o < 8 || (o >= 16 && o < 24);
      if constexpr (s_step) {
        constexpr int t = (o < 8 ? 0 : 2) + ((o & 7) >> 2);
        if constexpr (P::kQ8) {
          // a tile's 2 kQT products, each as long as two of the slots
          constexpr int slot = (o & 3) * kQT + j, jj = slot / 2 % kQT, term = slot / 2 / kQT;
          if constexpr (slot % 2 == 0) {
            mfma_s8<term>(sa[t][jj], st.pair[t & 1], st.q8[jj][term], term == 0 ? st.s_init[jj] : sa[t][jj],
                          static_cast<int>(c.k_exp), st.q_exp[jj]);
            if constexpr (term == 1) pin_v(sa[t][jj]);
          }
        } else {
          const bf16x8 a = st.ring[o & 3];
          if constexpr ((o & 3) == 0) mfma_s(sa[t][j], a, st.q[j][0], st.s_init[j]);
          else mfma_s(sa[t][j], a, st.q[j][o & 3], sa[t][j]);
          pin_v(sa[t][j]);
        }
      } else if constexpr (o < 16) {
        const bf16x8 a = pv_operand(oc);
        if constexpr (!kFirst) {
          mfma_o(st.o[o - 8][j], a, as_bf16x8(st.p1[j]));
          if constexpr (o == 15) mfma_o(st.l[j], as_bf16x8(st.ones), as_bf16x8(st.p1[j]));
        }
      } else {
        const bf16x8 a = pv_operand(oc);
        if constexpr (kFirst) mfma_o_first(st.o[o - 24][j], a, as_bf16x8(p0[j]));
        else mfma_o(st.o[o - 24][j], a, as_bf16x8(p0[j]));
        if constexpr (o == 31) {
          if constexpr (kFirst) mfma_o_first(st.l[j], as_bf16x8(st.ones), as_bf16x8(p0[j]));
          else mfma_o(st.l[j], as_bf16x8(st.ones), as_bf16x8(p0[j]));
        }
      }
      sched_fence();
      // ---- this slot's share of the rest ----
      if constexpr (kLazy && (o == 8 || o == 24)) take_max(jc, Const<o == 8 ? 0 : 2>{});
      if constexpr (kLazy && (o == 9 || o == 25)) take_top(jc);
      if constexpr (P::kQ8) {
        constexpr int n = (o & 15) < 4 ? -1 : o < 16 ? o : o - 4;
        if constexpr (j == 1 && n >= 0 && !(kFirst && n < 12)) q8_read(Const<(n < 0 ? 0 : n)>{});
      } else if constexpr (j == 1) {
        constexpr int n = o + kRingAhead;
        if constexpr (!(kFirst && n >= 8 && n < 16)) st.ring[n & 3] = oread(Const<n>{});
      }
      if constexpr (P::kQ8 && (o == 8 || o == 9)) {
        // V's conversions, where there are no exponentials
        constexpr int slot = (o - 8) * kQT + j, w0 = 8 * slot / kQT, w1 = 8 * (slot + 1) / kQT;
        static_for<w1 - w0>([&](auto n) __attribute__((always_inline)) {
          constexpr int word = 16 + w0 + decltype(n)::value;
          convert_word<word>(s, c, chunk[(word - 16) >> 2]);
          if constexpr ((word & 7) == 7) load_part<(word >> 3)>(s, c);
        });
      }
      // int8: 66 pieces, one in each odd slot of a step with exponentials in the even ones,
      // six and seven in the steps without any
      constexpr bool many = o == 8 || o == 9 || o == 24 || o == 25, one = o < 8 || (o >= 12 && o < 24);
      constexpr int first = o < 8 ? 2 * o : o < 10 ? 16 + 6 * (o - 8) : o < 24 ? 28 + 2 * (o - 12) : 52 + 7 * (o - 24);
      constexpr int n_step = o < 10 ? 6 : 7;
      constexpr int piece0 = first + (many ? n_step * j / kQT : one ? (j == 0 ? 0 : j == 1 ? 0 : j == last_odd ? 1 : 2) : 0);
      constexpr int piece1 = first + (many ? n_step * (j + 1) / kQT : one ? (j == 0 ? 0 : j == last_odd ? 2 : j == 1 ? 1 : 2) : 0);
      if constexpr (P::kPieces)
        static_for<piece1 - piece0>([&](auto n) __attribute__((always_inline)) {
          convert_piece<piece0 + decltype(n)::value>(s, c, pieces, chunk[0]);
        });
      if constexpr (even) {
        if constexpr (o < 8) exp_x(Const<k>{}, Const<24 + o>{});
        else if constexpr (o == 10) exp_x(Const<k>{}, Const<0>{});
        else if constexpr (o == 11) exp_x(Const<k>{}, Const<2>{});
        else if constexpr (o >= 12 && o < 24) exp_x(Const<k>{}, Const<o - 8>{});
        else if constexpr (o == 26) exp_x(Const<k>{}, Const<16>{});
        else if constexpr (o == 27) exp_x(Const<k>{}, Const<18>{});
        else if constexpr (o >= 28) exp_x(Const<k>{}, Const<o - 8>{});
      }
      if constexpr (!even || last) {
        if constexpr (o < 8 && (o & 1)) pack_x(Const<k>{}, Const<24 + o - 1>{});
        else if constexpr (o == 10) exp_x(Const<k>{}, Const<1>{});
        else if constexpr (o == 11) { exp_x(Const<k>{}, Const<3>{}); pack_x(Const<k>{}, Const<0>{}); }
        else if constexpr (o == 12) pack_x(Const<k>{}, Const<2>{});
        else if constexpr (o > 12 && o < 24 && (o & 1)) pack_x(Const<k>{}, Const<o - 9>{});
        else if constexpr (o == 26) exp_x(Const<k>{}, Const<17>{});
        else if constexpr (o == 27) { exp_x(Const<k>{}, Const<19>{}); pack_x(Const<k>{}, Const<16>{}); }
        else if constexpr (o == 28) pack_x(Const<k>{}, Const<18>{});
        else if constexpr (o > 28 && (o & 1)) pack_x(Const<k>{}, Const<o - 9>{});
      }
      if constexpr (P::kPieces && j == 1) next_ctx(Const<32 + o>{});  // (before the last slot's)
      if constexpr (last) {
        if constexpr (P::kQ8) {
          // the LDS writes: in steps that read no operand
          if constexpr (o == 0 || o == 2) stage_codes<o / 2, true>(s, c);
          if constexpr (o >= 16 && o < 20) write_chunk<o - 12>(c, chunk[o - 16]);
        } else if constexpr (!P::k8 && o < kDmaPerPage) {
          issue_load<o>(s, c);
        }
        next_ctx(oc);
        if constexpr (o == 14 || o == 30) pin_v(st.ones);
      }
      if constexpr (P::kPieces) end_pieces<piece0, piece1>(s, c, pieces);
      sched_fence();
    });
    if constexpr (o == 9) check_chunk(Const<0>{});
    if constexpr (o == 25) check_chunk(Const<2>{});
    if constexpr (kLazy && (o == 7 || o == 23)) scale_raised(st);
  });
#pragma unroll
  for (int j = 0; j < kQT; ++j) {
    st.s3[j] = sa[3][j];
    st.p1[j] = p1n[j];
  }
  // After a range's first page everything is waited for: a load the compiler
  // knows of and believes in flight on entry to the page loop would be waited
  // for in every iteration, with all the direct loads behind it.
  if constexpr (P::k8) wait_lds_but_ahead<P>();
  else if constexpr (kFirst) wait_dma_all();
  else wait_dma_all_but_last_page();
  s.c = nx;
  s.at += 1;
  s.stage = st_next;
  stream_reach(s);
}

// Finishes the last page of a range (its stage is the one before the
// stream's current): tile 3's exponentials, then the P*V of chunk 1.
template <int kQT, class P>
__device__ __forceinline__ void video_flush(VideoState<kQT, P>& st, const VideoStream<P>& s) {
  const uint32_t v1 = s.c.vp;
  mfma_drain();
#pragma unroll
  for (int j = 0; j < kQT; ++j)
#pragma unroll
    for (int r = 0; r < 4; r += 2)
      put_word(st.p1[j], 2 + (r >> 1), fast_exp2(st.s3[j][r]), fast_exp2(st.s3[j][r + 1]));
  bf16x8 v[8];
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) v[dt] = lds_read16(v1 + 2048u * dt);
  pin_v(st.ones);
  mfma_drain();
#pragma unroll
  for (int j = 0; j < kQT; ++j) mfma_o(st.l[j], as_bf16x8(st.ones), as_bf16x8(st.p1[j]));
#pragma unroll
  for (int dt = 0; dt < 8; ++dt)
#pragma unroll
    for (int j = 0; j < kQT; ++j) mfma_o(st.o[dt][j], v[dt], as_bf16x8(st.p1[j]));
  mfma_drain();
}

// One segment of a video workgroup's stream: the query tile of rows
// [q_lo, min(q_lo + 256, q_hi)) of head `head` against n pages of the stream,
// which are key range `seg` of the ranges that split this head's pages
// (`whole`: the only one; q_hi ends the tile's query class).  With one range
// the output is written in bf16; otherwise the softmax-normalised partial and
// its log-sum-exp go to the split-KV workspace for the combine kernel.
struct VideoSeg {
  int head, n, seg, q_lo, q_hi;
  bool whole;
};

// How a kernel's queries come: to be normed or scaled, prepared, or as the call says.
constexpr int kQueriesRaw = 0, kQueriesPrepared = 1, kQueriesAny = 2;
// First of the 8 dims that word group s of lane group g holds: 32 s + 8 g .., or, against
// e4m3 codes, s of the 16-dim chunks g and g + 4 (two groups each).
template <class P>
__device__ __forceinline__ int query_dim(int s, int g) {
  return P::kQ8 ? 64 * (s >> 1) + 8 * (s & 1) + 16 * g : 32 * s + 8 * g;
}
// A wave's query rows as the call gives them: raw[j][s] = Q[row j][query_dim(s, g) .. + 8].
template <int kQT>
struct RawQueries {
  u32x4 raw[kQT][4];
  bool rider[kQT];  // rider rows (at and past rq_row0): prepared rows of their own
  bool ok[kQT];
  int3 pos[kQT];
};
template <int kQT, int kQueries, class P>
__device__ __forceinline__ void fetch_queries(const AttnArgs& a, const VideoSeg& sg, int wrow, int lane,
                                              RawQueries<kQT>& x) {
  const int lane_o = opaque(lane), g = lane_o >> 4, i16 = lane_o & 15;
  // row j's pointer is the first row's plus 16 j token strides (uniform);
  // rows past the end read the zero block (zeros cost the matrix pipe little)
  const uint16_t* qp = a.q + sg.head * a.q_head_stride + (wrow + i16) * a.q_tok_stride + query_dim<P>(0, g);
#pragma unroll
  for (int j = 0; j < kQT; ++j) {
    const int row = wrow + 16 * j + i16;
    x.ok[j] = row < sg.q_hi;
    x.rider[j] = false;
    const uint16_t* p = x.ok[j] ? qp + 16 * j * a.q_tok_stride : a.zeros + query_dim<P>(0, g);
#pragma unroll
    for (int s = 0; s < 4; ++s) x.raw[j][s] = *reinterpret_cast<const u32x4*>(p + query_dim<P>(s, 0));
    x.pos[j] = make_int3(0, 0, 0);
    if (kQueries != kQueriesPrepared && a.mode == 1 && x.ok[j])
      x.pos[j] = make_int3(a.positions[3 * row], a.positions[3 * row + 1], a.positions[3 * row + 2]);
  }
  if (P::kPlain && a.n_rq > 0 && wrow + 16 * kQT > a.rq_row0) {  // rider rows among them
#pragma unroll
    for (int j = 0; j < kQT; ++j) {
      const int q = wrow + 16 * j + i16 - a.rq_row0;
      if (q >= 0 && q < a.n_rq) {
        const uint16_t* p = a.rq + q * a.rq_tok_stride + sg.head * a.rq_head_stride + 8 * g;
#pragma unroll
        for (int s = 0; s < 4; ++s) x.raw[j][s] = *reinterpret_cast<const u32x4*>(p + 32 * s);
        x.rider[j] = true;
      }
    }
  }
}

// The prepared queries, st.q[j][s] = Q''[row j][32 s + 8 g .. + 8], by the
// call's query mode (2: given as they are, else 0 or 1); rider rows
// (at and past rq_row0) come prepared.
template <int kQT, int kQueries, class P>
__device__ __forceinline__ void prepare_rows(const AttnArgs& a, const RawQueries<kQT>& x, int g, VideoState<kQT, P>& st) {
  if (kQueries == kQueriesPrepared || (kQueries == kQueriesAny && a.mode == 2)) {
#pragma unroll
    for (int j = 0; j < kQT; ++j)
#pragma unroll
      for (int s = 0; s < 4; ++s) st.q[j][s] = as_bf16x8(x.raw[j][s]);
    return;
  }
  if (a.mode == 0) {
#pragma unroll
    for (int j = 0; j < kQT; ++j) {
      const float sc = x.rider[j] ? 1.0f : a.scale_log2;  // riders: x 1 is exact
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16(bf16_lo(x.raw[j][s][i]) * sc, bf16_hi(x.raw[j][s][i]) * sc);
        st.q[j][s] = as_bf16x8(w);
      }
    }
    return;
  }
  // Norm and rotation.  The lane's 16 pairs are 16 s + 4 g + i; a pair's band
  // is a select on its index (no branch), the table rows' offsets are per row.
  const int p0 = a.rope.pairs[0], p01 = p0 + a.rope.pairs[1];
  float inv[kQT];
  const float2* row[kQT][3];
#pragma unroll
  for (int j = 0; j < kQT; ++j) {
    int pt = 0, ph = 0, pw = 0;
    if (x.ok[j] && !x.rider[j]) clamp_pos(a.rope, x.pos[j].x, x.pos[j].y, x.pos[j].z, a.flags, pt, ph, pw);
    row[j][0] = a.rope.tab[0] + static_cast<int64_t>(pt) * a.rope.pairs[0];
    row[j][1] = a.rope.tab[1] + static_cast<int64_t>(ph) * a.rope.pairs[1] - p0;
    row[j][2] = a.rope.tab[2] + static_cast<int64_t>(pw) * a.rope.pairs[2] - p01;
    float ss = 0.f;
#pragma unroll
    for (int s = 0; s < 4; ++s) ss += norm2_fma(x.raw[j][s]);
    ss = pair_sum<32>(pair_sum<16>(ss));
    inv[j] = rsqrtf(ss * (1.0f / kHeadDim) + a.eps);
  }
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int d = query_dim<P>(s, g);
    const float4 g0 = *reinterpret_cast<const float4*>(a.gamma + d);
    const float4 g1 = *reinterpret_cast<const float4*>(a.gamma + d + 4);
    const float gam[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
    float2 cs[kQT][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = d / 2 + i;
#pragma unroll
      for (int j = 0; j < kQT; ++j) cs[j][i] = (p < p0 ? row[j][0] : p < p01 ? row[j][1] : row[j][2])[p];
    }
#pragma unroll
    for (int j = 0; j < kQT; ++j) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y0 = bf16_lo(x.raw[j][s][i]) * inv[j] * gam[2 * i];
        const float y1 = bf16_hi(x.raw[j][s][i]) * inv[j] * gam[2 * i + 1];
        w[i] = pack_bf16((y0 * cs[j][i].x - y1 * cs[j][i].y) * a.scale_log2,
                         (y0 * cs[j][i].y + y1 * cs[j][i].x) * a.scale_log2);
      }
      // riders come prepared; a row past the call's end stays all zeros (with
      // eps = 0 its norm gives 0 * inf)
      st.q[j][s] = as_bf16x8(x.ok[j] ? w : x.raw[j][s]);
    }
  }
}

// e4m3 pages: the rows' two terms and exponents (StateQ8) from their bf16 words.
template <int kQT, class P>
__device__ __forceinline__ void split_queries(VideoState<kQT, P>& st) {
#pragma unroll
  for (int j = 0; j < kQT; ++j) {
    float v[32], top = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t w = __builtin_bit_cast(u32x4, st.q[j][i >> 2])[i & 3];
      v[2 * i] = bf16_lo(w);
      v[2 * i + 1] = bf16_hi(w);
      top = fmaxf(top, fmaxf(fabsf(v[2 * i]), fabsf(v[2 * i + 1])));
    }
    const uint32_t t = __float_as_uint(pair_max<32>(pair_max<16>(top)));
    // the least f with top <= 448 2^f (448 = 0.875 2^9), for exponent bytes above 0
    const int f = max(static_cast<int>(t >> 23) - 135 + ((t & 0x7fffffu) > 0x600000u ? 1 : 0), -122);
    const float inv = __uint_as_float(static_cast<uint32_t>(127 - f) << 23);
    st.q_exp[j] = (f + 127) | ((f + 123) << 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = v[4 * i + k] * inv;
      int c1 = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
      c1 = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], c1, true);
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(c1, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c1, true);
      int c2 = __builtin_amdgcn_cvt_pk_fp8_f32((x[0] - lo[0]) * 16.f, (x[1] - lo[1]) * 16.f, 0, false);
      c2 = __builtin_amdgcn_cvt_pk_fp8_f32((x[2] - hi[0]) * 16.f, (x[3] - hi[1]) * 16.f, c2, true);
      st.q8[j][0][i] = c1;
      st.q8[j][1][i] = c2;
    }
  }
}

template <int kQT, int kQueries, class P>
__device__ __forceinline__ void video_segment(const AttnArgs& a, const VideoSeg& sg, VideoStream<P>& s, int wave) {
  const int wrow = sg.q_lo + wave * 16 * kQT;
  VideoState<kQT, P> st;
  {
    RawQueries<kQT> raw;
    fetch_queries<kQT, kQueries, P>(a, sg, wrow, s.lane, raw);
    prepare_rows<kQT, kQueries, P>(a, raw, s.lane >> 4, st);
  }

  // ---- softmax shift ----
  // Logits arrive in the log2 domain (the scale and log2(e) are folded into
  // Q'').  By Cauchy-Schwarz every logit of row q is at most
  // B_q = |Q''_q| * max |k| over the segment's pages (knorm2 holds the
  // squared norms of the stored keys).  Softmax is shift invariant, so B_q
  // serves as the exp2 shift as it stands: p = exp2(s - B_q) <= 1, with no
  // running maximum and no rescale of O.  The row's largest p is at least
  // 2^(-2 B_q), so for B_q <= kShiftBoundMax every weight above 2^-46 of the
  // row maximum stays a normal bf16/fp32 number.  Rows with a larger bound run
  // under a running maximum (video_iter).
  float kn2 = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int idx = 64 * k + s.lane;
    if (idx >= s.at && idx < s.at + sg.n) kn2 = fmaxf(kn2, s.kn2[k]);
  }
  for (int k = max(s.at, 128) + s.lane; k < s.at + sg.n; k += 64)
    kn2 = fmaxf(kn2, a.knorm2[stream_entry(s, k) >> 7]);
  kn2 = fminf(wave_max(kn2), 3.0e38f);  // (finite: a zero query's bound is 0)
  bool lazy = false;
#pragma unroll
  for (int j = 0; j < kQT; ++j) {
    float qn2 = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t) qn2 = norm2_words(__builtin_bit_cast(u32x4, st.q[j][t]), qn2);
    const float bound = sqrtf(pair_sum<32>(pair_sum<16>(qn2)) * kn2);
    const bool is = a.fixed_shift == 0 || bound > kShiftBoundMax;
    lazy = lazy || is;
    st.m[j] = is ? (P::kWin ? kUnset : -1.f) : bound;  // (-1: to be set by the first keys)
    const float neg = is ? 0.f : -bound;
    st.s_init[j] = (f32x4){neg, neg, neg, neg};
  }
  if constexpr (P::kQ8) split_queries(st);
  st.any_lazy = __any(lazy);
  if constexpr (P::kWin) {
    st.any_unset = st.any_lazy;
    st.t_row = a.win.t0 + wrow + (s.lane & 15);
  }
  st.raised = 0;
  pin_queries(st);
  st.ones = (u32x4){0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  asm volatile("" : "+v"(st.ones));

  // ---- the segment's pages ----
  if constexpr (P::k8) {
    if (s.at == 0) wait_lds();
  } else {
    if (s.at == 0) wait_dma_all_but_last_page();
  }
  const int end = s.at + sg.n;
  video_iter<kQT, true, false, P>(st, s);
  // (one-armed branches in turn: of an if-else the compiler keeps both arms'
  // accumulators.  In this order, and with the last scaling in the second arm,
  // the first loop keeps its speed: 40 heads, 920 rows, 139 and 479 pages 132.5 and
  // 443.4 us a step; the other way round 133.8 and 448.0, with the scaling in the
  // flush as well; without the second loop 131.8 and 441.1.)
  if (!st.any_lazy)
    while (s.at < end) video_iter<kQT, false, false, P>(st, s);
  if (st.any_lazy) {
    while (s.at < end) video_iter<kQT, false, true, P>(st, s);
    mfma_drain();
    scale_raised(st);
  }
  video_flush<kQT>(st, s);
  if (!P::k8 && s.at == s.n) wait_dma_all();  // no direct load may still be writing this workgroup's LDS when it exits

  // ---- epilogue: lane holds O^T[16 dt + 4 g + r][q] ----
  const int lane_e = opaque(s.lane), ge = lane_e >> 4, ie = lane_e & 15;
  const bool riders = P::kPlain && a.n_rq > 0 && wrow + 16 * kQT > a.rq_row0;
  // bf16: the output itself, or the partial of a key range: the
  // softmax-normalised O (a convex combination of V rows, so bf16 keeps its
  // range; the merge adds at most one more bf16 rounding of the output's size)
  // and its fp32 log-sum-exp.
  const int64_t part_row = (static_cast<int64_t>(sg.seg) * a.num_heads + sg.head) * a.n_q;
  uint16_t* const base = sg.whole ? a.out + sg.head * a.out_head_stride
                                  : reinterpret_cast<uint16_t*>(a.part_o) + part_row * kHeadDim;
  const int64_t stride = sg.whole ? a.out_tok_stride : kHeadDim;
  if constexpr (P::kWin && !P::k8) {
    // a value that some row does not see may have reached it through a weight of 0
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < kQT; ++j)
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = max(top, __float_as_uint(st.o[dt][j][r]) << 1);
    if (__any(top >= 0xff000000u)) {
      const int first = s.at - sg.n;
      window_rows_plain(
          a, sg.head, wrow, min(16 * kQT, sg.q_hi - wrow), 0, sg.n, 1, lane_e,
          [&](int p) {
            const uint32_t x = s.lo + first + p;
            const int pi = stream_place(s, static_cast<int>(x - (sg.head - s.head0) * s.n_pages));
            return make_int2(s.pages[pi].x, s.pages[pi].y);
          },
          [&](int i, float m, float l, float o0, float o1) {
            const float inv = l > 0.f ? 1.0f / l : 0.f;
            *reinterpret_cast<uint32_t*>(base + (wrow + i) * stride + 2 * lane_e) = pack_bf16(o0 * inv, o1 * inv);
            if (!sg.whole && lane_e == 0) a.part_lse[part_row + wrow + i] = l > 0.f ? m + __log2f(l) : kNegInf;
          });
      return;
    }
  }
  uint16_t* const op = base + (wrow + ie) * stride + 16 * (ge & 1) + 8 * (ge >> 1);
#pragma unroll
  for (int j = 0; j < kQT; ++j) {
    const int row = wrow + 16 * j + ie;
    const float l = st.l[j][0];
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    const float lse = l > 0.f ? st.m[j] + __log2f(l) : kNegInf;
    if (riders) {  // always a partial, fp32, for the rider rows' own merge
      const int q = row - a.rq_row0;
      if (q >= 0 && q < a.n_rq) {
        const int64_t prow = (static_cast<int64_t>(sg.seg) * a.num_heads + sg.head) * a.n_rq + q;
        float* po = a.rpart_o + prow * kHeadDim + 4 * ge;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4*>(po + 16 * dt) = st.o[dt][j] * inv;
        if (ge == 0) a.rpart_lse[prow] = lse;
      }
    }
    // Lane groups trade halves of two neighbouring d tiles, so that each lane
    // writes 16 bytes: lane group g of (x[0], x[1]) -> groups (0, 2): d tile
    // dt, (1, 3): dt + 1.
    u32x4 w[4];
#pragma unroll
    for (int dt = 0; dt < 8; dt += 2) {
      uint32_t x[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 v = st.o[dt + h][j] * inv;
        x[h][0] = pack_bf16(v[0], v[1]);
        x[h][1] = pack_bf16(v[2], v[3]);
      }
      const auto w0 = __builtin_amdgcn_permlane16_swap(x[0][0], x[1][0], false, false);
      const auto w1 = __builtin_amdgcn_permlane16_swap(x[0][1], x[1][1], false, false);
      w[dt >> 1] = (u32x4){w0[0], w1[0], w0[1], w1[1]};
    }
    if (row < sg.q_hi) {
#pragma unroll
      for (int n = 0; n < 4; ++n) *reinterpret_cast<u32x4*>(op + 16 * j * stride + 32 * n) = w[n];
      if (!sg.whole && ge == 0) a.part_lse[part_row + row] = lse;
    }
  }
}

// The class table, read in place from the kernel arguments (the kernel's only
// argument is the AttnArgs; indexing the by-value argument at a run-time class
// would make the compiler copy it to private memory).
typedef const __attribute__((address_space(4))) AttnClass* const_class_table;
__device__ __forceinline__ const_class_table class_table() {
  const __attribute__((address_space(4))) char* seg =
      (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
  return (const_class_table)(seg + offsetof(AttnArgs, cls));
}
__device__ __forceinline__ ClassPages class_pages(int ci) {
  const __attribute__((address_space(4))) char* seg =
      (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
  const auto* p = (const __attribute__((address_space(4))) ClassPages*)(seg + offsetof(AttnArgs, cls_pages)) + ci;
  return ClassPages{p->head_pages, p->skip, p->count};
}
// ------------------------------------------------------------------------- //
// audio_attn: the few audio queries, memory-bound.  A workgroup of 4 waves
// takes one (head, 16-query tile, key range); wave w streams pages w, w + 4,
// ... of the range on its own (no LDS staging, no barriers), loading each
// page's valid K rows and V^T columns straight into registers in MFMA
// operand layout, and the four waves merge through LDS at the end.  Two
// workgroups fit a CU, so 8 independent waves per CU keep enough bytes in
// flight to stream the cache from HBM.  Each workgroup writes the partial of
// its key range; the combine kernel merges them.  Where a head is one range its
// workgroup writes the output itself, without the merge's launch (4 us): a CU
// takes 0.45 us per page, so that pays for up to 12 pages.  (On 8 waves
// instead of 4 the same 0.45 us: 8, 16 and 24 pages take 10.6, 13.4 and 17.2 us
// against 9.1, 12.7 and 16.5.)
//
// With lane l = 16 g + i (i = query column, g = lane group), per page:
//   S^T (16 keys x 16 queries) = K Q''^T  4 key tiles x 4 v_mfma_f32_16x16x32_bf16
//   O^T (16 d x 16 queries) += V^T P^T    8 d tiles x 2 key chunks, same MFMA
// Row m = 4 g' + r of key tile t holds key 32 (t/2) + 8 g' + 4 (t%2) + r, so
// that accumulator registers r of tiles 2c and 2c + 1 in lane group g are
// keys 32 c + 8 g + 0..7: exactly the B operand of the P*V MFMA of key chunk c.
// ------------------------------------------------------------------------- //
// Loads of one page's K operands, k[t][s] = K[key(t, i)][32 s + 8 g .. + 8],
// and V^T operands, v[dt][c] = V^T[16 dt + i][32 c + 8 g .. + 8].  Rows and
// columns past n_valid are read from the 1 KB zero block instead (a cache
// hit), so partly filled pages cost only their valid tokens in HBM traffic
// and no load is predicated.
__device__ __forceinline__ void audio_load_k(u32x4 (&k)[4][4], const uint16_t* kt, const uint16_t* zeros,
                                             int n_valid, int g, int i, int lane) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int key = audio_key(t, i);
    const uint16_t* src = key < n_valid ? kt + k_tile_index(key, 8 * g) : zeros + 8 * lane;
    const int step = key < n_valid ? k_tile_index(0, 32) : 0;  // next 32 d
#pragma unroll
    for (int s = 0; s < 4; ++s) k[t][s] = *reinterpret_cast<const u32x4*>(src + step * s);
  }
}
__device__ __forceinline__ void audio_load_v(u32x4 (&v)[8][2], const uint16_t* vt, const uint16_t* zeros,
                                             int n_valid, int g, int i, int lane) {
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const bool ok = 32 * c + 8 * g < n_valid;
    const uint16_t* src = ok ? vt + v_tile_index(32 * c + 8 * g, i) : zeros + 8 * lane;
    const int step = ok ? v_tile_index(0, 16) : 0;  // next 16 d
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) v[dt][c] = *reinterpret_cast<const u32x4*>(src + step * dt);
  }
}

// S^T of one page's four key tiles.
__device__ __forceinline__ void audio_scores(const u32x4 (&kreg)[4][4], const bf16x8 (&qreg)[4], f32x4 (&sacc)[4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    sacc[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 4; ++s)
      sacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kreg[t][s]), qreg[s], sacc[t], 0, 0, 0);
  }
}

// Softmax weights of one page (sacc, masked past n_valid here) as bf16 words
// pw (word c of chunk c: keys 32 c + 8 g + 0..7), with the running maximum,
// the row sum (over the same bf16 values the MFMAs consume) and O kept up to
// date.
__device__ __forceinline__ void audio_softmax(f32x4 (&sacc)[4], int n_valid, bool fixed_shift, int g, u32x4 (&pw)[2],
                                              f32x4 (&o)[8], float& m_run, float& l_run) {
  const bf16x2 ones = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
  if (n_valid < kPageTokens) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (audio_key(t, 4 * g + r) >= n_valid) sacc[t][r] = kNegInf;
  }
  float alpha = 1.f;
  if (!fixed_shift) {
    float mx = kNegInf;
#pragma unroll
    for (int t = 0; t < 4; ++t) mx = fmaxf(mx, fmaxf(fmaxf(sacc[t][0], sacc[t][1]), fmaxf(sacc[t][2], sacc[t][3])));
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float m_new = fmaxf(m_run, mx);
    alpha = m_new == kNegInf ? 1.f : fast_exp2(m_run - m_new);
    m_run = m_new;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) o[dt] *= alpha;
  }
  const float m_use = m_run == kNegInf ? 0.f : m_run;
  float psum = 0.f;
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4& sc = sacc[2 * c + h];
      const uint32_t w0 = pack_bf16(fast_exp2(sc[0] - m_use), fast_exp2(sc[1] - m_use));
      const uint32_t w1 = pack_bf16(fast_exp2(sc[2] - m_use), fast_exp2(sc[3] - m_use));
      pw[c][2 * h] = w0;
      pw[c][2 * h + 1] = w1;
      psum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w0), ones, psum, false);
      psum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w1), ones, psum, false);
    }
  l_run = l_run * alpha + psum;
}

__device__ __forceinline__ void audio_pv(const u32x4 (&vreg)[8][2], const u32x4 (&pw)[2], f32x4 (&o)[8]) {
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
      o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vreg[dt][c]), as_bf16x8(pw[c]), o[dt], 0, 0, 0);
}

// The page loop of the audio path, one wave: pages p_begin, p_begin + step,
// ... (< p_end) of the list, whose first page's operands kreg and vreg hold
// on entry.  Accumulates O^T (o), the running maximum and the row sum of the
// wave's 16 query columns (m_run and l_run as set up by the caller: the
// fixed shift, or -inf for a running maximum).
//
// Each page's K registers are reloaded (for the wave's next page) as soon as
// its S products are issued, and its V^T registers as soon as the P*V
// products are, so both loads of a page are in flight while the wave waits on
// the one before it.
__device__ __forceinline__ void audio_page_loop(const_page_list pages, int p_begin, int p_end, int step,
                                                const uint16_t* kpool, const uint16_t* vpool, int64_t page_stride,
                                                const uint16_t* zeros, const bf16x8 (&qreg)[4], bool fixed_shift,
                                                u32x4 (&kreg)[4][4], u32x4 (&vreg)[8][2], int g, int i16, int lane,
                                                f32x4 (&o)[8], float& m_run, float& l_run) {
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) o[dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
  for (int pi = p_begin; pi < p_end; pi += step) {
    const int n_valid = pages[pi].y;
    int2 nxt = make_int2(0, 0);  // past the last page: zeros
    if (pi + step < p_end) nxt = make_int2(pages[pi + step].x, pages[pi + step].y);
    f32x4 sacc[4];
    audio_scores(kreg, qreg, sacc);
    audio_load_k(kreg, kpool + nxt.x * page_stride, zeros, nxt.y, g, i16, lane);
    u32x4 pw[2];
    audio_softmax(sacc, n_valid, fixed_shift, g, pw, o, m_run, l_run);
    audio_pv(vreg, pw, o);
    audio_load_v(vreg, vpool + nxt.x * page_stride, zeros, nxt.y, g, i16, lane);
  }
}

// The softmax shift bound of the audio path: |Q''_q| times the largest key
// norm (squared: kn2, the lane's part of the pages), the same in all lane
// groups of a row.
__device__ __forceinline__ float audio_bound(const bf16x8 (&qreg)[4], float kn2) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) kn2 = fmaxf(kn2, __shfl_xor(kn2, off));
  float qn2 = 0.f;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const u32x4 w = __builtin_bit_cast(u32x4, qreg[s]);
#pragma unroll
    for (int k = 0; k < 4; ++k) qn2 += bf16_lo(w[k]) * bf16_lo(w[k]) + bf16_hi(w[k]) * bf16_hi(w[k]);
  }
  qn2 += __shfl_xor(qn2, 16);
  qn2 += __shfl_xor(qn2, 32);
  return sqrtf(qn2 * kn2);
}

// ------------------------------------------------------------------------- //
// The rider rows' own pages (entries rx_page0 .. of the page list, visible to
// them only), inside the video kernel: the last wave of the last query tile's
// workgroups attends them with the audio path's arithmetic; each of a head's
// first rx_ranges ranges takes its part of them and writes it as a key range of
// its own (after the head's ranges of the shared pages) of the rows' fp32
// partials.  A wave without rows does so between the page loads it issues
// anyway: one page's registers are requested in one iteration of the stream
// and consumed in the next (the request in the same iteration as a computation
// would hold up the page barrier), so the other waves never wait for it.  (With
// three such waves attending three pages each ahead of their first page
// barrier, the barrier waited 7 us.)  A wave with rows does it after its
// segments: a page or two, against a launch of the audio kernel (6 us).
// ------------------------------------------------------------------------- //
struct RiderWork {
  int head, range, p0, np;  // pages [p0, p0 + np) of the list
  int item, n_items;        // item: (16-row subtile, page), the pages innermost
  bool loaded;              // the item's operands are requested
  bool fixed_shift;
  float m, l;
  u32x4 k[4][4], v[8][2];
  f32x4 o[8];
  bf16x8 q[4];
};

__device__ __forceinline__ void rider_request(const AttnArgs& a, RiderWork& w, int lane) {
  const int g = lane >> 4, i16 = lane & 15;
  const const_page_list pages = page_list(a);
  const int per = max(w.np, 1), sub = w.item / per, pg = w.item - sub * per;
  if (pg == 0) {
    const int q = 16 * sub + i16;
    const bool ok = q < a.n_rq;
    const uint16_t* qp = a.rq + q * a.rq_tok_stride + w.head * a.rq_head_stride + 8 * g;
#pragma unroll
    for (int s = 0; s < 4; ++s)
      w.q[s] = as_bf16x8(ok ? *reinterpret_cast<const u32x4*>(qp + 32 * s) : (u32x4){0u, 0u, 0u, 0u});
    float kn2 = 0.f;
    for (int pi = w.p0 + lane; pi < w.p0 + w.np; pi += 64)
      kn2 = fmaxf(kn2, a.knorm2[static_cast<int64_t>(pages[pi].x) * a.num_heads + w.head]);
    const float bound = audio_bound(w.q, kn2);
    w.fixed_shift = a.fixed_shift != 0 && __all(bound <= kShiftBoundMax);
    w.m = w.fixed_shift ? bound : kNegInf;
    w.l = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) w.o[dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }
  int2 p = make_int2(0, 0);  // no page: zeros
  if (pg < w.np) p = make_int2(pages[w.p0 + pg].x, pages[w.p0 + pg].y);
  const int64_t tile = (static_cast<int64_t>(p.x) * a.num_heads + w.head) * kPageHeadElems;
  audio_load_k(w.k, a.kpool + tile, a.zeros, p.y, g, i16, lane);
  audio_load_v(w.v, a.vpool + tile, a.zeros, p.y, g, i16, lane);
  w.loaded = true;
}

__device__ __forceinline__ void rider_compute(const AttnArgs& a, RiderWork& w, int lane) {
  const int g = lane >> 4, i16 = lane & 15;
  const const_page_list pages = page_list(a);
  const int per = max(w.np, 1), sub = w.item / per, pg = w.item - sub * per;
  f32x4 sacc[4];
  u32x4 pw[2];
  audio_scores(w.k, w.q, sacc);
  audio_softmax(sacc, pg < w.np ? pages[w.p0 + pg].y : 0, w.fixed_shift, g, pw, w.o, w.m, w.l);
  audio_pv(w.v, pw, w.o);
  if (pg == per - 1) {  // lane holds O^T[16 dt + 4 g + r][q]
    float l = w.l + __shfl_xor(w.l, 16);
    l += __shfl_xor(l, 32);
    const int q = 16 * sub + i16;
    if (q < a.n_rq) {
      const int64_t row = (static_cast<int64_t>(w.range) * a.num_heads + w.head) * a.n_rq + q;
      const float inv = l > 0.f ? 1.0f / l : 0.f;
      float* po = a.rpart_o + row * kHeadDim + 4 * g;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4*>(po + 16 * dt) = w.o[dt] * inv;
      if (g == 0) a.rpart_lse[row] = l > 0.f ? w.m + __log2f(l) : kNegInf;
    }
  }
  ++w.item;
  w.loaded = false;
}

// The rider rows' pages that range sg.seg of the n_seg of its head takes.
__device__ __forceinline__ void rider_share(const AttnArgs& a, const VideoSeg& sg, int n_seg, RiderWork& w) {
  const int parts = min(n_seg, a.rx_ranges);
  w.item = 0;
  w.n_items = 0;
  w.loaded = false;
  if (sg.seg >= parts) return;
  w.head = sg.head;
  w.range = n_seg + sg.seg;
  w.p0 = a.rx_page0 + a.rx_pages * sg.seg / parts;
  w.np = a.rx_page0 + a.rx_pages * (sg.seg + 1) / parts - w.p0;
  w.n_items = ((a.n_rq + 15) / 16) * max(w.np, 1);
}
__device__ __forceinline__ void rider_rest(const AttnArgs& a, RiderWork& w, int lane) {
  while (w.item < w.n_items) {
    if (!w.loaded) rider_request(a, w, lane);
    rider_compute(a, w, lane);
  }
}

// A segment for a wave without query rows: it issues its share of the page
// loads and attends the rider rows' pages (n_seg > 0: the head's ranges).
template <class P>
__device__ __forceinline__ void video_idle_segment(const AttnArgs& a, const VideoSeg& sg, VideoStream<P>& s, int n_seg) {
  if constexpr (!P::kPlain) {
    if (s.at == 0) {
      if constexpr (P::k8) wait_lds();
      else wait_dma_all_but_last_page();
    }
    for (int k = 0; k < sg.n; ++k) {
      page_barrier();
      if constexpr (P::k8) stage_page<true>(s, s.c);
      else issue_page(s, s.c);
      const int at = min(s.at + 4, s.n - 1);
      s.at += 1;
      s.stage = ring_add(s.stage, 1);
      if constexpr (P::k8) {
        if constexpr (!P::kQ8) s.c.ks = s.c.ks_load;
        s.c.vs = s.c.vs_load;
        if constexpr (!P::kQ8) s.c.ks_load = peek_lanes(s.ks, at);
        s.c.vs_load = peek_lanes(s.vs, at);
        s.c.wk = s.wk + ring_add(s.stage, 2);
        s.c.wv = s.wv + ring_add(s.stage, 2);
        set_load(s, stream_peek(s, at), 0, s.c);
        wait_lds();
      } else {
        set_load(s, stream_peek(s, at), ring_add(s.stage, 3), s.c);
        wait_dma_all_but_last_page();
      }
      stream_reach(s);
    }
    return;
  }
  RiderWork w;
  w.item = w.n_items = 0;
  w.loaded = false;
  if (n_seg > 0) rider_share(a, sg, n_seg, w);
  if (s.at == 0) wait_dma_all_but_last_page();
  for (int k = 0; k < sg.n; ++k) {
    page_barrier();
    if (w.item < w.n_items) {
      if (w.loaded) rider_compute(a, w, s.lane);
      else rider_request(a, w, s.lane);
    }
    issue_page(s, s.c);
    const uint32_t e = stream_peek(s, min(s.at + 4, s.n - 1));
    s.at += 1;
    s.stage = ring_add(s.stage, 1);
    set_load(s, e, ring_add(s.stage, 3), s.c);
    wait_dma_all_but_last_page();
    stream_reach(s);
  }
  rider_rest(a, w, s.lane);  // a short segment's
}

// The segment at stream offset k of group `group`'s share.
__device__ __forceinline__ VideoPartition32 part_of(const __attribute__((address_space(4))) AttnClass& c) {
  const auto& p = c.part;
  return VideoPartition32{p.pages, p.cost, p.len, p.groups, p.quot, p.rem, p.fits,
                          {p.by_pages.mul, p.by_pages.shift}, {p.by_stride.mul, p.by_stride.shift},
                          {p.by_groups.mul, p.by_groups.shift}, {p.by_len.mul, p.by_len.shift}};
}
struct VideoWork {
  VideoPartition32 part;
  int group, q_lo, q_hi;
};
template <class P>
__device__ __forceinline__ VideoSeg video_seg(const VideoWork& w, const VideoStream<P>& s, int k) {
  const int x = s.lo + k;
  const int head = static_cast<int>(fast_div(x, s.div_pages)), h0 = head * s.n_pages;
  const int n = min(s.n - k, h0 + s.n_pages - x);
  const int seg = x == h0 ? 0 : w.group - static_cast<int>(part_group_of(w.part, h0));
  return VideoSeg{static_cast<int>(head_of(s, head)), n, seg, w.q_lo, w.q_hi, x == h0 && n == s.n_pages};
}

// Ranges of a head (for the rider rows' partials).
template <class P>
__device__ __forceinline__ int head_ranges(const VideoWork& w, const VideoStream<P>& s, int head) {
  const int h0 = head * s.n_pages;
  return static_cast<int>(part_group_of(w.part, h0 + s.n_pages - 1) - part_group_of(w.part, h0)) + 1;
}

template <int kQT, int kQueries, class P>
__device__ __forceinline__ void video_wave(const AttnArgs& a, const VideoWork& w, VideoStream<P>& s, int wave) {
  if constexpr (P::kWin) {
    const int t_first = a.win.t0 + w.q_lo + wave * 16 * kQT;
    const int t_last = a.win.t0 + min(w.q_lo + (wave + 1) * 16 * kQT, w.q_hi) - 1;
    s.hi_all = row_range(s.win, t_first).hi;
    s.lo_all = row_range(s.win, t_last).lo;
  }
  stream_start(a, s);
  while (s.at < s.n) video_segment<kQT, kQueries, P>(a, video_seg(w, s, s.at), s, wave);
}

// The rider rows' pages for a wave with rows of its own, after its segments.
__device__ __forceinline__ void rider_segments(const AttnArgs& a, const VideoWork& w, const VideoStream<PlainPath>& s) {
  for (int k = 0; k < s.n;) {
    const VideoSeg sg = video_seg(w, s, k);
    RiderWork r;
    rider_share(a, sg, head_ranges(w, s, sg.head), r);
    rider_rest(a, r, opaque(s.lane));
    k += sg.n;
  }
}

// Rows that see nothing: output 0.
__device__ __forceinline__ void video_empty(const AttnArgs& a, int head, int q_lo, int q_hi) {
  const int n = (q_hi - q_lo) * (kHeadDim / 8);
  for (int i = threadIdx.x; i < n; i += kVideoWaves * 64) {
    const int64_t q = q_lo + i / (kHeadDim / 8);
    *reinterpret_cast<u32x4*>(a.out + q * a.out_tok_stride + head * a.out_head_stride + 8 * (i % (kHeadDim / 8))) =
        (u32x4){0u, 0u, 0u, 0u};
  }
}

template <class P, int kQueries>
__device__ __forceinline__ void unit_attn(const AttnArgs& a) {
  // Work decode.  Each query class (the rows of one unit's queries, with the
  // pages its mask leaves visible) owns a block of workgroups: n_groups
  // groups of n_qtiles workgroups; group g takes a contiguous share of the
  // class's (head, page) units in head-major order (VideoPartition: even
  // shares of pages plus a cost per head started), one workgroup per query
  // tile, so the work fits a single round, and a share that crosses a head
  // boundary is processed as several segments.  Workgroups are dispatched
  // round-robin over the 8 XCDs; renumber so that consecutive work items
  // (the query tiles of a group, which read the same pages at the same time,
  // and neighbouring groups) run on one XCD and share its L2.  The divisions
  // are multiplications by host-made reciprocals: with the partition's own
  // integer divisions a workgroup spent 5 us before its first load.
  const int nblk = gridDim.x, bid = blockIdx.x;
  const int xcd = bid & 7, per = nblk >> 3, rem = nblk & 7;
  const int item = xcd * per + min(xcd, rem) + (bid >> 3);
  const const_class_table tab = class_table();
  int ci = 0;
  for (int k = 1; k < a.n_classes; ++k)
    if (item >= tab[k].wg0) ci = k;
  const int local = item - tab[ci].wg0;
  const int n_qtiles = tab[ci].n_qtiles;
  const int group = static_cast<int>(fast_div(local, FastDiv{tab[ci].by_qtiles.mul, tab[ci].by_qtiles.shift}));
  const int qt = local - group * n_qtiles;
  int q0 = tab[ci].q0, q_hi = q0 + tab[ci].n_q;
  int tile_rows = tab[ci].tile_rows, q_lo = q0 + qt * tile_rows;
  [[maybe_unused]] int head0 = 0;
  [[maybe_unused]] bool tiles = false;
  if constexpr (P::kWin) {
    if (a.n_tiles > 0) {
      tiles = true;
      head0 = static_cast<int>(fast_div(item, a.by_tiles));
      ci = item - head0 * a.n_tiles;
      tile_rows = a.tile_rows;
      q_lo = ci * tile_rows;
      q_hi = min(q_lo + tile_rows, a.n_q);
    }
  }
  // rider rows follow the video rows (a single class then)
  const int row_end = min(q_lo + tile_rows, P::kPlain && a.n_rq > 0 ? a.rq_row0 + a.n_rq : q_hi);
  const int wave_rows = video_wave_rows(tile_rows, row_end - q_lo);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));

  VideoWork w;
  w.group = group;
  w.q_lo = q_lo;
  w.q_hi = q_hi;
  VideoStream<P> s;
  s.pages = page_list(a);
  s.num_heads = a.num_heads;
  if constexpr (P::kWin) {
    s.win = a.win;
    const ClassPages cp = class_pages(ci);
    s.head_pages = cp.head_pages;
    s.skip = cp.skip;
    s.head0 = head0;
    s.n_pages = cp.count;
    s.page0 = tiles ? 0 : tab[ci].page0;
    s.hi_all = s.lo_all = 0;  // (a wave without rows asks for no edges)
  }
  if constexpr (P::k8) {
    s.kscale = a.kscale;
    s.vscale = a.vscale;
  }
  if constexpr (!P::kWin) {
    s.n_pages = tab[ci].n_pages;
    s.page0 = tab[ci].page0;
  }
  s.lane = lane;
  s.kpool = a.kpool;
  s.vpool = a.vpool;
  s.at = 0;
  s.stage = 0;
  s.valid = 0;
  if (s.n_pages == 0) {  // nothing visible: one group per head
    const int head = tiles ? head0 : group;
    if (head < a.num_heads) video_empty(a, head, q_lo, min(q_lo + tile_rows, q_hi));
    return;
  }
  w.part = part_of(tab[ci]);
  s.div_pages = w.part.by_pages;
  s.lo = static_cast<int>(part_group_lo(w.part, group));
  s.n = static_cast<int>(part_group_lo(w.part, group + 1)) - s.lo;
  if constexpr (P::kWin) {
    if (tiles) {
      s.div_pages = FastDiv{1, 0};  // (quotient 0)
      s.lo = 0;
      s.n = s.n_pages;
    }
  }
  if (s.n == 0) return;
  // the list entries of the window are under way while the lane's offsets are
  // computed; stream_start waits for them, and the first segment's queries are
  // loaded behind the direct loads it issues
  stream_request(s);
  {
    // K block wave: row 4 wave + lane / 16 of key tile 0, position lane % 16
    const int m = 4 * wave + (lane >> 4);
    s.dma_k = 2 * k_tile_index(audio_key(0, m), 8 * ((lane & 15) ^ m));
    // V^T block wave: row d = 8 wave + lane / 8, position lane % 8
    const int d = 8 * wave + (lane >> 3);
    s.dma_v = 2 * v_tile_index(8 * ((lane & 7) ^ ((d >> 1) & 7)), d);
    const uint32_t lds = lds_offset(g_stages);
    if constexpr (P::k8) {
      // A write takes 8 lanes at a time, over 128 bytes of banks: eight neighbours hold
      // two keys that are two apart, whose rows' swizzles send their chunks to even and
      // odd positions (e4m3 K: to the low and high ones).
      const uint32_t n = 64u * wave + lane, key = swap_low_bits(n >> 2), part = n & 3, t = 4 * key + part;
      const uint32_t tile = 2 * (key >> 5) + ((key >> 2) & 1), row = 4 * ((key >> 3) & 3) + (key & 3);
      s.load[0] = 16u * t;
      s.load[1] = opaque(16u * t + 4096u);  // (a register of its own: an offset beside a scalar base)
      // K: row 16 tile + m of the key, chunks 2 part (and 8 further, and the odd ones)
      s.wk = P::kQ8 ? lds + 128u * (16u * tile + row) + 16u * (part ^ codes_swizzle(row))
                    : lds + 256u * (16u * tile + row) + 16u * ((2u * part) ^ swap_low_bits(row));
      s.wv = lds + kStageV + 128u * key + 16u * ((2u * part) ^ ((key >> 1) & 7));  // (V^T: dim t / 4)
    }
    s.lds0 = __builtin_amdgcn_readfirstlane(lds + 1024u * wave);
    const int g = lane >> 4, i16 = lane & 15;
    s.k_read = P::kQ8  ? lds + 128u * i16 + 16u * (g ^ codes_swizzle(i16))
               : P::k8 ? lds + 256u * i16 + 16u * (g ^ swap_low_bits(i16))
                       : lds + 256u * i16 + 16u * (g ^ i16);
    s.v_read = lds + kStageV + 128u * i16 + 16u * (g ^ ((i16 >> 1) & 7));
  }
  const bool rx = P::kPlain && a.rx_pages > 0 && qt == n_qtiles - 1 && wave == kVideoWaves - 1;
  if (q_lo + wave * wave_rows >= row_end) {
    stream_start(a, s);
    while (s.at < s.n) {
      const VideoSeg sg = video_seg(w, s, s.at);
      video_idle_segment(a, sg, s, rx ? head_ranges(w, s, sg.head) : 0);
    }
    if (!P::k8) wait_dma_all();
    return;
  }
  if (wave_rows == 64) video_wave<4, kQueries>(a, w, s, wave);
  else if (wave_rows == 48) video_wave<3, kQueries>(a, w, s, wave);
  else video_wave<2, kQueries>(a, w, s, wave);
  if constexpr (P::kPlain)
    if (rx) rider_segments(a, w, s);
}

#define WS_ONE_WAVE_PER_SIMD __launch_bounds__(kVideoWaves * 64) __attribute__((amdgpu_waves_per_eu(1, 1)))

}  // namespace
}  // namespace ws
