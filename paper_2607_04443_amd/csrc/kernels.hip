// gfx950 (MI355X, CDNA4) kernels of the performer unit attention.
//
//  kv_append       writes a segment's K/V into its cache pages; NORM_ROPE keys
//                  get per-head RMS-norm, the gamma weight and (t,h,w) rotary
//                  positions in fp32 before the bf16 store; V is stored
//                  transposed per page ([d][slot]).
//  unit_attn       video queries: flash attention over the visible pages with
//                  v_mfma_f32_16x16x32_bf16, K/V pages staged through a ring
//                  of LDS stages, softmax in the exp2 domain under a shift
//                  fixed in advance or a lazily raised running maximum.
//  audio_attn      the few audio queries: memory-bound split-KV, one wave per
//                  key range, v_mfma_f32_16x16x32_bf16 straight from registers.
//  combine         log-sum-exp merge of split-KV partials.
//
// The attention is the performer's per-step attention over its K/V cache
// (Wan-Streamer v0.2, Sec. 3); block-causal visibility (Fig. 1 caption) is
// resolved on the host into the list of visible pages.
#include <hip/hip_ext.h>

#include <algorithm>
#include <cstddef>
#include <mutex>
#include <type_traits>
#include <utility>

#include "device_common.hpp"
#include "video_core.hpp"
#include "ws_kernels.hpp"

namespace ws {
namespace {

// ------------------------------------------------------------------------- //
// kv_append: one (item, head) tile of an append launch, an item being a K/V
// page or a 64-token chunk of a query set of one of up to
// AppendArgs::kMaxSegs segments.  256 threads; vt and wave_norm2 are the
// block's LDS, free again when the call returns.
//
// What bounds it: memory (a step of 924 queries and 1,180 new tokens over 40
// heads moves 67 MB, 10 us at the rate of a large copy) and, before that, the
// chain position -> table entry -> rotation of each row.  So a tile's loads are
// all issued first, its table entries two rows ahead by a select instead of a
// branch per band, and row sums are DPP rotations instead of LDS permutes.
// V is transposed through LDS: rows of 128 d, the 16-byte chunk d / 8 of row r
// at position (d / 8) ^ (r / 8), so that the 32-bit reads of a d pair over the
// eight row groups hit different banks; two rows of V^T per thread halve the
// LDS reads.  Measured (that step / its queries alone / 12 heads, 256
// queries and 320 tokens): 17.1 / 7.8 / 7.1 us before, 14.4 / 7.6 / 5.2 us.
// With registers for six blocks per CU it spills (25.7 us); grids of 3, 5 and 8
// blocks per CU take 15.6, 16.1 and 15.9 us for the first, 4 takes 14.9 in the
// same run.
// ------------------------------------------------------------------------- //
__device__ __forceinline__ void append_tile(const_append_args A, int item, int head, uint16_t (*vt)[kHeadDim],
                                            float* wave_norm2) {
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
  const int page = A->pages[item];
  const int64_t tok_stride = sg->tok_stride;
  const int n_tokens = sg->n_tokens;
  const bool norm_rope = sg->mode == 1;
  const int tok0 = A->blk_page[item] * kPageTokens;
  const int64_t tile = (static_cast<int64_t>(page) * num_heads + head) * kPageHeadElems;
  uint16_t* kdst = A->kpool + tile;
  uint16_t* vdst = A->vpool + tile;
  const int t = threadIdx.x, c = t & 15, rr = t >> 4;

  // all loads of the tile are issued up front: positions, K rows, V rows
  AppendRows r;
  load_rows(sg, tok0, head, norm_rope, c, rr, r);
  const uint16_t* const src_v = sg->v + head * sg->head_stride + 8 * c;
  u32x4 vx[4];
#pragma unroll
  for (int pass = 0; pass < 4; ++pass) {
    const int tok = tok0 + pass * 16 + rr;
    vx[pass] = tok < n_tokens ? *reinterpret_cast<const u32x4*>(src_v + tok * tok_stride) : (u32x4){0u, 0u, 0u, 0u};
  }

  // K: alongside, the largest squared norm of the stored rows of the tile.  It
  // only bounds scores (the softmax shift), so the dot product instruction does:
  // exact products, fp32 sums; squares it may flush (|k| < 1.1e-19) could move
  // a bound by less than 32 for the largest |q| whose square is finite.
  float norm2 = 0.f;
  auto put = [&](int, int slot, u32x4 y) {
    *reinterpret_cast<u32x4*>(kdst + k_tile_index(slot, 8 * c)) = y;
    norm2 = fmaxf(norm2, row_sum(norm2_words(y, 0.f)));
  };
  if (norm_rope) {
    // empty slots hold zeros whatever gamma and eps are
    rotate_rows(rope, flags, sg, tok0, 1.0f, c, rr, r, [&](int pass, int slot, u32x4 y) {
      put(pass, slot, tok0 + slot < n_tokens ? y : (u32x4){0u, 0u, 0u, 0u});
    });
  } else {
#pragma unroll
    for (int pass = 0; pass < 4; ++pass) put(pass, pass * 16 + rr, r.x[pass]);
  }
  norm2 = pair_max<32>(pair_max<16>(norm2));
  if ((t & 63) == 0) wave_norm2[t >> 6] = norm2;
#pragma unroll
  for (int pass = 0; pass < 4; ++pass) {
    const int row = pass * 16 + rr;
    *reinterpret_cast<u32x4*>(&vt[row][8 * (c ^ (row >> 3))]) = vx[pass];
  }
  __syncthreads();
  // thread: d pair d2 (two rows of V^T), slots 8 tc .. 8 tc + 7
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int ch = t + 256 * i, tc = ch & 7, d = 2 * (ch >> 3);
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      w[j] = *reinterpret_cast<const uint32_t*>(&vt[8 * tc + j][8 * ((d >> 3) ^ tc) + (d & 7)]);
    u32x4 lo, hi;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      lo[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x05040100u);
      hi[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x07060302u);
    }
    *reinterpret_cast<u32x4*>(vdst + v_tile_index(8 * tc, d)) = lo;
    *reinterpret_cast<u32x4*>(vdst + v_tile_index(8 * tc, d + 1)) = hi;
  }
  if (t == 0)
    A->knorm2[static_cast<int64_t>(page) * num_heads + head] =
        fmaxf(fmaxf(wave_norm2[0], wave_norm2[1]), fmaxf(wave_norm2[2], wave_norm2[3]));
}

// The launch: a grid of a few blocks per CU that loop over the launch's
// (item, head) tiles, consecutive tiles being the heads of one item.  (One
// block per tile made the launch as long as dispatching its ~1,400 short
// blocks: their average life was about an eighth of the launch.)
__global__ __launch_bounds__(256) void kv_append_kernel(const AppendArgs args) {
  (void)args;  // read in place, through append_args()
  __shared__ __attribute__((aligned(16))) uint16_t vt[kPageTokens][kHeadDim];
  __shared__ float wave_norm2[4];
  const const_append_args A = append_args();
  const int heads = A->num_heads;
  const int n_tiles = A->n_blocks * heads;
  for (int tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
    append_tile(A, tile / heads, tile % heads, vt, wave_norm2);
    __syncthreads();  // vt and wave_norm2 are rewritten by the next tile
  }
}

__global__ __launch_bounds__(256, 2) void audio_attn_kernel(const AttnArgs a) {
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
  const_page_list pages = page_list(a);
  const int64_t page_stride = static_cast<int64_t>(a.num_heads) * kPageHeadElems;
  const uint16_t* kpool = a.kpool + head * kPageHeadElems;
  const uint16_t* vpool = a.vpool + head * kPageHeadElems;

  // the wave's first page is requested before the query prologue
  u32x4 kreg[4][4], vreg[8][2];
  {
    int2 pg = make_int2(0, 0);  // no page: zeros
    if (p_begin < p_end) pg = make_int2(pages[p_begin].x, pages[p_begin].y);
    audio_load_k(kreg, kpool + pg.x * page_stride, a.zeros, pg.y, g, i16, lane);
    audio_load_v(vreg, vpool + pg.x * page_stride, a.zeros, pg.y, g, i16, lane);
  }

  // Q prologue: lane holds Q''[q][32 s + 8 g + j], s = 0..3, with the
  // softmax scale and log2(e) folded in
  const int q = qtile * kAudioQTile + i16;
  const bool q_ok = q < a.n_q;
  u32x4 qraw[4];
  const uint16_t* qp = a.q + q * a.q_tok_stride + head * a.q_head_stride + 8 * g;
#pragma unroll
  for (int s = 0; s < 4; ++s)
    qraw[s] = q_ok ? *reinterpret_cast<const u32x4*>(qp + 32 * s) : (u32x4){0u, 0u, 0u, 0u};
  bf16x8 qreg[4];
  if (a.mode == 1) {
    int pt = 0, ph = 0, pw = 0;
    if (q_ok) load_pos(a.rope, a.positions, q, a.flags, pt, ph, pw);
    float ss = 0.f;
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x0 = bf16_lo(qraw[s][k]), x1 = bf16_hi(qraw[s][k]);
        ss += x0 * x0 + x1 * x1;
      }
    ss += __shfl_xor(ss, 16);
    ss += __shfl_xor(ss, 32);
    const float inv = rsqrtf(ss * (1.0f / kHeadDim) + a.eps);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int d0 = 32 * s + 8 * g;
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
      qreg[s] = as_bf16x8(q_ok ? w : (u32x4){0u, 0u, 0u, 0u});
    }
  } else if (a.mode == 2) {  // prepared: Q'' as given
#pragma unroll
    for (int s = 0; s < 4; ++s) qreg[s] = as_bf16x8(qraw[s]);
  } else {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      u32x4 w;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[k] = pack_bf16(bf16_lo(qraw[s][k]) * a.scale_log2, bf16_hi(qraw[s][k]) * a.scale_log2);
      qreg[s] = as_bf16x8(w);
    }
  }

  // Softmax shift, as in the video kernel: the logit bound |Q''_q| max |k|
  // (log2 units) over the wave's pages when it is at most kShiftBoundMax for
  // all 16 queries, else a running maximum.
  float kn2 = 0.f;
  for (int pi = p_begin + 4 * lane; pi < p_end; pi += 256)
    kn2 = fmaxf(kn2, a.knorm2[static_cast<int64_t>(pages[pi].x) * a.num_heads + head]);
  const float bound = audio_bound(qreg, kn2);
  const bool fixed_shift = a.fixed_shift != 0 && __all(bound <= kShiftBoundMax);
  float m_run = fixed_shift ? bound : kNegInf, l_run = 0.f;

  f32x4 o[8];
  audio_page_loop(pages, p_begin, p_end, 4, kpool, vpool, page_stride, a.zeros, qreg, fixed_shift, kreg, vreg,
                  g, i16, lane, o, m_run, l_run);

  // merge the four waves: lane holds O^T[16 dt + 4 g + r][q] of its keys
  float l_w = l_run + __shfl_xor(l_run, 16);
  l_w += __shfl_xor(l_w, 32);
#pragma unroll
  for (int dt = 0; dt < 8; ++dt)
#pragma unroll
    for (int r = 0; r < 4; ++r) sm_o[wave][16 * dt + 4 * g + r][i16] = o[dt][r];
  if (g == 0) {
    sm_ml[wave][0][i16] = m_run;
    sm_ml[wave][1][i16] = l_w;
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
    ew[w] = big == kNegInf ? 0.f : fast_exp2(mw[w] - big);
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
      out0[k] = l_tot > 0.f ? out0[k] + 0.f : 0.f;  // (+ 0: the merge's sum turns -0 to 0)
      out1[k] = l_tot > 0.f ? out1[k] + 0.f : 0.f;
    }
    *reinterpret_cast<u32x4*>(a.out + qq * a.out_tok_stride + head * a.out_head_stride + d0) =
        (u32x4){pack_bf16(out0[0], out0[1]), pack_bf16(out0[2], out0[3]), pack_bf16(out1[0], out1[1]),
                pack_bf16(out1[2], out1[3])};
    return;
  }
  const int64_t row = (static_cast<int64_t>(split) * a.num_heads + head) * a.n_q + qq;
  float* po = a.part_o + row * kHeadDim + d0;
  *reinterpret_cast<f32x4*>(po) = out0;
  *reinterpret_cast<f32x4*>(po + 4) = out1;
  if (tid < 16) a.part_lse[row] = l_tot > 0.f ? big + __log2f(l_tot) : kNegInf;
}

__global__ WS_ONE_WAVE_PER_SIMD void unit_attn_kernel(const AttnArgs a) { unit_attn<PlainPath, kQueriesPrepared>(a); }
__global__ WS_ONE_WAVE_PER_SIMD void unit_attn_rows_kernel(const AttnArgs a) { unit_attn<PlainPath, kQueriesRaw>(a); }

// ------------------------------------------------------------------------- //
// combine (audio key ranges): 16 threads per (head, query) row, 8 d each, 16
// rows per block.  A thread reads the row's log-sum-exps, then requests the
// 8 values of kMergeBatch ranges before using any (one memory round trip per
// batch) and folds them against the largest.  The batch sets the registers a
// thread holds: the audio call's own merge takes 16 ranges at once; inside
// the merge launch of a step, whose video rows need few registers, 3 (more
// would cap the occupancy of the video rows' blocks).
// ------------------------------------------------------------------------- //
template <int kMergeBatch>
__device__ __forceinline__ void combine_block(const CombineArgs& a, int bid) {
  const int lane = threadIdx.x & 15;
  const int row = bid * 16 + (threadIdx.x >> 4);
  if (row >= a.num_heads * a.n_q) return;
  const int head = row / a.n_q, q = row % a.n_q;
  int n_splits = a.n_splits;
  if (a.r_groups > 0) {  // the ranges the video kernel wrote for rider rows
    const VideoPartition part{a.num_heads, a.r_pages, a.seg_cost, a.r_groups};
    const int64_t h0 = static_cast<int64_t>(head) * a.r_pages;
    const int ranges = static_cast<int>(video_group_of(part, h0 + a.r_pages - 1) - video_group_of(part, h0) + 1);
    n_splits += ranges + min(ranges, a.r_extra);  // and those of the rows' own pages
  }
  const int d0 = 8 * lane;
  const int64_t split_stride = static_cast<int64_t>(a.num_heads) * a.n_q;
  // The largest log-sum-exp first: every range is then weighted the same way
  // whatever the batch, so the step's merge launch and the audio call's own
  // give the same bits.  (With all ranges in one batch it comes from that
  // batch's loads.)
  float mx = kNegInf;
  for (int sp0 = 0; n_splits > kMergeBatch && sp0 < n_splits; sp0 += 16) {
    float lb[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) lb[i] = sp0 + i < n_splits ? a.part_lse[(sp0 + i) * split_stride + row] : kNegInf;
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, lb[i]);
  }
  float wsum = 0.f;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int sp0 = 0; sp0 < n_splits; sp0 += kMergeBatch) {
    float lb[kMergeBatch];
    f32x4 o0[kMergeBatch], o1[kMergeBatch];
#pragma unroll
    for (int i = 0; i < kMergeBatch; ++i) {
      const int sp = sp0 + i;
      const bool ok = sp < n_splits;
      const float* po = a.part_o + (sp * split_stride + row) * kHeadDim + d0;
      lb[i] = ok ? a.part_lse[sp * split_stride + row] : kNegInf;
      o0[i] = ok ? *reinterpret_cast<const f32x4*>(po) : (f32x4){0.f, 0.f, 0.f, 0.f};
      o1[i] = ok ? *reinterpret_cast<const f32x4*>(po + 4) : (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    if (n_splits <= kMergeBatch) {
#pragma unroll
      for (int i = 0; i < kMergeBatch; ++i) mx = fmaxf(mx, lb[i]);
    }
    if (mx == kNegInf) break;
#pragma unroll
    for (int i = 0; i < kMergeBatch; ++i) {
      const float w = lb[i] == kNegInf ? 0.f : fast_exp2(lb[i] - mx);
      wsum += w;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        acc[k] += w * o0[i][k];
        acc[4 + k] += w * o1[i][k];
      }
    }
  }
  const float inv = mx != kNegInf ? 1.0f / wsum : 0.f;
  u32x4 w;
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = pack_bf16(acc[2 * k] * inv, acc[2 * k + 1] * inv);
  *reinterpret_cast<u32x4*>(a.out + q * a.out_tok_stride + head * a.out_head_stride + d0) = w;
}

__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a) { combine_block<16>(a, blockIdx.x); }

// ------------------------------------------------------------------------- //
// video_combine: merges the key ranges of the video schedule.  A head's
// range count follows from the groups' shares (VideoPartition; a head
// in one range was written in bf16 by the attention kernel: nothing to
// merge).  16 threads per (head, query) row, 8 d each (16-byte loads), 16
// rows per block; all of a row's (at most kMaxVideoSplits) partials are
// requested before any is used.
// ------------------------------------------------------------------------- //
__device__ __forceinline__ void video_combine_block(const CombineArgs& a, const_class_table tab, int bid) {
  const int lane = threadIdx.x & 15;
  const int row = bid * 16 + (threadIdx.x >> 4);
  if (row >= a.num_heads * a.n_q) return;
  const int head = row / a.n_q, q = row % a.n_q;
  // the row's query class: every table entry is read with uniform (scalar)
  // loads and the row's fields are selected per lane
  int32_t cls_pages = tab[0].n_pages, cls_groups = tab[0].n_groups;
  for (int k = 1; k < a.n_classes; ++k) {
    const bool in = q >= tab[k].q0;
    cls_pages = in ? tab[k].n_pages : cls_pages;
    cls_groups = in ? tab[k].n_groups : cls_groups;
  }
  const int64_t n_pages = cls_pages;
  if (n_pages == 0) return;
  const VideoPartition part{a.num_heads, n_pages, a.seg_cost, cls_groups};
  const int64_t h0 = static_cast<int64_t>(head) * n_pages;
  const int n_ranges = static_cast<int>(video_group_of(part, h0 + n_pages - 1) - video_group_of(part, h0) + 1);
  if (n_ranges < 2) return;
  const int d0 = 8 * lane;
  const int64_t split_stride = static_cast<int64_t>(a.num_heads) * a.n_q;
  const uint16_t* po = reinterpret_cast<const uint16_t*>(a.part_o);
  float l[kMaxVideoSplits];
  u32x4 w[kMaxVideoSplits];
#pragma unroll
  for (int sp = 0; sp < kMaxVideoSplits; ++sp) {
    if (sp < n_ranges) {
      l[sp] = a.part_lse[sp * split_stride + row];
      w[sp] = *reinterpret_cast<const u32x4*>(po + (sp * split_stride + row) * kHeadDim + d0);
    } else {
      l[sp] = kNegInf;
      w[sp] = (u32x4){0u, 0u, 0u, 0u};
    }
  }
  float mx = kNegInf;
#pragma unroll
  for (int sp = 0; sp < kMaxVideoSplits; ++sp) mx = fmaxf(mx, l[sp]);
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (mx != kNegInf) {
    float wsum = 0.f;
#pragma unroll
    for (int sp = 0; sp < kMaxVideoSplits; ++sp) {
      if (l[sp] == kNegInf) continue;
      const float e = fast_exp2(l[sp] - mx);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[2 * i] += e * bf16_lo(w[sp][i]);
        acc[2 * i + 1] += e * bf16_hi(w[sp][i]);
      }
      wsum += e;
    }
    const float inv = 1.0f / wsum;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] *= inv;
  }
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = pack_bf16(acc[2 * i], acc[2 * i + 1]);
  *reinterpret_cast<u32x4*>(a.out + q * a.out_tok_stride + head * a.out_head_stride + d0) = o;
}

// The class table of the video CombineArgs, which is the first kernel
// argument of both merge kernels below, read in place.
__device__ __forceinline__ const_class_table combine_class_table() {
  const __attribute__((address_space(4))) char* seg =
      (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
  return (const_class_table)(seg + offsetof(CombineArgs, cls));
}

__global__ __launch_bounds__(256) void video_combine_kernel(const CombineArgs a) {
  video_combine_block(a, combine_class_table(), blockIdx.x);
}

// The merges of one step's video and audio calls in one launch: blocks below
// n_audio merge audio rows (they start first: their rows fold more ranges),
// the rest video rows.
__global__ __launch_bounds__(256) void step_combine_kernel(const CombineArgs v, const CombineArgs au,
                                                           int n_audio) {
  if (static_cast<int>(blockIdx.x) < n_audio)
    combine_block<3>(au, blockIdx.x);
  else
    video_combine_block(v, combine_class_table(), blockIdx.x - n_audio);
}

}  // namespace

// The no-allocation entry point's split-KV workspace.  Host code never
// passes this name to a kernel or a copy (in host code it is only a stand-in
// for the symbol): it uses the device address static_scratch() looks up.
static __device__ __align__(256) uint8_t scratch[kStaticScratchBytes];

hipError_t static_scratch(void** ptr) {
  constexpr int kMaxDevices = 64;
  static std::mutex mu;
  static void* addr[kMaxDevices] = {};
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (!addr[dev]) {
    void* p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return e;
    addr[dev] = p;
  }
  *ptr = addr[dev];
  return hipSuccess;
}

// With start or stop events, a launch goes through hipExtLaunchKernelGGL,
// whose events take the dispatch's own start and end timestamps (the
// kernel's execution, without the queue's event processing around it).
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream, hipEvent_t start, hipEvent_t stop) {
  const int tiles = a.n_blocks * a.num_heads;
  const int grid = std::min(tiles, std::max(1, a.grid_blocks));
  if (start || stop)
    hipExtLaunchKernelGGL(kv_append_kernel, dim3(grid), dim3(256), 0, stream, start, stop, 0, a);
  else
    hipLaunchKernelGGL(kv_append_kernel, dim3(grid), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_unit_attention(const AttnArgs& a, hipStream_t stream, hipEvent_t start, hipEvent_t stop) {
  const dim3 grid(a.n_wg), block(kVideoWaves * 64);
  const auto kernel = a.mode == 2 ? unit_attn_kernel : unit_attn_rows_kernel;
  if (start || stop)
    hipExtLaunchKernelGGL(kernel, grid, block, 0, stream, start, stop, 0, a);
  else
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_audio_attention(const AttnArgs& a, hipStream_t stream, hipEvent_t start, hipEvent_t stop) {
  const dim3 grid(a.num_heads * a.n_qtiles * a.n_splits);
  if (start || stop)
    hipExtLaunchKernelGGL(audio_attn_kernel, grid, dim3(256), 0, stream, start, stop, 0, a);
  else
    hipLaunchKernelGGL(audio_attn_kernel, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_step_combine(const CombineArgs& v, const CombineArgs& au, hipStream_t stream) {
  const int n_video = v.n_groups > 0 ? (v.num_heads * v.n_q + 15) / 16 : 0;
  const int n_audio = au.num_heads > 0 ? (au.num_heads * au.n_q + 15) / 16 : 0;
  if (n_video + n_audio == 0) return hipSuccess;
  hipLaunchKernelGGL(step_combine_kernel, dim3(n_video + n_audio), dim3(256), 0, stream, v, au, n_audio);
  return hipGetLastError();
}

hipError_t launch_combine(const CombineArgs& a, hipStream_t stream) {
  const int rows = a.num_heads * a.n_q;
  if (a.n_groups > 0)
    hipLaunchKernelGGL(video_combine_kernel, dim3((rows + 15) / 16), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(combine_kernel, dim3((rows + 15) / 16), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ws
