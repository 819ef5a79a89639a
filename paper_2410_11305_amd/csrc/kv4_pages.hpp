// Which pages of the 4-bit cache (kv4.hpp) a query is to read: bounds of each page's keys, and the choice of pages by them.
//
// Bounds.  Per page, key/value head and feature d the largest and the smallest key value of the page's tokens, U[d] and L[d], rounded
// outward to whole numbers of a grid e = 2^n, the smallest with max(|U|, |L|) <= 127 e over the features: 8 bits each.  For
// every token t of the page,
//   q . k[t] <= sum_d max(q[d] U[d], q[d] L[d]) = sum_d q+[d] U[d] + q-[d] L[d],     q+ = max(q, 0), q- = min(q, 0)
// which is a matrix product over 2 D features.  The rows of a query (its G heads that share a key/value head) are rounded to 8 bits, to nearest, on one
// grid of their own; the grid is the same for all pages, so its size does not matter for the choice.  The rounding does: a score can lie below what the
// unrounded query bounds, and of 32 pages of 512 (random keys of 128 features, one or eight heads) 98 to 99 % are those that unrounded queries choose.
//
// Everything that decides is a whole number times a power of two: the sums are below 2^21 and exact in any order, and so is their
// product with the grid in binary32.  Pages with equal scores are taken in their order.
//
// Layout: per page, Hkv rows of D upper and D lower codes (int8), then Hkv grids (binary32), filled up to 16 bytes.
#pragma once
#include "attn_kv4.hpp"
#include "common.hpp"
#include "kv4.hpp"

namespace qspec {

constexpr int kBlockTokens = 64;                       // of a page at least: a step of the attention lies inside one

__host__ __device__ inline size_t bounds_page_bytes(int Hkv, int D) { return (size_t)Hkv * 2 * D + (((size_t)Hkv * 4 + 15) & ~(size_t)15); }

// The smallest power of two with top <= 127 of it; 1 for zeros.
__device__ inline float grid_of(float top) {
  if (!(top > 0.0f)) return 1.0f;
  const int e = __builtin_amdgcn_frexp_expf(top);      // top = m 2^e, 1/2 <= m < 1
  return __builtin_amdgcn_ldexpf(1.0f, e - 7 + (__builtin_amdgcn_frexp_mantf(top) > 127.0f / 128.0f ? 1 : 0));
}

struct BoundsArgs {
  KvShape kv;
  const uint8_t* cache;
  uint8_t* bounds;
  int touched;               // pages that a sequence's rows can lie in
};

// The i-th page that rows pos .. pos + T - 1 lie in, and its tokens up to the last of them; tokens 0: there is none.
struct TouchedPage { int number, tokens; };
__device__ inline TouchedPage touched_page(const KvShape& kv, int b, int i) {
  const long long first = kv.pos[b], last = min(first + kv.T, (long long)kv.max_pages << kv.page_shift) - 1;
  const long long number = (max(first, 0LL) >> kv.page_shift) + i, from = number << kv.page_shift;
  if (from > last) return TouchedPage{0, 0};
  return TouchedPage{(int)number, (int)min(last + 1 - from, 1LL << kv.page_shift)};
}

// grid (B * touched, Hkv): a workgroup takes a page of a head.  A row of D/8 lanes reads a key, a code word a lane, 256 / (D/8) keys at
// a time; the folds over them stay in registers until the end.  The bounds are worked out anew from the page's codes, not carried on from what stands there:
// what a rejected draft left must go, and a page is 4 KB.  Bound by launch and latency (one page of 32 heads 3.2 us; 34 pages of 32 heads 5.6).
template <int D>
__global__ __launch_bounds__(256) void kv4_bounds_kernel(BoundsArgs p) {
  constexpr int LANES = D / 8, PER = 256 / LANES;
  __shared__ float tops[4][D], lows[4][D];
  __shared__ int odd_waves[4];
  const int b = blockIdx.x / p.touched, head = blockIdx.y;
  const TouchedPage here = touched_page(p.kv, b, blockIdx.x - b * p.touched);
  if (here.tokens == 0) return;
  const int page = kv_page(p.kv, b, (long long)here.number << p.kv.page_shift);
  if (page < 0) return;
  const int P = 1 << p.kv.page_shift, tid = threadIdx.x, w = tid & (LANES - 1);
  const uint8_t* const region = p.cache + ((size_t)page * p.kv.Hkv + head) * ((size_t)P * (D + 8));
  float hi[8], lo[8], odd = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) { hi[e] = -__builtin_inff(); lo[e] = __builtin_inff(); }
#pragma unroll 4
  for (int t = tid / LANES; t < here.tokens; t += PER) {
    const uint32_t word = reinterpret_cast<const uint32_t*>(region + (size_t)t * (D / 2))[w];
    const v2h par = *reinterpret_cast<const v2h*>(region + (size_t)P * D + (size_t)t * 8);
    const float step = (float)par.x, low = (float)par.y;
    odd += step * 0.0f + low * 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = fmaf((float)((word >> (4 * nibble_pos(e))) & 15u), step, low);
      hi[e] = fmaxf(hi[e], x);
      lo[e] = fminf(lo[e], x);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    hi[e] = column_max(hi[e]);
    lo[e] = -column_max(-lo[e]);
    if (LANES == 8) {
      hi[e] = fmaxf(hi[e], dpp_f32<0x128>(hi[e]));
      lo[e] = fminf(lo[e], dpp_f32<0x128>(lo[e]));
    }
  }
  const int wave = tid >> 6, lane = tid & 63;
  const bool any_odd = __builtin_amdgcn_ballot_w64(!(odd == 0.0f)) != 0;
  if (lane < LANES) {
#pragma unroll
    for (int e = 0; e < 8; ++e) { tops[wave][8 * w + e] = hi[e]; lows[wave][8 * w + e] = lo[e]; }
  }
  if (lane == 0) odd_waves[wave] = any_odd;
  __syncthreads();
  if (wave > 0) return;
  constexpr int EACH = D / 64;
  float up[EACH], down[EACH], top = 0.0f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int d = lane * EACH + i;
    up[i] = fmaxf(fmaxf(tops[0][d], tops[1][d]), fmaxf(tops[2][d], tops[3][d]));
    down[i] = fminf(fminf(lows[0][d], lows[1][d]), fminf(lows[2][d], lows[3][d]));
    top = fmaxf(top, fmaxf(fabsf(up[i]), fabsf(down[i])));
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  const bool number = (odd_waves[0] | odd_waves[1] | odd_waves[2] | odd_waves[3]) == 0;
  const float grid = grid_of(top), inverse = 1.0f / grid;        // (a power of two: exact)
  uint8_t* const out = p.bounds + (size_t)page * bounds_page_bytes(p.kv.Hkv, D);
  uint8_t* const row = out + (size_t)head * (2 * D);
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int d = lane * EACH + i;
    row[d] = number ? (uint8_t)(int8_t)(int)ceilf(up[i] * inverse) : 0;
    row[D + d] = number ? (uint8_t)(int8_t)(int)floorf(down[i] * inverse) : 0;
  }
  if (lane == 0) reinterpret_cast<float*>(out + (size_t)p.kv.Hkv * 2 * D)[head] = number ? grid : __builtin_nanf("");
}

struct BoundsReadArgs {
  KvShape kv;
  const uint8_t* bounds;
  float4* upper;             // [B][touched][Hkv][D]
  float4* lower;
  int touched;
};

// grid (B * touched, parts of Hkv D / 4): four features a thread, code * grid (34 pages of 32 heads 1.8 us: a launch)
template <int D>
__global__ __launch_bounds__(256) void kv4_bounds_read_kernel(BoundsReadArgs p) {
  const int i = blockIdx.y * 256 + threadIdx.x, head = i / (D / 4), d = i & (D / 4 - 1);
  if (head >= p.kv.Hkv) return;
  const int b = blockIdx.x / p.touched;
  const TouchedPage here = touched_page(p.kv, b, blockIdx.x - b * p.touched);
  const int page = here.tokens == 0 ? -1 : kv_page(p.kv, b, (long long)here.number << p.kv.page_shift);
  float4 hi = {0.0f, 0.0f, 0.0f, 0.0f}, lo = hi;
  if (page >= 0) {
    const uint8_t* const in = p.bounds + (size_t)page * bounds_page_bytes(p.kv.Hkv, D);
    const float grid = reinterpret_cast<const float*>(in + (size_t)p.kv.Hkv * 2 * D)[head];
    const uint32_t u = reinterpret_cast<const uint32_t*>(in + (size_t)head * (2 * D))[d], l = reinterpret_cast<const uint32_t*>(in + (size_t)head * (2 * D) + D)[d];
    const auto value = [&](uint32_t w, int n) { return (float)(int8_t)(w >> (8 * n)) * grid; };
    hi = float4{value(u, 0), value(u, 1), value(u, 2), value(u, 3)};
    lo = float4{value(l, 0), value(l, 1), value(l, 2), value(l, 3)};
  }
  const size_t o = (size_t)blockIdx.x * p.kv.Hkv * (D / 4) + i;
  p.upper[o] = hi;
  p.lower[o] = lo;
}

struct SelectArgs {
  KvShape kv;
  const uint16_t* q;         // fp16 [B][T][Hq][D]
  const uint8_t* bounds;
  uint32_t* keys;            // [B * T][Hkv][pitch]
  int32_t* pages;            // [B * T][Hkv][count]
  int Hq, G;
  int width, columns;        // log2 of the columns that a query's heads take in a block of 16, blocks of a workgroup
  int queries, sets, batch;  // queries of a workgroup, workgroups that a sequence's queries take, sequences
  int first, last, count;
  int pitch;
};
__host__ __device__ inline int select_row_keys(int max_pages) { return (max_pages + 63) & ~63; }

// Pages that row j of sequence b sees.
__device__ inline int pages_in_sight(const KvShape& kv, int b, int j) {
  const long long at = (long long)kv.pos[b] + j;
  return at < 0 ? 0 : (int)min(at >> kv.page_shift, (long long)kv.max_pages - 1) + 1;
}

// A score as a number that orders alike.  0: no such page;  the largest: one that is taken in any case;  below it: a page with a key that is
// no number, which must not be passed over.
constexpr uint32_t kKeyForced = 0xFFFFFFFFu, kKeyOdd = 0xFFFFFFFEu, kKeyNone = 0u;
__device__ inline uint32_t key_of(float score) {
  const uint32_t u = __builtin_bit_cast(uint32_t, score);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Largest over the 2^width neighbouring lanes of a row of 16 that hold a query's heads.
__device__ inline float head_max(float v, int width) {
  if (width > 0) v = fmaxf(v, dpp_f32<0xB1>(v));
  if (width > 1) v = fmaxf(v, dpp_f32<0x4E>(v));
  if (width > 2) v = fmaxf(v, dpp_f32<0x141>(v));
  if (width > 3) v = fmaxf(v, dpp_f32<0x140>(v));
  return v;
}
template <int CTRL>
__device__ inline int dpp_max(int v) { return max(v, __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false)); }
__device__ inline int head_max(int v, int width) {
  if (width > 0) v = dpp_max<0xB1>(v);
  if (width > 1) v = dpp_max<0x4E>(v);
  if (width > 2) v = dpp_max<0x141>(v);
  if (width > 3) v = dpp_max<0x140>(v);
  return v;
}

constexpr int kScoreColumns = 4;                       // blocks of 16 columns of a workgroup (as many as one query takes, where that is more)

// grid (B * sets * Hkv, chunks): a product of pages by heads over 2 D features, 16 by 16 a matrix instruction.  A query's heads take the next
// power of two of columns (repeating the last one), so their largest score is a fold in a row of lanes; more than 16 take several
// blocks.  The queries' codes are worked out once a workgroup and shared through LDS.  A wavefront runs through its pages 16 at a time, the next ones'
// bounds on their way; the heads of a sequence follow each other on one XCD, whose L2 then has the lines that they share (512 pages of 32 sequences and 8 heads: 12
// us for 16).  Bound by latency (position, table, bounds one after the other: 2048 pages of 8 heads 3.7 us), then by the loads of 260 bytes that lie 2 KB
// apart (128 queries of up to 512 pages: 21 MB in 10.4 us).  Runs of 64 pages with all their loads at once were slower (14): fewer wavefronts fit.
// Lane (row, k): row = lane & 15, 16 codes from 16 (lane >> 4) on in each 64.
template <int D>
__global__ __launch_bounds__(256) void kv4_score_kernel(SelectArgs p) {
  constexpr int NI = D / 64;                           // matrix instructions of a half
  extern __shared__ __align__(16) uint8_t score_lds[];       // [columns][2 NI][64] of 16 bytes
  v4i* const codes = reinterpret_cast<v4i*>(score_lds);
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 15, kb = lane >> 4;
  const uint32_t place = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);      // neighbours in one L2
  const int set = (int)(place / (uint32_t)p.kv.Hkv), head = (int)place - set * p.kv.Hkv, b = set / p.sets, j0 = (set - b * p.sets) * p.queries;
  if (b >= p.batch) return;
  const int queries = min(p.queries, p.kv.T - j0);
  const int n = pages_in_sight(p.kv, b, j0 + queries - 1);
  if (n <= p.count) return;                            // all of them are taken
  if ((int)blockIdx.y * 64 >= n) return;
  const size_t row_bytes = bounds_page_bytes(p.kv.Hkv, D);
  // ---- the bounds of 16 pages
  v4i u[NI], l[NI];
  float grid;                                          // of page i0 + col; below zero: there is none
  const auto load_pages = [&](int i0) {
    const int mine = i0 + col;
    const int page = mine < n ? kv_page(p.kv, b, (long long)mine << p.kv.page_shift) : -1;
    const uint8_t* const in = p.bounds + (size_t)max(page, 0) * row_bytes;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      u[i] = *reinterpret_cast<const v4i*>(in + (size_t)head * (2 * D) + 64 * i + 16 * kb);
      l[i] = *reinterpret_cast<const v4i*>(in + (size_t)head * (2 * D) + D + 64 * i + 16 * kb);
    }
    const float g = reinterpret_cast<const float*>(in + (size_t)p.kv.Hkv * 2 * D)[head];
    grid = page >= 0 ? g : -1.0f;
  };
  int i0 = (blockIdx.y * 4 + wave) * 16;
  load_pages(i0);                                      // (past the last page: there is none)
  // ---- the codes of the queries: block c by wavefront c % 4
  const int per = 16 >> p.width;                       // queries of a block, where they take one
  const auto load_row = [&](int c, uint4 (&x)[2 * NI]) {       // 16 features from 16 kb + 64 i on
    const int j = p.G > 16 ? 0 : min(c * per + (col >> p.width), queries - 1), g = p.G > 16 ? min(c * 16 + col, p.G - 1) : min(col & ((1 << p.width) - 1), p.G - 1);
    const uint16_t* const src = p.q + (((size_t)b * p.kv.T + j0 + j) * p.Hq + (size_t)head * p.G + g) * D + kb * 16;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      x[2 * i] = reinterpret_cast<const uint4*>(src + 64 * i)[0];
      x[2 * i + 1] = reinterpret_cast<const uint4*>(src + 64 * i)[1];
    }
  };
  const auto top_of = [&](const uint4 (&x)[2 * NI]) {          // of a block's queries; infinite where one feature is no finite number
    float top = 0.0f, odd = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * NI; ++i) {
      const v8h h = __builtin_bit_cast(v8h, x[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) { top = fmaxf(top, fabsf((float)h[e])); odd += (float)h[e] * 0.0f; }
    }
    return head_max(column_max(odd == 0.0f ? top : __builtin_inff()), p.width);
  };
  const int blocks = p.G > 16 ? p.columns : (queries + per - 1) / per;
  float all_heads = 0.0f;
  for (int c = 0; c < (p.G > 16 ? blocks : 0); ++c) {
    uint4 x[2 * NI];
    load_row(c, x);
    all_heads = fmaxf(all_heads, top_of(x));
  }
  for (int c = wave; c < blocks; c += 4) {
    uint4 x[2 * NI];
    load_row(c, x);
    const float top = p.G > 16 ? all_heads : top_of(x), inverse = top < __builtin_inff() ? 1.0f / grid_of(top) : 0.0f;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      v4i plus, minus;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const v8h h = __builtin_bit_cast(v8h, x[2 * i + w / 2]);
        uint32_t a = 0, m = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int k = inverse > 0.0f ? (int)rintf((float)h[4 * (w & 1) + e] * inverse) : 0;
          a |= (uint32_t)max(k, 0) << (8 * e);
          m |= ((uint32_t)min(k, 0) & 255u) << (8 * e);
        }
        plus[w] = (int)a;
        minus[w] = (int)m;
      }
      codes[(c * 2 * NI + i) * 64 + lane] = plus;
      codes[(c * 2 * NI + NI + i) * 64 + lane] = minus;
    }
  }
  __syncthreads();
  for (; i0 < n; i0 += gridDim.y * 64) {
    v4i now_u[NI], now_l[NI];
    float g4[4];                                       // of this lane's four pages
#pragma unroll
    for (int i = 0; i < NI; ++i) { now_u[i] = u[i]; now_l[i] = l[i]; }
#pragma unroll
    for (int r = 0; r < 4; ++r) g4[r] = __shfl(grid, 4 * kb + r);
    if (i0 + (int)gridDim.y * 64 < n) load_pages(i0 + gridDim.y * 64);
    v4i best = {};
    for (int c = 0; c < blocks; ++c) {
      v4i dot = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(now_u[i], codes[(c * 2 * NI + i) * 64 + lane], dot, 0, 0, 0);
        dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(now_l[i], codes[(c * 2 * NI + NI + i) * 64 + lane], dot, 0, 0, 0);
      }
      if (p.G > 16) {
#pragma unroll
        for (int r = 0; r < 4; ++r) best[r] = c == 0 ? dot[r] : max(best[r], dot[r]);
        if (c + 1 < blocks) continue;
        dot = best;
      }
      uint32_t key[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float score = (float)head_max(dot[r], p.width) * g4[r];
        key[r] = g4[r] < 0.0f ? kKeyNone : g4[r] == g4[r] ? key_of(score) : kKeyOdd;
      }
      const int j = p.G > 16 ? 0 : c * per + (col >> p.width);
      if ((col & ((1 << p.width) - 1)) == 0 && j < queries)      // (up to the end of 16 pages: rows have room for whole sets of 64)
        *reinterpret_cast<uint4*>(p.keys + (((size_t)b * p.kv.T + j0 + j) * p.kv.Hkv + head) * p.pitch + i0 + 4 * kb) = uint4{key[0], key[1], key[2], key[3]};
    }
  }
}

constexpr int kChooseThreads = 256, kChooseBins = 2048;        // (threads: where there are many pages)

// A wavefront's values folded up to and with each lane's: sums inside rows of 16 lanes, then the rows before.  NONE: what changes nothing.
template <uint32_t NONE, class Fold>
__device__ __forceinline__ uint32_t folded(uint32_t v, Fold fold) {
#define QSPEC_FOLD(ctrl, rows) v = fold(v, (uint32_t)__builtin_amdgcn_update_dpp((int)NONE, (int)v, ctrl, rows, 0xf, false))
  QSPEC_FOLD(0x111, 0xf);                              // row_shr 1, 2, 4, 8
  QSPEC_FOLD(0x112, 0xf);
  QSPEC_FOLD(0x114, 0xf);
  QSPEC_FOLD(0x118, 0xf);
  QSPEC_FOLD(0x142, 0xa);                              // row_bcast 15 into rows 1 and 3
  QSPEC_FOLD(0x143, 0xc);                              // row_bcast 31 into rows 2 and 3
#undef QSPEC_FOLD
  return v;
}
__device__ __forceinline__ uint32_t sum_up_to(uint32_t v) { return folded<0u>(v, [](uint32_t a, uint32_t b) { return a + b; }); }
__device__ __forceinline__ uint32_t last_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 63); }
__device__ __forceinline__ uint32_t least_of_wave(uint32_t v) { return last_lane(folded<0xFFFFFFFFu>(v, [](uint32_t a, uint32_t b) { return min(a, b); })); }
__device__ __forceinline__ uint32_t most_of_wave(uint32_t v) { return last_lane(folded<0u>(v, [](uint32_t a, uint32_t b) { return max(a, b); })); }
__device__ __forceinline__ uint32_t sum_of_wave(uint32_t v) { return last_lane(sum_up_to(v)); }

// Sum of v over the threads before this one, and over all.
template <int THREADS>
__device__ inline uint32_t scan_before(uint32_t v, uint32_t* waves, uint32_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t upto = sum_up_to(v);
  __syncthreads();                                     // (what an earlier scan left has been read)
  if (lane == 63) waves[wave] = upto;
  __syncthreads();
  uint32_t before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    before += w < wave ? waves[w] : 0u;
    all += waves[w];
  }
  return before + upto - v;
}

// The need-th key from the top of low .. low + 2^width - 1 narrowed down by a histogram over 2048 parts of that range, in `bins`: the part it lies
// in, which of its keys it is, and how many it has, in found.  A thread's own parts are neighbours, from the top.
template <int THREADS>
__device__ inline void find_part(const uint32_t* bins, uint32_t* waves, uint32_t* found, uint32_t need) {
  constexpr int OWN = kChooseBins / THREADS;
  const int from = kChooseBins - OWN * ((int)threadIdx.x + 1);
  uint32_t part[OWN], mine = 0, all;
#pragma unroll
  for (int k = 0; k < OWN; ++k) {
    part[k] = bins[from + OWN - 1 - k];
    mine += part[k];
  }
  uint32_t before = scan_before<THREADS>(mine, waves, all);
  if (before < need && before + mine >= need) {
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
      if (before < need && before + part[k] >= need) {
        found[0] = (uint32_t)(from + OWN - 1 - k);
        found[1] = need - before;
        found[2] = part[k];
      }
      before += part[k];
    }
  }
  __syncthreads();
}

// grid (B * T * Hkv), up to THREADS * KEYS pages: one row's `count` best pages, in their order.  A thread's keys stay in its registers, key k that of
// page THREADS k + thread.  One histogram over their range leaves few keys beside the one looked for, as a rule; these are ranked by comparing each with all.
// What is taken is written by its rank among the taken: their number in front of each set of 64 pages, and the lanes in front.
// Bound by the chain of steps and barriers (8 rows of 2048 pages 3.8 us, 1024 rows of up to 512 4.5).
template <int THREADS, int KEYS>
__global__ __launch_bounds__(THREADS) void kv4_choose_kernel(SelectArgs p) {
  constexpr int WAVES = THREADS / 64;
  constexpr int kList = 64;                            // keys that are ranked by comparing
  __shared__ __align__(16) uint32_t bins[kChooseBins];
  __shared__ uint32_t waves[WAVES], found[4], tops[3][WAVES], list_key[kList], list_page[kList], sets[KEYS * WAVES];
  const int row = blockIdx.x / p.kv.Hkv, b = row / p.kv.T, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = pages_in_sight(p.kv, b, row - b * p.kv.T);
  int32_t* const out = p.pages + (size_t)blockIdx.x * p.count;
  if (n <= p.count) {
    for (int i = tid; i < p.count; i += THREADS) out[i] = i < n ? i : -1;
    return;
  }
  const uint32_t* const keys = p.keys + (size_t)blockIdx.x * p.pitch;
  uint32_t key[KEYS];
#pragma unroll
  for (int k = 0; k < KEYS; ++k) key[k] = THREADS * k + tid < n ? keys[THREADS * k + tid] : 0u;
#pragma unroll
  for (int i = 0; i < kChooseBins / THREADS; ++i) bins[i * THREADS + tid] = 0u;
  uint32_t least = 0xFFFFFFFFu, most = 0u, odd = 0u, taken = 0u;      // taken: a bit a key
#pragma unroll
  for (int k = 0; k < KEYS; ++k) {
    const int i = THREADS * k + tid;
    const bool forced = i < p.first || i >= n - p.last, there = i < n;
    taken |= there && forced ? 1u << k : 0u;
    const uint32_t own = there && !forced ? key[k] : 0u;
    odd += own == kKeyOdd ? 1u : 0u;
    least = min(least, there && !forced ? own : 0xFFFFFFFFu);
    most = max(most, own < kKeyOdd ? own : 0u);
  }
  least = least_of_wave(least);
  most = most_of_wave(most);
  odd = sum_of_wave(odd);
  if (lane == 0) { tops[0][wave] = least; tops[1][wave] = most; tops[2][wave] = odd; }
  if (tid == 0) found[3] = 0u;
  __syncthreads();
  odd = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    least = min(least, tops[0][w]);
    most = max(most, tops[1][w]);
    odd += tops[2][w];
  }
  // The keys that may be taken: neither forced ones nor absent ones.  key >= low and < low + 2^width hold the need-th; larger ones are taken.
  uint32_t low = kKeyOdd, need = (uint32_t)(p.count - p.first - p.last), inside = odd;
  int width = 0;
  const auto open = [&](int k) { return THREADS * k + tid < n && !(taken >> k & 1u); };
  if (odd < need) {
    need -= odd;
    low = least;
    width = 32 - __builtin_clz(max(most - least, 1u));
    inside = 0xFFFFFFFFu;
    while (width > 0 && inside > (uint32_t)kList && inside != need) {
      const int shift = max(width - 11, 0);
      if (inside != 0xFFFFFFFFu) {                     // (the bins are clear the first time)
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kChooseBins / THREADS; ++i) bins[i * THREADS + tid] = 0u;
        __syncthreads();
      }
#pragma unroll
      for (int k = 0; k < KEYS; ++k) {
        if (!open(k) || key[k] < low || key[k] > most) continue;
        const uint32_t part = (key[k] - low) >> shift;
        if (part < 1u << (width - shift)) atomicAdd(&bins[part], 1u);
      }
      __syncthreads();
      find_part<THREADS>(bins, waves, found, need);
      low += found[0] << shift;
      need = found[1];
      inside = found[2];
      width = shift;
    }
  }
  // keys from low on that are inside: all of them taken (as many as are needed), equal to each other (width 0: the first of them), or few
  const uint32_t high = width < 32 ? low + (1u << width) - 1u : 0xFFFFFFFFu;      // (no range reaches past the largest number)
  const bool whole = inside == need, ranked = !whole && width > 0;
  uint32_t ties = 0u;
#pragma unroll
  for (int k = 0; k < KEYS; ++k) {
    if (!open(k) || need == 0) continue;
    const bool in = key[k] >= low && key[k] <= high;
    taken |= key[k] > high || (in && whole) ? 1u << k : 0u;
    ties |= in && !whole ? 1u << k : 0u;
  }
  if (ranked) {
#pragma unroll
    for (int k = 0; k < KEYS; ++k) {
      if (!(ties >> k & 1u)) continue;
      const uint32_t at = atomicAdd(&found[3], 1u);
      list_key[at] = key[k];
      list_page[at] = (uint32_t)(THREADS * k + tid);
    }
    __syncthreads();
    const uint32_t listed = found[3];
#pragma unroll
    for (int k = 0; k < KEYS; ++k) {
      if (!(ties >> k & 1u)) continue;
      uint32_t rank = 0;
#pragma unroll 8
      for (uint32_t i = 0; i < listed; ++i)
        rank += list_key[i] > key[k] || (list_key[i] == key[k] && list_page[i] < (uint32_t)(THREADS * k + tid)) ? 1u : 0u;
      taken |= rank < need ? 1u << k : 0u;
    }
    ties = 0u;
  }
  // ---- by rank: taken ones in the lower half of a word, ties in the upper
#pragma unroll
  for (int k = 0; k < KEYS; ++k) {
    const uint64_t a = __builtin_amdgcn_ballot_w64(taken >> k & 1u), t = __builtin_amdgcn_ballot_w64(ties >> k & 1u);
    if (lane == 0) sets[WAVES * k + wave] = (uint32_t)__builtin_popcountll(a) | (uint32_t)__builtin_popcountll(t) << 16;
  }
  __syncthreads();
  constexpr int EACH = (KEYS * WAVES + 63) / 64;           // sets of 64 pages a lane
  uint32_t mine[EACH], upto = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    mine[i] = lane * EACH + i < KEYS * WAVES ? sets[lane * EACH + i] : 0u;
    upto += mine[i];
  }
  const uint32_t before = sum_up_to(upto) - upto;
  const int first_set = uniform(wave);
#pragma unroll
  for (int k = 0; k < KEYS; ++k) {
    const int set = WAVES * k + first_set;
    uint32_t in_front = (uint32_t)__builtin_amdgcn_readlane((int)before, set / EACH);
#pragma unroll
    for (int i = 0; i + 1 < EACH; ++i) in_front += i < set % EACH ? (uint32_t)__builtin_amdgcn_readlane((int)mine[i], set / EACH) : 0u;
    const uint64_t a = __builtin_amdgcn_ballot_w64(taken >> k & 1u), t = __builtin_amdgcn_ballot_w64(ties >> k & 1u), lower = (1ull << lane) - 1;
    const uint32_t taken_before = (in_front & 0xFFFFu) + (uint32_t)__builtin_popcountll(a & lower), ties_before = (in_front >> 16) + (uint32_t)__builtin_popcountll(t & lower);
    const bool tie = (ties >> k & 1u) && ties_before < need;
    if ((taken >> k & 1u) || tie) out[taken_before + min(ties_before, need)] = THREADS * k + tid;
  }
}

// grid (B * T * Hkv), any number of pages: one row's `count` best pages, in their order.  The key that the last of them has is found by histograms over the range
// that is left, 2048 parts of it at a time; the pages with larger keys, and as many of those with that key as there is room for, are
// written by their rank.  (The keys do not fit the registers: they are read again in every step.)
__global__ __launch_bounds__(kChooseThreads) void kv4_choose_many_kernel(SelectArgs p) {
  __shared__ __align__(16) uint32_t bins[kChooseBins];
  __shared__ uint32_t waves[4], found[3];
  const int row = blockIdx.x / p.kv.Hkv, b = row / p.kv.T, tid = threadIdx.x;
  const int n = pages_in_sight(p.kv, b, row - b * p.kv.T);
  int32_t* const out = p.pages + (size_t)blockIdx.x * p.count;
  if (n <= p.count) {
    for (int i = tid; i < p.count; i += kChooseThreads) out[i] = i < n ? i : -1;
    return;
  }
  const uint32_t* const keys = p.keys + (size_t)blockIdx.x * p.pitch;
  const auto fetch = [&](int i) { return i < p.first || i >= n - p.last ? kKeyForced : keys[i]; };
  uint32_t least = 0xFFFFFFFFu, most = 0u, odd = 0u;
  for (int i = tid; i < n; i += kChooseThreads) {
    const uint32_t key = fetch(i);
    least = min(least, key);
    most = max(most, key < kKeyOdd ? key : 0u);
    odd += key == kKeyOdd ? 1u : 0u;
  }
  least = least_of_wave(least);
  most = most_of_wave(most);
  odd = sum_of_wave(odd);
  if ((tid & 63) == 0) { waves[tid >> 6] = least; bins[tid >> 6] = most; bins[4 + (tid >> 6)] = odd; }
  __syncthreads();
  least = min(min(waves[0], waves[1]), min(waves[2], waves[3]));
  most = max(max(bins[0], bins[1]), max(bins[2], bins[3]));
  odd = bins[4] + bins[5] + bins[6] + bins[7];
  // The key looked for is the need-th from the top of low .. low + 2^width - 1; larger ones are taken.  whole: all from low on are.
  const uint32_t forced = (uint32_t)(p.first + p.last), count = (uint32_t)p.count;       // (fewer than n)
  uint32_t low = kKeyOdd, need = count - forced;
  bool whole = false;
  if (need == 0) {
    low = kKeyForced;
    whole = true;
  } else if (odd < need) {
    low = least;
    need -= odd;
    int width = 32 - __builtin_clz(max(most - least, 1u));
    while (width > 0 && !whole) {
      const int shift = max(width - 11, 0);
      __syncthreads();
      for (int i = tid; i < kChooseBins; i += kChooseThreads) bins[i] = 0u;
      __syncthreads();
      for (int i = tid; i < n; i += kChooseThreads) {
        const uint32_t key = fetch(i);
        if (key < low || key > most) continue;
        const uint32_t part = (key - low) >> shift;
        if (part < 1u << (width - shift)) atomicAdd(&bins[part], 1u);
      }
      __syncthreads();
      find_part<kChooseThreads>(bins, waves, found, need);
      low += found[0] << shift;
      need = found[1];
      whole = found[2] == need;
      width = shift;
    }
  }
  // ---- by rank: a thread's neighbouring pages (an odd number of them: in banks of their own)
  const int per = ((n + kChooseThreads - 1) / kChooseThreads) | 1, begin = min(tid * per, n), end = min(begin + per, n);
  uint32_t larger = 0, equal = 0, all;
  for (int i = begin; i < end; ++i) {
    const uint32_t key = fetch(i);
    larger += key > low || (whole && key == low) ? 1u : 0u;
    equal += !whole && key == low ? 1u : 0u;
  }
  const uint32_t equal_before = scan_before<kChooseThreads>(equal, waves, all);
  uint32_t at = scan_before<kChooseThreads>(larger, waves, all) + min(equal_before, need), room = need - min(equal_before, need);
  for (int i = begin; i < end; ++i) {
    const uint32_t key = fetch(i);
    const bool tie = !whole && key == low && room > 0;
    if (tie) --room;
    if (tie || key > low || (whole && key == low)) out[at++] = i;
  }
}

}  // namespace qspec
