// Which pages of the 4-bit cache (kv4.hpp) a query is to read: bounds of each page's keys, and the choice of pages by them.
//
// Bounds.  Per page, key/value head and feature d the largest and the smallest key value of the page's tokens, U[d] and L[d], rounded
// outward to whole numbers of a grid e = 2^n, the smallest with max(|U|, |L|) <= 127 e over the features: 8 bits each.  For
// every token t of the page,
//   q . k[t] <= sum_d max(q[d] U[d], q[d] L[d]) = sum_d q+[d] U[d] + q-[d] L[d],     q+ = max(q, 0), q- = min(q, 0)
// which is a matrix product over 2 D features.  The rows of a query (its G heads that share a key/value head) are rounded to 8 bits on one
// grid of their own, the same for all pages, so it does not matter for the choice.
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
// a time; the folds over them stay in registers until the end.
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

// grid (B * touched, parts of Hkv D / 4): four features a thread, code * grid
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
  int queries, sets;         // queries of a block of 16 columns, blocks of a sequence
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

// grid (B * sets * Hkv, chunks): 16 pages and 16 columns (heads of `queries` queries, or 16 of one query's heads at a time) a
// wavefront, one matrix product over 2 D features.  Lane (row, k): row = lane & 15, 16 codes from 16 (lane >> 4) on in each of the 64.
template <int D>
__global__ __launch_bounds__(256) void kv4_score_kernel(SelectArgs p) {
  constexpr int NI = D / 64;                           // matrix instructions of a half
  __shared__ int dots[4][16][17];
  __shared__ float tops[4][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 15, kb = lane >> 4;
  const int head = blockIdx.x % p.kv.Hkv, set = blockIdx.x / p.kv.Hkv, b = set / p.sets, j0 = (set - b * p.sets) * p.queries;
  const int queries = min(p.queries, p.kv.T - j0);
  const int n = pages_in_sight(p.kv, b, j0 + queries - 1);
  if (n <= p.count) return;                            // all of them are taken
  int i0 = (blockIdx.y * 4 + wave) * 16;
  if (i0 >= n) return;                                 // (wavefronts are on their own from here on)
  const int passes = (min(p.queries, 16) * p.G + 15) / 16;       // of the heads: one, or one query's in sets of 16
  const int columns = queries * p.G;
  typedef uint4 Rows[2 * NI];
  const auto load = [&](int pass, Rows& x) {           // 16 features from 16 kb + 64 i on
    const int c = min(pass * 16 + col, columns - 1), j = c / p.G, g = c - j * p.G;
    const uint16_t* const src = p.q + (((size_t)b * p.kv.T + j0 + j) * p.Hq + (size_t)head * p.G + g) * D + kb * 16;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      x[2 * i] = reinterpret_cast<const uint4*>(src + 64 * i)[0];
      x[2 * i + 1] = reinterpret_cast<const uint4*>(src + 64 * i)[1];
    }
  };
  // ---- the grid of each query
  Rows x;
  for (int pass = 0; pass < passes; ++pass) {
    load(pass, x);
    float top = 0.0f, odd = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * NI; ++i) {
      const v8h h = __builtin_bit_cast(v8h, x[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) { top = fmaxf(top, fabsf((float)h[e])); odd += (float)h[e] * 0.0f; }
    }
    top = odd == 0.0f ? top : __builtin_inff();
    top = column_max(top);
    if (kb == 0) tops[wave][pass * 16 + col] = top;
  }
  wave_lds_order();
  const auto inverse_of = [&](int pass) {              // of a column's query: 1 / grid, or 0 for one that holds what is no number
    const int c = min(pass * 16 + col, columns - 1), j = c / p.G;
    float top = 0.0f;
    for (int g = 0; g < p.G; ++g) top = fmaxf(top, tops[wave][j * p.G + g]);
    return top < __builtin_inff() ? 1.0f / grid_of(top) : 0.0f;
  };
  const auto codes = [&](const Rows& x, float inverse, v4i (&plus)[NI], v4i (&minus)[NI]) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const v8h h = __builtin_bit_cast(v8h, x[2 * i + w / 2]);
        uint32_t a = 0, m = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float f = (float)h[4 * (w & 1) + e];
          const int c = inverse > 0.0f ? (int)rintf(f * inverse) : 0;
          a |= (uint32_t)max(c, 0) << (8 * e);
          m |= ((uint32_t)min(c, 0) & 255u) << (8 * e);
        }
        plus[i][w] = (int)a;
        minus[i][w] = (int)m;
      }
    }
  };
  v4i plus[NI], minus[NI];
  if (passes == 1) codes(x, inverse_of(0), plus, minus);
  const size_t row_bytes = bounds_page_bytes(p.kv.Hkv, D);
  for (; i0 < n; i0 += gridDim.y * 64) {
    // ---- the bounds of 16 pages
    const int mine = i0 + col;
    const int page = mine < n ? kv_page(p.kv, b, (long long)mine << p.kv.page_shift) : -1;
    const uint8_t* const in = p.bounds + (size_t)max(page, 0) * row_bytes;
    v4i u[NI], l[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      u[i] = *reinterpret_cast<const v4i*>(in + (size_t)head * (2 * D) + 64 * i + 16 * kb);
      l[i] = *reinterpret_cast<const v4i*>(in + (size_t)head * (2 * D) + D + 64 * i + 16 * kb);
    }
    const float grid = page >= 0 ? reinterpret_cast<const float*>(in + (size_t)p.kv.Hkv * 2 * D)[head] : 0.0f;
    int best = -0x7fffffff;                            // (several passes: of one query)
    for (int pass = 0; pass < passes; ++pass) {
      if (passes > 1) {
        load(pass, x);
        codes(x, inverse_of(pass), plus, minus);
      }
      v4i dot = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(u[i], plus[i], dot, 0, 0, 0);
        dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(l[i], minus[i], dot, 0, 0, 0);
      }
      wave_lds_order();
#pragma unroll
      for (int r = 0; r < 4; ++r) dots[wave][4 * kb + r][col] = dot[r];
      wave_lds_order();
      if (passes > 1) {
        for (int c = 0; c < min(16, columns - pass * 16); ++c) best = max(best, dots[wave][col][c]);
      }
    }
    // ---- the best of a query's heads: lane (page, query)
    for (int j = kb; j < queries; j += 4) {
      if (passes == 1) {
        best = dots[wave][col][j * p.G];
        for (int g = 1; g < p.G; ++g) best = max(best, dots[wave][col][j * p.G + g]);
      }
      const uint32_t key = page < 0 ? kKeyNone : grid == grid ? key_of((float)best * grid) : kKeyOdd;
      if (mine < n) p.keys[(((size_t)b * p.kv.T + j0 + j) * p.kv.Hkv + head) * p.pitch + mine] = key;
    }
    wave_lds_order();
  }
}

constexpr int kChooseThreads = 256, kChooseKeys = 8192, kChooseBins = 2048;

// Sum of v over the threads before this one, and over all.
__device__ inline uint32_t scan_before(uint32_t v, uint32_t* waves, uint32_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t upto = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t other = __shfl_up(upto, d);
    upto += lane >= d ? other : 0u;
  }
  __syncthreads();                                     // (what an earlier scan left has been read)
  if (lane == 63) waves[wave] = upto;
  __syncthreads();
  uint32_t before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kChooseThreads / 64; ++w) {
    before += w < wave ? waves[w] : 0u;
    all += waves[w];
  }
  return before + upto - v;
}

// grid (B * T * Hkv): one row's `count` best pages, in their order.  The key that the last of them has is found by histograms over the range
// that is left, 2048 parts of it at a time; the pages with larger keys, and as many of those with that key as there is room for, are
// written by their rank.
__global__ __launch_bounds__(kChooseThreads) void kv4_choose_kernel(SelectArgs p) {
  __shared__ __align__(16) uint32_t held[kChooseKeys];
  __shared__ uint32_t bins[kChooseBins], waves[4], found[3];
  const int row = blockIdx.x / p.kv.Hkv, b = row / p.kv.T, tid = threadIdx.x;
  const int n = pages_in_sight(p.kv, b, row - b * p.kv.T);
  int32_t* const out = p.pages + (size_t)blockIdx.x * p.count;
  if (n <= p.count) {
    for (int i = tid; i < p.count; i += kChooseThreads) out[i] = i < n ? i : -1;
    return;
  }
  const uint32_t* const keys = p.keys + (size_t)blockIdx.x * p.pitch;
  const auto fetch = [&](int i) { return i < p.first || i >= n - p.last ? kKeyForced : keys[i]; };
  const bool fits = n <= kChooseKeys;
  uint32_t least = 0xFFFFFFFFu, most = 0u, odd = 0u;
  for (int i = tid; i < n; i += kChooseThreads) {
    const uint32_t key = fetch(i);
    if (fits) held[i] = key;
    least = min(least, key);
    most = max(most, key < kKeyOdd ? key : 0u);
    odd += key == kKeyOdd ? 1u : 0u;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    least = min(least, (uint32_t)__shfl_xor((int)least, d));
    most = max(most, (uint32_t)__shfl_xor((int)most, d));
    odd += (uint32_t)__shfl_xor((int)odd, d);
  }
  if ((tid & 63) == 0) { waves[tid >> 6] = least; bins[tid >> 6] = most; bins[4 + (tid >> 6)] = odd; }
  __syncthreads();
  least = min(min(waves[0], waves[1]), min(waves[2], waves[3]));
  most = max(max(bins[0], bins[1]), max(bins[2], bins[3]));
  odd = bins[4] + bins[5] + bins[6] + bins[7];
  const auto key_at = [&](int i) { return fits ? held[i] : fetch(i); };
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
        const uint32_t key = key_at(i);
        if (key < low || key > most) continue;
        const uint32_t part = (key - low) >> shift;
        if (part < 1u << (width - shift)) atomicAdd(&bins[part], 1u);
      }
      __syncthreads();
      uint32_t mine = 0, all;                          // a thread's 8 parts, from the top
#pragma unroll
      for (int k = 0; k < 8; ++k) mine += bins[kChooseBins - 1 - (8 * tid + k)];
      uint32_t before = scan_before(mine, waves, all);
      if (before < need && before + mine >= need) {
        for (int k = 0; k < 8; ++k) {
          const uint32_t part = (uint32_t)(kChooseBins - 1 - (8 * tid + k)), c = bins[part];
          if (before < need && before + c >= need) {
            found[0] = part;
            found[1] = need - before;
            found[2] = c;
          }
          before += c;
        }
      }
      __syncthreads();
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
    const uint32_t key = key_at(i);
    larger += key > low || (whole && key == low) ? 1u : 0u;
    equal += !whole && key == low ? 1u : 0u;
  }
  const uint32_t equal_before = scan_before(equal, waves, all);
  uint32_t at = scan_before(larger, waves, all) + min(equal_before, need), room = need - min(equal_before, need);
  for (int i = begin; i < end; ++i) {
    const uint32_t key = key_at(i);
    const bool tie = !whole && key == low && room > 0;
    if (tie) --room;
    if (tie || key > low || (whole && key == low)) out[at++] = i;
  }
}

}  // namespace qspec
