// Key/value cache held in 4 bits: its layout, rotary positions with the append to it, and reading it back.
//
// Quantisation, per token and head over its D features (asymmetric: the rotated keys of a token are far from
// symmetric, and the extra fp16 per row is 3 % of it), everything that decides a code exact:
//   low = min x, step = fp16((max x - low) / 15), code = clamp(rne((x - low) / step), 0, 15); step 0 gives codes 0
// A value is code * step + low.  A row that holds a NaN or an infinity has NaN for step and low and codes 0: none of its values is a number.
//
// A page holds P tokens of every key/value head; per head, one region of P (D + 8) bytes:
//   keys    P rows of D/2 bytes, word w holding features 8w .. 8w+7
//   values  P/16 tiles of 8 D bytes: word w (features 8w .. 8w+7) of token t of the tile at word w * 16 + t
//   rows    P times {key step, key low, value step, value low}, fp16
// Codes of a word stand in the order of nibble_pos.  Both products of the attention contract over what a lane can load
// in 16 bytes: features of one token for q k^T, four tokens of one word for p v.
#pragma once
#include "common.hpp"
#include "producers.hpp"
#include "quant_act.hpp"

namespace qspec {

struct KvShape {
  const int32_t* pos;        // [B]: position of each sequence's first row of this call
  const int32_t* table;      // [B][max_pages], or null: sequence b holds pages b * max_pages ..
  int T, Hkv, page_shift, max_pages, n_pages;
};

// 4-byte values that no launch in flight writes, at an address the whole wavefront shares: a scalar load
typedef const __attribute__((address_space(4))) int32_t* scalar_i32_ptr;
__device__ __forceinline__ int32_t scalar_load(const int32_t* p, size_t i) { return ((scalar_i32_ptr)(uintptr_t)p)[i]; }

// Page of position at of sequence b, or -1 where there is none (positions outside the sequence's pages, table
// entries outside the cache).
__device__ __forceinline__ int kv_page(const KvShape& s, int b, long long at) {
  if (at < 0 || (at >> s.page_shift) >= s.max_pages) return -1;
  const size_t i = (size_t)b * s.max_pages + (size_t)(at >> s.page_shift);
  const int page = s.table != nullptr ? s.table[i] : (int)i;
  return page >= 0 && page < s.n_pages ? page : -1;
}

// A binary64 value (NaN: an infinity) to fp16 in one rounding: cut to 20 bits of significand with a last bit that remembers what was
// cut off (9 bits more than fp16 has; round to odd), put together as binary32, then to nearest even.  Whole-number operations: the
// conversions from and to binary64 take four times as long as any of them.
__device__ inline _Float16 half_of_f64(double v) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t high = (uint32_t)(bits >> 32) | min((uint32_t)bits, 1u);
  // exponents below binary32's become zero, exponents past fp16's stay past them
  const int magnitude = min(max((int)(high & 0x7FFFFFFFu) - (896 << 20), 0), 200 << 20);
  return (_Float16)__builtin_bit_cast(float, (high & 0x80000000u) | (uint32_t)magnitude << 3);
}

// A value in fp16.  A step that was rounded up can carry the 15th code of a row that fills fp16's range past its end: the largest finite
// value then.  What is no number, or infinite, stays so.
__device__ __forceinline__ _Float16 held_to_half(float x) {
  return (_Float16)(fabsf(x) < __builtin_inff() ? fminf(fmaxf(x, -65504.0f), 65504.0f) : x);
}

// cos and sin of `turns` whole turns, to a few units in the last place of binary64: the nearest quarter turn off, then
// the Taylor series on +-pi/4 (the first terms left out are below 2^-58).
__device__ inline void cos_sin_turns(double turns, double& c, double& s) {
  const double r = turns - rint(turns);
  const double quarter = rint(r * 4.0);
  const double y = fma(quarter, -0.25, r) * 6.283185307179586477;
  const double z = y * y;
  double ps = 1.0 / 355687428096000.0;
  ps = fma(ps, z, -1.0 / 1307674368000.0);
  ps = fma(ps, z, 1.0 / 6227020800.0);
  ps = fma(ps, z, -1.0 / 39916800.0);
  ps = fma(ps, z, 1.0 / 362880.0);
  ps = fma(ps, z, -1.0 / 5040.0);
  ps = fma(ps, z, 1.0 / 120.0);
  ps = fma(ps, z, -1.0 / 6.0);
  const double sy = fma(ps * z, y, y);
  double pc = 1.0 / 20922789888000.0;
  pc = fma(pc, z, -1.0 / 87178291200.0);
  pc = fma(pc, z, 1.0 / 479001600.0);
  pc = fma(pc, z, -1.0 / 3628800.0);
  pc = fma(pc, z, 1.0 / 40320.0);
  pc = fma(pc, z, -1.0 / 720.0);
  pc = fma(pc, z, 1.0 / 24.0);
  pc = fma(pc, z, -0.5);
  const double cy = fma(pc, z, 1.0);
  const int q = (int)quarter & 3;
  const double u = (q & 1) ? sy : cy, v = (q & 1) ? cy : sy;
  c = (q == 1 || q == 2) ? -u : u;
  s = (q & 2) ? -v : v;
}

struct AppendArgs {
  KvShape kv;
  const uint4* qkv;          // fp16 [B*T][(Hq + 2 Hkv) D]
  const double* inv_freq;    // [rot/2], radians per position
  uint4* q;                  // fp16 [B*T][Hq D]
  uint8_t* cache;
  int Hq, rot, interleaved;
  float mscale;
};

// Largest and smallest of a head's values, over the row of LANES = D / 8 lanes that holds it.
template <int LANES>
__device__ inline float row_max(float a) {
  a = fmaxf(a, dpp_f32<0xB1>(a));
  a = fmaxf(a, dpp_f32<0x4E>(a));
  a = fmaxf(a, dpp_f32<0x141>(a));
  if (LANES == 16) a = fmaxf(a, dpp_f32<0x140>(a));
  return a;
}

// Code word of 8 values of a head, and the head's step and minimum.  A quotient in binary32 is off by less than 2^-18; where one of the
// 8 lies nearer to half way between two integers than that, all are formed in binary64, where the difference of two
// fp16 values is exact and a quotient that is not itself half way is far enough from it to stay on its side.
template <int LANES>
__device__ inline uint32_t kv_code_word(const float (&v)[8], _Float16& step, _Float16& low) {
  float hi = v[0], lo = v[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) { hi = fmaxf(hi, v[e]); lo = fminf(lo, v[e]); }
  hi = row_max<LANES>(hi) + 0.0f;                           // (a zero is +0, here and in the step)
  lo = -row_max<LANES>(-lo) + 0.0f;
  low = (_Float16)lo;                                       // exact: one of the values
  // a fifteenth: one remainder step from the rounded reciprocal (halves of fp16 units come out exactly)
  const double range = (double)hi - (double)lo, fifteenth = range * (1.0 / 15.0);
  step = half_of_f64(fma(fma(-15.0, fifteenth, range), 1.0 / 15.0, fifteenth));
  const float s = (float)step;
  if (!(s > 0.0f)) return 0u;
  const float y = 1.0f / s;
  uint32_t w = 0;
  float nearest = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = (v[e] - lo) * y, t = rintf(q);
    nearest = fmaxf(nearest, fabsf(q - t));
    w |= (uint32_t)fminf(t, 15.0f) << (4 * nibble_pos(e));
  }
  if (nearest > 0.49999f) {
    const double s64 = (double)s, lo64 = (double)lo;
    double y64 = __builtin_amdgcn_rcp(s64);
    y64 = fma(fma(-s64, y64, 1.0), y64, y64);
    y64 = fma(fma(-s64, y64, 1.0), y64, y64);
    w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double d = (double)v[e] - lo64;
      double t = d * y64;
      t = fma(fma(-t, s64, d), y64, t);
      w |= (uint32_t)min((int)rint(t), 15) << (4 * nibble_pos(e));
    }
  }
  return w;
}

// grid (B*T, parts): a workgroup takes one token and every parts-th set of 256 / (D/8) of its Hq + 2 Hkv heads, a row of D/8
// lanes a head, 8 features a lane: 16 bytes in, a code word out, and the folds over a head stay in a row of lanes.  The angles
// of a token are worked out once a workgroup.  Measured: 2050 tokens of 32 heads and 32 key/value heads of 128 25 us, the vector unit at 54 % of its
// cycles.  The binary64 rotation and the stores share the bound: a token's value words lie 64 bytes apart and each costs a sector of 32, 58 MB
// written where 26 are needed.  512 tokens of 64 and 8 heads 9.1 us (10.9 MB written for 9.0), one token 3.7 us, a launch and four dependent trips to memory.
template <int D>
__global__ __launch_bounds__(256) void rope_kv4_append_kernel(AppendArgs p) {
  constexpr int LANES = D / 8, PER = 256 / LANES;
  __shared__ double2 turn[D / 2];                           // cos, sin of each pair's angle, times mscale
  const int token = blockIdx.x, b = token / p.kv.T, j = token - b * p.kv.T;
  const int l = threadIdx.x & (LANES - 1);
  const int heads = p.Hq + 2 * p.kv.Hkv;
  const int half = p.rot >> 1;
  const bool in_rot = 8 * l < p.rot, upper = 8 * l >= half;
  const uint4* const rows = p.qkv + (size_t)token * heads * LANES + l;
  const int partner = in_rot && !p.interleaved ? (upper ? -(half >> 3) : half >> 3) : 0;
  int head = blockIdx.y * PER + (int)threadIdx.x / LANES;
  uint4 mine = rows[(size_t)min(head, heads - 1) * LANES], other = rows[(size_t)min(head, heads - 1) * LANES + partner];
  const long long at = (long long)p.kv.pos[b] + j;
  const int page = kv_page(p.kv, b, at);
  if ((int)threadIdx.x < half) {
    double c, s;
    cos_sin_turns((double)at * (p.inv_freq[threadIdx.x] * 0.15915494309189533577), c, s);
    turn[threadIdx.x] = double2{c * (double)p.mscale, s * (double)p.mscale};
  }
  __syncthreads();
  const int P = 1 << p.kv.page_shift, slot = (int)(at & (P - 1));
  uint8_t* const regions = p.cache + (size_t)max(page, 0) * p.kv.Hkv * ((size_t)P * (D + 8));
  for (int base = blockIdx.y * PER; base < heads; base += gridDim.y * PER) {
    const v8h x = __builtin_bit_cast(v8h, mine), z = __builtin_bit_cast(v8h, other);
    const int now = head, next = min(head + (int)gridDim.y * PER, heads - 1);
    head += gridDim.y * PER;
    mine = rows[(size_t)next * LANES];                      // (the last one's loads repeat a head)
    other = rows[(size_t)next * LANES + partner];
    v8h h = x;
    if (in_rot && now < p.Hq + p.kv.Hkv) {
      if (p.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const double2 t = turn[4 * l + e / 2];
          const double a = (double)(float)x[e], c = (double)(float)x[e + 1];
          h[e] = half_of_f64(a * t.x - c * t.y);
          h[e + 1] = half_of_f64(c * t.x + a * t.y);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double2 t = turn[8 * l + e - (upper ? half : 0)];
          const double a = (double)(float)x[e], c = (double)(float)z[e];
          h[e] = half_of_f64(a * t.x + (upper ? c : -c) * t.y);
        }
      }
    }
    // What is no finite number: a lane that has any, of the whole wavefront.  Rare, so what has to be done about it stands apart.
    const v2h nothing = {(_Float16)0.0f, (_Float16)0.0f};
    float odd = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) odd = __builtin_amdgcn_fdot2(v2h{h[e], h[e + 1]}, nothing, odd, false);
    const uint64_t odd_lanes = __builtin_amdgcn_ballot_w64(!(odd == 0.0f));
    if (odd_lanes != 0 && in_rot && now < p.Hq + p.kv.Hkv) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {                         // (rounding has made infinities of the NaN among them)
        const double2 t = turn[p.interleaved ? 4 * l + e / 2 : 8 * l + e - (upper ? half : 0)];
        const double a = (double)(float)x[e], c = (double)(float)(p.interleaved ? x[e ^ 1] : z[e]);
        const double r = a * t.x + ((p.interleaved ? (e & 1) != 0 : upper) ? c : -c) * t.y;
        h[e] = r == r ? h[e] : (_Float16)__builtin_nanf("");
      }
    }
    if (now < p.Hq) p.q[((size_t)token * p.Hq + now) * LANES + l] = __builtin_bit_cast(uint4, h);
    if (now >= p.Hq && now < heads) {                       // (whole rows of lanes: the folds see each other)
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
      _Float16 step, low;
      uint32_t word = kv_code_word<LANES>(v, step, low);
      if (odd_lanes != 0 && (odd_lanes >> (threadIdx.x & 63 & ~(LANES - 1)) & ((1u << LANES) - 1)) != 0) {      // in one of the row's lanes
        word = 0u;
        step = low = __builtin_bit_cast(_Float16, (uint16_t)0x7E00);
      }
      if (page >= 0) {
        const bool value = now >= p.Hq + p.kv.Hkv;
        uint8_t* const region = regions + (size_t)(now - p.Hq - (value ? p.kv.Hkv : 0)) * ((size_t)P * (D + 8));
        uint32_t* const place = value ? reinterpret_cast<uint32_t*>(region + (size_t)P * (D / 2) + (size_t)(slot >> 4) * (8 * D)) + l * 16 + (slot & 15)
                                      : reinterpret_cast<uint32_t*>(region + (size_t)slot * (D / 2)) + l;
        *place = word;
        if (l == 0) *reinterpret_cast<v2h*>(region + (size_t)P * D + (size_t)slot * 8 + (value ? 4 : 0)) = v2h{step, low};
      }
    }
  }
}

struct KvReadArgs {
  KvShape kv;
  const uint8_t* cache;
  uint4* k;                  // fp16 [B*T][Hkv D]
  uint4* v;
};

// 8 codes of a word times step plus low, each rounded once to binary32 and once to fp16.
__device__ inline v8h kv_values(uint32_t w, _Float16 step, _Float16 low) {
  v8h h;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    h[e] = held_to_half(rounded_f32(fmaf((float)((w >> (4 * nibble_pos(e))) & 15u), (float)step, (float)low)));
  }
  return h;
}

// grid (B*T, parts of Hkv D / 8 words of a token).  A copy that widens 4 bits to 16: memory bounds it (2050 tokens of 32
// heads of 128: 51 MB in 13 us, 3.9 TB/s; one token 2.4 us, a launch).  Rows without a place in the cache come back as zeros.
template <int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(KvReadArgs p) {
  constexpr int LANES = D / 8;
  const int token = blockIdx.x, b = token / p.kv.T;
  const int i = blockIdx.y * 256 + threadIdx.x, head = i / LANES, w = i & (LANES - 1);
  if (head >= p.kv.Hkv) return;
  const long long at = (long long)p.kv.pos[b] + (token - b * p.kv.T);
  const int page = kv_page(p.kv, b, at);
  const size_t o = ((size_t)token * p.kv.Hkv + head) * LANES + w;
  if (page < 0) {
    p.k[o] = p.v[o] = uint4{0u, 0u, 0u, 0u};
    return;
  }
  const int P = 1 << p.kv.page_shift, slot = (int)(at & (P - 1));
  const uint8_t* const region = p.cache + ((size_t)page * p.kv.Hkv + head) * ((size_t)P * (D + 8));
  typedef _Float16 v4h __attribute__((ext_vector_type(4)));
  const v4h par = *reinterpret_cast<const v4h*>(region + (size_t)P * D + (size_t)slot * 8);
  const uint32_t kw = reinterpret_cast<const uint32_t*>(region + (size_t)slot * (D / 2))[w];
  const uint32_t vw = reinterpret_cast<const uint32_t*>(region + (size_t)P * (D / 2) + (size_t)(slot >> 4) * (8 * D))[w * 16 + (slot & 15)];
  p.k[o] = __builtin_bit_cast(uint4, kv_values(kw, par.x, par.y));
  p.v[o] = __builtin_bit_cast(uint4, kv_values(vw, par.z, par.w));
}

}  // namespace qspec
