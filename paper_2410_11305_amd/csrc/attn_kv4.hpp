// Attention over the 4-bit cache (layout and quantisation: kv4.hpp):
//   o[r] = sum_t softmax_t(scale q[r] . k[t]) v[t],   k[t] = code * step + low, likewise v
// over the tokens t that row r sees.  One pass over the cache with a running reference m and sums of 2^(s - m).
//
// The rows that share a key/value head (T tokens times G query heads) fill the columns of the matrix instructions,
// 16 to a block, so a code is loaded and widened once for all of them.  Both products run on the bare codes:
//   s[t, r] = step_k[t] (code_k[t] . q[r]) + low_k[t] sum(q[r])
//   o[r]    = sum_t w[t, r] code_v[t] - 8 sum_t w[t, r] + sum_t p[t, r] (low_v[t] + 8 step_v[t]),   w = fp16(p step_v)
// (the middle term takes the same rounded weights as the first, so that their rounding meets a code about its middle
// and not one of 0 to 15: half the error).
// A masked nibble in the low bits of a half word IS an fp16 number, code * 2^-24 or 16 * code * 2^-24 (subnormal: exact
// in the matrix unit, which keeps subnormal operands), so widening a word of 8 codes takes 5 bit operations; the
// factor of 16 is taken out of q (a power of two that q's row is scaled by first, so that nothing is lost) and out of
// the finished sums.  The token order of the second product is that of the first one's results: p goes from the
// accumulators into the next operand without crossing lanes, and a lane's codes of four tokens are 16 bytes of the
// cache (kv4.hpp).
//
// Work: an item is one block of rows of one sequence and one key/value head, a step 32 tokens.  The workgroups share
// the steps of all items evenly, whatever the lengths, each taking one run of them; the wavefronts of a workgroup
// take its steps in turn and join their sums through LDS.  An item that several workgroups share is joined by the last of them
// to finish (last_arrival), from partial sums in the workspace.  The lengths are known on the device only: every
// workgroup works the division out for itself.
#pragma once
#include "common.hpp"
#include "exchange.hpp"
#include "kv4.hpp"

namespace qspec {

constexpr int kAttnStep = 32;                // tokens
constexpr int kAttnWhole = 16;               // items of up to so many steps are not shared out
constexpr int kAttnMinSteps = 8;             // a workgroup is not given fewer steps on average
constexpr int kAttnMaxWorkgroups = 512;
constexpr size_t kAttnTicketBytes = 16384;   // arrival counters at the head of the workspace

// Wavefronts of a workgroup, by blocks of 16 rows that each of them carries.
__host__ __device__ constexpr int attn_waves(int nb) { return nb == 1 ? 8 : 4; }

struct AttnArgs {
  KvShape kv;
  const uint16_t* q;         // fp16 [B][T][Hq][D]
  const uint8_t* cache;
  uint16_t* out;             // fp16 [B][T][Hq][D]
  unsigned* tickets;
  float* parts;
  int B, Hq, G, blocks;      // blocks: blocks of rows of a sequence
  uint32_t G_inverse;        // ceil(2^32 / G) for G > 1: r / G is the upper half of r * G_inverse while r G < 2^32
  int window, sinks;
  float scale_log2;          // scale * log2(e)
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

__device__ __forceinline__ int over_group(const AttnArgs& p, int r) { return p.G == 1 ? r : (int)__umulhi((uint32_t)r, p.G_inverse); }

// What one block of rows reads: sink steps from token 0 on, then the others from step `first` on.
struct AttnSpan {
  int steps, sink_steps, first;
  int lo, hi;                // positions of its first and its last row
};

// pos: position of the sequence's first row.  (Held to +-2^30, far outside of any cache, so that sums stay in 32 bits.)
__device__ __forceinline__ AttnSpan attn_span(const AttnArgs& p, int pos, int block, int rows_per_block) {
  const int r0 = block * rows_per_block, r1 = min(p.kv.T * p.G, r0 + rows_per_block) - 1;
  pos = min(max(pos, -(1 << 30)), 1 << 30);
  AttnSpan s;
  s.lo = pos + over_group(p, r0);
  s.hi = pos + over_group(p, r1);
  const int end = min(s.hi + 1, p.kv.max_pages << p.kv.page_shift);      // tokens 0 .. end - 1
  s.first = p.window > 0 ? max(s.lo - p.window + 1, 0) / kAttnStep : 0;
  s.sink_steps = p.window > 0 ? max(min((min(p.sinks, end) + kAttnStep - 1) / kAttnStep, s.first), 0) : 0;
  // at least one: rows that see nothing have their zeros written
  s.steps = max(s.sink_steps + max((end + kAttnStep - 1) / kAttnStep - s.first, 0), 1);
  return s;
}

// Sum and maximum over the four lanes that hold one column.
__device__ __forceinline__ float column_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ float column_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

__device__ __forceinline__ v8h half_frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(v8h, uint4{a, b, c, d});
}

// A row of an item as its workgroups hand it over: reference, sum, (two unused), o
__host__ __device__ constexpr int attn_part_floats(int D) { return D + 4; }

// D features a head, NB blocks of 16 rows.
template <int D, int NB>
__global__ __launch_bounds__(64 * attn_waves(NB), NB == 1 ? 4 : 2) void attn_kv4_kernel(AttnArgs p) {
  constexpr int WAVES = attn_waves(NB), THREADS = 64 * WAVES;
  constexpr int NK = D / 32;                  // matrix instructions of a 16-token tile of q k^T; words of a lane of a key
  constexpr int NV = D / 16;                  // matrix instructions of a step of p v
  constexpr int RB = 16 * NB;
  constexpr int PITCH = D + 4;                // floats of a row in LDS
  constexpr int OWN = 16 * D / THREADS;       // features of a thread where the wavefronts' sums are joined
  constexpr int LANES = D / OWN;              // threads of a row there
  constexpr int PART = attn_part_floats(D);
  constexpr bool Q_LDS = NB == 4;             // the rows' registers would not leave room for the sums
  constexpr float kNone = -1e30f;             // reference of a row that has seen nothing: below every score
  __shared__ float o_lds[WAVES][16][PITCH];
  __shared__ float m_lds[WAVES][16], l_lds[WAVES][16], c_lds[WAVES][16];
  __shared__ uint4 q_lds[Q_LDS ? NB * NK * 64 : 1];
  __shared__ float2 f_lds[Q_LDS ? RB : 1];
  __shared__ uint32_t scan[WAVES];
  __shared__ int found[2][3];                 // entry, head, step in the item: begin and end of this workgroup's run
  __shared__ uint32_t found_at;               // the begin, counted over all steps
  __shared__ unsigned ticket;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int col = lane & 15, kb = lane >> 4;
  const int P = 1 << p.kv.page_shift, R = p.kv.T * p.G, Hkv = p.kv.Hkv;
  const uint32_t region_bytes = (uint32_t)P * (D + 8);
  const int row_of = tid / LANES, own = (tid & (LANES - 1)) * OWN;     // join: row of a block, first feature
  const auto sequence_of = [&](int e) { return p.blocks == 1 ? e : e / p.blocks; };

  // ---- the division of the work: entries are (sequence, block of rows), each of Hkv items of equal length
  const int entries = p.B * p.blocks;
  const int per = (entries + THREADS - 1) / THREADS;
  const int e0 = tid * per, e1 = min(entries, e0 + per);
  const auto steps_of = [&](int e) {
    const int b = sequence_of(e);
    return attn_span(p, p.kv.pos[b], e - b * p.blocks, RB).steps;
  };
  uint32_t mine = 0;
  for (int e = e0; e < e1; ++e) mine += steps_of(e);
  mine *= Hkv;
  uint32_t upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t up = __shfl_up(upto, d);
    if (lane >= d) upto += up;
  }
  if (lane == 63) scan[wave] = upto;
  if (tid == 0) { found[1][0] = entries; found[1][1] = 0; found[1][2] = 0; }
  __syncthreads();
  uint32_t total = 0;
  upto -= mine;                               // steps before this thread's entries
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) upto += scan[w];
    total += scan[w];
  }
  total = uniform(total);
  const uint32_t groups = uniform(max(1u, min((uint32_t)gridDim.x, total / kAttnMinSteps)));
  const uint32_t me = blockIdx.x;
  if (me >= groups) return;
  // workgroup w begins at step w * share, and the first `more` of them take one more each
  const uint32_t share = uniform(total / groups), more = total - share * groups;
  const auto start_of = [&](uint32_t w) { return w * share + min(w, more); };
  const auto group_of = [&](uint32_t x) {     // the workgroup that takes step x
    const uint32_t wide = more * (share + 1);
    return uniform(x < wide ? x / (share + 1) : more + (x - wide) / share);
  };
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const uint32_t x = start_of(me + side);
    if (x - upto < mine) {                    // (unsigned: upto <= x < upto + mine)
      uint32_t at = upto;
      for (int e = e0; e < e1; ++e) {
        const uint32_t n = steps_of(e);
        if (x - at < n * Hkv) {
          const uint32_t h = (x - at) / n, s = n <= kAttnWhole ? 0 : x - at - h * n;
          found[side][0] = e; found[side][1] = (int)h; found[side][2] = (int)s;
          if (side == 0) found_at = at + h * n + s;
          break;
        }
        at += n * Hkv;
      }
    }
  }
  __syncthreads();
  int entry = uniform(found[0][0]), head = uniform(found[0][1]), begin = uniform(found[0][2]);
  const int last_entry = uniform(found[1][0]), last_head = uniform(found[1][1]), last_step = uniform(found[1][2]);
  uint32_t at = uniform(found_at);            // of `begin` of this item
  bool first_run = true;

  while (entry < last_entry || (entry == last_entry && (head < last_head || (head == last_head && begin < last_step)))) {
    const int b = uniform(sequence_of(entry)), block = entry - b * p.blocks;
    AttnSpan span = attn_span(p, uniform(scalar_load(p.kv.pos, b)), block, RB);
    span.steps = uniform(span.steps); span.sink_steps = uniform(span.sink_steps); span.first = uniform(span.first);
    span.lo = uniform(span.lo); span.hi = uniform(span.hi);
    const int stop = entry == last_entry && head == last_head ? last_step : span.steps;
    const int rows = min(RB, R - block * RB);

    // ---- loads of a step: keys, rows of steps and lows, values, from the regions of its two 16-token tiles
    struct Raw { uint32_t k[2][NK]; uint4 v[2], par[2][2]; };
    Raw raw;
    const auto first_token = [&](int s) { return kAttnStep * (s < span.sink_steps ? s : s - span.sink_steps + span.first); };
    // page of the 16 tokens from t on, or -1
    const auto page_of = [&](int t) {
      const int i = t >> p.kv.page_shift;
      if (i >= p.kv.max_pages) return -1;
      const int page = p.kv.table != nullptr ? uniform(scalar_load(p.kv.table, (size_t)b * p.kv.max_pages + i)) : b * p.kv.max_pages + i;
      return page >= 0 && page < p.kv.n_pages ? page : -1;
    };
    const auto region_of = [&](int page) { return p.cache + (size_t)(uint32_t)(max(page, 0) * Hkv + head) * region_bytes; };
    const uint32_t k_off = (uint32_t)(col * (D / 2) + kb * (4 * NK)), par_off = (uint32_t)(kb * 32);
    const uint32_t v_off = (uint32_t)((col & (D / 8 - 1)) * 64 + kb * 16);
    const auto load_keys = [&](int i, int t, const uint8_t* region) {
      const uint8_t* const src = region + (uint32_t)(t & (P - 1)) * (D / 2);
      if (NK == 4) {
        const uint4 w = *reinterpret_cast<const uint4*>(src + k_off);
        raw.k[i][0] = w.x; raw.k[i][1] = w.y; raw.k[i][NK - 2] = w.z; raw.k[i][NK - 1] = w.w;
      } else {
        const uint2 w = *reinterpret_cast<const uint2*>(src + k_off);
        raw.k[i][0] = w.x; raw.k[i][1] = w.y;
      }
    };
    const auto load_rest = [&](int i, int t, const uint8_t* region) {
      const uint32_t slot = (uint32_t)(t & (P - 1));
      const uint8_t* const par = region + (uint32_t)P * D + slot * 8;
      raw.par[i][0] = *reinterpret_cast<const uint4*>(par + par_off);
      raw.par[i][1] = *reinterpret_cast<const uint4*>(par + par_off + 16);
      raw.v[i] = *reinterpret_cast<const uint4*>(region + (uint32_t)P * (D / 2) + slot * (D / 2) + v_off);
    };
    int s = begin + wave;
    int t = 0, page0 = -1, page1 = -1;
    if (s < stop) {
      t = first_token(s);
      page0 = page_of(t);
      page1 = P >= kAttnStep ? page0 : page_of(t + 16);
      const uint8_t* const region0 = region_of(page0);
      const uint8_t* const region1 = region_of(page1);
      load_keys(0, t, region0);
      load_keys(1, t + 16, region1);
      load_rest(0, t, region0);
      load_rest(1, t + 16, region1);
    }

    // ---- the rows: scaled to 2^13 .. 2^14, a sixteenth where the codes come 16 times too large
    v8h qf[Q_LDS ? 1 : NB][NK];
    float f[NB], shift[NB], m[NB], l[NB], c[NB];      // l: sum of p; c: the part of o that all features share
    int row_pos[NB];
    v4f o[NB][NV];
    const auto row_of_q = [&](int nb, v8h (&x)[NK], float& factor, float& sum_of) {
      const int r = min(nb * 16 + col, rows - 1) + block * RB;             // (columns without a row repeat the last one)
      const int j = over_group(p, r), g = r - j * p.G;
      const uint16_t* const src = p.q + (((size_t)b * p.kv.T + j) * p.Hq + (size_t)head * p.G + g) * D + kb * 8 * NK;
      float top = 0.0f, sum = 0.0f;
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        x[i] = __builtin_bit_cast(v8h, reinterpret_cast<const uint4*>(src)[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) { top = fmaxf(top, fabsf((float)x[i][e])); sum += (float)x[i][e]; }
      }
      top = column_max(top);
      sum = column_sum(sum);
      const int ex = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) : 0;
      const float up = __builtin_amdgcn_ldexpf(1.0f, 14 - ex);
#pragma unroll
      for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = (_Float16)((float)x[i][e] * (e & 2 ? up * 0.0625f : up));
      factor = p.scale_log2 * __builtin_amdgcn_ldexpf(1.0f, ex + 10);
      sum_of = sum * __builtin_amdgcn_ldexpf(1.0f, -ex - 10);
    };
    if (Q_LDS) {
      if (wave < NB) {
        v8h x[NK];
        float factor, sum_of;
        row_of_q(wave, x, factor, sum_of);
#pragma unroll
        for (int i = 0; i < NK; ++i) q_lds[(wave * NK + i) * 64 + lane] = __builtin_bit_cast(uint4, x[i]);
        if (kb == 0) f_lds[wave * 16 + col] = float2{factor, sum_of};
      }
      __syncthreads();
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (Q_LDS) {
        const float2 both = f_lds[nb * 16 + col];
        f[nb] = both.x;
        shift[nb] = both.y;
      } else {
        row_of_q(nb, qf[nb], f[nb], shift[nb]);
      }
      row_pos[nb] = span.lo + over_group(p, min(nb * 16 + col, rows - 1) + block * RB) - over_group(p, block * RB);
      m[nb] = kNone;
      l[nb] = c[nb] = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) o[nb][v] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const auto q_frag = [&](int nb, int w) {
      if (Q_LDS) return __builtin_bit_cast(v8h, q_lds[(nb * NK + w) * 64 + lane]);
      return qf[Q_LDS ? 0 : nb][w];
    };
    int vexp = -30;                           // exponent of the largest value step so far

    // ---- the steps of this wavefront
    for (; s < stop; s += WAVES) {
      const int t_next = first_token(min(s + WAVES, span.steps - 1));       // (the last one's loads repeat a step)
      const int next0 = page_of(t_next), next1 = P >= kAttnStep ? next0 : page_of(t_next + 16);
      const uint8_t* const region0 = region_of(next0);
      const uint8_t* const region1 = region_of(next1);
      // every token of the step in sight of every row
      const bool whole = page0 >= 0 && page1 >= 0 && t + kAttnStep - 1 <= span.lo &&
                         (p.window == 0 || t > span.hi - p.window || t + kAttnStep <= p.sinks);
      v4f sc[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) sc[nb][0] = sc[nb][1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < NK; ++w) {
        const auto widen = [](uint32_t x) {
          const uint32_t y = x >> 8;
          return half_frag(x & 0x000F000Fu, x & 0x00F000F0u, y & 0x000F000Fu, y & 0x00F000F0u);
        };
        const v8h k0 = widen(raw.k[0][w]), k1 = widen(raw.k[1][w]);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const v8h x = q_frag(nb, w);
          sc[nb][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, x, sc[nb][0], 0, 0, 0);
          sc[nb][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, x, sc[nb][1], 0, 0, 0);
        }
      }
      load_keys(0, t_next, region0);
      load_keys(1, t_next + 16, region1);

      // steps and lows of this lane's 8 tokens
      v2h kp[8], vp[8];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t w[8] = {raw.par[i][0].x, raw.par[i][0].y, raw.par[i][0].z, raw.par[i][0].w,
                               raw.par[i][1].x, raw.par[i][1].y, raw.par[i][1].z, raw.par[i][1].w};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          kp[4 * i + x] = __builtin_bit_cast(v2h, w[2 * x]);
          vp[4 * i + x] = __builtin_bit_cast(v2h, w[2 * x + 1]);
        }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int x = 0; x < 8; ++x)
          sc[nb][x >> 2][x & 3] = fmaf(sc[nb][x >> 2][x & 3], (float)kp[x].x, (float)kp[x].y * shift[nb]);
      if (!whole) {
        uint32_t any = 0;                     // bit x: a row of this lane sees its token x
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            const int tok = t + (x >> 2) * 16 + 4 * kb + (x & 3);
            const bool in = (x < 4 ? page0 : page1) >= 0 && tok <= row_pos[nb] &&
                            (p.window == 0 || tok > row_pos[nb] - p.window || tok < p.sinks);
            any |= in ? 1u << x : 0u;
            sc[nb][x >> 2][x & 3] = in ? sc[nb][x >> 2][x & 3] : -__builtin_inff();
          }
        }
        // whatever stands in rows that nobody sees (infinities, NaN) must not meet a weight, not even one of zero
#pragma unroll
        for (int x = 0; x < 8; ++x) vp[x] = any >> x & 1u ? vp[x] : v2h{(_Float16)0.0f, (_Float16)0.0f};
      }
      // The reference: 2^(s - m) times the value steps has to stay inside fp16's range, with its largest terms well above its
      // smallest numbers, so m is the largest score less 8, plus the exponent of the largest value step.  It moves
      // when a term could pass 2^14, which after the first step is rare.
      v2h vmax2 = vp[0];
#pragma unroll
      for (int x = 1; x < 8; ++x) vmax2 = __builtin_elementwise_max(vmax2, vp[x]);
      const float vtop = (float)vmax2.x;
      bool reset = vtop > __builtin_amdgcn_ldexpf(1.0f, vexp);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float top = sc[nb][0][0];
#pragma unroll
        for (int x = 1; x < 8; ++x) top = fmaxf(top, sc[nb][x >> 2][x & 3]);
        reset |= fmaf(top, f[nb], -m[nb]) > (float)(14 - vexp);
      }
      if (__builtin_amdgcn_ballot_w64(reset) != 0) {
        float vwide = vtop;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) vwide = fmaxf(vwide, __shfl_xor(vwide, d));
        const int before = vexp;
        vexp = uniform(max(vexp, vwide > 0.0f ? __builtin_amdgcn_frexp_expf(vwide) : vexp));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float top = sc[nb][0][0];
#pragma unroll
          for (int x = 1; x < 8; ++x) top = fmaxf(top, sc[nb][x >> 2][x & 3]);
          const float to = fmaxf(m[nb] + (float)(vexp - before), fmaf(column_max(top), f[nb], (float)(vexp - 8)));
          const float by = __builtin_amdgcn_exp2f(m[nb] - to);
          m[nb] = to;
          l[nb] *= by;
          c[nb] *= by;
#pragma unroll
          for (int v = 0; v < NV; ++v) o[nb][v] *= by;
        }
      }
      v8h pf[NB];
      typedef float v2f __attribute__((ext_vector_type(2)));
      const v2h minus8 = {(_Float16)-8.0f, (_Float16)-8.0f};
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        v2h w[4];
#pragma unroll
        for (int x = 0; x < 8; x += 2) {
          const float e0 = __builtin_amdgcn_exp2f(fmaf(sc[nb][x >> 2][x & 3], f[nb], -m[nb]));
          const float e1 = __builtin_amdgcn_exp2f(fmaf(sc[nb][x >> 2][(x & 3) + 1], f[nb], -m[nb]));
          l[nb] += e0;
          l[nb] += e1;
          c[nb] = fmaf(e0, fmaf(8.0f, (float)vp[x].x, (float)vp[x].y), c[nb]);
          c[nb] = fmaf(e1, fmaf(8.0f, (float)vp[x + 1].x, (float)vp[x + 1].y), c[nb]);
          // 11 bits of a weight: what an fp16 probability keeps
          w[x / 2] = __builtin_convertvector((v2f{e0 * (float)vp[x].x, e1 * (float)vp[x + 1].x}), v2h);
          c[nb] = __builtin_amdgcn_fdot2(w[x / 2], minus8, c[nb], false);
        }
        pf[nb] = __builtin_bit_cast(v8h, uint4{__builtin_bit_cast(uint32_t, w[0]), __builtin_bit_cast(uint32_t, w[1]),
                                               __builtin_bit_cast(uint32_t, w[2]), __builtin_bit_cast(uint32_t, w[3])});
      }
      // values: token pairs of one half of the words, nibble by nibble
      const auto values = [&](uint32_t sel, int v0) {
        const uint4 a = raw.v[0], d = raw.v[1];
        const uint32_t x[4] = {__builtin_amdgcn_perm(a.y, a.x, sel), __builtin_amdgcn_perm(a.w, a.z, sel),
                               __builtin_amdgcn_perm(d.y, d.x, sel), __builtin_amdgcn_perm(d.w, d.z, sel)};
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const uint32_t mask = n & 1 ? 0x00F000F0u : 0x000F000Fu;
          const int by = n & 2 ? 8 : 0;
          const v8h vf = half_frag(x[0] >> by & mask, x[1] >> by & mask, x[2] >> by & mask, x[3] >> by & mask);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) o[nb][v0 + n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[nb], o[nb][v0 + n], 0, 0, 0);
        }
      };
      if (D == 128) {
        values(0x05040100u, 0);
        values(0x07060302u, NV - 4);
      } else {
        values(col & 8 ? 0x07060302u : 0x05040100u, 0);        // lanes 8 .. 15 of a row take the upper halves of the same words
      }
      load_rest(0, t_next, region0);
      load_rest(1, t_next + 16, region1);
      t = t_next;
      page0 = next0;
      page1 = next1;
    }

    // ---- the wavefronts' sums, 16 rows at a time
    const bool shared = begin > 0 || stop < span.steps;
    const uint32_t item = at - begin;
    const uint32_t w0 = shared ? group_of(item) : me, w1 = shared ? group_of(item + span.steps - 1) : me;   // the workgroups that hold a part of it
    const auto write_row = [&](int r, const float (&v)[OWN], float sum) {
      const int j = over_group(p, r), g = r - j * p.G;
      const float by = sum > 0.0f ? 1.0f / sum : 0.0f;
      typedef _Float16 vh __attribute__((ext_vector_type(OWN)));
      vh h;
#pragma unroll
      for (int x = 0; x < OWN; ++x) h[x] = (_Float16)(sum > 0.0f ? fminf(fmaxf(v[x] * by, -65504.0f), 65504.0f) : 0.0f);   // (a 15th code may lie past fp16's end)
      *reinterpret_cast<vh*>(p.out + (((size_t)b * p.kv.T + j) * p.Hq + (size_t)head * p.G + g) * D + own) = h;
    };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (nb * 16 >= rows) break;
      l[nb] = column_sum(l[nb]);
      c[nb] = column_sum(c[nb]);
      if (kb == 0) { m_lds[wave][col] = m[nb]; l_lds[wave][col] = l[nb]; c_lds[wave][col] = c[nb]; }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float* const dst = &o_lds[wave][col][8 * ((4 * kb + i) & (D / 8 - 1))];
        if (D == 128) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = o[nb][((e & 1) * 4 + e / 2) % NV][i] * (e & 2 ? 1048576.0f : 16777216.0f);
          reinterpret_cast<float4*>(dst)[0] = float4{x[0], x[1], x[2], x[3]};
          reinterpret_cast<float4*>(dst)[1] = float4{x[4], x[5], x[6], x[7]};
        } else {
#pragma unroll
          for (int n = 0; n < 4; ++n) dst[2 * n + (kb >> 1)] = o[nb][n][i] * (n & 1 ? 1048576.0f : 16777216.0f);
        }
      }
      __syncthreads();
      const int r = nb * 16 + row_of;
      if (r < rows) {
        float v[OWN], by[WAVES], total_l = 0.0f, total_c = 0.0f, ref = kNone;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) ref = fmaxf(ref, m_lds[w][row_of]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          by[w] = __builtin_amdgcn_exp2f(m_lds[w][row_of] - ref);
          total_l = fmaf(l_lds[w][row_of], by[w], total_l);
          total_c = fmaf(c_lds[w][row_of], by[w], total_c);
        }
#pragma unroll
        for (int x = 0; x < OWN; ++x) {
          v[x] = total_c;
#pragma unroll
          for (int w = 0; w < WAVES; ++w) v[x] = fmaf(o_lds[w][row_of][own + x], by[w], v[x]);
        }
        if (!shared) {
          write_row(block * RB + r, v, total_l);
        } else {
          float* const part = p.parts + ((size_t)(2 * me + (first_run ? 0 : 1)) * RB + r) * PART;
          if (own == 0) store_shared_f2(part, ref, total_l);
#pragma unroll
          for (int x = 0; x < OWN; x += 2) store_shared_f2(part + 4 + own + x, v[x], v[x + 1]);
        }
      }
      __syncthreads();
    }

    // ---- the last of the item's workgroups joins their parts
    if (shared && last_arrival(p.tickets, (int)(w1 - w0 + 1), w0, &ticket)) {
      const int n = (int)(w1 - w0 + 1);
      const uint32_t slot0 = 2 * w0 + (start_of(w0) < item ? 1 : 0);
      // few rows: several threads take a row's parts in turn
      const int taken = rows > 8 ? 16 : rows > 4 ? 8 : rows > 2 ? 4 : rows > 1 ? 2 : 1;
      const int sub = row_of & (taken - 1), lot = row_of / taken, lots = 16 / taken;
      for (int r0 = 0; r0 < rows; r0 += 16) {
        const int r = r0 + sub;
        float ref = kNone, sum = 0.0f, v[OWN];
#pragma unroll
        for (int x = 0; x < OWN; ++x) v[x] = 0.0f;
        if (r < rows) {
#pragma unroll 2
          for (int i = lot; i < n; i += lots) {
            const float* const part = p.parts + ((size_t)(i == 0 ? slot0 : 2 * (w0 + i)) * RB + r) * PART;
            const float2 head2 = load_shared_f2(part);
            float2 in[OWN / 2];
#pragma unroll
            for (int x = 0; x < OWN / 2; ++x) in[x] = load_shared_f2(part + 4 + own + 2 * x);
            const float to = fmaxf(ref, head2.x), a = __builtin_amdgcn_exp2f(ref - to), d = __builtin_amdgcn_exp2f(head2.x - to);
            ref = to;
            sum = sum * a + head2.y * d;
#pragma unroll
            for (int x = 0; x < OWN / 2; ++x) {
              v[2 * x] = v[2 * x] * a + in[x].x * d;
              v[2 * x + 1] = v[2 * x + 1] * a + in[x].y * d;
            }
          }
        }
        if (lots > 1) {
          if (own == 0) { m_lds[0][row_of] = ref; l_lds[0][row_of] = sum; }
#pragma unroll
          for (int x = 0; x < OWN; ++x) o_lds[0][row_of][own + x] = v[x];
          __syncthreads();
          if (lot == 0 && r < rows) {
            for (int k = 1; k < lots; ++k) {
              const int from = k * taken + sub;
              const float to = fmaxf(ref, m_lds[0][from]), a = __builtin_amdgcn_exp2f(ref - to), d = __builtin_amdgcn_exp2f(m_lds[0][from] - to);
              ref = to;
              sum = sum * a + l_lds[0][from] * d;
#pragma unroll
              for (int x = 0; x < OWN; ++x) v[x] = v[x] * a + o_lds[0][from][own + x] * d;
            }
          }
        }
        if (lot == 0 && r < rows) write_row(block * RB + r, v, sum);
        __syncthreads();
      }
    }
    at += stop - begin;
    begin = 0;
    first_run = false;
    if (++head == Hkv) { head = 0; ++entry; }
  }
}

}  // namespace qspec
