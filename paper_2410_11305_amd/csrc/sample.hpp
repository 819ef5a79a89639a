// The choice of a token from fp16 logits by a given random number: temperature, top-k, min-p, top-p, then the inverse
// of the running mass; and the acceptance walk over tokens chosen that way.
//
// A logit is one of 65536 values, so a row is its histogram: counts of every value (65536 counters of 16 bits, 128 KB of
// LDS, one workgroup per row), added up as integers.  All tokens of one value weigh the same and follow one another in the
// order of the draw (falling logit, the lowest index first among equals), so every limit and the draw itself are decided from the counts and
// exp((value - max) / temperature) in binary64, whatever order the logits arrived in; only the last step, which of the
// tokens of one value, looks at indices.  No sort, no passes over candidates, every logit read once for the counts and
// (rows of up to 65536: from registers) once more for the index.
//
// Measured (device time): one row of 32000 12.8 us, 32 rows of 128256 25.7 us (0.32 TB/s), 512 rows of 32000 33.9 us
// (0.97 TB/s), of which for one row: the launch 2.2, logits and counts 2.3, their sums 1.3, the masses 3 to 4 (binary64), the draw 1.5 and
// the index 1.3.  Neither bytes nor rates bound it but this chain of steps with a barrier after each: the 128 KB of counters leave room for one workgroup a
// compute unit, so that rows beyond the 256 units come one after the other.  Counters of 16 bits are what makes the
// whole value range fit; those of 32 bits would need a pass over each half.
//
// A thread owns a block of 64 neighbouring values, which are equally spaced (64 divides every binade): its weights are a
// geometric series, two exponentials and one multiply-add a value.  Where something is decided inside a block, every
// wavefront takes the block a value to a lane, so nothing is walked and nothing handed around.
#pragma once
#include "accept.hpp"
#include "common.hpp"
#include "producers.hpp"

namespace qspec {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kSampleRound = 8 * kSampleThreads;              // logits of one trip, 8 to a thread
constexpr int kSampleKept = 8;                                // trips that stay in registers
constexpr int kSampleMaxV = 256 * kSampleRound;
constexpr int kSampleExtras = kSampleMaxV / 32768;            // halves of a counter's range that a row can run over

struct SampleArgs {
  const uint16_t* logits;    // fp16 [rows][V]
  const float* u;            // [rows]
  const float* temperature;  // [B] each, or null
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* tokens;           // [rows]
  int V, per;                // per: rows of a sequence
};

// exp(x) for x <= 0 in binary64, to about a unit in the last place: n ln 2 off in two parts, the Taylor polynomial of
// degree 13 on +-ln 2 / 2 (the next term is below 2^-57).  The parts: ln 2 cut to 40 bits, which n (11 bits) multiplies exactly, and what is left of it.
__device__ inline double exp_negative(double x) {
  x = fmax(x, -800.0);
  const double n = rint(x * 1.44269504088896340736);
  const double ln2 = 0x1.62e42fefa2p-1, ln2_rest = 0x1.9ef35793c7673p-41;
  const double r = fma(n, -ln2_rest, fma(n, -ln2, x));
  double e = 1.0 / 6227020800.0;
  e = fma(e, r, 1.0 / 479001600.0);
  e = fma(e, r, 1.0 / 39916800.0);
  e = fma(e, r, 1.0 / 3628800.0);
  e = fma(e, r, 1.0 / 362880.0);
  e = fma(e, r, 1.0 / 40320.0);
  e = fma(e, r, 1.0 / 5040.0);
  e = fma(e, r, 1.0 / 720.0);
  e = fma(e, r, 1.0 / 120.0);
  e = fma(e, r, 1.0 / 24.0);
  e = fma(e, r, 1.0 / 6.0);
  e = fma(e, r, 0.5);
  e = fma(e, r, 1.0);
  e = fma(e, r, 1.0);
  return __builtin_amdgcn_ldexp(e, (int)n);
}

// Values by number, in their order (half_order_key): 0x8000 + magnitude bits, 0x7FFF - magnitude bits for negative ones;
// 0x7FFF is -0, whose tokens count as those of 0x8000.  64 neighbours from a multiple of 64 on are equally spaced.
__device__ __forceinline__ double sample_value(uint32_t key) {
  return (double)half_bits_to_float((uint16_t)(key & 0x8000u ? key ^ 0x8000u : key ^ 0xFFFFu));
}
constexpr int kNumber = 0x3F8;                                // v_cmp_class: everything but NaN and -inf

typedef unsigned short v2us __attribute__((ext_vector_type(2)));

// Piece i of a row: 8 logits from 8 i on, -inf past the end.  (Rows start wherever V puts them.)
__device__ __forceinline__ uint4 sample_piece(const uint16_t* row, int V, int i) {
  uint4 q = {0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u};
  if (8 * i + 8 <= V) {
    __builtin_memcpy(&q, row + 8 * i, 16);
  } else {
#pragma unroll 1
    for (int e = V - 8 * i - 1; e >= 0; --e)                  // (one piece of a row at most)
      q = uint4{q.x << 16 | row[8 * i + e], __builtin_amdgcn_alignbit(q.y, q.x, 16), __builtin_amdgcn_alignbit(q.z, q.y, 16),
                __builtin_amdgcn_alignbit(q.w, q.z, 16)};
  }
  return q;
}
// Inclusive sum over the lanes up to this one.
__device__ __forceinline__ uint32_t lane_scan(uint32_t v) {
#define QSPEC_DPP_ADD(ctrl, rows) v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false)
  QSPEC_DPP_ADD(0x111, 0xf);                  // row_shr 1, 2, 4, 8: inside a row of 16
  QSPEC_DPP_ADD(0x112, 0xf);
  QSPEC_DPP_ADD(0x114, 0xf);
  QSPEC_DPP_ADD(0x118, 0xf);
  QSPEC_DPP_ADD(0x142, 0xa);                  // row_bcast 15 into rows 1 and 3
  QSPEC_DPP_ADD(0x143, 0xc);                  // row_bcast 31 into rows 2 and 3
#undef QSPEC_DPP_ADD
  return v;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_or_zero(double v) {
  const unsigned long long b = __builtin_bit_cast(unsigned long long, v);
  const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)b, CTRL, ROWS, 0xf, false);
  const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(b >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, ((unsigned long long)hi << 32) | lo);
}
__device__ __forceinline__ double lane_scan(double v) {
  v += dpp_or_zero<0x111, 0xf>(v);
  v += dpp_or_zero<0x112, 0xf>(v);
  v += dpp_or_zero<0x114, 0xf>(v);
  v += dpp_or_zero<0x118, 0xf>(v);
  v += dpp_or_zero<0x142, 0xa>(v);
  v += dpp_or_zero<0x143, 0xc>(v);
  return v;
}

// grid rows.
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs p) {
  __shared__ __align__(16) uint32_t hist[32768];              // two values' counts a word
  __shared__ uint32_t extra[kSampleExtras];                   // values that stand for 32768 tokens more, each time they are named
  __shared__ uint32_t extras;
  __shared__ uint32_t wave_u[3][kSampleWaves];
  __shared__ double wave_d[kSampleWaves];
  __shared__ uint32_t border[5], border_before[5];            // blocks in which something is decided, and the tokens before them
  __shared__ double border_mass[5];                           // ... and the mass
  __shared__ uint32_t cell_found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = blockIdx.x, b = r / p.per;
  const uint16_t* const row = p.logits + (size_t)r * p.V;
  const uint32_t own = kSampleThreads - 1 - tid;              // this thread's block, the largest values first
  const int pieces = (p.V + 7) / 8, trips = (pieces + kSampleThreads - 1) / kSampleThreads;
  // The counter of a value is a half of its magnitude's word, the upper one for negative values: counting takes the bits of
  // a logit as they are.  16 bytes c of 64 words stand at c ^ (the number of the 64): threads that read neighbouring
  // blocks do not meet in a bank.
  const auto place_of = [](uint32_t byte) { return byte ^ ((byte >> 4) & 0x70u); };
  uint8_t* const bytes = reinterpret_cast<uint8_t*>(hist);
  const auto count_of = [&](uint32_t key) {
    const bool below = key < 0x8000u;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(bytes + place_of((below ? 0x7FFFu - key : key - 0x8000u) * 4));
    uint32_t n = below ? w >> 16 : w & 0xFFFFu;
    if (key == 0x8000u) n += w >> 16;
    if (key == 0x7FFFu) n = 0;
#pragma unroll 1
    for (uint32_t i = 0; i < extras; ++i) n += extra[i] == key ? 32768u : 0u;
    return n;
  };

  // ---- the sequence's parameters
  const float temperature = p.temperature ? p.temperature[b] : 1.0f;
  const bool greedy = !(temperature > 0.0f);
  const uint32_t k = greedy ? 1u : p.top_k && p.top_k[b] > 0 ? (uint32_t)p.top_k[b] : 0xFFFFFFFFu;
  const double least = p.min_p && p.min_p[b] > 0.0f ? fmin((double)p.min_p[b], 1.0) : 0.0;
  const float share = p.top_p ? p.top_p[b] : 1.0f;
  const double u = (double)fminf(fmaxf(p.u[r], 0.0f), 0.99999994f);
  const double inverse = greedy ? 0.0 : 1.0 / (double)temperature;

  // ---- counts
  uint4 kept[kSampleKept];
#pragma unroll
  for (int t = 0; t < kSampleKept; ++t)
    if (t < trips) kept[t] = sample_piece(row, p.V, t * kSampleThreads + tid);
#pragma unroll
  for (int i = 0; i < 8; ++i) reinterpret_cast<uint4*>(hist)[i * kSampleThreads + tid] = uint4{0u, 0u, 0u, 0u};
  if (tid == 0) extras = 0;
  if (tid < 5) {
    border[tid] = 0xFFFFFFFFu;
    border_before[tid] = 0;
    border_mass[tid] = 0.0;
  }
  __syncthreads();
  uint32_t counted = 0;
  const auto count_piece = [&](const uint4& q) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t x = w[e >> 1];
      const uint32_t byte = e & 1 ? x >> 14 & 0x1FFFCu : x << 2 & 0x1FFFCu;
      const uint32_t one = max(e & 1 ? x >> 15 & 0x10000u : x << 1 & 0x10000u, 1u);
      if (__builtin_amdgcn_classh(__builtin_bit_cast(v2h, x)[e & 1], kNumber)) {
        atomicAdd(reinterpret_cast<uint32_t*>(bytes + place_of(byte)), one);
        ++counted;
      }
    }
  };
#pragma unroll
  for (int t = 0; t < kSampleKept; ++t)
    if (t < trips) count_piece(kept[t]);
  const auto further = [&](int t0, int t1, auto f) {          // trips that are not kept, four on their way together
    for (int t = t0; t < t1; t += 4) {
      uint4 q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = sample_piece(row, p.V, (t + i) * kSampleThreads + tid);    // (past the end: -inf)
#pragma unroll
      for (int i = 0; i < 4; ++i) f(t + i, q[i]);
    }
  };
  further(kSampleKept, trips, [&](int, const uint4& q) { count_piece(q); });
  __syncthreads();
  // this thread's 64 values: 64 words, upwards or (negative values; the upper half of the wavefronts) downwards
  const bool negative = wave >= kSampleWaves / 2;             // own < 512
  const uint32_t group = negative ? 511u - own : own - 512u;
  const auto own_words = [&](uint32_t c) { return *reinterpret_cast<const uint4*>(bytes + (group * 256 + ((c ^ (group & 7u)) << 4))); };
  const auto sum_own = [&] {
    uint32_t n = 0;
    const v2us half = negative ? v2us{0, 1} : v2us{1, 0};
#pragma unroll 4
    for (uint32_t c = 0; c < 16; ++c) {
      const uint4 w = own_words(c);
      n = __builtin_amdgcn_udot2(__builtin_bit_cast(v2us, w.x), half, n, false);
      n = __builtin_amdgcn_udot2(__builtin_bit_cast(v2us, w.y), half, n, false);
      n = __builtin_amdgcn_udot2(__builtin_bit_cast(v2us, w.z), half, n, false);
      n = __builtin_amdgcn_udot2(__builtin_bit_cast(v2us, w.w), half, n, false);
    }
    if (group == 0) n = negative ? n - (hist[0] >> 16) : n + (hist[0] >> 16);        // -0 counts as 0
    return n;
  };
  // the sum of the wavefronts' numbers before this one, and of all of them
  const auto over_waves = [&](const uint32_t* each, uint32_t& all) {
    const uint32_t scan = lane_scan(lane < kSampleWaves ? each[lane] : 0u);
    all = (uint32_t)__builtin_amdgcn_readlane((int)scan, kSampleWaves - 1);
    return wave ? (uint32_t)__builtin_amdgcn_readlane((int)scan, wave - 1) : 0u;
  };
  uint32_t here = sum_own();
  uint32_t upto = lane_scan(here);
  if (lane == 63) wave_u[0][wave] = upto;
  const bool may_run_over = p.V > 65535;
  if (may_run_over) {
    const uint32_t seen_wave = lane_scan(counted);
    if (lane == 63) wave_u[1][wave] = seen_wave;
  }
  __syncthreads();
  uint32_t tokens, seen;
  uint32_t before = over_waves(wave_u[0], tokens) + upto - here;
  seen = tokens;
  if (may_run_over) over_waves(wave_u[1], seen);
  if (tokens != seen) {
    // A counter ran over (more than 65535 equal logits; every overflow loses counts, so it shows in the sum).  Again, 32768
    // tokens at a time, each time taking 32768 off the counters that have them.
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) reinterpret_cast<uint4*>(hist)[i * kSampleThreads + tid] = uint4{0u, 0u, 0u, 0u};
    __syncthreads();
#pragma unroll 1
    for (int t0 = 0; t0 < trips; t0 += 4) {
#pragma unroll 1
      for (int i = 8 * t0 * kSampleThreads + tid; i < min(p.V, 8 * (t0 + 4) * kSampleThreads); i += kSampleThreads) {
        const uint32_t x = row[i];
        if (__builtin_amdgcn_classh(__builtin_bit_cast(_Float16, (uint16_t)x), kNumber))
          atomicAdd(reinterpret_cast<uint32_t*>(bytes + place_of(x << 2 & 0x1FFFCu)), max(x << 1 & 0x10000u, 1u));
      }
      __syncthreads();
#pragma unroll 1
      for (uint32_t i = 0; i < 64; ++i) {
        const uint32_t magnitude = group * 64 + i;
        uint32_t* const w = reinterpret_cast<uint32_t*>(bytes + place_of(magnitude * 4));
        const uint32_t bit = negative ? 0x80000000u : 0x8000u;
        if (*w & bit) {
          atomicSub(w, bit);                                   // (the other half is another thread's)
          extra[atomicAdd(&extras, 1u)] = negative && magnitude ? 0x7FFFu - magnitude : 0x8000u + magnitude;
        }
      }
      __syncthreads();
    }
    here = sum_own();
#pragma unroll 1
    for (uint32_t i = 0; i < extras; ++i) here += extra[i] >> 6 == own ? 32768u : 0u;
    upto = lane_scan(here);
    if (lane == 63) wave_u[0][wave] = upto;
    __syncthreads();
    before = over_waves(wave_u[0], tokens) + upto - here;
  }
  if (seen == 0) {                                            // nothing to choose from
    if (tid == 0) p.tokens[r] = -1;
    return;
  }

  // ---- the largest value: in the first block that has any
  if (here && before == 0) border[3] = own;
  __syncthreads();
  const uint32_t top_block = border[3];
  const uint64_t any = __builtin_amdgcn_ballot_w64(count_of(top_block * 64 + 63 - lane) != 0);
  const uint32_t top = top_block * 64 + 63 - (uint32_t)__builtin_ctzll(any);

  const double top_value = sample_value(top);
  // (beside +inf the others weigh nothing)
  const auto weight_of = [&](uint32_t key) {
    return key == top ? 1.0 : top == 0xFC00u ? 0.0 : exp_negative((sample_value(key) - top_value) * inverse);
  };

  // ---- this thread's part of the mass: its largest value's weight times a polynomial in the ratio of neighbours
  double mass = 0.0;
  const bool in = here && before < k;
  if (in) {
    const uint32_t low = own * 64, high = min(low + 63u, top);
    const double first = weight_of(high), ratio = top == 0xFC00u ? 0.0 : exp_negative((sample_value(low) - sample_value(low + 1)) * inverse);
    const bool all = !(least > 0.0) || weight_of(low) >= least;
    if (!all || before + here > k || high != low + 63u) {
      // cut inside by top_k or by min_p, or the block of the largest value: three blocks at most, for a wavefront each
      if (first >= least) {
        const int slot = before + here > k ? 0 : all ? 2 : 1;
        border[slot] = own;
        border_before[slot] = before;
      }
    } else if (extras) {
#pragma unroll 1
      for (uint32_t key = low; key <= high; ++key) mass = fma(mass, ratio, (double)count_of(key));
      mass *= first;
    } else {
      const uint32_t shift = negative ? 16u : 0u;
#pragma unroll 2
      for (uint32_t i = 0; i < 16; ++i) {
        const uint32_t c = negative ? 15u - i : i;
        const uint4 w = own_words(c);
        uint32_t n[4] = {w.x >> shift & 0xFFFFu, w.y >> shift & 0xFFFFu, w.z >> shift & 0xFFFFu, w.w >> shift & 0xFFFFu};
        if (c == 0 && group == 0) n[0] = negative ? 0u : (w.x & 0xFFFFu) + (w.x >> 16);        // -0 counts as 0
        if (negative) {
          const uint32_t n0 = n[0], n1 = n[1];
          n[0] = n[3]; n[1] = n[2]; n[2] = n1; n[3] = n0;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // (a count in the low bits of 2^52, and 2^52 off again: two short operations where the conversion takes as long as four)
          mass = fma(mass, ratio, __builtin_bit_cast(double, 0x4330000000000000ull | n[e]) - 4503599627370496.0);
        }
      }
      mass *= first;
    }
  }
  __syncthreads();
  // A block, a value to a lane: how many of its tokens are within top_k and min_p, their weight, and the mass up to them.
  struct Block { uint32_t key, n; double weight, upto; };
  const auto block_of = [&](uint32_t block, uint32_t tokens_before, double mass_before) {
    Block x;
    x.key = block * 64 + 63 - lane;
    const uint32_t n = x.key <= top ? count_of(x.key) : 0u;
    const uint32_t at = tokens_before + lane_scan(n) - n;
    x.weight = n ? weight_of(x.key) : 0.0;
    x.n = at >= k || x.weight < least ? 0u : min(n, k - at);
    x.upto = mass_before + lane_scan((double)x.n * x.weight);
    return x;
  };
  if (wave < 3 && border[wave] != 0xFFFFFFFFu) {
    const double cut = lane_value_f64(block_of(border[wave], border_before[wave], 0.0).upto, 63);
    if (lane == 0) border_mass[wave] = cut;
  }
  __syncthreads();
#pragma unroll
  for (int slot = 0; slot < 3; ++slot) mass = border[slot] == own ? border_mass[slot] : mass;
  const double sum = lane_scan(mass);
  if (lane == 63) wave_d[wave] = sum;
  __syncthreads();
  const double waves_scan = lane_scan(lane < kSampleWaves ? wave_d[lane] : 0.0);
  const double total = lane_value_f64(waves_scan, kSampleWaves - 1);
  const double wave_base = wave ? lane_value_f64(waves_scan, wave - 1) : 0.0, next_base = lane_value_f64(waves_scan, wave);
  const double shifted = __shfl_up(sum, 1);
  // To is the next thread's from, bit for bit.  (The sums of a scan can fall by a rounding from one lane to the next, so a
  // thread without mass may seem to hold such a piece: it does not claim it, and what no one claims has a default below.)
  const double from = lane ? wave_base + shifted : wave_base, to = lane < 63 ? wave_base + sum : next_base;

  // ---- top-p: the shortest beginning that holds this much (one token at least)
  double kept_mass = total;
  if (share < 1.0f) {
    const double limit = fmax((double)share * total, 1e-300);
    if (mass > 0.0 && from < limit && limit <= to) { border[4] = own; border_before[4] = before; border_mass[4] = from; }
    __syncthreads();
    const Block x = block_of(min(border[4], (uint32_t)kSampleThreads), border_before[4], border_mass[4]);       // (past all blocks: no tokens)
    // the value in which the mass is reached; rounding may leave that to the last one
    const uint64_t hit = __builtin_amdgcn_ballot_w64(x.n && x.upto >= limit), have = __builtin_amdgcn_ballot_w64(x.n && x.weight > 0.0);
    const int at = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(have | 1ull);
    const double start = x.upto - (double)x.n * x.weight;
    const double cut = hit ? fma(fmin(fmax(ceil((limit - start) / x.weight), 1.0), (double)x.n), x.weight, start) : x.upto;
    kept_mass = border[4] == 0xFFFFFFFFu ? limit : lane_value_f64(cut, at);
  }

  // ---- the draw
  const double target = u * kept_mass;
  if (mass > 0.0 && from <= target && target < to) { border[3] = own; border_before[3] = before; border_mass[3] = from; }       // (else: the first block)
  __syncthreads();
  const Block x = block_of(border[3], border_before[3], border_mass[3]);
  const uint64_t hit = __builtin_amdgcn_ballot_w64(x.n && x.upto > target), have = __builtin_amdgcn_ballot_w64(x.n && x.weight > 0.0);
  const int at = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(have | 1ull);
  const double into = fmax(target - (x.upto - (double)x.n * x.weight), 0.0) / x.weight;
  // (none: a block whose weights are below binary64 one by one, though not in the polynomial, and which the scans' rounding gave the target.  The
  // largest value then: every value that is looked for below has a token.)
  const bool some = (hit | have) != 0;
  const uint32_t key = some ? (uint32_t)__builtin_amdgcn_readlane((int)x.key, at) : top;
  const uint32_t rank = some ? (uint32_t)__builtin_amdgcn_readlane((int)(x.n ? min((uint32_t)fmin(into, 4e9), x.n - 1) : 0u), at) : 0u;

  // ---- which of the tokens of that value: matches of every wavefront and trip, in the order of the indices
  __syncthreads();
  uint32_t* const table = hist;
  for (int i = tid; i < (trips + 3) * kSampleWaves; i += kSampleThreads) table[i] = 0u;      // (trips go by fours)
  __syncthreads();
  // the value's bits, and the bits of a logit that count (either zero is the value 0)
  const uint32_t wanted = (key & 0x8000u ? key ^ 0x8000u : key ^ 0xFFFFu) * 0x10001u, counts = wanted ? 0xFFFFFFFFu : 0x7FFF7FFFu;
  const auto matches = [&](const uint4& q) {
    const uint32_t w[4] = {(q.x ^ wanted) & counts, (q.y ^ wanted) & counts, (q.z ^ wanted) & counts, (q.w ^ wanted) & counts};
    uint32_t zeros = 0, found = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) zeros |= (w[i] - 0x00010001u) & ~w[i] & 0x80008000u;        // a half that is zero shows
    if (zeros) {
#pragma unroll
      for (int e = 0; e < 8; ++e) found |= (e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu) == 0 ? 1u << e : 0u;
    }
    return found;
  };
  const auto note = [&](int t, const uint4& q) {
    const uint32_t found = matches(q);
    if (found) atomicAdd(&table[t * kSampleWaves + wave], (uint32_t)__popc(found));
  };
#pragma unroll
  for (int t = 0; t < kSampleKept; ++t)
    if (t < trips) note(t, kept[t]);
  further(kSampleKept, trips, note);
  __syncthreads();
  if (wave == 0) {
    const int cells = trips * kSampleWaves, per = (cells + 63) / 64;
    uint32_t n = 0;
    for (int i = 0; i < per; ++i) n += lane * per + i < cells ? table[lane * per + i] : 0u;
    const uint32_t sum_n = lane_scan(n);
    uint32_t before_n = sum_n - n;
    if (before_n <= rank && rank < sum_n) {
      int i = lane * per;
      while (before_n + table[i] <= rank) before_n += table[i++];
      cell_found[0] = (uint32_t)i;
      cell_found[1] = rank - before_n;
    }
  }
  __syncthreads();
  const int cell = (int)cell_found[0];
  if (wave == (cell & (kSampleWaves - 1))) {
    const int piece = cell / kSampleWaves * kSampleThreads + tid;
    uint32_t found = matches(sample_piece(row, p.V, piece));
    const uint32_t n = (uint32_t)__popc(found), sum_n = lane_scan(n);
    uint32_t left = cell_found[1];
    if (sum_n - n <= left && left < sum_n) {
      for (left -= sum_n - n; left; --left) found &= found - 1;        // the lowest set bit off
      p.tokens[r] = 8 * piece + __builtin_ctz(found);
    }
  }
}

struct AcceptTokensArgs {
  const int32_t* chosen;     // [B][gamma+1]
  const int32_t* draft;      // [B][gamma]
  int32_t* n_accept;         // [B]
  int32_t* out_tokens;       // [B][gamma+1]
  int gamma;
};

// The walk of accept_kernel over tokens that are there already: grid B, one wavefront a sequence, 64 rows at a time.
__global__ __launch_bounds__(64) void accept_tokens_kernel(AcceptTokensArgs p) {
  const int b = blockIdx.x, lane = threadIdx.x, rows = p.gamma + 1;
  bool open = true;                       // no draft rejected so far
  for (int base = 0; base < rows; base += 64) {
    const int j = base + lane;
    const int32_t token = j < rows ? p.chosen[(size_t)b * rows + j] : 0;
    const bool same = j < p.gamma && p.draft[(size_t)b * p.gamma + j] == token;
    const uint64_t miss = __ballot(j < rows && !same);
    const int stop = miss ? __builtin_ctzll(miss) : 64;
    if (j < rows) p.out_tokens[(size_t)b * rows + j] = open && lane <= stop ? token : -1;
    if (open && miss && lane == 0) p.n_accept[b] = base + stop;
    if (miss) open = false;
  }
}

}  // namespace qspec
