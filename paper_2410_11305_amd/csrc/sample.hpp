// The choice of a token from fp16 logits by a given random number: temperature, top-k, min-p, top-p, then the inverse
// of the running mass; and the acceptance walk over tokens chosen that way.
//
// A logit is one of 65536 values, so a row is its histogram: counts of every value (65536 counters of 16 bits, 128 KB of
// LDS, one workgroup per row), added up as integers.  All tokens of one value weigh the same and follow one another in the
// order of the draw (falling logit, the lowest index first among equals), so every limit and the draw itself are decided from the counts and
// exp((value - max) / temperature) in binary64, whatever order the logits arrived in; only the last step, which of the
// tokens of one value, looks at indices.  No sort, no passes over candidates, every logit read once for the counts and
// once more for the index.
//
// A thread owns 64 neighbouring values, which are equally spaced (64 divides every binade): two exponentials give it all 64 weights.
#pragma once
#include "accept.hpp"
#include "common.hpp"

namespace qspec {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kSampleOwn = 64;                                // values of a thread
constexpr int kSampleCounts = 65535;                          // logits whose counts fit 16 bits, whatever they are
constexpr int kSampleRound = 8 * kSampleThreads;              // logits of one trip
constexpr int kSampleMaxV = 256 * kSampleRound;               // a table of 16 counters per trip takes the histogram's place

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
// degree 13 on +-ln 2 / 2 (the next term is below 2^-57).
__device__ inline double exp_negative(double x) {
  x = fmax(x, -800.0);
  const double n = rint(x * 1.44269504088896340736);
  const double r = fma(n, -1.90821492927058770002e-10, fma(n, -6.93147180369123816490e-01, x));
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

// Order of the values as 16 bits (half_order_key); 0 for what cannot be drawn, -inf and NaN.
__device__ __forceinline__ uint32_t sample_key(uint32_t bits) {
  return (bits & 0x7FFFu) > 0x7C00u || bits == 0xFC00u ? 0u : half_order_key(bits);
}
__device__ __forceinline__ double sample_value(uint32_t key) {
  return (double)half_bits_to_float((uint16_t)(key & 0x8000u ? key ^ 0x8000u : key ^ 0xFFFFu));
}

// Piece i of a row: 8 logits from 8 i on, -inf past the end.  VEC: rows start on 16 bytes and V % 8 == 0.
template <bool VEC>
__device__ __forceinline__ uint4 sample_piece(const uint16_t* row, int V, int i) {
  uint4 q = {0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u};
  if (VEC) {
    if (8 * i < V) q = reinterpret_cast<const uint4*>(row)[i];
  } else {
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = 8 * i + e < V ? row[8 * i + e] : 0xFC00u;
    q = uint4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
  }
  return q;
}
__device__ __forceinline__ uint32_t piece_bits(const uint4& q, int e) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  return e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu;
}

// grid rows.
template <bool VEC>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs p) {
  __shared__ uint32_t hist[32768];                            // two values' counts a word
  __shared__ uint32_t wave_u[kSampleWaves];
  __shared__ double wave_d[kSampleWaves];
  __shared__ double shared_mass;
  __shared__ uint32_t shared_key, shared_rank;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = blockIdx.x, b = r / p.per;
  const uint16_t* const row = p.logits + (size_t)r * p.V;
  const int own = kSampleThreads - 1 - tid;                   // block of values, the largest first
  // (word i of a block stands at i ^ block: a wavefront reads 32 blocks at once without meeting in a bank)
  const auto word_of = [](uint32_t d) { return (d & ~31u) | ((d ^ (d >> 5)) & 31u); };

  // ---- counts
#pragma unroll
  for (int i = 0; i < 32; ++i) hist[i * kSampleThreads + tid] = 0u;
  uint32_t count[kSampleOwn];
#pragma unroll
  for (int i = 0; i < kSampleOwn; ++i) count[i] = 0u;
  __syncthreads();
  const int pieces = (p.V + 7) / 8;
  for (int base = 0; base < pieces; base += kSampleCounts / 8) {
    const int end = min(pieces, base + kSampleCounts / 8);
    for (int i = base + tid; i < end; i += kSampleThreads) {
      const uint4 q = sample_piece<VEC>(row, p.V, i);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t key = sample_key(piece_bits(q, e));
        if (key) atomicAdd(&hist[word_of(key >> 1)], key & 1u ? 0x10000u : 1u);
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      uint32_t* const w = &hist[own * 32 + ((i ^ own) & 31)];
      count[2 * i] += *w & 0xFFFFu;
      count[2 * i + 1] += *w >> 16;
      *w = 0u;
    }
    __syncthreads();
  }

  // ---- the largest value, and how many tokens come before this thread's
  uint32_t here = 0, top = 0;
#pragma unroll
  for (int i = 0; i < kSampleOwn; ++i) {
    here += count[i];
    if (count[i]) top = (uint32_t)(own * kSampleOwn + i);
  }
  top = wave_max_u32(top);
  if (lane == 0) wave_u[wave] = top;
  __syncthreads();
  for (int w = 0; w < kSampleWaves; ++w) top = max(top, wave_u[w]);
  __syncthreads();
  if (top == 0) {                                             // nothing to choose from
    if (tid == 0) p.tokens[r] = -1;
    return;
  }
  uint32_t upto = here;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t up = __shfl_up(upto, d);
    if (lane >= d) upto += up;
  }
  if (lane == 63) wave_u[wave] = upto;
  __syncthreads();
  uint32_t before = upto - here;
  for (int w = 0; w < wave; ++w) before += wave_u[w];

  // ---- this thread's part of the mass
  const float temperature = p.temperature ? p.temperature[b] : 1.0f;
  const bool greedy = !(temperature > 0.0f);
  const uint32_t k = greedy ? 1u : p.top_k && p.top_k[b] > 0 ? (uint32_t)p.top_k[b] : 0xFFFFFFFFu;
  const double least = p.min_p && p.min_p[b] > 0.0f ? fmin((double)p.min_p[b], 1.0) : 0.0;
  const double inverse = greedy ? 0.0 : 1.0 / (double)temperature;
  const double top_value = sample_value(top);
  const bool infinite = top == 0xFC00u;                        // +inf: the others weigh nothing beside it
  const uint32_t high = min((uint32_t)(own * kSampleOwn + kSampleOwn - 1), top);
  double first = 0.0, ratio = 0.0;
  if (here && before < k) {
    first = high == top ? 1.0 : infinite ? 0.0 : exp_negative((sample_value(high) - top_value) * inverse);
    ratio = infinite ? 0.0 : exp_negative((sample_value(own * kSampleOwn) - sample_value(own * kSampleOwn + 1)) * inverse);
  }
  // f(value, tokens of it, weight) for this thread's values from the largest on, within top_k and min_p, until it returns true
  const auto walk = [&](auto f) {
    double w = first;
    uint32_t at = before;
#pragma unroll
    for (int i = kSampleOwn - 1; i >= 0; --i) {
      const uint32_t key = (uint32_t)(own * kSampleOwn + i);
      if (key <= high) {
        const uint32_t n = at >= k ? 0u : min(count[i], k - at);
        if (n && w > 0.0 && !(w < least)) {
          if (f(key, n, w)) return;
        }
        at += count[i];
        w *= ratio;
      }
    }
  };
  double mass = 0.0;
  if (here && before < k) walk([&](uint32_t, uint32_t n, double w) { mass = fma((double)n, w, mass); return false; });
  double sum = mass;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double up = __shfl_up(sum, d);
    if (lane >= d) sum += up;
  }
  if (lane == 63) wave_d[wave] = sum;
  __syncthreads();
  double wave_base = 0.0, total = 0.0;
  for (int w = 0; w < kSampleWaves; ++w) {
    if (w == wave) wave_base = total;
    total += wave_d[w];
  }
  const double up = __shfl_up(sum, 1);
  const double from = lane ? wave_base + up : wave_base, to = wave_base + sum;     // (to is the next thread's from, bit for bit)

  // ---- top-p: the shortest beginning that holds this much
  const float share = p.top_p ? p.top_p[b] : 1.0f;
  double kept = total;
  if (share < 1.0f) {
    const double limit = fmax((double)share * total, 1e-300);              // (the first token is always kept)
    if (from < limit && limit <= to) {
      double cum = from, cut = from;
      walk([&](uint32_t, uint32_t n, double w) {
        const double all = fma((double)n, w, cum);
        cut = all;
        if (all >= limit) {
          cut = fma(fmin(fmax(ceil((limit - cum) / w), 1.0), (double)n), w, cum);
          return true;
        }
        cum = all;
        return false;
      });
      shared_mass = cut;
    }
    __syncthreads();
    kept = shared_mass;
  }

  // ---- the draw
  const double u = (double)fminf(fmaxf(p.u[r], 0.0f), 0.99999994f);
  const double target = u * kept;
  if (from <= target && target < to) {
    double cum = from;
    uint32_t key = 0, rank = 0;
    walk([&](uint32_t v, uint32_t n, double w) {
      const double all = fma((double)n, w, cum);
      key = v;
      rank = min((uint32_t)fmin((target - cum) / w, 4e9), n - 1);
      cum = all;
      return all > target;
    });
    shared_key = key;
    shared_rank = rank;
  }
  __syncthreads();
  const uint32_t key = shared_key, rank = shared_rank;

  // ---- which of the tokens of that value: matches of every wavefront and trip, in the order of the indices
  uint32_t* const table = hist;
  const int trips = (pieces + kSampleThreads - 1) / kSampleThreads;
  for (int t = 0; t < trips; ++t) {
    const uint4 q = sample_piece<VEC>(row, p.V, t * kSampleThreads + tid);
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) n += (uint32_t)__popcll(__ballot(sample_key(piece_bits(q, e)) == key));
    if (lane == 0) table[t * kSampleWaves + wave] = n;
  }
  __syncthreads();
  if (wave == 0) {
    const int cells = trips * kSampleWaves, per = (cells + 63) / 64;
    uint32_t n = 0;
    for (int i = 0; i < per; ++i) n += lane * per + i < cells ? table[lane * per + i] : 0u;
    uint32_t sum_n = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t below = __shfl_up(sum_n, d);
      if (lane >= d) sum_n += below;
    }
    uint32_t at = sum_n - n;
    if (at <= rank && rank < sum_n) {
      int i = lane * per;
      while (at + table[i] <= rank) at += table[i++];
      wave_u[0] = (uint32_t)i;
      wave_u[1] = rank - at;
    }
  }
  __syncthreads();
  const int cell = (int)wave_u[0];
  if (wave == (cell & (kSampleWaves - 1))) {
    const int piece = cell / kSampleWaves * kSampleThreads + tid;
    const uint4 q = sample_piece<VEC>(row, p.V, piece);
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) n += sample_key(piece_bits(q, e)) == key ? 1u : 0u;
    uint32_t sum_n = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t below = __shfl_up(sum_n, d);
      if (lane >= d) sum_n += below;
    }
    uint32_t left = wave_u[1];
    if (sum_n - n <= left && left < sum_n) {
      left -= sum_n - n;
      int found = 0;
#pragma unroll
      for (int e = 7; e >= 0; --e) {
        // matches of this piece before element e
        uint32_t first_of = 0;
        for (int i = 0; i < e; ++i) first_of += sample_key(piece_bits(q, i)) == key ? 1u : 0u;
        if (sample_key(piece_bits(q, e)) == key && first_of == left) found = e;
      }
      p.tokens[r] = 8 * piece + found;
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
