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
// factor of 16 is taken out of q (its row is scaled by a power of two first, so that only features 2^23 times smaller than its largest
// lose bits, which the sums in binary32 do not keep either); the values'
// codes are shifted to 16 * code * 2^-24 all alike, and the finished sums scaled.  The token order of the second product
// is that of the first one's results: p goes from the accumulators into the next operand without crossing lanes, and a
// lane's codes of four tokens are 16 bytes of the cache (kv4.hpp).
//
// Work: an item is one block of rows of one sequence and one key/value head, a step 32 or 64 tokens.  The workgroups share
// the steps of all items evenly, whatever the lengths, each taking one run of them; the wavefronts of a workgroup
// take its steps in turn and join their sums through LDS.  An item that several workgroups share is joined by the last of them
// to finish (last_arrival), from partial sums in the workspace.  Where there are more items than workgroups and sorted by length they come
// out as even, they are dealt out whole.  The lengths are known on the device only: every
// workgroup works the division out for itself.
//
// Measured (device time; bytes of the cache, queries and results): 8 sequences of up to 2048 tokens, one row of 32 heads, 21.8 us
// (2.9 TB/s); 131071 tokens, one row of 64 over 8 heads, 38.8 us (3.7 TB/s); 32 sequences through a window of 4096, 64 over 8 heads of
// 64, 26.8 us (2.8 TB/s); 128 sequences of 200 to 2048 tokens, 4 rows of 64 over 8 heads, 59.5 us (2.9 TB/s, 320 TF/s); a prompt of
// 2050 tokens of 32 heads 77.7 us (445 TF/s), a chunk of 2050 rows over 4096 tokens of 64 over 8 heads 331 us (620 TF/s).  Short passes are bound by
// the start (1.4 us of division, 3 us to the first scores) and the joins.  Long ones of few rows wait (36 to 43 % of a wavefront's life) as much
// as they issue, the vector unit works in 27 to 34 % of its cycles.  From 17 rows on it works in 55 % (32 rows), 37 % (64: two wavefronts a SIMD,
// in which the products and the exponentials of a step wait for one another), the matrix unit in 12 %: it takes 5 to 7 vector
// instructions a word to widen and a dozen a score.
#pragma once
#include "common.hpp"
#include "exchange.hpp"
#include "kv4.hpp"

namespace qspec {

constexpr size_t kAttnTicketBytes = 16384;   // arrival counters at the head of the workspace, two a workgroup
constexpr int kAttnRounds = 8;               // rounds of whole items (more have little left to gain: one part of many)
// The shape of an instance.  NB: blocks of 16 columns a wavefront carries; F: token tiles that share a block (below).
// Two workgroups of four wavefronts to a compute unit: the loop is free of spills (a reload inside it waits for every load
// under way), and one workgroup's start and end of an item stand beside the other's steps.  Workgroups of eight wavefronts, one
// to a unit, halve the parts of a shared item but leave those gaps open (64 sequences of up to 2000 tokens, 8 heads of
// 64, 4 rows: 33 us and 24); three of four, where the registers allow them, bring more parts than they hide (131071 tokens: 62 and 47).
template <int NB, int F>
struct AttnForm {
  static constexpr int waves = 4;
  static constexpr int workgroups = 512;                           // of a launch; two parts of an item each in the workspace at most
  static constexpr int tiles = F > 1 ? 4 : 2;                      // 16-token tiles of a step (8 at F = 4: 27 us for 22 at 8 x 2048 tokens)
  static constexpr int step = 16 * tiles;                          // tokens of a step
  static constexpr int rows = 16 * NB / F;                         // rows of a block of an item
  // In steps: what the start and the end of an item cost beside its steps (measured: 3 us and more, of which an item's
  // steps of 1024 tokens take as much), items that are not shared out, and what a workgroup gets on average at least.
  static constexpr int over = (NB == 1 ? 1024 : NB == 2 ? 768 : 512) / step;
  static constexpr int whole = 1024 / step;
  static constexpr int least = (NB == 1 ? 512 : NB == 2 ? 640 : 1280) / step;
  static_assert(over >= 2 * waves && least >= 2 * waves, "no workgroup's share rounds down to nothing");
  static_assert(2 * workgroups * sizeof(unsigned) <= kAttnTicketBytes, "two counters for every workgroup");
};

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

// The position that a row of a block's window begins behind.  (A row in front of the sequence sees nothing, whatever its window.)
__device__ __forceinline__ int behind_window(const AttnArgs& p, int at) { return max(at, 0) - p.window; }

// pos: position of the sequence's first row.  (Held, so that sums stay in 32 bits: from below far in front of the sequence, where rows see nothing,
// from above to the last positions that there are.)
template <int STEP>
__device__ __forceinline__ AttnSpan attn_span(const AttnArgs& p, int pos, int block, int rows_per_block) {
  const int r0 = block * rows_per_block, r1 = min(p.kv.T * p.G, r0 + rows_per_block) - 1;
  pos = min(max(pos, -(1 << 30)), 0x7fffffff - p.kv.T);
  AttnSpan s;
  s.lo = pos + over_group(p, r0);
  s.hi = pos + over_group(p, r1);
  const int end = min(s.hi + 1, p.kv.max_pages << p.kv.page_shift);      // tokens 0 .. end - 1
  s.first = p.window > 0 ? max(behind_window(p, s.lo) + 1, 0) / STEP : 0;
  s.sink_steps = p.window > 0 ? max(min((min(p.sinks, end) + STEP - 1) / STEP, s.first), 0) : 0;
  // at least one: rows that see nothing have their zeros written
  s.steps = max(s.sink_steps + max((end + STEP - 1) / STEP - s.first, 0), 1);
  return s;
}

// Sum and maximum over the four lanes that hold one column of an accumulator (lanes 16 and 32 apart).
__device__ __forceinline__ float column_sum(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  v = __builtin_bit_cast(float, (uint32_t)a[0]) + __builtin_bit_cast(float, (uint32_t)a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return __builtin_bit_cast(float, (uint32_t)b[0]) + __builtin_bit_cast(float, (uint32_t)b[1]);
}
__device__ __forceinline__ float column_max(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  v = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}
// Sum and maximum over the F columns that hold one row (16 / F columns apart).
template <int F>
__device__ __forceinline__ float group_sum(float v) {
  if (F > 1) v += dpp_f32<0x128>(v);            // rotation by 8 in a row of 16 lanes
  if (F > 2) v += dpp_f32<0x124>(v);            // and by 4: the two sums of pairs alternate
  return v;
}
template <int F>
__device__ __forceinline__ float group_max(float v) {
  if (F > 1) v = fmaxf(v, dpp_f32<0x128>(v));
  if (F > 2) v = fmaxf(v, dpp_f32<0x124>(v));
  return v;
}

__device__ __forceinline__ v8h half_frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(v8h, uint4{a, b, c, d});
}
__device__ __forceinline__ v8h widen_codes(uint32_t x) {       // a word's 8 codes, in the order of the features
  const uint32_t y = x >> 8;
  return half_frag(x & 0x000F000Fu, x & 0x00F000F0u, y & 0x000F000Fu, y & 0x00F000F0u);
}

// A row of an item as its workgroups hand it over: reference, sum, (two unused), o
__host__ __device__ constexpr int attn_part_floats(int D) { return D + 4; }

// The workspace of an instance: what its launch indexes.
template <int D, int NB, int F>
constexpr size_t attn_workspace() {
  typedef AttnForm<NB, F> Form;
  return kAttnTicketBytes + (size_t)2 * Form::workgroups * Form::rows * attn_part_floats(D) * sizeof(float);
}

// D features a head, NB blocks of 16 columns, F tiles of tokens to a block.
//
// With up to 16 / F rows, F > 1, the columns of a block hold the rows F times over, and column c takes the tokens of tile
// c / (16 / F) of a step only: the scores of the F tiles are computed for all columns and each column keeps its own, which
// costs a selection and saves (F - 1) / F of the exponentials and all that goes with them; in the second product a
// column's weights are zero for the tiles of the others.  Each column ends with its own sums, joined like those of the wavefronts.
template <int D, int NB, int F>
__global__ __launch_bounds__((64 * AttnForm<NB, F>::waves), 2) void attn_kv4_kernel(AttnArgs p) {
  typedef AttnForm<NB, F> Form;
  constexpr int WAVES = Form::waves, THREADS = 64 * WAVES, TILES = Form::tiles, STEP = Form::step, RB = Form::rows, OVER = Form::over;
  constexpr int NK = D / 32;                  // matrix instructions of a tile of q k^T; words of a lane of a key
  constexpr int NV = D / 16;                  // matrix instructions of two tiles of p v
  constexpr int COLS = 16 / F;                // rows of a block of columns
  constexpr int NX = 4 * TILES / F;           // scores of a lane in a step and block
  constexpr int NP = NX / 4;                  // tiles of a lane
  constexpr int PITCH = D + 4;                // floats of a row in LDS
  constexpr int LANES = D / 4;                // threads of a row where sums are joined, 4 features each
  constexpr int PART = attn_part_floats(D);
  constexpr bool Q_LDS = NB == 4;             // the rows' registers would not leave room for the sums
  constexpr bool TIGHT = NB == 4;                        // registers for the sums and the loads under way, none for widening ahead
  constexpr int kPass = 0x108;                // past the fences: matrix instructions and LDS reads (us, prompts: 80 -> 77, 342 -> 331)
  constexpr float kNone = -1e30f;             // reference of a row that has seen nothing: below every score
  __shared__ __align__(16) float o_lds[WAVES][COLS][PITCH];
  __shared__ float m_lds[WAVES][COLS], l_lds[WAVES][COLS], c_lds[WAVES][COLS];
  __shared__ float join_m[THREADS / LANES], join_l[THREADS / LANES];
  __shared__ uint4 q_lds[Q_LDS ? NB * NK * 64 : 1];
  __shared__ float4 f_lds[Q_LDS ? RB : 1];    // factor, sum, position of a row
  __shared__ unsigned ticket;
  __shared__ uint32_t taken[kAttnRounds];     // this workgroup's items where they are dealt out whole
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int col = lane & 15, kb = lane >> 4, mine_tile = F > 1 ? col / COLS : 0;
  const int P = 1 << p.kv.page_shift, R = p.kv.T * p.G, Hkv = p.kv.Hkv;
  const uint32_t region_bytes = (uint32_t)P * (D + 8);
  const int row_of = tid / LANES, own = (tid & (LANES - 1)) * 4;       // join: row, first feature
  const auto sequence_of = [&](int e) { return p.blocks == 1 ? e : e / p.blocks; };

  // ---- the division of the work: entries are (sequence, block of rows), each of Hkv items of equal size, OVER + steps.
  // Every wavefront works it out by itself, a run of entries to a lane: no barrier stands before the first loads.
  const int entries = p.B * p.blocks;
  const int per = (entries + 63) / 64;
  const auto size_of = [&](int e, int pos) {
    return (uint32_t)(OVER + attn_span<STEP>(p, pos, e - sequence_of(e) * p.blocks, RB).steps) * (uint32_t)Hkv;
  };
  uint32_t mine = 0;
  for (int e = lane * per; e < min(entries, (lane + 1) * per); ++e) mine += size_of(e, p.kv.pos[sequence_of(e)]);
  uint32_t upto = mine;                       // of the entries up to this lane's
#define QSPEC_DPP_ADD(ctrl, rows) upto += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)upto, ctrl, rows, 0xf, false)
  QSPEC_DPP_ADD(0x111, 0xf);                  // row_shr 1, 2, 4, 8: sums inside a row of 16
  QSPEC_DPP_ADD(0x112, 0xf);
  QSPEC_DPP_ADD(0x114, 0xf);
  QSPEC_DPP_ADD(0x118, 0xf);
  QSPEC_DPP_ADD(0x142, 0xa);                  // row_bcast 15 into rows 1 and 3
  QSPEC_DPP_ADD(0x143, 0xc);                  // row_bcast 31 into rows 2 and 3
#undef QSPEC_DPP_ADD
  const uint32_t total = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  const uint32_t groups = uniform(min((uint32_t)gridDim.x, max((uint32_t)(entries * Hkv), (total - (uint32_t)(entries * Hkv) * OVER) / Form::least)));
  const uint32_t me = blockIdx.x;
  if (me >= groups) return;
  // workgroup w begins at w * share, and the first `more` of them take one more each; inside an item it begins a whole
  // number of rounds of its wavefronts in, or with the item in one that is not shared out
  const uint32_t share = uniform(total / groups), more = total - share * groups;
  const auto start_of = [&](uint32_t w) { return w * share + min(w, more); };
  const auto group_of = [&](uint32_t x) {     // the last workgroup that begins at x or before
    const uint32_t wide = more * (share + 1);
    return uniform(x < wide ? x / (share + 1) : more + (x - wide) / share);
  };
  struct Place { int entry, head, step; uint32_t item; };     // item: where its item starts
  const auto place_of = [&](uint32_t x) {
    if (x >= total) return Place{entries, 0, 0, total};
    const int owner = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > x));
    uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), owner), n = (uint32_t)__builtin_amdgcn_readlane((int)mine, owner);
    int e = owner * per;
    if (per > 1) {
      for (;; ++e) {
        n = uniform(size_of(e, uniform(scalar_load(p.kv.pos, sequence_of(e)))));
        if (x - at < n) break;
        at += n;
      }
    }
    const uint32_t each = uniform(n / (uint32_t)Hkv), head = uniform((x - at) / each), in = x - at - head * each;
    return Place{e, (int)head, each <= Form::whole + OVER || in < OVER ? 0 : (int)((in - OVER) & ~(WAVES - 1u)), at + head * each};
  };
  // Whole items instead, where they come out as even: in the order of falling length, dealt out in rounds, first to last
  // workgroup, last to first, and so on, long ones and short ones add up.  A run that begins inside an item pays one more
  // start and end, so much may the fullest workgroup have on top of an even share here.  (us: prompt of 2050 tokens,
  // 32 heads 81 for 99, 4 of 512 46 for 57; 128 sequences of 200 to 2048 tokens, 4 rows of 64 over 8 heads 60 for 67.)
  const uint32_t items = (uint32_t)(entries * Hkv);
  const auto dealt = [&](uint32_t round, uint32_t w) { return round * gridDim.x + (round & 1 ? gridDim.x - 1 - w : w); };
  bool whole_items = false;
  if (items > gridDim.x && items <= kAttnRounds * gridDim.x && (NB == 4 || entries <= THREADS)) {
    // Prompts of one length and history are in order by their blocks; the fullest workgroup is one of the ends, or at the
    // end of the last round.  Few rows: one block, or a few, a sequence, and the lengths are sorted, in the LDS of the sums to come.
    uint32_t* const lengths = reinterpret_cast<uint32_t*>(&o_lds[0][0][0]);
    uint16_t* const order = reinterpret_cast<uint16_t*>(lengths + THREADS);
    static_assert(sizeof(o_lds) >= THREADS * 6, "room for both");
    const auto load_of = [&](uint32_t w, auto length_of) {
      uint32_t load = 0;
      for (uint32_t round = 0; round * gridDim.x < items; ++round) {
        const uint32_t i = dealt(round, w);
        if (i < items) load += length_of(i / (uint32_t)Hkv);
      }
      return load;
    };
    bool even = true;
    if (NB == 4) {
      const int pos = uniform(scalar_load(p.kv.pos, 0));
      for (int e = lane; e < p.B; e += 64) even &= p.kv.pos[e] == pos;
      const uint32_t rest = max(items % gridDim.x, 1u);
      const uint32_t load = load_of(lane == 0 ? 0 : lane == 1 ? gridDim.x - 1 : lane == 2 ? rest - 1 : gridDim.x - rest, [&](uint32_t place) {
        return (uint32_t)(OVER + attn_span<STEP>(p, pos, p.blocks - 1 - (int)(place / (uint32_t)p.B), RB).steps);
      });
      even &= lane > 3 || load <= share + OVER;
      even = __builtin_amdgcn_ballot_w64(!even) == 0;
    } else {
      const int seq = sequence_of(tid);
      const uint32_t length = tid < entries ? (uint32_t)(OVER + attn_span<STEP>(p, p.kv.pos[seq], tid - seq * p.blocks, RB).steps) : 0u;
      lengths[tid] = length;
      __syncthreads();
      uint32_t rank = 0;
#pragma unroll 4
      for (int j = 0; j < entries; j += 4) {
        const uint4 other = *reinterpret_cast<const uint4*>(lengths + j);
        rank += other.x > length || (other.x == length && j < tid) ? 1u : 0u;
        rank += other.y > length || (other.y == length && j + 1 < tid) ? 1u : 0u;
        rank += other.z > length || (other.z == length && j + 2 < tid) ? 1u : 0u;
        rank += other.w > length || (other.w == length && j + 3 < tid) ? 1u : 0u;
      }
      __syncthreads();
      if (tid < entries) {
        lengths[rank] = length;
        order[rank] = (uint16_t)tid;
      }
      __syncthreads();
      for (uint32_t w = tid; w < gridDim.x; w += THREADS) even &= load_of(w, [&](uint32_t place) { return lengths[place]; }) <= share + OVER;
    }
    if (tid < kAttnRounds) {
      const uint32_t i = dealt(tid, me), place = i / (uint32_t)Hkv, from_top = place / (uint32_t)p.B;
      const uint32_t e = NB == 4 ? (place - from_top * (uint32_t)p.B) * (uint32_t)p.blocks + (uint32_t)p.blocks - 1 - from_top : i < items ? order[place] : 0u;
      taken[tid] = i < items ? e * (uint32_t)Hkv + i - place * (uint32_t)Hkv : items;
    }
    whole_items = __syncthreads_and(even);
  }
  // item: where it starts; or, for whole ones (last_head is -1), the round
  int entry, head, begin = 0, last_entry = entries, last_head = -1, last_step = 0;
  uint32_t item = 0;
  const auto take = [&] {
    const uint32_t i = item < (uint32_t)kAttnRounds ? uniform(taken[item]) : (uint32_t)(entries * Hkv);
    entry = (int)uniform(i / (uint32_t)Hkv);
    head = (int)(i - (uint32_t)entry * (uint32_t)Hkv);
  };
  if (whole_items) {
    take();
  } else {
    const Place from = place_of(start_of(me)), to = place_of(start_of(me + 1));
    entry = from.entry; head = from.head; begin = from.step; item = from.item;
    last_entry = to.entry; last_head = to.head; last_step = to.step;
  }
  bool first_run = true;

  while (entry < last_entry || (entry == last_entry && (head < last_head || (head == last_head && begin < last_step)))) {
    const int b = uniform(sequence_of(entry)), block = entry - b * p.blocks;
    AttnSpan span = attn_span<STEP>(p, uniform(scalar_load(p.kv.pos, b)), block, RB);
    span.steps = uniform(span.steps); span.sink_steps = uniform(span.sink_steps); span.first = uniform(span.first);
    span.lo = uniform(span.lo); span.hi = uniform(span.hi);
    const int stop = entry == last_entry && head == last_head ? last_step : span.steps;
    const int rows = min(RB, R - block * RB);

    // ---- loads of a step: keys and values of its tiles, steps and lows of this lane's tiles
    struct Raw { uint32_t k[TILES][NK]; uint4 v[TILES], par[NP][2]; };
    Raw raw;
    struct Pages { int page[TILES]; uint32_t there; };    // of every tile, and a bit for each that exists
    const auto first_token = [&](int s) { return STEP * (s < span.sink_steps ? s : s - span.sink_steps + span.first); };
    // Pages of the next 64 tiles of this wavefront, BATCH steps, a tile to a lane: they are looked up a batch ahead.
    constexpr int BATCH = 64 / TILES;
    const auto look_up = [&](int s) {
      const int i = (first_token(min(s + lane / TILES * WAVES, span.steps - 1)) + lane % TILES * 16) >> p.kv.page_shift;
      if (i >= p.kv.max_pages) return -1;
      const size_t at_page = (size_t)b * p.kv.max_pages + i;
      return p.kv.table != nullptr ? p.kv.table[at_page] : (int)at_page;
    };
    int known = look_up(begin + wave), ahead = -1;
    const auto pages_of = [&](int k) {        // of the batch's step k
      Pages g;
      g.there = 0;
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const int page = i > 0 && P >= STEP ? g.page[0] : __builtin_amdgcn_readlane(known, k * TILES + i);
        const bool there = page >= 0 && page < p.kv.n_pages;
        g.page[i] = there ? page : 0;
        g.there |= there ? 1u << i : 0u;
      }
      return g;
    };
    const auto region_of = [&](int page) { return p.cache + (size_t)(uint32_t)(page * Hkv + head) * region_bytes; };
    const uint32_t k_off = (uint32_t)(col * (D / 2) + kb * (4 * NK)), par_off = (uint32_t)(kb * 32);
    const uint32_t v_off = (uint32_t)((col & (D / 8 - 1)) * 64 + kb * 16);
    const auto load_keys = [&](int t, const Pages& g) {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const uint8_t* const src = region_of(g.page[i]) + (uint32_t)((t + 16 * i) & (P - 1)) * (D / 2);
        if (NK == 4) {
          const uint4 w = *reinterpret_cast<const uint4*>(src + k_off);
          raw.k[i][0] = w.x; raw.k[i][1] = w.y; raw.k[i][NK - 2] = w.z; raw.k[i][NK - 1] = w.w;
        } else {
          const uint2 w = *reinterpret_cast<const uint2*>(src + k_off);
          raw.k[i][0] = w.x; raw.k[i][1] = w.y;
        }
      }
    };
    const auto load_rest = [&](int t, const Pages& g, int k) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {                   // its tiles: i * F + mine_tile
        const uint8_t* par;
        if (F == 1 || P >= STEP) {
          par = region_of(g.page[i * F]) + (uint32_t)P * D + (uint32_t)((t + 16 * F * i) & (P - 1)) * 8 + (par_off + (uint32_t)mine_tile * 128);
        } else {                                     // pages that end inside a step: a lane's tile has a region of its own
          const int page = __shfl(known, k * TILES + i * F + mine_tile);
          par = region_of(page >= 0 && page < p.kv.n_pages ? page : 0) + (uint32_t)P * D + (uint32_t)((t + 16 * (i * F + mine_tile)) & (P - 1)) * 8 + par_off;
        }
        raw.par[i][0] = reinterpret_cast<const uint4*>(par)[0];
        raw.par[i][1] = reinterpret_cast<const uint4*>(par)[1];
      }
#pragma unroll
      for (int i = 0; i < TILES; ++i)
        raw.v[i] = *reinterpret_cast<const uint4*>(region_of(g.page[i]) + (uint32_t)P * (D / 2) + (uint32_t)((t + 16 * i) & (P - 1)) * (D / 2) + v_off);
    };
    // ---- the rows: scaled to 2^13 .. 2^14, a sixteenth where the codes come 16 times too large
    v8h qf[Q_LDS ? 1 : NB][NK];
    float f_own[Q_LDS ? 1 : NB], shift_own[Q_LDS ? 1 : NB], m[NB], l[NB], c[NB];      // l: sum of p; c: the part of o that all features share
    int pos_own[Q_LDS ? 1 : NB];
    v4f o[NB][NV];
    const auto row_of_column = [&](int nb) { return block * RB + min(nb * COLS + (col & (COLS - 1)), rows - 1); };     // (columns without a row repeat the last one)
    const auto load_row = [&](int nb, v8h (&x)[NK]) {
      const int r = row_of_column(nb), j = over_group(p, r), g = r - j * p.G;
      const uint16_t* const src = p.q + (((size_t)b * p.kv.T + j) * p.Hq + (size_t)head * p.G + g) * D + kb * 8 * NK;
#pragma unroll
      for (int i = 0; i < NK; ++i) x[i] = __builtin_bit_cast(v8h, reinterpret_cast<const uint4*>(src)[i]);
    };
    const auto scale_row = [&](v8h (&x)[NK], float& factor_of, float& sum_of) {
      float top = 0.0f, sum = 0.0f;
#pragma unroll
      for (int i = 0; i < NK; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { top = fmaxf(top, fabsf((float)x[i][e])); sum += (float)x[i][e]; }
      }
      top = column_max(top);
      sum = column_sum(sum);
      sum += sum - sum;                       // no number if one of the features is none, and then no score is
      const int ex = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) : 0;
      const float up = __builtin_amdgcn_ldexpf(1.0f, 14 - ex);
#pragma unroll
      for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = (_Float16)((float)x[i][e] * (e & 2 ? up * 0.0625f : up));
      factor_of = p.scale_log2 * __builtin_amdgcn_ldexpf(1.0f, ex + 10);
      sum_of = sum * __builtin_amdgcn_ldexpf(1.0f, -ex - 10);
    };
    const auto position_of = [&](int nb) { return span.lo + over_group(p, row_of_column(nb)) - over_group(p, block * RB); };
    if (!Q_LDS) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) load_row(nb, qf[Q_LDS ? 0 : nb]);
    }
    int s = begin + wave, t = 0;
    Pages pages;
    if (s < stop) {
      t = first_token(s);
      pages = pages_of(0);
      load_keys(t, pages);
      load_rest(t, pages, 0);
      ahead = look_up(s + BATCH * WAVES);
    }
    if (Q_LDS) {
      if (wave < NB) {
        v8h x[NK];
        float factor_of, sum_of;
        load_row(wave, x);
        scale_row(x, factor_of, sum_of);
#pragma unroll
        for (int i = 0; i < NK; ++i) q_lds[(wave * NK + i) * 64 + lane] = __builtin_bit_cast(uint4, x[i]);
        if (kb == 0) f_lds[wave * 16 + col] = float4{factor_of, sum_of, __builtin_bit_cast(float, position_of(wave)), 0.0f};
      }
      __syncthreads();
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (!Q_LDS) {
        scale_row(qf[Q_LDS ? 0 : nb], f_own[Q_LDS ? 0 : nb], shift_own[Q_LDS ? 0 : nb]);
        pos_own[Q_LDS ? 0 : nb] = position_of(nb);
      }
      m[nb] = kNone;
      l[nb] = c[nb] = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) o[nb][v] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const auto q_frag = [&](int nb, int w) {
      if (Q_LDS) return __builtin_bit_cast(v8h, q_lds[(nb * NK + w) * 64 + lane]);
      return qf[Q_LDS ? 0 : nb][w];
    };
    const auto factor = [&](int nb) { return Q_LDS ? f_lds[nb * 16 + col].x : f_own[Q_LDS ? 0 : nb]; };
    const auto shift = [&](int nb) { return Q_LDS ? f_lds[nb * 16 + col].y : shift_own[Q_LDS ? 0 : nb]; };
    const auto position = [&](int nb) { return Q_LDS ? __builtin_bit_cast(int, f_lds[nb * 16 + col].z) : pos_own[Q_LDS ? 0 : nb]; };
    int vexp = -30;                           // exponent of the largest value step so far

    // ---- the steps of this wavefront
    for (int k = 1; s < stop; s += WAVES, ++k) {
      const int t_next = first_token(min(s + WAVES, span.steps - 1));       // (the last one's loads repeat a step)
      if (k == BATCH) {
        k = 0;
        known = ahead;
        ahead = look_up(s + (BATCH + 1) * WAVES);
      }
      const Pages next = pages_of(k);
      // every token of the step in sight of every row
      const bool whole = pages.there == (1u << TILES) - 1 && t + STEP - 1 <= span.lo && (p.window == 0 || t > behind_window(p, span.hi) || t + STEP <= p.sinks);
      v4f sc[NB][TILES];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < TILES; ++i) sc[nb][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < NK; ++w) {
        v8h kf[TILES];
#pragma unroll
        for (int i = 0; i < TILES; ++i) kf[i] = widen_codes(raw.k[i][w]);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const v8h x = q_frag(nb, w);
#pragma unroll
          for (int i = 0; i < TILES; ++i) sc[nb][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i], x, sc[nb][i], 0, 0, 0);
        }
        if (TIGHT) __builtin_amdgcn_sched_barrier(kPass);          // (widening ahead would cost the registers of the sums)
      }
      load_keys(t_next, next);

      // steps and lows of this lane's tokens, and its scores
      v2h kp[NX], vp[NX];
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const uint32_t w[8] = {raw.par[i][0].x, raw.par[i][0].y, raw.par[i][0].z, raw.par[i][0].w,
                               raw.par[i][1].x, raw.par[i][1].y, raw.par[i][1].z, raw.par[i][1].w};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          kp[4 * i + x] = __builtin_bit_cast(v2h, w[2 * x]);
          vp[4 * i + x] = __builtin_bit_cast(v2h, w[2 * x + 1]);
        }
      }
      float sv[NB][NX];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float sum_of = shift(nb);
#pragma unroll
        for (int x = 0; x < NX; ++x) {
          float dot = sc[nb][(x >> 2) * F][x & 3];
#pragma unroll
          for (int i = 1; i < F; ++i) dot = mine_tile == i ? sc[nb][(x >> 2) * F + i][x & 3] : dot;
          sv[nb][x] = fmaf(dot, (float)kp[x].x, (float)kp[x].y * sum_of);
        }
      }
      if (!whole) {
        uint32_t any = 0;                     // bit x: a row of this lane sees its token x
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int at_row = position(nb), behind = p.window > 0 ? behind_window(p, at_row) : -1;
#pragma unroll
          for (int x = 0; x < NX; ++x) {
            const int tok = t + ((x >> 2) * F + mine_tile) * 16 + 4 * kb + (x & 3);
            const bool in = ((pages.there >> ((x >> 2) * F + mine_tile) & 1u) != 0) & (tok <= at_row) & ((tok > behind) | (tok < p.sinks));
            any |= in ? 1u << x : 0u;
            sv[nb][x] = in ? sv[nb][x] : -__builtin_inff();
          }
        }
        // whatever stands in rows that nobody sees (infinities, NaN) must not meet a weight, not even one of zero
#pragma unroll
        for (int x = 0; x < NX; ++x) vp[x] = any >> x & 1u ? vp[x] : v2h{(_Float16)0.0f, (_Float16)0.0f};
        if (NB > 1) {
          // nor, in a token that only some of the lane's rows see, the weights of zero of the others: it is taken out, and its NaN left with the rows that see it
          const v2h zero = {(_Float16)0.0f, (_Float16)0.0f};
          v2h odd = vp[0] * zero;
#pragma unroll
          for (int x = 1; x < NX; ++x) odd += vp[x] * zero;
          if (__builtin_amdgcn_ballot_w64(!((float)odd.x + (float)odd.y == 0.0f)) != 0) {
#pragma unroll
            for (int x = 0; x < NX; ++x) {
              const float none = (float)vp[x].x * 0.0f + (float)vp[x].y * 0.0f;
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) c[nb] += sv[nb][x] == -__builtin_inff() ? 0.0f : none;
              vp[x] = none == 0.0f ? vp[x] : zero;
            }
          }
        }
      }
      // The reference: 2^(s - m) times the value steps has to stay inside fp16's range, with its largest terms well above its
      // smallest numbers, so m is the largest score less 8, plus the exponent of the largest value step.  It moves
      // when a term could pass 2^14, which after the first step is rare.
      v2h vmax2 = vp[0];
#pragma unroll
      for (int x = 1; x < NX; ++x) vmax2 = __builtin_elementwise_max(vmax2, vp[x]);
      const float vtop = (float)vmax2.x;
      bool reset = vtop > __builtin_amdgcn_ldexpf(1.0f, vexp);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float top = sv[nb][0];
#pragma unroll
        for (int x = 1; x < NX; ++x) top = fmaxf(top, sv[nb][x]);
        reset |= fmaf(top, factor(nb), -m[nb]) > (float)(14 - vexp);
      }
      if (__builtin_amdgcn_ballot_w64(reset) != 0) {
        float vwide = vtop;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) vwide = fmaxf(vwide, __shfl_xor(vwide, d));
        const int before = vexp;
        vexp = uniform(max(vexp, vwide > 0.0f ? __builtin_amdgcn_frexp_expf(vwide) : vexp));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float top = sv[nb][0];
#pragma unroll
          for (int x = 1; x < NX; ++x) top = fmaxf(top, sv[nb][x]);
          const float to = fmaxf(m[nb] + (float)(vexp - before), fmaf(column_max(top), factor(nb), (float)(vexp - 8)));
          const float by = __builtin_amdgcn_exp2f(m[nb] - to);
          m[nb] = to;
          l[nb] *= by;
          c[nb] *= by;
#pragma unroll
          for (int v = 0; v < NV; ++v) o[nb][v] *= by;
        }
      }
      uint32_t w[NB][NX / 2];                 // the weights, two a word
      typedef float v2f __attribute__((ext_vector_type(2)));
      const v2h minus8 = {(_Float16)-8.0f, (_Float16)-8.0f};
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float by = factor(nb);
#pragma unroll
        for (int x = 0; x < NX; x += 2) {
          const float e0 = __builtin_amdgcn_exp2f(fmaf(sv[nb][x], by, -m[nb]));
          const float e1 = __builtin_amdgcn_exp2f(fmaf(sv[nb][x + 1], by, -m[nb]));
          l[nb] += e0;
          l[nb] += e1;
          c[nb] = fmaf(e0, fmaf(8.0f, (float)vp[x].x, (float)vp[x].y), c[nb]);
          c[nb] = fmaf(e1, fmaf(8.0f, (float)vp[x + 1].x, (float)vp[x + 1].y), c[nb]);
          // 11 bits of a weight, what an fp16 probability keeps, since the matrix unit takes fp16: results are off by 2.4e-4 to 2.8e-4 where
          // their own rounding makes 2.1e-4.  (A second number for what is cut off cost drafts 5 %.)
          const v2h both = __builtin_convertvector((v2f{e0 * (float)vp[x].x, e1 * (float)vp[x + 1].x}), v2h);
          c[nb] = __builtin_amdgcn_fdot2(both, minus8, c[nb], false);
          w[nb][x / 2] = __builtin_bit_cast(uint32_t, both);
        }
        if (TIGHT) __builtin_amdgcn_sched_barrier(kPass);
      }
      // values, two tiles at a time: token pairs of one half of the words, nibble by nibble
#pragma unroll
      for (int pair = 0; pair < TILES / 2; ++pair) {
        v8h pf[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          if (F == 1) {
            pf[nb] = half_frag(w[nb][4 * pair], w[nb][4 * pair + 1], w[nb][4 * pair + 2], w[nb][4 * pair + 3]);
          } else {
            const uint32_t first = mine_tile == 2 * pair % F ? ~0u : 0u, second = mine_tile == 2 * pair % F + 1 ? ~0u : 0u;
            const uint32_t lo = w[nb][2 * (2 * pair / F)], hi = w[nb][2 * (2 * pair / F) + 1];
            pf[nb] = half_frag(lo & first, hi & first, lo & second, hi & second);
          }
        }
        const auto values = [&](uint32_t sel, int v0) {
          const uint4 a = raw.v[2 * pair], d = raw.v[2 * pair + 1];
          const uint32_t x[4] = {__builtin_amdgcn_perm(a.y, a.x, sel), __builtin_amdgcn_perm(a.w, a.z, sel),
                                 __builtin_amdgcn_perm(d.y, d.x, sel), __builtin_amdgcn_perm(d.w, d.z, sel)};
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            // nibbles 0 to 3 of the half words, each as 16 * code * 2^-24.  (As code * 2^-24, one shift less, the unit's sums
            // lose more bits: with 131071 tokens the result is off by 3.3e-4 for 2.9e-4, of which 2.1e-4 is its own rounding.)
            const auto nibble = [&](uint32_t w) { return (n == 0 ? w << 4 : w >> (n > 0 ? 4 * n - 4 : 0)) & 0x00F000F0u; };
            const v8h vf = half_frag(nibble(x[0]), nibble(x[1]), nibble(x[2]), nibble(x[3]));
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) o[nb][v0 + n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[nb], o[nb][v0 + n], 0, 0, 0);
            if (TIGHT) __builtin_amdgcn_sched_barrier(kPass);
          }
        };
        if (D == 128) {
          values(0x05040100u, 0);
          values(0x07060302u, NV - 4);
        } else {
          values(col & 8 ? 0x07060302u : 0x05040100u, 0);      // lanes 8 .. 15 of a row take the upper halves of the same words
        }
      }
      load_rest(t_next, next, k);
      t = t_next;
      pages = next;
    }

    // ---- the wavefronts' sums, a block of columns at a time
    const bool shared = begin > 0 || stop < span.steps;
    const uint32_t w0 = shared ? group_of(item + OVER + WAVES - 1) : me, w1 = shared ? group_of(item + OVER + span.steps - 1) : me;   // the workgroups that hold a part of it
    const auto write_row = [&](int r, const float (&v)[4], float sum, float ref) {
      const int j = over_group(p, r), g = r - j * p.G;
      // From 2^27 on, where binary32 goes by 16, a reference can be 8 off and the largest weight past fp16's range; further on all weights zero or infinite.
      const bool none = sum == 0.0f && ref == kNone;
      const float by = fabsf(ref) < 134217728.0f ? 1.0f / sum : __builtin_nanf("");
      typedef _Float16 v4h __attribute__((ext_vector_type(4)));
      v4h h;
#pragma unroll
      for (int x = 0; x < 4; ++x) h[x] = none ? (_Float16)0.0f : held_to_half(v[x] * by);
      *reinterpret_cast<v4h*>(p.out + (((size_t)b * p.kv.T + j) * p.Hq + (size_t)head * p.G + g) * D + own) = h;
    };
    const auto write_part = [&](uint32_t slot, int r, float ref, float sum, const float (&v)[4]) {
      float* const part = p.parts + ((size_t)slot * RB + r) * PART;
      if (own == 0) store_shared_f2(part, ref, sum);
      store_shared_f2(part + 4 + own, v[0], v[1]);
      store_shared_f2(part + 6 + own, v[2], v[3]);
    };
    // (Code that runs once an item comes from memory at every launch: one copy of what can be shared, few unrolled loops.)
    const auto hand_over = [&](int nb) {
      if (F > 1) {                            // the columns of a row
        const float to = group_max<F>(m[nb]), by = __builtin_amdgcn_exp2f(m[nb] - to);
        m[nb] = to;
        l[nb] = group_sum<F>(l[nb] * by);
        c[nb] = group_sum<F>(c[nb] * by);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[nb][v][i] = group_sum<F>(o[nb][v][i] * by);
      }
      l[nb] = column_sum(l[nb]);
      c[nb] = column_sum(c[nb]);
      if (lane < COLS) { m_lds[wave][lane] = m[nb]; l_lds[wave][lane] = l[nb]; c_lds[wave][lane] = c[nb]; }
      if (F == 1 || col < COLS) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float* const dst = &o_lds[wave][col & (COLS - 1)][8 * ((4 * kb + i) & (D / 8 - 1))];
          if (D == 128) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = o[nb][((e & 1) * 4 + e / 2) % NV][i] * 1048576.0f;
            reinterpret_cast<float4*>(dst)[0] = float4{x[0], x[1], x[2], x[3]};
            reinterpret_cast<float4*>(dst)[1] = float4{x[4], x[5], x[6], x[7]};
          } else {
#pragma unroll
            for (int n = 0; n < 4; ++n) dst[2 * n + (kb >> 1)] = o[nb][n][i] * 1048576.0f;
          }
        }
      }
    };
#pragma unroll 1
    for (int nb = 0; nb < NB && nb * COLS < rows; ++nb) {
      if (NB == 1 || nb == 0) hand_over(0);
      else if (NB == 2 || nb == 1) hand_over(NB > 1 ? 1 : 0);
      else if (nb == 2) hand_over(NB > 2 ? 2 : 0);
      else hand_over(NB > 2 ? 3 : 0);
      __syncthreads();
      for (int in = row_of; in < COLS; in += THREADS / LANES) {
        const int r = nb * COLS + in;
        if (r >= rows) break;
        float v[4], total_l = 0.0f, total_c = 0.0f, ref = kNone;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) ref = fmaxf(ref, m_lds[w][in]);
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          const float by = __builtin_amdgcn_exp2f(m_lds[w][in] - ref);
          const float4 x = *reinterpret_cast<const float4*>(&o_lds[w][in][own]);
          total_l = fmaf(l_lds[w][in], by, total_l);
          total_c = fmaf(c_lds[w][in], by, total_c);
          v[0] = fmaf(x.x, by, v[0]); v[1] = fmaf(x.y, by, v[1]); v[2] = fmaf(x.z, by, v[2]); v[3] = fmaf(x.w, by, v[3]);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] += total_c;
        if (!shared) {
          write_row(block * RB + r, v, total_l, ref);
        } else {
          write_part(2 * me + (first_run ? 0 : 1), r, ref, total_l, v);
        }
      }
      __syncthreads();
    }

    // ---- the last of the item's workgroups joins their parts; of many parts, the last of each eight theirs first (a
    // workgroup reads parts past the caches at tens of GB/s: 64 parts of 8 rows in one go take 14 us)
    const uint32_t parts = w1 - w0 + 1;
    const auto slot_of = [&](uint32_t w) { return w == w0 ? 2 * w0 + (start_of(w0) < item ? 1 : 0) : 2 * w; };
#pragma unroll 1
    for (int stage = parts > 16 ? 0 : 1; shared && stage < 2; ++stage) {
      uint32_t first = w0, stride = 1, n = parts, counter = w0;
      if (stage == 0) {
        first = w0 + ((me - w0) & ~7u);
        n = min(8u, w1 + 1 - first);
        // One on its own has its part in place already.  It must not count: the next item's first eight may begin with this
        // workgroup, and would count at the same place.  (Sets of two or more begin with a workgroup that is inside their item.)
        if (n == 1) continue;
        counter = Form::workgroups + first;
      } else if (parts > 16) {
        stride = 8;
        n = (parts + 7) / 8;
      }
      if (!last_arrival(p.tickets, (int)n, counter, &ticket)) break;
      constexpr int SETS = THREADS / LANES;            // rows at a time
      // few rows: several threads take a row's parts in turn
      int taken = 1;
      while (taken < min(rows, SETS)) taken *= 2;
      const int sub = row_of & (taken - 1), lot = row_of / taken, lots = SETS / taken;
      for (int r0 = 0; r0 < rows; r0 += SETS) {
        const int r = r0 + sub;
        float ref = kNone, sum = 0.0f, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const auto add = [&](float m2, float l2, float a, float b2, float c2, float d2) {
          const float to = fmaxf(ref, m2), x = __builtin_amdgcn_exp2f(ref - to), y = __builtin_amdgcn_exp2f(m2 - to);
          ref = to;
          sum = sum * x + l2 * y;
          v[0] = v[0] * x + a * y; v[1] = v[1] * x + b2 * y; v[2] = v[2] * x + c2 * y; v[3] = v[3] * x + d2 * y;
        };
        if (r < rows) {
          constexpr int FLY = 4;                       // parts on their way together: each is a trip past the caches (more only lengthen the code)
          for (int i0 = lot; i0 < (int)n; i0 += FLY * lots) {
            float2 ml[FLY], in[FLY][2];
#pragma unroll
            for (int y = 0; y < FLY; ++y) {
              const uint32_t i = min((uint32_t)(i0 + y * lots), n - 1);
              const float* const part = p.parts + ((size_t)slot_of(first + i * stride) * RB + r) * PART;
              ml[y] = load_shared_f2(part);
              in[y][0] = load_shared_f2(part + 4 + own);
              in[y][1] = load_shared_f2(part + 6 + own);
            }
#pragma unroll
            for (int y = 0; y < FLY; ++y)
              if (i0 + y * lots < (int)n) add(ml[y].x, ml[y].y, in[y][0].x, in[y][0].y, in[y][1].x, in[y][1].y);
          }
        }
        if (lots > 1) {
          float* const lot_rows = &o_lds[0][0][0];       // (as many rows as the wavefronts' sums had)
          if (own == 0) { join_m[row_of] = ref; join_l[row_of] = sum; }
          if (lot > 0) *reinterpret_cast<float4*>(lot_rows + (size_t)(row_of - taken) * PITCH + own) = float4{v[0], v[1], v[2], v[3]};
          __syncthreads();
          if (lot == 0 && r < rows) {
            for (int k = 1; k < lots; ++k) {
              const int from = k * taken + sub;
              const float4 x = *reinterpret_cast<const float4*>(lot_rows + (size_t)(from - taken) * PITCH + own);
              add(join_m[from], join_l[from], x.x, x.y, x.z, x.w);
            }
          }
        }
        if (lot == 0 && r < rows) {
          if (stage == 1) write_row(block * RB + r, v, sum, ref);
          else write_part(slot_of(first), r, ref, sum, v);
        }
        __syncthreads();
      }
    }
    if (last_head < 0) {
      ++item;
      take();
      continue;
    }
    item += (uint32_t)(OVER + span.steps);
    begin = 0;
    first_run = false;
    if (++head == Hkv) { head = 0; ++entry; }
  }
}

}  // namespace qspec
