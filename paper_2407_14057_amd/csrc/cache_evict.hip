// Eviction from K,V caches by accumulated attention weight: of a request's n tokens the `budget` best stay, protected
// ones (position below `sinks`, or among the `recent` last positions) first, then by weight, ties to the lower slot.
//
// The kept tokens end up in slots 0 .. budget-1, but not in order: a kept token that lies below the budget already stays
// where it is, and the slots that lose theirs are filled, in order, with the kept tokens from behind the budget.  Exactly
// the rows that have to move move (one per step in a cache that is full), no source is another row's destination, and
// attention does not depend on the order of the slots (positions move along).
//
// Up to 16384 slots one workgroup per request selects (latency bound: a few KB of tables, some ten barriers), and a second
// launch moves the rows of K and V at the rate of a copy; where the caches have room for a few evictions only, the
// selecting workgroup moves them itself.  Where only a few tokens leave, as in a cache that is full, it finds them
// directly.  From more slots many workgroups select, six launches for any number of tokens that leave.
#include "common.h"

namespace lz {

namespace {

constexpr int FUSED_MOVES = 512;                    // most rows that a selecting workgroup moves itself
constexpr int FEW = 8;                              // most tokens that are looked for one after the other

constexpr uint32_t PROTECTED = 0xfffffffeu, NOBODY = 0xffffffffu;

// sorts like the weight; above every weight: a protected token; lowest: NaN
__device__ __forceinline__ uint32_t eviction_key(float w, int pos, int sinks, bool any_recent, int recent_from) {
  const uint32_t u = __float_as_uint(w + 0.f);               // -0 counts as 0
  const uint32_t key = w != w ? 0u : u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
  return pos < sinks || (any_recent && pos >= recent_from) ? PROTECTED : key;
}

// lowest of the lanes' values, in every lane
__device__ __forceinline__ uint32_t wave_lowest(uint32_t v) {
  v = min(v, (uint32_t)__builtin_amdgcn_update_dpp(-1, (int)v, 0x111, 0xf, 0xf, false));      // (the steps of wave_scan)
  v = min(v, (uint32_t)__builtin_amdgcn_update_dpp(-1, (int)v, 0x112, 0xf, 0xf, false));
  v = min(v, (uint32_t)__builtin_amdgcn_update_dpp(-1, (int)v, 0x114, 0xf, 0xf, false));
  v = min(v, (uint32_t)__builtin_amdgcn_update_dpp(-1, (int)v, 0x118, 0xf, 0xf, false));
  v = min(v, (uint32_t)__builtin_amdgcn_update_dpp(-1, (int)v, 0x142, 0xa, 0xf, false));
  v = min(v, (uint32_t)__builtin_amdgcn_update_dpp(-1, (int)v, 0x143, 0xc, 0xf, false));
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Adds every lane with `on` to its bin; where all of them have the same bin (ties), at once: LDS atomics on one address
// take a turn per lane.
__device__ __forceinline__ void count_bins(int* hist, uint32_t bin, bool on) {
  const unsigned long long who = __ballot(on);
  if (who == 0ull) return;
  const int lead = __builtin_ctzll(who);
  const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)bin, lead);
  if (__ballot(on && bin == first) == who) {
    if ((int)(threadIdx.x & 63) == lead) atomicAdd(&hist[first], __popcll(who));
  } else if (on) {
    atomicAdd(&hist[bin], 1);
  }
}

// The radix select, most significant bits first: 11, 11 and 10 of the key.  (The first 11 bits of a weight are its
// exponent and two bits more, so that few lanes of a wave meet in a bin; by 8 bits the weights of a prompt fall into
// five bins.)
constexpr int PASSES = 3, BINS = 2048;
__device__ __forceinline__ int pass_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ int pass_bins(int pass) { return pass == 2 ? 1024 : 2048; }
__device__ __forceinline__ uint32_t pass_bin(uint32_t key, int pass) { return (key >> pass_shift(pass)) & (uint32_t)(pass_bins(pass) - 1); }

// What a select has found out: the key of rank `need` among those that begin with `prefix` (bits of `mask`), and at the
// end how many keys equal it.
struct Found {
  uint32_t prefix = 0u, mask = 0u;
  int need = 0, same = 0;
};
// Goes on by one pass, given its histogram.  A wave does it for itself; every lane gets the result.  Counted from the top:
// lane L owns the `per` bins below bins - per * L, then lane l one of the bins of the lane that the rank falls to.
__device__ __forceinline__ void next_digit(Found& f, const int* hist, int pass) {
  const int lane = threadIdx.x & 63, bins = pass_bins(pass), per = bins / 64;
  int mine = 0;
  for (int u = 0; u < per / 4; ++u) {
    const int4 h = *(const int4*)&hist[bins - per * (lane + 1) + 4 * ((u + lane) % (per / 4))];   // (staggered over the banks)
    mine += (h.x + h.y) + (h.z + h.w);
  }
  int incl = wave_scan(mine);
  int at = __builtin_ctzll(__ballot(incl >= f.need));
  f.need -= __builtin_amdgcn_readlane(incl - mine, at);
  const int top = bins - per * at - 1;
  mine = lane < per ? hist[top - lane] : 0;
  incl = wave_scan(mine);
  at = __builtin_ctzll(__ballot(incl >= f.need));
  f.need -= __builtin_amdgcn_readlane(incl - mine, at);
  f.same = __builtin_amdgcn_readlane(mine, at);
  f.prefix |= (uint32_t)(top - at) << pass_shift(pass);
  f.mask |= (uint32_t)(bins - 1) << pass_shift(pass);
}

__device__ __forceinline__ int first_recent(int top, int recent) {
  return (int)max((long long)top + 1 - (recent > 0 ? recent : 1), (long long)INT32_MIN);
}

// From the bit masks of the keys above the threshold (keep) and equal to it: which of the equal ones stay (the first
// `need`), and the list of moves.  Holes are slots below the budget that lose their token, movers kept tokens from behind
// it; as many of each, returned.  All threads of the workgroup; keep is complete on return, the lists after a barrier.
// SPREAD: the words are dealt out again to write the lists, `equal` takes the counts (eight prompts of 1 - 8 k tokens to
// 1100: 6 k cycles instead of the 13 k of a thread a word).  Not for small caches, where one barrier more costs as much as
// it saves (2049 slots: 9.7 us, 9.2 without).
template <int THREADS, bool SPREAD>
__device__ __forceinline__ int resolve_moves(unsigned long long* keep, unsigned long long* equal, int W, int kept, int need,
                                             bool all_equal, int32_t* hole_at, int32_t* mover_at, int2* part) {
  constexpr int WAVES = THREADS / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // exclusive sums over the words, a thread a word, of two counts at once; total: of all of them.  Up to 64 words every
  // wave makes for itself.
  auto over_words = [&](int x, int y, int2& total) {
    const int sx = wave_scan(x), sy = wave_scan(y);
    if (W <= 64) {
      total = make_int2(__builtin_amdgcn_readlane(sx, 63), __builtin_amdgcn_readlane(sy, 63));
      return make_int2(sx - x, sy - y);
    }
    __syncthreads();
    if (lane == 63) part[wave] = make_int2(sx, sy);
    __syncthreads();
    int2 before = make_int2(0, 0);
    total = make_int2(0, 0);
#pragma unroll
    for (int u = 0; u < WAVES; ++u) {
      const int2 v = part[u];
      if (u < wave) before = make_int2(before.x + v.x, before.y + v.y);
      total = make_int2(total.x + v.x, total.y + v.y);
    }
    return make_int2(before.x + sx - x, before.y + sy - y);
  };
  const bool one = W <= 64;               // word of this thread: lane, in every wave alike
  const int own = one ? lane : threadIdx.x, stride = one ? 64 : THREADS;
  if (!all_equal) {
    int base = 0;
    for (int w0 = 0; w0 < W; w0 += stride) {
      const int at = w0 + own;
      unsigned long long eq = at < W ? equal[at] : 0ull;
      int2 total;
      int left = need - (base + over_words(__popcll(eq), 0, total).x);
      base += total.x;
      unsigned long long take = 0ull;
      if (left >= 64) take = eq;
      else
        for (; left > 0 && eq != 0ull; --left) {
          take |= eq & (~eq + 1ull);
          eq &= eq - 1ull;
        }
      if (at < W && (!one || wave == 0)) keep[at] |= take;
    }
    __syncthreads();
  }
  // holes and movers of a word
  auto split = [&](int at, unsigned long long& hole, unsigned long long& mover) {
    const unsigned long long mine = at < W ? keep[at] : 0ull;
    const int below = min(max(kept - 64 * at, 0), 64);         // slots of this word below the budget
    const unsigned long long front = below == 64 ? ~0ull : (1ull << below) - 1ull;
    hole = at < W ? ~mine & front : 0ull;
    mover = mine & ~front;
  };
  int2 done = make_int2(0, 0);            // holes, movers
  for (int w0 = 0; w0 < W; w0 += stride) {
    const int at = w0 + own;
    unsigned long long hole, mover;
    split(at, hole, mover);
    int2 total;
    const int2 first = over_words(__popcll(hole), __popcll(mover), total);
    int h = done.x + first.x, m = done.y + first.y;
    done = make_int2(done.x + total.x, done.y + total.y);
    if (SPREAD) {
      if (at < W && (!one || wave == 0)) equal[at] = (unsigned long long)(unsigned)m << 32 | (unsigned)h;
    } else if (!one || wave == 0) {
      for (; hole != 0ull; hole &= hole - 1ull) hole_at[h++] = 64 * at + __builtin_ctzll(hole);
      for (; mover != 0ull; mover &= mover - 1ull) mover_at[m++] = 64 * at + __builtin_ctzll(mover);
    }
  }
  if (SPREAD) {
    // the words dealt out to the waves, eight at a time; one word after the other, with a lane a slot
    __syncthreads();
    for (int w0 = wave * 8; w0 < W; w0 += WAVES * 8) {
      const int at = w0 + (lane & 7);
      unsigned long long hole, mover;
      split(at, hole, mover);
      const unsigned long long before = at < W ? equal[at] : 0ull;
      for (unsigned long long busy = __ballot(lane < 8 && (hole | mover) != 0ull); busy != 0ull; busy &= busy - 1ull) {
        const int l = __builtin_ctzll(busy);
        auto emit = [&](unsigned long long bits, uint32_t from, int32_t* to) {
          const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)(bits >> 32), l);
          const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)bits, l);
          if (((lane < 32 ? lo : hi) >> (lane & 31)) & 1u)
            to[__builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, (unsigned)__builtin_amdgcn_readlane((int)from, l)))] =
                64 * (w0 + l) + lane;
        };
        emit(hole, (uint32_t)before, hole_at);
        emit(mover, (uint32_t)(before >> 32), mover_at);
      }
    }
  }
  return done.x;
}

}  // namespace

__device__ __forceinline__ void move_tables(const EvictArgs& a, int b, int to, int from) {
  const size_t at = (size_t)b * a.capacity;
  a.weight_out[at + to] = a.weight[at + from];
  a.pos_out[at + to] = a.pos[at + from];
  if (a.kept != nullptr) a.kept[(size_t)b * a.budget + to] = from;
}

// THREADS threads, ITEMS slots per thread in registers.  Every wave reads the histograms for itself: a barrier a pass.
template <int THREADS, int ITEMS>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(EvictArgs a) {
  constexpr int WAVES = THREADS / 64;
  __shared__ unsigned long long keep[THREADS * ITEMS / 64], equal[THREADS * ITEMS / 64];
  __shared__ __attribute__((aligned(16))) int hist[PASSES][BINS];
  __shared__ int2 part[WAVES];
  __shared__ int list[2][FUSED_MOVES];
  __shared__ uint2 low[2][WAVES];
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float* weight = a.weight + (size_t)b * a.capacity;
  const int32_t* pos = a.pos + (size_t)b * a.capacity;
  float* weight_out = a.weight_out + (size_t)b * a.capacity;
  int32_t* pos_out = a.pos_out + (size_t)b * a.capacity;
  int32_t* kept_from = a.kept != nullptr ? a.kept + (size_t)b * a.budget : nullptr;
  // the tables are on their way before the length is known
  float w[ITEMS];
  int p[ITEMS];
  uint32_t keys[ITEMS];
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const int i = u * THREADS + threadIdx.x;
    w[u] = i < a.capacity ? weight[i] : 0.f;
    p[u] = i < a.capacity ? pos[i] : 0;
  }
  const int given = a.lengths[b], n = min(given, a.capacity), kept = min(n, a.budget);
  for (int i = threadIdx.x; i < PASSES * BINS / 4; i += THREADS) ((int4*)hist)[i] = make_int4(0, 0, 0, 0);
  // calls f(item, slot) for the items that any thread has a slot below n for; all lanes of a wave together
  auto each = [&](auto f) {
#pragma unroll
    for (int u = 0; u < ITEMS; ++u)
      if (u * THREADS < n) f(u, u * THREADS + (int)threadIdx.x);
  };
  int top = INT32_MIN;
  each([&](int u, int i) { top = max(top, i < n ? p[u] : INT32_MIN); });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = max(top, __shfl_xor(top, o, 64));
  if (lane == 0) part[wave].x = top;
  __syncthreads();                       // (also: every thread has read the length, which may be overwritten now)
#pragma unroll
  for (int v = 0; v < WAVES; ++v) top = max(top, part[v].x);
  if (threadIdx.x == 0) {
    a.lengths_out[b] = kept;
    if (given > a.capacity && a.status != nullptr) atomicOr(a.status, ST_BAD_CU);
  }
  const bool new_weight = weight_out != weight, new_pos = pos_out != pos;
  auto stay = [&](int u, int i) {
    if (new_weight) weight_out[i] = w[u];
    if (new_pos) pos_out[i] = p[u];
    if (kept_from != nullptr) kept_from[i] = i;
  };
  if (n <= a.budget) {
    each([&](int u, int i) { if (i < kept) stay(u, i); });
    if (threadIdx.x == 0 && !a.fused) a.moves[b] = 0;
    return;
  }
  const int recent_from = first_recent(top, a.recent);
  each([&](int u, int) { keys[u] = eviction_key(w[u], p[u], a.sinks, a.recent > 0, recent_from); });
  int holes;
  const int leave = n - kept;
  if (leave <= FEW) {
    // A full cache that gives a token up for every new one: the lowest keys, of equal ones the higher slot, are found one
    // after the other, and their rows moved by this workgroup (32 caches, of 2049 tokens one: 6.7 us, by the histograms 9.3;
    // of 2056 eight: 9.3, 9.8; 16 caches, one of 8192: 8.4, 17.7).
    int gone = INT32_MAX;                // the slot that was found j-th, in lane j
    uint32_t behind = 0u;                // those from the budget on, as bits
    auto all = [&](auto f) {             // (no branch an item, as `each` has, where there is so little to do)
#pragma unroll
      for (int u = 0; u < ITEMS; ++u) f(u, u * THREADS + (int)threadIdx.x);
    };
    all([&](int u, int i) { keys[u] = i < n ? keys[u] : NOBODY; });
    for (int j = 0; j < leave; ++j) {
      // (slots as their complement)
      uint32_t key = NOBODY, from = NOBODY;
      all([&](int u, int) { key = min(key, keys[u]); });
      key = wave_lowest(key);
      all([&](int u, int i) { from = min(from, keys[u] == key ? ~(uint32_t)i : NOBODY); });
      from = wave_lowest(from);
      if (lane == 0) low[j & 1][wave] = make_uint2(key, from);
      __syncthreads();
      const uint2 said = lane < WAVES ? low[j & 1][lane] : make_uint2(NOBODY, NOBODY);
      key = wave_lowest(said.x);
      const int slot = (int)~wave_lowest(said.x == key ? said.y : NOBODY);
      all([&](int u, int i) { keys[u] = i == slot ? NOBODY : keys[u]; });
      if (lane == j) gone = slot;
      if (slot >= kept) behind |= 1u << (slot - kept);
    }
    holes = __popcll(__ballot(gone < kept));
    int rank = 0;
    for (int j = 0; j < leave; ++j) rank += __builtin_amdgcn_readlane(gone, j) < gone;
    if (wave == 0 && gone < kept) list[0][rank] = gone;
    if (wave == 0 && lane < leave && !((behind >> lane) & 1u)) list[1][__popc(~behind & ((1u << lane) - 1u))] = kept + lane;
    if (new_weight || new_pos || kept_from != nullptr)
      each([&](int u, int i) { if (i < kept && keys[u] != NOBODY) stay(u, i); });
    if (threadIdx.x == 0 && !a.fused) a.moves[b] = 0;
  } else {
    Found f;
    f.need = kept;
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
      each([&](int u, int i) { count_bins(hist[pass], pass_bin(keys[u], pass), i < n && (keys[u] & f.mask) == f.prefix); });
      __syncthreads();
      next_digit(f, hist[pass], pass);
    }

    // kept set as a bit mask: keys above the threshold, and the first `need` equal to it
    const int W = (n + 63) / 64;
    const bool all_equal = f.need == f.same;
    each([&](int u, int i) {
      const unsigned long long hi = __ballot(i < n && (all_equal ? keys[u] >= f.prefix : keys[u] > f.prefix));
      const unsigned long long eq = __ballot(i < n && keys[u] == f.prefix);
      const int at = u * WAVES + wave;
      if (lane == 0 && at < W) {
        keep[at] = hi;
        equal[at] = eq;
      }
    });
    __syncthreads();
    int32_t* hole_at = a.fused ? list[0] : a.moves + a.batch + (size_t)b * 2 * a.max_moves;
    int32_t* mover_at = a.fused ? list[1] : hole_at + a.max_moves;
    holes = resolve_moves<THREADS, (ITEMS > 8)>(keep, equal, W, kept, f.need, all_equal, hole_at, mover_at, part);
    if (new_weight || new_pos || kept_from != nullptr)
      each([&](int u, int i) { if (i < kept && ((keep[i >> 6] >> (i & 63)) & 1ull)) stay(u, i); });
    if (!a.fused) {
      if (threadIdx.x == 0) a.moves[b] = holes;
      return;
    }
  }
  __syncthreads();                       // the lists are read by other threads
  for (int i = threadIdx.x; i < holes; i += THREADS) move_tables(a, b, list[0][i], list[1][i]);
  uint16_t* k = a.k + b * a.batch_stride;
  uint16_t* v = a.v + b * a.batch_stride;
  for (int i = threadIdx.x; i < holes * a.row_chunks; i += THREADS) {
    const int row = i / a.row_chunks, ch = i % a.row_chunks * 8;
    const long long to = list[0][row] * a.row_stride + ch, from = list[1][row] * a.row_stride + ch;
    const uint4 x = *(const uint4*)(k + from), y = *(const uint4*)(v + from);
    *(uint4*)(k + to) = x;
    *(uint4*)(v + to) = y;
  }
}

// ------------------------------------------------------------------------------------------
// Caches of more slots: a workgroup per SEG slots, a launch per pass (131000 slots brought down to 16000, 8 K,V heads: 48 us, 24 of
// them the moves; in segments of 8192 slots and with the list of moves by one workgroup 72; all by one workgroup 176, nearly all
// of it waiting for its own loads and LDS).  Segments are cut at the budget, so that one has either holes or movers.  Per request the workspace holds the segments' highest positions, the
// histograms, the bit masks, how many bits those have, and what was found.
constexpr int SEG = 2048, SEG_THREADS = 512, SEG_ITEMS = SEG / SEG_THREADS, SEG_WORDS = SEG / 64;

namespace {

struct LongState {                       // of one request, in the workspace
  int32_t *top, *hist, *found;           // found: duplicates of the threshold to keep, all of them, tokens kept
  int2* counts;                          // of a segment: keys above the threshold (all that stay, if all duplicates do), equal to it
  unsigned long long *keep, *equal;
};
// segments up to the budget
__host__ __device__ inline int front_segs(int capacity, int budget) { return ((budget < capacity ? budget : capacity) + SEG - 1) / SEG; }
__host__ __device__ inline int long_segs(int capacity, int budget) {
  return front_segs(capacity, budget) + (budget < capacity ? (capacity - budget + SEG - 1) / SEG : 0);
}
__host__ __device__ inline size_t long_state_bytes(int capacity, int budget) {
  const size_t segs = long_segs(capacity, budget);
  return PASSES * BINS * 4 + segs * SEG_WORDS * 16 + (segs * 12 + 12 + 255) / 256 * 256;
}
__device__ __forceinline__ LongState long_state(const EvictArgs& a, int b) {
  const size_t segs = long_segs(a.capacity, a.budget);
  char* at = (char*)a.long_state + b * long_state_bytes(a.capacity, a.budget);
  LongState s;
  s.hist = (int32_t*)at;
  s.keep = (unsigned long long*)(at + PASSES * BINS * 4);
  s.equal = s.keep + segs * SEG_WORDS;
  s.counts = (int2*)(s.equal + segs * SEG_WORDS);
  s.top = (int32_t*)(s.counts + segs);
  s.found = s.top + segs;
  return s;
}
// First slot of a segment, and the slot behind its last one of a request of n tokens.
struct Range {
  int lo, hi;
};
__device__ __forceinline__ Range seg_range(const EvictArgs& a, int seg, int n) {
  const int front = front_segs(a.capacity, a.budget), lo = seg < front ? seg * SEG : a.budget + (seg - front) * SEG;
  return {lo, min(min(lo + SEG, seg < front ? a.budget : n), n)};
}
// Highest position of a request, from its segments'; all threads of a wave together.
__device__ __forceinline__ int highest(const LongState& s, int segs) {
  const int lane = threadIdx.x & 63;
  int top = INT32_MIN;
  for (int i = lane; i < segs; i += 64) top = max(top, s.top[i]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = max(top, __shfl_xor(top, o, 64));
  return top;
}

}  // namespace

// Highest position of a segment; the histograms are cleared.
__global__ void __launch_bounds__(SEG_THREADS) evict_long_top_kernel(EvictArgs a) {
  __shared__ int part[SEG_THREADS / 64];
  const int b = blockIdx.y, seg = blockIdx.x;
  const Range r = seg_range(a, seg, min(a.lengths[b], a.capacity));
  const LongState s = long_state(a, b);
  for (int i = seg * SEG_THREADS + threadIdx.x; i < PASSES * BINS / 4; i += gridDim.x * SEG_THREADS)
    ((int4*)s.hist)[i] = make_int4(0, 0, 0, 0);
  const int32_t* pos = a.pos + (size_t)b * a.capacity;
  int top = INT32_MIN;
#pragma unroll
  for (int u = 0; u < SEG_ITEMS; ++u) {
    const int i = r.lo + u * SEG_THREADS + threadIdx.x;
    top = max(top, i < r.hi ? pos[i] : INT32_MIN);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = max(top, __shfl_xor(top, o, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int v = 1; v < SEG_THREADS / 64; ++v) top = max(top, part[v]);
    s.top[seg] = top;
  }
}

// PASS < PASSES: counts a segment's keys of that pass; PASS == PASSES: writes its bit masks.
template <int PASS>
__global__ void __launch_bounds__(SEG_THREADS) evict_long_pass_kernel(EvictArgs a) {
  __shared__ __attribute__((aligned(16))) int hist[BINS];
  __shared__ int2 part[SEG_THREADS / 64];
  const int b = blockIdx.y, seg = blockIdx.x, n = min(a.lengths[b], a.capacity);
  const Range r = seg_range(a, seg, n);
  if (n <= a.budget || r.lo >= r.hi) return;
  const LongState s = long_state(a, b);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float* weight = a.weight + (size_t)b * a.capacity;
  const int32_t* pos = a.pos + (size_t)b * a.capacity;
  float w[SEG_ITEMS];
  int p[SEG_ITEMS];
#pragma unroll
  for (int u = 0; u < SEG_ITEMS; ++u) {
    const int i = min(r.lo + u * SEG_THREADS + (int)threadIdx.x, r.hi - 1);
    w[u] = weight[i];
    p[u] = pos[i];
  }
  if (PASS < PASSES) {
    for (int i = threadIdx.x; i < BINS / 4; i += SEG_THREADS) ((int4*)hist)[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
  }
  const int recent_from = first_recent(highest(s, gridDim.x), a.recent);
  Found f;
  f.need = a.budget;
#pragma unroll
  for (int pass = 0; pass < PASS; ++pass) next_digit(f, s.hist + pass * BINS, pass);
  int2 count = make_int2(0, 0);
#pragma unroll
  for (int u = 0; u < SEG_ITEMS; ++u) {
    const int i = r.lo + u * SEG_THREADS + threadIdx.x;
    const uint32_t key = eviction_key(w[u], p[u], a.sinks, a.recent > 0, recent_from);
    if (PASS < PASSES) {
      count_bins(hist, pass_bin(key, PASS), i < r.hi && (key & f.mask) == f.prefix);
    } else {
      const unsigned long long hi = __ballot(i < r.hi && (f.need == f.same ? key >= f.prefix : key > f.prefix));
      const unsigned long long eq = __ballot(i < r.hi && key == f.prefix);
      count = make_int2(count.x + __popcll(hi), count.y + __popcll(eq));
      if (lane == 0) {
        const int at = seg * SEG_WORDS + u * (SEG_THREADS / 64) + wave;
        s.keep[at] = hi;
        s.equal[at] = eq;
      }
    }
  }
  if (PASS < PASSES) {
    __syncthreads();
    for (int i = threadIdx.x; i < pass_bins(PASS); i += SEG_THREADS)
      if (hist[i] != 0) atomicAdd(&s.hist[PASS * BINS + i], hist[i]);
  } else {
    if (lane == 0) part[wave] = count;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int v = 1; v < SEG_THREADS / 64; ++v) count = make_int2(count.x + part[v].x, count.y + part[v].y);
      s.counts[seg] = count;
      if (seg == 0) {
        s.found[0] = f.need;
        s.found[1] = f.same;
      }
    }
  }
}

// A segment's holes or movers, and which of its duplicates of the threshold stay (the first of the request's); by the first
// one also how many moves there are.  The new length is written by the launch behind: others read the old one here.
__global__ void __launch_bounds__(256) evict_long_moves_kernel(EvictArgs a) {
  const int b = blockIdx.y, seg = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const LongState s = long_state(a, b);
  const int given = a.lengths[b], n = min(given, a.capacity), front = front_segs(a.capacity, a.budget);
  if (seg == 0 && threadIdx.x == 0) {
    s.found[2] = min(n, a.budget);
    if (n <= a.budget) a.moves[b] = 0;
    if (given > a.capacity && a.status != nullptr) atomicOr(a.status, ST_BAD_CU);
  }
  const Range r = seg_range(a, seg, n);
  if (n <= a.budget || r.lo >= r.hi) return;
  const int need = s.found[0] == s.found[1] ? 0 : s.found[0];
  // sums over the segments before this one: duplicates, holes, movers; a lane a segment, every wave for itself
  int equals = 0, holes = 0, movers = 0, mine = 0, left = 0;
  for (int t0 = 0; t0 < (int)gridDim.x; t0 += 64) {
    const int t = t0 + lane;
    const Range q = seg_range(a, t, n);
    const bool live = t < (int)gridDim.x && q.lo < q.hi;
    const int2 count = live ? s.counts[t] : make_int2(0, 0);
    const int eq = wave_scan(count.y), before = equals + eq - count.y;
    const int stay = count.x + min(max(need - before, 0), count.y);
    const int hole = live && t < front ? q.hi - q.lo - stay : 0, mover = live && t >= front ? stay : 0;
    const int h = wave_scan(hole), m = wave_scan(mover);
    if (seg >= t0 && seg < t0 + 64) {
      left = need - __builtin_amdgcn_readlane(before, seg - t0);
      mine = __builtin_amdgcn_readlane(seg < front ? holes + h - hole : movers + m - mover, seg - t0);
    }
    equals += __builtin_amdgcn_readlane(eq, 63);
    holes += __builtin_amdgcn_readlane(h, 63);
    movers += __builtin_amdgcn_readlane(m, 63);
  }
  if (seg == 0 && threadIdx.x == 0) a.moves[b] = holes;
  // a lane a word of the masks (a wave that comes after the first one's store finds the same bits again)
  unsigned long long keep = lane < SEG_WORDS ? s.keep[seg * SEG_WORDS + lane] : 0ull;
  unsigned long long eq = lane < SEG_WORDS ? s.equal[seg * SEG_WORDS + lane] : 0ull;
  const int equal_here = __popcll(eq);
  left -= wave_scan(equal_here) - equal_here;
  if (left >= equal_here) keep |= eq;
  else
    for (; left > 0; --left) {
      keep |= eq & (~eq + 1ull);
      eq &= eq - 1ull;
    }
  if (wave == 0 && lane < SEG_WORDS) s.keep[seg * SEG_WORDS + lane] = keep;
  const int size = min(max(r.hi - r.lo - 64 * lane, 0), 64);
  const unsigned long long bits = seg < front ? ~keep & (size == 64 ? ~0ull : (1ull << size) - 1ull) : keep;
  const int from = mine + wave_scan(__popcll(bits)) - __popcll(bits);
  int32_t* to = a.moves + a.batch + (size_t)b * 2 * a.max_moves + (seg < front ? 0 : a.max_moves);
  // the words dealt out to the waves, with a lane a slot
#pragma unroll
  for (int u = 0; u < SEG_WORDS / 4; ++u) {
    const int l = wave * (SEG_WORDS / 4) + u;
    const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)(bits >> 32), l);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)bits, l);
    if (((lane < 32 ? lo : hi) >> (lane & 31)) & 1u)
      to[__builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, (unsigned)__builtin_amdgcn_readlane(from, l)))] = r.lo + 64 * l + lane;
  }
}

__host__ __device__ inline int rows_at_once(int row_chunks) { return row_chunks < 256 ? 256 / row_chunks : 1; }

// The tokens that move, a row of K and V at a time, narrow ones several, their old rows by non-temporal loads (eight prompts of
// 1 - 8 k tokens brought down to 1100, 176 MB: 30 us; 38 by cached loads in a quarter of the workgroups; 32 caches of 8000, rows of
// 512 bytes, to 1000: 29.8 us in all, one row at a time 44.7).  LONG: the tables of those that stay, unless a table is its own
// output, and the new length are written here too.
template <bool LONG>
__global__ void __launch_bounds__(256) evict_move_kernel(EvictArgs a) {
  const int b = blockIdx.y, count = a.moves[b];
  const int32_t* hole_at = a.moves + a.batch + (size_t)b * 2 * a.max_moves;
  const int32_t* mover_at = hole_at + a.max_moves;
  uint16_t* k = a.k + b * a.batch_stride;
  uint16_t* v = a.v + b * a.batch_stride;
  // narrow rows several at a time
  const int at_once = rows_at_once(a.row_chunks), sub = at_once > 1 ? threadIdx.x / a.row_chunks : 0;
  const int first_ch = threadIdx.x - sub * a.row_chunks;
  for (int i = blockIdx.x * at_once + sub; i < count && sub < at_once; i += gridDim.x * at_once) {
    const int to = hole_at[i], from = mover_at[i];
    const long long k_to = to * a.row_stride, k_from = from * a.row_stride;
    for (int ch = first_ch; ch < a.row_chunks; ch += 512) {
      const bool more = ch + 256 < a.row_chunks;
      uint4 x2 = make_uint4(0u, 0u, 0u, 0u), y2 = x2;
      const uint4 x = load_once((const uint4*)(k + k_from) + ch), y = load_once((const uint4*)(v + k_from) + ch);
      if (more) {
        x2 = load_once((const uint4*)(k + k_from) + ch + 256);
        y2 = load_once((const uint4*)(v + k_from) + ch + 256);
      }
      ((uint4*)(k + k_to))[ch] = x;
      ((uint4*)(v + k_to))[ch] = y;
      if (more) {
        ((uint4*)(k + k_to))[ch + 256] = x2;
        ((uint4*)(v + k_to))[ch + 256] = y2;
      }
    }
    if (first_ch == 0) move_tables(a, b, to, from);
  }
  if (LONG && blockIdx.x == 0 && threadIdx.x == 0) a.lengths_out[b] = long_state(a, b).found[2];
  if (!LONG || (a.weight_out == a.weight && a.pos_out == a.pos && a.kept == nullptr)) return;
  const LongState s = long_state(a, b);
  const size_t at = (size_t)b * a.capacity;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < s.found[2]; i += gridDim.x * 256)
    if (count == 0 || ((s.keep[i >> 6] >> (i & 63)) & 1ull)) {          // (without moves all of them stay)
      if (a.weight_out != a.weight) a.weight_out[at + i] = a.weight[at + i];
      if (a.pos_out != a.pos) a.pos_out[at + i] = a.pos[at + i];
      if (a.kept != nullptr) a.kept[(size_t)b * a.budget + i] = i;
    }
}

// The largest capacity that one workgroup selects from (its registers end here): so far its launch is the quicker form, or as
// quick.  One workgroup / many, in us, a quarter of the slots kept: one request of 4096 16.5 / 25.2, 8192 21.0 / 26.4, 16384 31.3 /
// 30.1; eight 25.0 / 35.3, 37.0 / 43.2, 63.0 / 63.2; 32 54 / 65, 104 / 113, 193 / 195; 16100 of 16384 kept 28.7 / 26.3, 31.1 / 30.8,
// 42.0 / 46.8.  Where one token leaves the limit costs most: one request of 16384 10.4, of 16400 25.8; 32 requests 11.2, 35.2.
constexpr int SELECT_CAPACITY = 16384;

static size_t move_bytes(int batch, int capacity, int budget) {
  const int most = budget < capacity - budget ? budget : capacity - budget;
  return ((size_t)batch * (1 + 2 * (size_t)(most > 0 ? most : 0)) * 4 + 255) & ~(size_t)255;
}

size_t evict_workspace_bytes(int batch, int capacity, int budget) {
  return move_bytes(batch, capacity, budget) + (capacity > SELECT_CAPACITY ? (size_t)batch * long_state_bytes(capacity, budget) : 0);
}

hipError_t launch_cache_evict(EvictArgs a, void* workspace, hipStream_t st) {
  const int most = a.budget < a.capacity - a.budget ? a.budget : a.capacity - a.budget;
  a.max_moves = most > 0 ? most : 0;
  a.moves = (int32_t*)workspace;
  if (a.capacity > SELECT_CAPACITY) {
    a.long_state = (char*)workspace + move_bytes(a.batch, a.capacity, a.budget);
    const dim3 grid(long_segs(a.capacity, a.budget), a.batch);
    hipLaunchKernelGGL(evict_long_top_kernel, grid, dim3(SEG_THREADS), 0, st, a);
    hipLaunchKernelGGL(evict_long_pass_kernel<0>, grid, dim3(SEG_THREADS), 0, st, a);
    hipLaunchKernelGGL(evict_long_pass_kernel<1>, grid, dim3(SEG_THREADS), 0, st, a);
    hipLaunchKernelGGL(evict_long_pass_kernel<2>, grid, dim3(SEG_THREADS), 0, st, a);
    hipLaunchKernelGGL(evict_long_pass_kernel<PASSES>, grid, dim3(SEG_THREADS), 0, st, a);
    hipLaunchKernelGGL(evict_long_moves_kernel, grid, dim3(256), 0, st, a);
  } else {
    // up to 128 KB of K and V to move for a request: by its selecting workgroup, a launch less (32 caches, 32 rows of 4 KB each:
    // 13.4 us, with the launch 14.6; 64 rows 19.1 / 17.7; 8 caches, 16 rows of 16 KB 14.5 / 13.4; 32 caches, 128 rows of 1 KB 14.3 /
    // 17.2)
    a.fused = a.max_moves <= FUSED_MOVES && (long long)a.max_moves * a.row_chunks * 32 <= 128 * 1024;
    if (a.capacity <= 1024) hipLaunchKernelGGL((evict_select_kernel<256, 4>), dim3(a.batch), dim3(256), 0, st, a);
    else if (a.capacity <= 4096) hipLaunchKernelGGL((evict_select_kernel<512, 8>), dim3(a.batch), dim3(512), 0, st, a);
    else hipLaunchKernelGGL((evict_select_kernel<1024, 16>), dim3(a.batch), dim3(1024), 0, st, a);
  }
  const bool one_workgroup = a.capacity <= SELECT_CAPACITY;
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (one_workgroup && (a.max_moves == 0 || a.fused))) return e;
  int groups = 8192 / a.batch;
  if (groups < 16) groups = 16;
  const int at_once = rows_at_once(a.row_chunks), iterations = (a.max_moves + at_once - 1) / at_once;
  const int useful = one_workgroup ? iterations : iterations + (a.capacity + 255) / 256;
  if (groups > useful) groups = useful;
  if (one_workgroup) hipLaunchKernelGGL(evict_move_kernel<false>, dim3(groups, a.batch), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(evict_move_kernel<true>, dim3(groups, a.batch), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace lz
