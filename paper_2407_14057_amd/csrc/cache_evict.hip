// Eviction from K,V caches by accumulated attention weight: of a request's n tokens the `budget` best stay, protected
// ones (position below `sinks`, or among the `recent` last positions) first, then by weight, ties to the lower slot.
//
// The kept tokens end up in slots 0 .. budget-1, but not in order: a kept token that lies below the budget already stays
// where it is, and the slots that lose theirs are filled, in order, with the kept tokens from behind the budget.  Exactly
// the rows that have to move move (one per step in a cache that is full), no source is another row's destination, and
// attention does not depend on the order of the slots (positions move along).
//
// One workgroup per request selects (latency bound: a few KB of tables, some ten barriers), a second launch moves the
// rows of K and V at the rate of a copy; where the caches have room for a few evictions only, the selecting workgroup
// moves them itself.
#include "common.h"

namespace lz {

namespace {

constexpr int FUSED_MOVES = 512;                    // most rows that a selecting workgroup moves itself

// sorts like the weight; above every weight: a protected token; lowest: NaN
__device__ __forceinline__ uint32_t eviction_key(float w, int pos, int sinks, bool any_recent, int recent_from) {
  const uint32_t u = __float_as_uint(w + 0.f);               // -0 counts as 0
  const uint32_t key = w != w ? 0u : u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
  return pos < sinks || (any_recent && pos >= recent_from) ? 0xffffffffu : key;
}

// inclusive sum over the lanes of a wave (DPP: rows of 16, then the rows' totals handed on)
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);    // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);    // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);    // row_bcast:31 into rows 2 and 3
  return v;
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

}  // namespace

// THREADS threads; ITEMS slots per thread are kept in registers (0: any number, read again from memory where needed).
// Threshold: MSB-first radix select by 11, 11 and 10 bits, a barrier each: every wave reads the histogram for itself.  (The
// first 11 bits of a weight are its exponent and two bits more, so that few lanes of a wave meet in a bin; by 8 bits the
// weights of a prompt fall into five bins.)
template <int THREADS, int ITEMS>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(EvictArgs a) {
  constexpr int WAVES = THREADS / 64, BINS = 2048;
  extern __shared__ __attribute__((aligned(16))) unsigned long long words[];   // keep[W], equal[W]
  __shared__ __attribute__((aligned(16))) int hist[3][BINS];
  __shared__ int2 part[WAVES];
  __shared__ int list[2][FUSED_MOVES];
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float* weight = a.weight + (size_t)b * a.capacity;
  const int32_t* pos = a.pos + (size_t)b * a.capacity;
  float* weight_out = a.weight_out + (size_t)b * a.capacity;
  int32_t* pos_out = a.pos_out + (size_t)b * a.capacity;
  int32_t* kept_from = a.kept != nullptr ? a.kept + (size_t)b * a.budget : nullptr;
  const int given = a.lengths[b], n = min(given, a.capacity), kept = min(n, a.budget);
  for (int i = threadIdx.x; i < 3 * BINS / 4; i += THREADS) ((int4*)hist)[i] = make_int4(0, 0, 0, 0);

  float w[ITEMS > 0 ? ITEMS : 1];
  int p[ITEMS > 0 ? ITEMS : 1];
  uint32_t keys[ITEMS > 0 ? ITEMS : 1];
  int top = INT32_MIN;
  // calls f(item, slot, weight, position) for this thread's slots below n; all lanes of a wave together where f needs it
  auto each = [&](auto f) {
    if (ITEMS > 0) {
#pragma unroll
      for (int u = 0; u < ITEMS; ++u)
        if (u * THREADS < n) f(u, u * THREADS + (int)threadIdx.x, w[u], p[u]);
    } else {
      constexpr int AHEAD = 8;             // loads in flight
      for (int u0 = 0; u0 * THREADS < n; u0 += AHEAD) {
        float wi[AHEAD];
        int pi[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          const int i = min((u0 + u) * THREADS + (int)threadIdx.x, n - 1);
          wi[u] = weight[i];
          pi[u] = pos[i];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
          if ((u0 + u) * THREADS < n) f(u0 + u, (u0 + u) * THREADS + (int)threadIdx.x, wi[u], pi[u]);
      }
    }
  };
  if (ITEMS > 0) {
#pragma unroll
    for (int u = 0; u < ITEMS; ++u)
      if (u * THREADS < n) {
        const int i = u * THREADS + threadIdx.x;
        w[u] = i < n ? weight[i] : 0.f;
        p[u] = i < n ? pos[i] : INT32_MIN;
      }
  }
  each([&](int, int i, float, int at) { if (i < n) top = max(top, at); });
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
  auto stay = [&](int i, float wi, int pi) {
    if (new_weight) weight_out[i] = wi;
    if (new_pos) pos_out[i] = pi;
    if (kept_from != nullptr) kept_from[i] = i;
  };
  if (n <= a.budget) {
    each([&](int, int i, float wi, int pi) { if (i < kept) stay(i, wi, pi); });
    if (threadIdx.x == 0 && !a.fused) a.moves[b] = 0;
    return;
  }
  const bool any_recent = a.recent > 0;
  const int recent_from = (int)max((long long)top + 1 - (any_recent ? a.recent : 1), (long long)INT32_MIN);
  if (ITEMS > 0)
    each([&](int u, int i, float wi, int pi) { keys[u] = eviction_key(wi, pi, a.sinks, any_recent, recent_from); });
  auto key_of = [&](int u, float wi, int pi) {
    return ITEMS > 0 ? keys[u] : eviction_key(wi, pi, a.sinks, any_recent, recent_from);
  };

  // the key of rank `kept` from above, and how many of its duplicates are kept
  uint32_t threshold = 0u, mask = 0u;
  int need = kept, same = 0;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
    each([&](int u, int i, float wi, int pi) {
      const uint32_t key = key_of(u, wi, pi);
      count_bins(hist[pass], (key >> shift) & (bins - 1), i < n && (key & mask) == threshold);
    });
    __syncthreads();
    // counted from the top: lane L owns the `per` bins below bins - per * L, then lane l one of the bins of the lane
    // that the rank falls to
    const int per = bins / 64;
    int mine = 0;
#pragma unroll
    for (int u = 0; u < per / 4; ++u) {
      const int4 h = *(const int4*)&hist[pass][bins - per * (lane + 1) + 4 * ((u + lane) % (per / 4))];   // (staggered over the banks)
      mine += (h.x + h.y) + (h.z + h.w);
    }
    int incl = wave_scan(mine);
    int at = __builtin_ctzll(__ballot(incl >= need));
    need -= __builtin_amdgcn_readlane(incl - mine, at);
    const int top_bin = bins - per * at - 1;
    mine = lane < per ? hist[pass][top_bin - lane] : 0;
    incl = wave_scan(mine);
    at = __builtin_ctzll(__ballot(incl >= need));
    need -= __builtin_amdgcn_readlane(incl - mine, at);
    same = __builtin_amdgcn_readlane(mine, at);
    threshold |= (uint32_t)(top_bin - at) << shift;
    mask |= (uint32_t)(bins - 1) << shift;
  }

  // kept set as a bit mask: keys above the threshold, and the first `need` equal to it
  const int W = (n + 63) / 64;
  unsigned long long* keep = words;
  unsigned long long* equal = words + (a.capacity + 63) / 64;
  const bool all_equal = need == same;
  each([&](int u, int i, float wi, int pi) {
    const uint32_t key = key_of(u, wi, pi);
    const unsigned long long hi = __ballot(i < n && (all_equal ? key >= threshold : key > threshold));
    const unsigned long long eq = __ballot(i < n && key == threshold);
    const int at = u * WAVES + wave;
    if (lane == 0 && at < W) {
      keep[at] = hi;
      equal[at] = eq;
    }
  });
  __syncthreads();
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

  // moves: holes are slots below the budget that lose their token, movers kept tokens from behind it; as many of each
  int32_t* hole_at = a.fused ? list[0] : a.moves + a.batch + (size_t)b * 2 * a.max_moves;
  int32_t* mover_at = a.fused ? list[1] : hole_at + a.max_moves;
  int2 done = make_int2(0, 0);            // holes, movers
  for (int w0 = 0; w0 < W; w0 += stride) {
    const int at = w0 + own;
    const unsigned long long mine = at < W ? keep[at] : 0ull;
    const int below = min(max(kept - 64 * at, 0), 64);         // slots of this word below the budget
    const unsigned long long front = below == 64 ? ~0ull : (1ull << below) - 1ull;
    unsigned long long hole = at < W ? ~mine & front : 0ull, mover = mine & ~front;
    int2 total;
    const int2 first = over_words(__popcll(hole), __popcll(mover), total);
    int h = done.x + first.x, m = done.y + first.y;
    done = make_int2(done.x + total.x, done.y + total.y);
    if (!one || wave == 0) {
      for (; hole != 0ull; hole &= hole - 1ull) hole_at[h++] = 64 * at + __builtin_ctzll(hole);
      for (; mover != 0ull; mover &= mover - 1ull) mover_at[m++] = 64 * at + __builtin_ctzll(mover);
    }
  }
  const int holes = done.x;
  if (threadIdx.x == 0 && !a.fused) a.moves[b] = holes;
  if (new_weight || new_pos || kept_from != nullptr)
    each([&](int, int i, float wi, int pi) { if (i < kept && ((keep[i >> 6] >> (i & 63)) & 1ull)) stay(i, wi, pi); });
  __syncthreads();                        // the lists are read by other threads of this workgroup
  for (int i = threadIdx.x; i < holes; i += THREADS) {
    const int to = hole_at[i], from = mover_at[i];
    weight_out[to] = weight[from];
    pos_out[to] = pos[from];
    if (kept_from != nullptr) kept_from[to] = from;
  }
  if (!a.fused) return;
  uint16_t* k = a.k + b * a.batch_stride;
  uint16_t* v = a.v + b * a.batch_stride;
  for (int i = threadIdx.x; i < holes * a.row_chunks; i += THREADS) {
    const int row = i / a.row_chunks, ch = i % a.row_chunks * 8;
    const long long to = hole_at[row] * a.row_stride + ch, from = mover_at[row] * a.row_stride + ch;
    const uint4 x = *(const uint4*)(k + from), y = *(const uint4*)(v + from);
    *(uint4*)(k + to) = x;
    *(uint4*)(v + to) = y;
  }
}

// K and V of the tokens that move, a row at a time.
__global__ void __launch_bounds__(256) evict_move_kernel(EvictArgs a) {
  const int b = blockIdx.y, count = a.moves[b];
  const int32_t* hole_at = a.moves + a.batch + (size_t)b * 2 * a.max_moves;
  const int32_t* mover_at = hole_at + a.max_moves;
  uint16_t* k = a.k + b * a.batch_stride;
  uint16_t* v = a.v + b * a.batch_stride;
  for (int i = blockIdx.x; i < count; i += gridDim.x) {
    const long long to = hole_at[i] * a.row_stride, from = mover_at[i] * a.row_stride;
    for (int ch = threadIdx.x; ch < a.row_chunks; ch += 256) {
      const uint4 x = *(const uint4*)(k + from + 8 * ch), y = *(const uint4*)(v + from + 8 * ch);
      *(uint4*)(k + to + 8 * ch) = x;
      *(uint4*)(v + to + 8 * ch) = y;
    }
  }
}

size_t evict_workspace_bytes(int batch, int capacity, int budget) {
  const int most = budget < capacity - budget ? budget : capacity - budget;
  return ((size_t)batch * (1 + 2 * (size_t)(most > 0 ? most : 0)) * 4 + 255) & ~(size_t)255;
}

hipError_t launch_cache_evict(EvictArgs a, void* workspace, hipStream_t st) {
  const int most = a.budget < a.capacity - a.budget ? a.budget : a.capacity - a.budget;
  a.max_moves = most > 0 ? most : 0;
  a.moves = (int32_t*)workspace;
  // up to 256 KB of K and V to move for a request: by its selecting workgroup, a launch less
  a.fused = a.max_moves <= FUSED_MOVES && (long long)a.max_moves * a.row_chunks * 32 <= 256 * 1024;
  const int lds = (a.capacity + 63) / 64 * 16;
#define LZ_EVICT(THREADS, ITEMS)                                                                                   \
  do {                                                                                                             \
    auto kern = evict_select_kernel<THREADS, ITEMS>;                                                               \
    if (lds > 32768) {                                                                                             \
      hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);      \
      if (e != hipSuccess) return e;                                                                               \
    }                                                                                                              \
    hipLaunchKernelGGL(kern, dim3(a.batch), dim3(THREADS), lds, st, a);                                            \
  } while (0)
  if (a.capacity <= 1024) LZ_EVICT(256, 4);
  else if (a.capacity <= 4096) LZ_EVICT(512, 8);
  else if (a.capacity <= 16384) LZ_EVICT(1024, 16);
  else LZ_EVICT(1024, 0);
#undef LZ_EVICT
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.max_moves == 0 || a.fused) return e;
  int groups = 2048 / a.batch;
  if (groups < 16) groups = 16;
  if (groups > a.max_moves) groups = a.max_moves;
  hipLaunchKernelGGL(evict_move_kernel, dim3(groups, a.batch), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace lz
