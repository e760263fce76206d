// Eviction from K,V caches by accumulated attention weight: of a request's n tokens the `budget` best stay, protected
// ones (position below `sinks`, or among the `recent` last positions) first, then by weight, ties to the lower slot.
//
// The kept tokens end up in slots 0 .. budget-1, but not in order: a kept token that lies below the budget already stays
// where it is, and the slots that lose theirs are filled, in order, with the kept tokens from behind the budget.  Exactly
// the rows that have to move move (one per step in a cache that is full), no source is another row's destination, and
// attention does not depend on the order of the slots (positions move along).
#include "common.h"

namespace lz {

namespace {

constexpr int THREADS = 1024;

// sorts like the weight; above every weight: a protected token; lowest: NaN
__device__ __forceinline__ uint32_t eviction_key(float w, int pos, int sinks, long long recent_from) {
  if (pos < sinks || pos >= recent_from) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);               // -0 counts as 0
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// exclusive prefix over the threads of the workgroup; total: the sum.  part: LDS int[THREADS / 64].
__device__ __forceinline__ int block_scan(int v, int* part, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(incl, o, 64);
    if (lane >= o) incl += t;
  }
  __syncthreads();
  if (lane == 63) part[wave] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) before += part[w];
    total += part[w];
  }
  return before + incl - v;
}

}  // namespace

// One workgroup per request: the threshold by a radix select over the keys, the kept set as a bit mask in LDS, the list
// of moves (slot, source) into the workspace, and the tables of the kept tokens.
__global__ void __launch_bounds__(THREADS) evict_select_kernel(EvictArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned long long words[];   // above[W], equal[W]
  __shared__ int hist[256], part[THREADS / 64], chosen[2];
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float* weight = a.weight + (size_t)b * a.capacity;
  const int32_t* pos = a.pos + (size_t)b * a.capacity;
  float* weight_out = a.weight_out + (size_t)b * a.capacity;
  int32_t* pos_out = a.pos_out + (size_t)b * a.capacity;
  int n = a.lengths[b];
  if (n > a.capacity) {
    if (threadIdx.x == 0 && a.status != nullptr) atomicOr(a.status, ST_BAD_CU);
    n = a.capacity;
  }
  const int kept = min(n, a.budget);
  __syncthreads();                                  // every thread has the length before it may be overwritten
  if (threadIdx.x == 0) a.lengths_out[b] = kept;
  if (n <= a.budget) {
    for (int i = threadIdx.x; i < kept; i += THREADS) {
      const float w = weight[i];
      const int p = pos[i];
      weight_out[i] = w;
      pos_out[i] = p;
      if (a.kept != nullptr) a.kept[(size_t)b * a.budget + i] = i;
    }
    if (threadIdx.x == 0) a.moves[b] = 0;
    return;
  }
  const int W = (n + 63) / 64;
  unsigned long long* above = words;
  unsigned long long* equal = words + (a.capacity + 63) / 64;

  int top = INT32_MIN;
  for (int i = threadIdx.x; i < n; i += THREADS) top = max(top, pos[i]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = max(top, __shfl_xor(top, o, 64));
  if (lane == 0) part[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) top = max(top, part[w]);
  const long long recent_from = (long long)top + 1 - a.recent;
  auto key_at = [&](int i) { return eviction_key(weight[i], pos[i], a.sinks, recent_from); };

  // the key of rank `kept` from above, and how many of its duplicates are kept
  uint32_t threshold = 0u, mask = 0u;
  int need = kept;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (threadIdx.x < 256) hist[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) {
      const uint32_t key = key_at(i);
      if ((key & mask) == threshold) atomicAdd(&hist[(key >> shift) & 255u], 1);
    }
    __syncthreads();
    // thread i: bin 255 - i, counted from the top
    int total;
    const int mine = threadIdx.x < 256 ? hist[255 - threadIdx.x] : 0;
    const int over = block_scan(mine, part, total);
    if (over < need && need <= over + mine) {
      chosen[0] = 255 - threadIdx.x;
      chosen[1] = need - over;
    }
    __syncthreads();
    threshold |= (uint32_t)chosen[0] << shift;
    mask |= 255u << shift;
    need = chosen[1];
    __syncthreads();
  }

  // kept set: keys above the threshold, and the first `need` equal to it
  for (int w = wave; w < W; w += THREADS / 64) {
    const int i = w * 64 + lane;
    const uint32_t key = i < n ? key_at(i) : 0u;
    const unsigned long long hi = __ballot(i < n && key > threshold), eq = __ballot(i < n && key == threshold);
    if (lane == 0) {
      above[w] = hi;
      equal[w] = eq;
    }
  }
  __syncthreads();
  int base = 0;
  for (int w0 = 0; w0 < W; w0 += THREADS) {
    const int w = w0 + threadIdx.x;
    unsigned long long eq = w < W ? equal[w] : 0ull;
    int total;
    int left = need - (base + block_scan(__popcll(eq), part, total));
    base += total;
    if (w < W) {
      unsigned long long take = 0ull;
      if (left >= 64) take = eq;
      else
        for (; left > 0 && eq != 0ull; --left) {
          take |= eq & (~eq + 1ull);
          eq &= eq - 1ull;
        }
      above[w] |= take;
    }
  }
  __syncthreads();

  // moves: holes are slots below the budget that lose their token, movers kept tokens from behind it; as many of each
  int32_t* hole_at = a.moves + a.batch + (size_t)b * 2 * a.max_moves;
  int32_t* mover_at = hole_at + a.max_moves;
  int holes = 0, movers = 0;
  for (int w0 = 0; w0 < W; w0 += THREADS) {
    const int w = w0 + threadIdx.x;
    const unsigned long long keep = w < W ? above[w] : 0ull;
    const int below = min(max(kept - 64 * w, 0), 64);          // slots of this word below the budget
    const unsigned long long front = below == 64 ? ~0ull : (1ull << below) - 1ull;
    unsigned long long hole = w < W ? ~keep & front : 0ull, mover = keep & ~front;
    int total_h, total_m;
    int h = holes + block_scan(__popcll(hole), part, total_h);
    int m = movers + block_scan(__popcll(mover), part, total_m);
    holes += total_h;
    movers += total_m;
    for (; hole != 0ull; hole &= hole - 1ull) hole_at[h++] = 64 * w + __builtin_ctzll(hole);
    for (; mover != 0ull; mover &= mover - 1ull) mover_at[m++] = 64 * w + __builtin_ctzll(mover);
  }
  if (threadIdx.x == 0) a.moves[b] = holes;
  __syncthreads();                                             // (the lists are read by other threads of this workgroup)
  for (int i = threadIdx.x; i < kept; i += THREADS)
    if ((above[i >> 6] >> (i & 63)) & 1ull) {
      const float w = weight[i];
      const int p = pos[i];
      weight_out[i] = w;
      pos_out[i] = p;
      if (a.kept != nullptr) a.kept[(size_t)b * a.budget + i] = i;
    }
  for (int i = threadIdx.x; i < holes; i += THREADS) {
    const int to = hole_at[i], from = mover_at[i];
    weight_out[to] = weight[from];
    pos_out[to] = pos[from];
    if (a.kept != nullptr) a.kept[(size_t)b * a.budget + to] = from;
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
  const int lds = (a.capacity + 63) / 64 * 16;
  hipError_t e = hipFuncSetAttribute((const void*)evict_select_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(evict_select_kernel, dim3(a.batch), dim3(THREADS), lds, st, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.max_moves == 0) return e;
  int groups = 2048 / a.batch;
  if (groups < 16) groups = 16;
  if (groups > a.max_moves) groups = a.max_moves;
  hipLaunchKernelGGL(evict_move_kernel, dim3(groups, a.batch), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace lz
