// Attention of a batch's new tokens over per-request K,V caches, optionally behind a prefix that all requests share,
// with Eq. 1's head-averaged weight of every cached token kept up to date.
//
// Request b has n_b cached tokens and Q new ones; the new tokens' K,V are appended at slots n_b .. n_b+Q-1 by this
// launch.  Token t sees the prefix (P keys) and the slots up to n_b + t:
//   z = q . k / sqrt(hd),  p = exp(z) / sum exp(z),  o = sum p v,  weight[slot] += 1/H sum_{t,h} p[t][h][slot].
//
// One pass over K and V with a running maximum and sum.  A work item is a K,V head, a block of its query rows and a
// range of keys; the query rows of a K,V head are the (token, query head of the group) pairs of one request for a
// range of its own cache, and those of ALL requests for a range of the prefix, which is therefore read once for a block of rows.
// The partial results (output, maximum, sum) of the ranges are merged by a second launch.
#include <algorithm>
#include <type_traits>

#include "common.h"


namespace lz {

namespace {

constexpr int STEP = 32;              // keys of a wave's step
constexpr int WAVES = 4;
constexpr int SLOTS = 2;              // slots of a lane, for the weights
constexpr int SPLIT_BATCH = 256;      // most requests whose ranges follow the lengths

// Ranges are multiples of what the four waves take in turn.
__host__ __device__ __forceinline__ int round_range(int keys) { return (keys + STEP * WAVES - 1) / (STEP * WAVES) * (STEP * WAVES); }

// Row r of an item is token tok0 + r / group, query head kvh * group + r % group.
struct Item {
  const uint16_t *k, *v;              // first key of the segment, this K,V head
  const uint16_t *k_tail, *v_tail;    // keys n and up: the new tokens (the prefix: its last row again, masked)
  long long stride, tail_stride;      // elements from key to key
  int n, n_tail;                      // keys in the segment, keys behind it
  int lo, hi;                         // range of this item
  int kvh, row0, n_rows, tok0, part;
  bool own;
};

__device__ __forceinline__ int cached_tokens(const CacheAttentionArgs& a, int b) {
  return min(a.lengths[b], a.max_len);            // negative: the request takes no part
}

// parts that a request left, given its number of cached tokens
__device__ __forceinline__ int parts_of(const CacheAttentionArgs& a, int b, int n) {
  if (n < 0) return 0;
  return a.prefix_parts + (a.own_split > 0 ? a.counts[b] : (n + a.q_len + a.own_range - 1) / a.own_range);
}

typedef short short4_t __attribute__((ext_vector_type(4)));
typedef short short8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

// Of four rows' 16 elements, read by 16 lanes 8 bytes each (four lanes a row), lane c gets element c of the four.  The
// restrict says that no copy into LDS under way writes here: without it the compiler waits for all of them.
__device__ __forceinline__ short4_t read_transposed(__attribute__((address_space(3))) short4_t* __restrict__ p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
}

__device__ __forceinline__ uint32_t pack_halves(uint32_t hi, uint32_t lo, bool upper) {
  return __builtin_amdgcn_perm(hi, lo, upper ? 0x07060302u : 0x05040100u);
}

}  // namespace

// A wave takes 32 keys at a time, the four waves of a workgroup in turn over the range; both products run on 16x16x32 MFMAs,
// transposed so that a lane owns a query column: S^T = K Q^T, O^T = V^T P^T.
//   K: row by row into 32 rows of LDS that are the wave's own (no barrier: the copies of the next step start when this
//      step's operands have been read, and have this step's first product and softmax to land in: they stand under a
//      condition, so the compiler, which cannot count them, waits for all that is under way, logit stores too, in front
//      of the second product), read as operands: lane (c = lane % 16, g = lane / 16) takes dimensions
//      32 s + 8 g .. + 7 of key c.  Straight into operand registers, 64 bytes of 16 rows a load, was level without and 10 %
//      slower with non-temporal loads (113.7 against 101 us below).
//   V: straight into registers.  Lane (c, g) holds dimensions HD/16 c .. of the eight keys that its S^T accumulators belong
//      to (4 g + r of each block of 16), whole rows of 256 bytes per 16 lanes; pairs of keys are put together by v_perm.
//      Output tile i then has dimension HD/16 c + i in row c, and no value of P changes its lane.
// P goes into the second product as two bf16 terms (value and remainder): one alone would add an error as large as the
// rounding of the output itself, and the matrix cores idle here anyway, the kernel is bound by reading K and V (8 requests
// of 1 - 8 k tokens, 32 heads: 554 MB in 101 us with the merge; 16 of 8000, 8 K,V heads: 524 MB in 113).
// STREAM: non-temporal loads.  0: none, row blocks share what is read; 1: V (8 requests of 1 - 8 k tokens 121 us without,
// 113 with, before K went through LDS); 2: K too, for more than the last-level cache can hold from one call to the next
// (launch_cache_attention).
template <int HD, int T, int STREAM>
__global__ void __launch_bounds__(256, 2) cache_attention_kernel(CacheAttentionArgs a) {
  constexpr int KS = HD / 32;          // k-steps of the first product
  constexpr int NT = HD / 16;          // tiles of 16 output dimensions = dimensions a lane holds of a V row
  constexpr int VW = NT / 2;           // dwords of that
  constexpr int PITCH = HD + 4;
  typedef uint32_t words_t __attribute__((ext_vector_type(VW)));
  extern __shared__ __attribute__((aligned(16))) float lds[];   // [WAVES][16 T][PITCH], then float2 [WAVES][16 T]
  float2* ml = (float2*)(lds + WAVES * 16 * T * PITCH);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int kvd = a.n_kv * HD;

  // The K,V head varies fastest: workgroups are dealt out to the XCDs in turn, so that all of them get as much of every
  // request, and row blocks of one range share an L2.
  int id = blockIdx.x;
  const int prefix_items = a.shared_tiles ? 0 : a.prefix_parts * a.n_kv * a.prefix_blocks;
  Item it;
  it.own = id >= prefix_items;
  if (it.own) id -= prefix_items;
  it.kvh = id % a.n_kv;
  id /= a.n_kv;
  const int blocks = it.own ? a.own_blocks : a.prefix_blocks;
  it.row0 = 0;
  if (blocks > 1) {
    it.row0 = id % blocks * 16 * T;
    id /= blocks;
  }
  int b = 0, part = id, own_range = a.own_range, own_parts = 0, given = 0;
  if (it.own && a.own_split > 0) {
    // Of all requests' keys every range gets about its share: a lane a request, 64 requests at a time.
    int length[SPLIT_BATCH / 64], keys[SPLIT_BATCH / 64];
    uint32_t total = 0;                                          // (below 2^31, as batch * capacity)
#pragma unroll
    for (int u = 0; u < SPLIT_BATCH / 64; ++u) length[u] = 64 * u + lane < a.batch ? a.lengths[64 * u + lane] : -1;
#pragma unroll
    for (int u = 0; u < SPLIT_BATCH / 64; ++u)
      if (64 * u < a.batch) {
        keys[u] = length[u] >= 0 ? min(length[u], a.max_len) + a.q_len : 0;
        total += (uint32_t)__builtin_amdgcn_readlane(wave_scan(keys[u]), 63);
      }
    const int range = max(own_range, round_range((int)min((total + a.own_split - 1) / a.own_split, 1u << 30)));
    int before = 0;                                              // parts of the 64s before
    b = -1;
#pragma unroll
    for (int u = 0; u < SPLIT_BATCH / 64; ++u)
      if (b < 0 && 64 * u < a.batch) {
        const int parts = (keys[u] + range - 1) / range, upto = before + wave_scan(parts);
        const int at = __popcll(__ballot(upto <= id));
        before = __builtin_amdgcn_readlane(upto, 63);
        if (at < 64) {
          b = 64 * u + at;
          given = __builtin_amdgcn_readlane(length[u], at);
          part = id - __builtin_amdgcn_readlane(upto - parts, at);
          // equal ranges of this request
          const int mine = __builtin_amdgcn_readlane(keys[u], at), n_parts = __builtin_amdgcn_readlane(parts, at);
          own_range = round_range((mine + n_parts - 1) / n_parts);
          own_parts = (mine + own_range - 1) / own_range;
        }
      }
    if (b < 0) return;                 // (more workgroups than parts)
  } else if (it.own && a.batch > 1) {
    b = id % a.batch;
    part = id / a.batch;
  }
  it.tok0 = b * a.q_len;
  it.n_rows = (it.own ? 1 : a.batch) * a.q_len * a.group;

  // (on its way while the length is, where the request was not found from the lengths above)
  bf16x8_t qf[T][KS];
  int tok[T];
  size_t out_row[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int r = min(it.row0 + 16 * t + c, it.n_rows - 1);
    tok[t] = r / a.group;
    out_row[t] = (size_t)(it.tok0 + tok[t]) * a.n_heads + it.kvh * a.group + r - tok[t] * a.group;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[t][s] = *(const bf16x8_t*)(a.q + out_row[t] * HD + 32 * s + 8 * g);
  }

  if (!it.own) {
    it.part = part;
    it.stride = a.prefix_stride;
    it.k = a.prefix_k + it.kvh * HD;
    it.v = a.prefix_v + it.kvh * HD;
    it.n = a.prefix_len;
    it.n_tail = 1;
    it.k_tail = it.k + (a.prefix_len - 1) * it.stride;
    it.v_tail = it.v + (a.prefix_len - 1) * it.stride;
    it.tail_stride = 0;
    it.lo = part * a.prefix_range;
    it.hi = min(it.lo + a.prefix_range, a.prefix_len);
  } else {
    it.part = a.prefix_parts + part;
    if (a.own_split == 0) given = a.lengths[b];
    it.n = min(given, a.max_len);
    if (it.n < 0) {
      // no partial results: the output rows are zero (with more than one part the second launch clears them)
      if (a.merge == 0)
        for (int i = threadIdx.x; i < min(16 * T, it.n_rows - it.row0) * (HD / 8); i += 256) {
          const int r = it.row0 + i / (HD / 8);
          ((uint4*)(a.o + ((size_t)(it.tok0 + r / a.group) * a.n_heads + it.kvh * a.group + r % a.group) * HD))[i % (HD / 8)] =
              make_uint4(0, 0, 0, 0);
        }
      return;
    }
    if (part == 0 && it.kvh == 0 && it.row0 == 0 && threadIdx.x == 0) {
      if (a.status != nullptr && given > a.max_len) atomicOr(a.status, ST_BAD_CU);
      if (a.own_split > 0) a.counts[b] = own_parts;
    }
    it.stride = a.row_stride;
    it.k = a.k + b * a.batch_stride + it.kvh * HD;
    it.v = a.v + b * a.batch_stride + it.kvh * HD;
    it.n_tail = a.q_len;
    it.k_tail = a.k_new + ((size_t)it.tok0 * a.n_kv + it.kvh) * HD;
    it.v_tail = a.v_new + ((size_t)it.tok0 * a.n_kv + it.kvh) * HD;
    it.tail_stride = kvd;
    it.lo = part * own_range;
    it.hi = min(it.lo + own_range, it.n + a.q_len);
  }
  if (it.lo >= it.hi) return;
  int last[T];                          // the last key that a query row sees
#pragma unroll
  for (int t = 0; t < T; ++t) last[t] = it.own ? it.n + tok[t] : it.n - 1;

  floatx4_t acc[T][NT];
  float m_run[T], l_run[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    m_run[t] = -INFINITY;
    l_run[t] = 0.f;
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[t][i] = {0.f, 0.f, 0.f, 0.f};
  }

  // rows of a step that reaches beyond key n: the new tokens' (the prefix: its last one again, masked)
  auto tail_row = [&](const uint16_t* base, const uint16_t* behind, int key) {
    if (key < it.n) return base + key * it.stride;
    return behind + min(key - it.n, it.n_tail - 1) * it.tail_stride;
  };
  // K of a step goes through 32 rows of LDS of this wave's own: copied row by row, read as operands
  constexpr int CHK = HD / 8, ROWS = 64 / CHK;        // 16-byte chunks of a row, rows of a copy
  constexpr int COPIES = STEP / ROWS;
  char* mine = (char*)lds + wave * STEP * HD * 2;
  auto swz = [](int r) { return CHK == 16 ? swz128(r) : swz64(r); };
  uint32_t k_from[COPIES];                            // this lane's part of a copy's address, in bytes
#pragma unroll
  for (int u = 0; u < COPIES; ++u) {
    const int r = u * ROWS + lane / CHK;
    k_from[u] = (uint32_t)(lane / CHK) * (uint32_t)it.stride * 2u + ((lane % CHK) ^ swz(r)) * 16;
  }
  const uint32_t v_from = 4u * g * (uint32_t)it.stride * 2u + NT * c * 2;
  auto copy_k = [&](int k0) {
    if (k0 + STEP <= it.n) {
      const char* base = (const char*)(it.k + k0 * it.stride);
#pragma unroll
      for (int u = 0; u < COPIES; ++u)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base + u * ROWS * 2 * it.stride + k_from[u]),
                                         (__attribute__((address_space(3))) void*)(mine + u * 1024), 16, 0, STREAM == 2 ? 2 : 0);
    } else {
#pragma unroll
      for (int u = 0; u < COPIES; ++u) {
        const int r = u * ROWS + lane / CHK;
        g2l16(tail_row(it.k, it.k_tail, k0 + r) + ((lane % CHK) ^ swz(r)) * 8, mine + u * 1024);
      }
    }
  };
  // q is here before the first copy starts: waited for inside the loop, it would have every copy waited for
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < KS; ++i) asm volatile("" : "+v"(qf[t][i]));
  int k0 = it.lo + STEP * wave;
  if (k0 < it.hi) copy_k(k0);
  auto step = [&](auto reaches_beyond) {
    constexpr bool tail = decltype(reaches_beyond)::value;
    uint32_t vf[8][VW];
    const char* vbase = (const char*)(it.v + k0 * it.stride);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const words_t* vp;
      if (tail) vp = (const words_t*)(tail_row(it.v, it.v_tail, k0 + 16 * (j >> 2) + 4 * g + (j & 3)) + NT * c);
      else vp = (const words_t*)(vbase + (16 * (j >> 2) + (j & 3)) * 2 * it.stride + v_from);
      *(words_t*)vf[j] = STREAM > 0 ? __builtin_nontemporal_load(vp) : *vp;
    }
    // K has landed (the eight loads of V are behind it)
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    bf16x8_t kf[2][KS];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int i = 0; i < KS; ++i)
        kf[sub][i] = *(const bf16x8_t*)(mine + (16 * sub + c) * HD * 2 + (((4 * i + g) ^ swz(16 * sub + c)) * 16));
    // read: the next step's K may come
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (k0 + STEP * WAVES < it.hi) copy_k(k0 + STEP * WAVES);
    __builtin_amdgcn_sched_barrier(0);
    float s[T][8];                      // s[t][4 sub + r]: key k0 + 16 sub + 4 g + r, not scaled
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        floatx4_t s4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KS; ++i) s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[sub][i], qf[t][i], s4, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[t][4 * sub + r] = s4[r];
      }
    uint4 p_hi[T], p_lo[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      if (tail)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (k0 + 16 * (i >> 2) + 4 * g + (i & 3) > last[t]) s[t][i] = -INFINITY;
      if (a.z != nullptr && it.own && it.row0 + 16 * t + c < it.n_rows) {
        float* zp = a.z + out_row[t] * a.z_ld + k0 + 4 * g;
        *(float4*)zp = make_float4(s[t][0] * a.scale_log2e, s[t][1] * a.scale_log2e, s[t][2] * a.scale_log2e, s[t][3] * a.scale_log2e);
        *(float4*)(zp + 16) = make_float4(s[t][4] * a.scale_log2e, s[t][5] * a.scale_log2e, s[t][6] * a.scale_log2e, s[t][7] * a.scale_log2e);
      }
      float top = s[t][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, s[t][i]);
      top *= a.scale_log2e;
      // the reference point of the exponentials follows only when a logit exceeds it by 2^8
      if (__any(top > m_run[t] + 8.f)) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m_new = fmaxf(m_run[t], top);
        const float f = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[t] - m_new);
        m_run[t] = m_new;
        l_run[t] *= f;
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[t][i] *= f;
      }
      const float m_use = m_run[t] == -INFINITY ? 0.f : m_run[t];
      float p[8], rest[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], a.scale_log2e, -m_use));
        l_run[t] += p[i];
      }
      p_hi[t] = pack8(p);
      unpack8(p_hi[t], rest);
#pragma unroll
      for (int i = 0; i < 8; ++i) rest[i] = p[i] - rest[i];
      p_lo[t] = pack8(rest);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      uint4 w;
      w.x = pack_halves(vf[1][i / 2], vf[0][i / 2], i & 1);
      w.y = pack_halves(vf[3][i / 2], vf[2][i / 2], i & 1);
      w.z = pack_halves(vf[5][i / 2], vf[4][i / 2], i & 1);
      w.w = pack_halves(vf[7][i / 2], vf[6][i / 2], i & 1);
      const bf16x8_t vt = *(const bf16x8_t*)&w;
#pragma unroll
      for (int t = 0; t < T; ++t) {
        acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, *(const bf16x8_t*)&p_hi[t], acc[t][i], 0, 0, 0);
        acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, *(const bf16x8_t*)&p_lo[t], acc[t][i], 0, 0, 0);
      }
    }
    k0 += STEP * WAVES;
  };
  while (k0 < it.hi && k0 + STEP <= it.n) step(std::false_type{});
  while (k0 < it.hi) step(std::true_type{});

  // the new tokens of this range into the cache (nobody reads slots n and up from it in this launch)
  if (it.own && it.row0 == 0 && it.hi > it.n) {
    const int first = max(it.lo, it.n);
    for (int i = threadIdx.x; i < (it.hi - first) * (HD / 8) * 2; i += 256) {
      const int slot = first + i / (HD / 4), ch = i % (HD / 8) * 8;
      const bool is_v = (i / (HD / 8)) & 1;
      uint16_t* dst = (is_v ? a.v : a.k) + b * a.batch_stride + slot * a.row_stride + it.kvh * HD + ch;
      *(uint4*)dst = *(const uint4*)((is_v ? it.v_tail : it.k_tail) + (slot - it.n) * it.tail_stride + ch);
    }
    if (a.pos != nullptr && it.kvh == 0 && (int)threadIdx.x < it.hi - first)
      a.pos[(size_t)b * a.capacity + first + threadIdx.x] = a.pos_new[b] + first - it.n + threadIdx.x;
  }

  __syncthreads();                      // (K's rows are read: the waves' results go where they were)
  // the four waves, merged through LDS
#pragma unroll
  for (int t = 0; t < T; ++t) {
    float l = l_run[t];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) ml[wave * 16 * T + 16 * t + c] = make_float2(m_run[t], l);
    float* row = lds + (wave * 16 * T + 16 * t + c) * PITCH;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < NT; i += 4)
        *(float4*)(row + NT * (4 * g + r) + i) = make_float4(acc[t][i][r], acc[t][i + 1][r], acc[t][i + 2][r], acc[t][i + 3][r]);
  }
  __syncthreads();
  const int rows = min(16 * T, it.n_rows - it.row0);
  const size_t all_rows = (size_t)a.batch * a.q_len * a.n_heads;
  for (int i = threadIdx.x; i < rows * (HD / 8); i += 256) {
    const int r = i / (HD / 8), ch = i % (HD / 8) * 8, gr = it.row0 + r;
    float m = -INFINITY, l = 0.f, w[WAVES];
#pragma unroll
    for (int u = 0; u < WAVES; ++u) m = fmaxf(m, ml[u * 16 * T + r].x);
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < WAVES; ++u) {
      const float2 s = ml[u * 16 * T + r];
      w[u] = s.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.x - m);
      l += w[u] * s.y;
      const float* src = lds + (u * 16 * T + r) * PITCH + ch;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += w[u] * src[e];
    }
    const size_t orow = (size_t)(it.tok0 + gr / a.group) * a.n_heads + it.kvh * a.group + gr % a.group;
    if (a.merge == 0) {
      const float inv = 1.0f / l;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= inv;
      *(uint4*)(a.o + orow * HD + ch) = pack8(x);
    } else {
      float* dst = a.part + (it.part * all_rows + orow) * HD + ch;
      *(float4*)dst = make_float4(x[0], x[1], x[2], x[3]);
      *(float4*)(dst + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
    if (ch == 0 && a.stat != nullptr) a.stat[it.part * all_rows + orow] = make_float2(m, l);
  }
}

// (maximum, sum) of one row over its parts, by eight consecutive lanes together; every one of them gets the result.
__device__ __forceinline__ float2 merged_stat(const float2* __restrict__ st, size_t pitch, int parts, int sub) {
  float m = -INFINITY, l = 0.f;
  for (int s0 = 0; s0 < parts; s0 += 32) {
    float2 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = s0 + 8 * u + sub;
      v[u] = s < parts ? st[s * pitch] : make_float2(-INFINITY, 0.f);
    }
    const float top = fmaxf(fmaxf(fmaxf(v[0].x, v[1].x), fmaxf(v[2].x, v[3].x)), m);
    const float at = top == -INFINITY ? 0.f : top;
    l *= __builtin_amdgcn_exp2f(m - at);
#pragma unroll
    for (int u = 0; u < 4; ++u) l += v[u].y * __builtin_amdgcn_exp2f(v[u].x - at);
    m = top;
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    const float m2 = __shfl_xor(m, o, 64), l2 = __shfl_xor(l, o, 64);
    const float top = fmaxf(m, m2), at = top == -INFINITY ? 0.f : top;
    l = l * __builtin_amdgcn_exp2f(m - at) + l2 * __builtin_amdgcn_exp2f(m2 - at);
    m = top;
  }
  return make_float2(m, l);
}

// Merges the partial results and adds the weights.  The first workgroups take an output row each (its parts dealt out to
// the waves) or, with few parts, one row a wave; the others 128 slots of a request each: a lane two slots, every wave a
// share of its rows, in a fixed order.  (64 slots: 60.5 us for 16 requests of 0.7 - 8 k, five tokens each, where this took
// 59.4, and 108 for 106.4 on 16 of 8000.)  MW waves: 16 where a slot gets the weights of 64 rows or more, which they read
// sooner, 4 elsewhere, where the workgroups are many and short.  4 / 16 waves: 8 tokens of one request of 1900 24.4 / 18.3 us,
// 17 requests of 2 - 63 20.0 / 14.5, five of 16 of 0.7 - 8 k 58.1 / 57.0, two (64 rows) of 44 of 80 - 640 24.8 / 24.3; one token (32 rows) of
// one of 131071 109 / 114, of 32 of 150 - 2100 25.6 / 26.5.
template <int HD, int MW>
__global__ void __launch_bounds__(64 * MW) cache_merge_kernel(CacheAttentionArgs a) {
  constexpr int E = HD / 64;           // output dimensions of a lane
  constexpr int RB = MW == 16 ? 4 : 8; // rows whose logits a wave reads at a time
  __shared__ float2 stats[256];
  __shared__ float sums[MW][HD], slot_sums[MW][SLOTS][64];
  const int all_rows = a.batch * a.q_len * a.n_heads;
  const int merge_groups = a.merge == 0 ? 0 : a.merge == 1 ? (all_rows + MW - 1) / MW : all_rows;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if ((int)blockIdx.x < merge_groups) {
    const int row = a.merge == 1 ? blockIdx.x * MW + wave : blockIdx.x;
    const int first = a.merge == 1 ? 0 : wave, step = a.merge == 1 ? 1 : MW;
    if (row >= all_rows) return;       // (of whole waves, and only where no barrier follows)
    const float2* st = a.stat + row;
    const float* src = a.part + (size_t)row * HD + E * lane;
    const int most = a.prefix_parts + a.own_parts;
    // the parts' outputs four at a time, the next four on their way before the sum of these (and the first before anything
    // is known about the request: those it does not have are not added)
    float x[E], v[4][E], top[4];
    auto fetch = [&](int s0) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const size_t s = min(s0 + u * step, most - 1);
        top[u] = st[s * all_rows].x;
#pragma unroll
        for (int e = 0; e < E; ++e) v[u][e] = src[s * all_rows * HD + e];
      }
    };
    fetch(first);
    const int request = row / (a.q_len * a.n_heads), parts = parts_of(a, request, cached_tokens(a, request));
    const float2 ml = merged_stat(st, all_rows, parts, lane & 7);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = 0.f;
    for (int s0 = first; s0 < parts; s0 += 4 * step) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (s0 + u * step < parts) {
          const float w = __builtin_amdgcn_exp2f(top[u] - ml.x);
#pragma unroll
          for (int e = 0; e < E; ++e) x[e] += w * v[u][e];
        }
      if (s0 + 4 * step < parts) fetch(s0 + 4 * step);
    }
    if (a.merge != 1) {
#pragma unroll
      for (int e = 0; e < E; ++e) sums[wave][E * lane + e] = x[e];
      __syncthreads();
      if (wave != 0) return;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int u = 1; u < MW; ++u) x[e] += sums[u][E * lane + e];
    }
    const float inv = parts == 0 ? 0.f : 1.0f / ml.y;
    if (E == 2) ((uint32_t*)(a.o + (size_t)row * HD))[lane] = pack_bf16(x[0] * inv, x[E - 1] * inv);
    else a.o[(size_t)row * HD + lane] = to_bf16(x[0] * inv);
    return;
  }
  const int id = blockIdx.x - merge_groups;
  const int chunks = (a.max_len + a.q_len + 64 * SLOTS - 1) / (64 * SLOTS);
  const int b = id / chunks, slot0 = id % chunks * (64 * SLOTS), slot = slot0 + SLOTS * lane;
  const int n = cached_tokens(a, b);
  if (n < 0 || slot0 >= n + a.q_len) return;
  const int rows = a.q_len * a.n_heads, row0 = b * rows;
  const int parts = parts_of(a, b, n);
  typedef float slots_t __attribute__((ext_vector_type(SLOTS)));
  const float* zp = a.z + (size_t)row0 * a.z_ld + min(slot, a.z_ld - SLOTS);
  float sum[SLOTS];
#pragma unroll
  for (int e = 0; e < SLOTS; ++e) sum[e] = 0.f;
  for (int base = 0; base < rows; base += 256) {
    const int count = min(256, rows - base);
    __syncthreads();
    for (int r = threadIdx.x >> 3; r < count; r += 8 * MW) {
      const float2 ml = merged_stat(a.stat + row0 + base + r, all_rows, parts, threadIdx.x & 7);
      if ((threadIdx.x & 7) == 0) stats[r] = make_float2(ml.x, 1.0f / ml.y);
    }
    __syncthreads();
    // every wave its share of the rows
    const int share = (count + MW - 1) / MW, end = min(count, (wave + 1) * share);
    for (int r = wave * share; r < end; r += RB) {
      slots_t z[RB];
#pragma unroll
      for (int u = 0; u < RB; ++u) z[u] = *(const slots_t*)(zp + (size_t)(base + min(r + u, end - 1)) * a.z_ld);
#pragma unroll
      for (int u = 0; u < RB; ++u) {
        const float2 ml = stats[min(r + u, end - 1)];
        const float inv = r + u < end ? ml.y : 0.f;
#pragma unroll
        for (int e = 0; e < SLOTS; ++e) sum[e] += __builtin_amdgcn_exp2f(z[u][e] - ml.x) * inv;
      }
    }
  }
#pragma unroll
  for (int e = 0; e < SLOTS; ++e) slot_sums[wave][e][lane] = sum[e];
  __syncthreads();
  if (wave < SLOTS) {
    const int s = slot + wave;
    if (s < n + a.q_len) {
      float x = slot_sums[0][wave][lane];
#pragma unroll
      for (int u = 1; u < MW; ++u) x += slot_sums[u][wave][lane];
      a.weight_out[(size_t)b * a.capacity + s] = (s < n ? a.weight[(size_t)b * a.capacity + s] : 0.f) + x / (float)a.n_heads;
    }
  }
}

// ------------------------------------------------------------------------------------------
// The prefix for many query rows of a K,V head: the matrix cores bound it.  A workgroup is eight waves of 32 query rows
// of one K,V head; tiles of 64 keys go through LDS, copied three stages deep by global_load_lds, and every wave reads
// all of a tile.  Products and layout as above, but V's operand comes out of LDS through the transposing read
// (ds_read_b64_tr_b16: of four keys' 16 dimensions, lane c gets dimension c of the four), so no vector instruction is
// spent on it.  The sum of the exponentials is one more row tile of the second product (V = 1): it costs the
// matrix pipe 1/13 and spares the vector unit an addition per probability.  P goes into the second product as two bf16
// terms, as above, so that a request's accuracy does not depend on how many others are in its batch: 2048 rows of 8 K,V
// heads behind 32768 keys 353 us and 1.66e-3 off (the rounding of the output), with one term 264 us and 2.33e-3.
// What bounds it there: of the 5.5 k cycles that a step takes a SIMD, 3.3 k are the matrix pipe's; 420 vector instructions,
// 128 of them exponentials, go on beside it.  With one term, the two waves of a SIMD kept in opposite phases by two
// barriers a step, or with the next scores under the exponentials, were no faster (300, 280 us where this took 268); nor
// were three row tiles a wave (314).
template <int HD>
__global__ void __launch_bounds__(512, 2) prefix_attention_kernel(CacheAttentionArgs a) {
  constexpr int KS = HD / 32, NT = HD / 16, BN = 64, T = 2, NW = 8;
  constexpr int CHK = HD / 8;                        // 16-byte chunks of a row
  constexpr int TILE = BN * HD * 2;                  // bytes of a K or V tile
  constexpr int STAGE = 2 * TILE, NS = 3;
  constexpr int COPIES = TILE / 1024 / NW;           // of each tile per wave
  constexpr int ROWS_PER_COPY = 64 / CHK;
  extern __shared__ __attribute__((aligned(1024))) char tiles[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  int id = blockIdx.x;
  const int kvh = id % a.n_kv;
  id /= a.n_kv;
  const int row0 = id % a.prefix_blocks * (16 * T * NW) + 16 * T * wave;
  const int part = id / a.prefix_blocks;
  const int n_rows = a.batch * a.q_len * a.group;
  const int lo = part * a.prefix_range, hi = min(lo + a.prefix_range, a.prefix_len);
  const uint16_t* kbase = a.prefix_k + kvh * HD;
  const uint16_t* vbase = a.prefix_v + kvh * HD;

  // Chunk ch of row r lies at chunk ch ^ swizzle(r).  K is read 16 rows x 16 bytes at a time: 16 rows take 16 different
  // 16-byte units of a 256-byte line; V 8 rows x 32 bytes: eight rows take eight different 32-byte units.
  auto swz_k = [](int r) { return CHK == 16 ? swz128(r) : swz64(r); };
  auto swz_v = [](int r) { return CHK == 16 ? (r & 7) << 1 : (r >> 1 & 3) << 1; };
  // copies of a wave: rows r0 + u * ROWS_PER_COPY of a tile, as byte offsets from the tile's first row
  const int r0 = wave * COPIES * ROWS_PER_COPY + lane / CHK;
  uint32_t k_from[COPIES], v_from[COPIES];
#pragma unroll
  for (int u = 0; u < COPIES; ++u) {
    const int r = r0 + u * ROWS_PER_COPY;
    const uint32_t row = (uint32_t)r * (uint32_t)a.prefix_stride * 2u;
    k_from[u] = row + ((lane % CHK) ^ swz_k(r)) * 16;
    v_from[u] = row + ((lane % CHK) ^ swz_v(r)) * 16;
  }
  auto issue = [&](int stage, int k0) {
    char* to = tiles + stage * STAGE + wave * COPIES * 1024;
    const long long row = (long long)k0 * a.prefix_stride;
    const int last_row = a.prefix_len - 1 - k0;          // rows behind it: the last one again
#pragma unroll
    for (int u = 0; u < COPIES; ++u) {
      uint32_t kf = k_from[u], vf = v_from[u];
      if (last_row < BN - 1) {
        const int r = r0 + u * ROWS_PER_COPY;
        const uint32_t back = (uint32_t)max(r - last_row, 0) * (uint32_t)a.prefix_stride * 2u;
        kf -= back;
        vf -= back;
      }
      g2l16((const char*)(kbase + row) + kf, to + u * 1024);
      g2l16((const char*)(vbase + row) + vf, to + TILE + u * 1024);
    }
  };
  // byte offsets of this lane's operand reads in a stage; 16 rows further on: 32 HD bytes
  uint32_t k_at[KS], v_at[NT];
#pragma unroll
  for (int i = 0; i < KS; ++i) k_at[i] = c * HD * 2 + (((4 * i + g) ^ swz_k(c)) * 16);
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int r = 4 * g + (c >> 2);
    v_at[i] = TILE + r * HD * 2 + (((2 * i + (c >> 1 & 1)) ^ swz_v(r)) * 16) + (c & 1) * 8;
  }

  bf16x8_t qf[T][KS];
  size_t out_row[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int r = min(row0 + 16 * t + c, n_rows - 1);
    out_row[t] = (size_t)(r / a.group) * a.n_heads + kvh * a.group + r % a.group;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[t][s] = *(const bf16x8_t*)(a.q + out_row[t] * HD + 32 * s + 8 * g);
  }
  floatx4_t acc[T][NT], sum[T];
  float m_run[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    m_run[t] = -INFINITY;
    sum[t] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[t][i] = {0.f, 0.f, 0.f, 0.f};
  }
  // q is here before the first copy starts: waited for inside the loop, it would have every copy waited for
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[t][s]));
  const uint4 ones4 = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
  const bf16x8_t ones = *(const bf16x8_t*)&ones4;

  const int steps = (hi - lo + BN - 1) / BN;
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (i < steps) issue(i, lo + i * BN);
  int stage = 0;
  for (int it = 0; it < steps; ++it) {
    const int k0 = lo + it * BN;
    // this step's copies have landed (those of the next one may be under way), and the stage that the copies
    // issued below overwrite, the previous step's, is no longer read
    if (it + 1 < steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * COPIES) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (it + NS - 1 < steps) issue(stage == 0 ? NS - 1 : stage - 1, k0 + (NS - 1) * BN);
    lds_char* st = (lds_char*)tiles + stage * STAGE;
    stage = stage + 1 == NS ? 0 : stage + 1;

    floatx4_t s[T][4];                               // s[t][sub][r]: key k0 + 16 sub + 4 g + r
#pragma unroll
    for (int sub = 0; sub < 4; ++sub)
#pragma unroll
      for (int t = 0; t < T; ++t) s[t][sub] = {0.f, 0.f, 0.f, 0.f};
    // (two key blocks at a time: four accumulators in turn, so that no product waits for the one before it)
#pragma unroll
    for (int pair = 0; pair < 2; ++pair)
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int sub = 2 * pair; sub < 2 * pair + 2; ++sub) {
          const bf16x8_t kf = *(const __attribute__((address_space(3))) bf16x8_t*)(st + k_at[i] + sub * 32 * HD);
#pragma unroll
          for (int t = 0; t < T; ++t) s[t][sub] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][i], s[t][sub], 0, 0, 0);
        }
    // operand reads run six ahead of the products that take them
    __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
    for (int u = 0; u < 4 * KS - 6; ++u) {
      __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 12, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (k0 + BN > a.prefix_len)
#pragma unroll
      for (int sub = 0; sub < 4; ++sub)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (k0 + 16 * sub + 4 * g + r >= a.prefix_len)
#pragma unroll
            for (int t = 0; t < T; ++t) s[t][sub][r] = -INFINITY;
    uint4 p_hi[T][2], p_lo[T][2];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      float top = s[t][0][0];
#pragma unroll
      for (int sub = 0; sub < 4; ++sub)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, s[t][sub][r]);
      top *= a.scale_log2e;
      if (__any(top > m_run[t] + 8.f)) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m_new = fmaxf(m_run[t], top);
        const float f = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[t] - m_new);
        m_run[t] = m_new;
        asm volatile("; raise the running maximum" ::: "memory");
        sum[t] *= f;
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[t][i] *= f;
      }
      const float neg_m = m_run[t] == -INFINITY ? 0.f : -m_run[t];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          e[j] = __builtin_amdgcn_exp2f(fmaf(s[t][2 * u + (j >> 2)][j & 3], a.scale_log2e, neg_m));
        float rest[8];
        p_hi[t][u] = pack8(e);
        unpack8(p_hi[t][u], rest);
#pragma unroll
        for (int j = 0; j < 8; ++j) rest[j] = e[j] - rest[j];
        p_lo[t][u] = pack8(rest);
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int t = 0; t < T; ++t) sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, *(const bf16x8_t*)&p_hi[t][u], sum[t], 0, 0, 0);
#pragma unroll
      for (int t = 0; t < T; ++t) sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, *(const bf16x8_t*)&p_lo[t][u], sum[t], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        short4_t half[2];
#pragma unroll
        for (int w = 0; w < 2; ++w)
          half[w] = read_transposed((__attribute__((address_space(3))) short4_t*)(st + v_at[i] + (2 * u + w) * 32 * HD));
        const short8_t both = __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int t = 0; t < T; ++t)
          acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8_t*)&both, *(const bf16x8_t*)&p_hi[t][u], acc[t][i], 0, 0, 0);
#pragma unroll
        for (int t = 0; t < T; ++t)
          acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8_t*)&both, *(const bf16x8_t*)&p_lo[t][u], acc[t][i], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 12, 0);
#pragma unroll
    for (int u = 0; u < 2 * NT - 6; ++u) {
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 32, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
  const size_t all_rows = (size_t)a.batch * a.q_len * a.n_heads;
#pragma unroll
  for (int t = 0; t < T; ++t)
    if (row0 + 16 * t + c < n_rows) {
      float* dst = a.part + (part * all_rows + out_row[t]) * HD + 4 * g;
#pragma unroll
      for (int i = 0; i < NT; ++i) *(float4*)(dst + 16 * i) = make_float4(acc[t][i][0], acc[t][i][1], acc[t][i][2], acc[t][i][3]);
      if (g == 0) a.stat[part * all_rows + out_row[t]] = make_float2(m_run[t], sum[t][0]);
    }
}

// How a call is cut, measured (us):
//  - the prefix through shared tiles (blocks of 256 query rows) from 42 M logits on: keys x K,V heads x query rows, less the
//    rows that are missing in the last block, which cost as much.  Below, the launch more costs more than the tiles save.
//    Direct / shared, at 36, 44 and 66 M: 256 rows of 8 K,V heads of 128: 50 / 50, 59 / 55, 87 / 70; 512: 45 / 46, 51 / 51, 72 / 65;
//    2048: 56 / 57, 61 / 62, 76 / 72; 256 of 32 heads: 63 / 66, 71 / 71, 94 / 86; 2048 of one: 44 / 47, 51 / 52, 72 / 65; 256 of 4
//    heads of 64: 36 / 40, 41 / 43, 58 / 50; 1024: 35 / 36, 41 / 39, 56 / 47; 2048 of 8 heads of 64: 35 / 41, 39 / 45, 50 / 52.  Blocks in part
//    empty, at 44 and 66 M without that: 128 rows of 8 heads: 71 / 78, 98 / 107; 192: 67 / 63, 96 / 82; 288: 66 / 72, 97 / 96.
//  - row tiles: one up to 16 rows, else two (a prefix of 3376 for 128 rows: 20.1 with one, 16.6 with two).
//  - ranges of the caches, up to 256 requests: by the lengths, which the host does not know; every workgroup finds its range
//    from all of them.  About 256 ranges x K,V heads a request, at most 2048 (one row tile) or 512 (two: as many workgroups
//    as run at once).  By max_len / by the lengths: 32 x 150 - 2100 tokens 28.4 / 25.5; 16 x 0.7 - 8 k, 20 rows 69.1 / 60.3;
//    64 x 5 - 2000 39.6 / 34.1; 2 x 20 and 64 k 109 / 89; 4 x 4 - 30 k, 20 rows 90 / 76; one of 4000, the bound itself, 11.8 / 12.3.
//    Ranges in all 512 / 1024 / 2048 / 4096: 8 x 1 - 8 k of 32 heads 112 / 104 / 101 / 99; 16 x 8000 109 / 108 / 109 / 117; 64 x 0.5 -
//    2 k 76 / 73 / 72 / 72; two row tiles, 4 x 4 - 30 k: 76 / 82 / 93; one request of 30000, 32 rows, from 256 on: 49 / 60 / 65 / 75.
//    At least 256 keys, 512 with more than 8 rows of a K,V head, since a range leaves a partial result of each row (16 x 0.7 -
//    8 k, 20 rows: 256 keys 63.5, 512 60.3, 768 60.4; 32 x 150 - 2100, 4 rows: 25.3, 25.1, 28.1; one of 4000: 12.5, 14.3, 17.2).
//    More requests: equal ranges by max_len.
//  - an output row merged by a wave up to 16 parts, or 64 where there are 256 rows, else by a workgroup.  Wave / workgroup: 8
//    requests of 2 - 16 k, five tokens, 1280 rows of up to 32 parts 65.5 / 74.5; 4 of 4 - 30 k, 640 rows 72.9 / 77.8; 128 rows behind a
//    prefix of 25000, 33 parts 28.0 / 25.6; one of 131071, 32 rows of 32 106.9 / 105.0; by their number, 16 x 0.7 - 8 k of 16 56.6 / 69.4.
//  - ranges of the prefix: about 256 workgroups, at least 256 keys per row tile (128 rows, 3376 keys: 256 keys 17.3, 512
//    16.9, 1024 20.7; 8 rows of 32 heads, 1000 keys: 19, 21, 27).
//  - K by non-temporal loads (V always, where no row blocks share them) from 400 MB of K and V on, by the bound that the host
//    knows of the lengths: the last-level cache holds 256 MB, and what can be there from the call before is read from
//    there.  K cached / streamed: 8 x 1 - 8 k tokens of 32 heads (1074 MB at most, 554 in fact) 108 / 101; 8 x 4000 (524) 100
//    / 95; 16 x 8000 of 8 K,V heads (524) 116 / 113; 131 k (537) 115 / 112; 32 x 150 - 2100 (275, 86 in fact, three sets of
//    caches in turn) 28 / 31; a prefix of 8192 of 32 heads and 16 x 50 - 500 (265, 166 in fact) 34.5 / 36.5.
CacheAttentionPlan cache_attention_plan(int batch, int n_heads, int n_kv, int head_dim, int q_len, int max_len,
                                        int prefix_len, bool weights) {
  CacheAttentionPlan p{};
  const int group = n_heads / n_kv;
  const long long own_rows = (long long)q_len * group, prefix_rows = prefix_len > 0 ? own_rows * batch : 0;
  const long long missing = (prefix_rows + 255) / 256 * 256 - prefix_rows;
  p.shared_tiles = (double)(prefix_rows - missing) * prefix_len * n_kv >= 42e6;
  p.tiles = (p.shared_tiles || prefix_rows < own_rows ? own_rows : prefix_rows) <= 16 ? 1 : 2;
  const int rows = 16 * p.tiles, shared_rows = p.shared_tiles ? 256 : rows;
  p.own_blocks = (int)((own_rows + rows - 1) / rows);
  p.prefix_blocks = (int)((prefix_rows + shared_rows - 1) / shared_rows);
  auto cut = [](long long keys, long long items, long long groups, long long least, int& range, int& parts) {
    const long long want = groups > items ? groups / items : 1;
    long long r = (keys + want - 1) / want;
    if (r < least) r = least;
    r = range = round_range((int)r);
    parts = (int)((keys + r - 1) / r);
  };
  const long long least = own_rows > 8 ? 512 : 256, most_keys = (long long)max_len + q_len, per_range = (long long)n_kv * p.own_blocks;
  const long long split = std::min(256ll * batch, p.tiles == 1 ? 2048ll : 512ll) / per_range;
  if (batch <= SPLIT_BATCH && split > 1 && most_keys > least) {
    p.own_split = (int)split;
    p.own_range = (int)least;
    p.own_parts = (int)std::min((most_keys + least - 1) / least, split);
  } else {
    cut(most_keys, batch * per_range, 4096, least, p.own_range, p.own_parts);
  }
  if (prefix_len > 0) cut(prefix_len, (long long)n_kv * p.prefix_blocks, 256, p.shared_tiles ? 256 : 256 * p.tiles, p.prefix_range,
                          p.prefix_parts);
  const bool once = p.own_blocks == 1 && (p.shared_tiles || p.prefix_blocks <= 1);
  const double keys = (double)batch * (max_len + q_len) + (p.shared_tiles ? 0 : prefix_len);
  p.stream = !once ? 0 : keys * n_kv * head_dim * 4 >= 400e6 ? 2 : 1;
  const size_t all_rows = (size_t)batch * q_len * n_heads;
  const int parts = p.own_parts + p.prefix_parts;
  p.merge = parts == 1 ? 0 : parts <= 16 || (parts <= 64 && all_rows >= 256) ? 1 : 2;
  p.merge_waves = weights && q_len * n_heads >= 64 ? 16 : 4;
  p.z_ld = (max_len + q_len + STEP - 1) / STEP * STEP;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  p.part_bytes = p.merge ? up(all_rows * parts * head_dim * 4) : 0;
  p.stat_bytes = p.merge || weights ? up(all_rows * parts * 8) : 0;
  p.z_bytes = weights ? up(all_rows * p.z_ld * 4) : 0;
  p.count_bytes = p.own_split ? up(batch * 4) : 0;
  const size_t prefix_items = (size_t)p.prefix_parts * n_kv * p.prefix_blocks;
  const size_t own_items = (size_t)per_range * std::min((size_t)batch * p.own_parts, p.own_split ? (size_t)(p.own_split + batch) : SIZE_MAX);
  const size_t items = own_items + (p.shared_tiles ? 0 : prefix_items);
  const size_t merge_items = (p.merge == 0 ? 0 : p.merge == 1 ? (all_rows + p.merge_waves - 1) / p.merge_waves : all_rows) +
                             (weights ? (size_t)batch * ((max_len + q_len + 64 * SLOTS - 1) / (64 * SLOTS)) : 0);
  const size_t most = 0xffffffffull / 1024;          // threads of a launch are counted in 32 bits
  p.fits = prefix_items <= most && items <= most && merge_items <= most && all_rows <= 0x7fffffff;
  p.prefix_groups = p.shared_tiles ? (unsigned)prefix_items : 0;
  p.groups = (unsigned)items;
  p.merge_groups = (unsigned)merge_items;
  return p;
}

hipError_t launch_cache_attention(CacheAttentionArgs a, const CacheAttentionPlan& p, int head_dim, void* workspace, hipStream_t st) {
  a.group = a.n_heads / a.n_kv;
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)head_dim);
  a.own_blocks = p.own_blocks; a.own_range = p.own_range; a.own_split = p.own_split; a.own_parts = p.own_parts;
  a.prefix_blocks = p.prefix_blocks; a.prefix_range = p.prefix_range; a.prefix_parts = p.prefix_parts;
  a.shared_tiles = p.shared_tiles;
  a.merge = p.merge;
  a.z_ld = p.z_ld;
  char* ws = (char*)workspace;
  a.part = p.part_bytes ? (float*)ws : nullptr;
  a.stat = p.stat_bytes ? (float2*)(ws + p.part_bytes) : nullptr;
  a.z = p.z_bytes ? (float*)(ws + p.part_bytes + p.stat_bytes) : nullptr;
  a.counts = p.count_bytes ? (int32_t*)(ws + p.part_bytes + p.stat_bytes + p.z_bytes) : nullptr;
  if (p.shared_tiles) {
#define LZ_PATT(HD)                                                                                                \
  do {                                                                                                             \
    constexpr int LDS_BYTES = 3 * 2 * 64 * HD * 2;                                                                 \
    auto kern = prefix_attention_kernel<HD>;                                                                       \
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, LDS_BYTES);  \
    if (e != hipSuccess) return e;                                                                                 \
    hipLaunchKernelGGL(kern, dim3(p.prefix_groups), dim3(512), LDS_BYTES, st, a);                           \
    e = hipGetLastError();                                                                                         \
    if (e != hipSuccess) return e;                                                                                 \
  } while (0)
    if (head_dim == 128) LZ_PATT(128);
    else LZ_PATT(64);
#undef LZ_PATT
  }
#define LZ_CATT(HD, T, STREAM)                                                                                     \
  do {                                                                                                             \
    constexpr int K_BYTES = WAVES * STEP * HD * 2, MERGE_BYTES = WAVES * 16 * T * (HD + 4) * 4 + WAVES * 16 * T * 8; \
    constexpr int LDS_BYTES = K_BYTES > MERGE_BYTES ? K_BYTES : MERGE_BYTES;                                       \
    auto kern = cache_attention_kernel<HD, T, STREAM>;                                                             \
    if (LDS_BYTES > 65536) {                                                                                       \
      hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, LDS_BYTES); \
      if (e != hipSuccess) return e;                                                                               \
    }                                                                                                              \
    hipLaunchKernelGGL(kern, dim3(p.groups), dim3(64 * WAVES), LDS_BYTES, st, a);                                  \
  } while (0)
#define LZ_CATT_HD(HD)                                                                                             \
  do {                                                                                                             \
    if (p.tiles == 1 && p.stream == 2) LZ_CATT(HD, 1, 2);                                                          \
    else if (p.tiles == 1) LZ_CATT(HD, 1, 1);                                                                      \
    else if (p.stream == 2) LZ_CATT(HD, 2, 2);                                                                     \
    else if (p.stream == 1) LZ_CATT(HD, 2, 1);                                                                     \
    else LZ_CATT(HD, 2, 0);                                                                                        \
  } while (0)
  if (head_dim == 128) LZ_CATT_HD(128);
  else LZ_CATT_HD(64);
#undef LZ_CATT_HD
#undef LZ_CATT
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.merge_groups == 0) return e;
#define LZ_MERGE(HD, MW) hipLaunchKernelGGL((cache_merge_kernel<HD, MW>), dim3(p.merge_groups), dim3(64 * MW), 0, st, a)
  if (p.merge_waves == 16) {
    if (head_dim == 128) LZ_MERGE(128, 16);
    else LZ_MERGE(64, 16);
  } else {
    if (head_dim == 128) LZ_MERGE(128, 4);
    else LZ_MERGE(64, 4);
  }
#undef LZ_MERGE
  return hipGetLastError();
}

}  // namespace lz
