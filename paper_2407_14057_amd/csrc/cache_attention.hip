// Attention of a batch's new tokens over per-request K,V caches, optionally behind a prefix that all requests share,
// with Eq. 1's head-averaged weight of every cached token kept up to date.
//
// Request b has n_b cached tokens and Q new ones; the new tokens' K,V are appended at slots n_b .. n_b+Q-1 by this
// launch.  Token t sees the prefix (P keys) and the slots up to n_b + t:
//   z = q . k / sqrt(hd),  p = exp(z) / sum exp(z),  o = sum p v,  weight[slot] += 1/H sum_{t,h} p[t][h][slot].
//
// One pass over K and V with a running maximum and sum.  A work item is a K,V head, a block of its query rows and a
// range of keys; the query rows of a K,V head are the (token, query head of the group) pairs of one request for a
// range of its own cache, and those of ALL requests for a range of the prefix, which is therefore read once.
// The partial results (output, maximum, sum) of the ranges are merged by a second launch.
#include "common.h"

namespace lz {

namespace {

constexpr int STEP = 32;              // keys of a wave's step
constexpr int WAVES = 4;

// (row of q, query head) of row r of an item: tok = tok0 + r / group, head = kvh * group + r % group
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

__device__ __forceinline__ uint32_t pack_halves(uint32_t hi, uint32_t lo, bool upper) {
  return __builtin_amdgcn_perm(hi, lo, upper ? 0x07060302u : 0x05040100u);
}

}  // namespace

// A wave takes 32 keys at a time straight from memory into MFMA operands (16x16x32, both products transposed so that a
// lane owns a query column: S^T = K Q^T, O^T = V^T P^T), the four waves of a workgroup take turns over the range.
//   K: lane (c = lane % 16, g = lane / 16) holds dimensions 32 s + 8 g .. + 7 of key c: the A operand as it lies.
//   V: lane (c, g) holds dimensions HD/16 c .. of the eight keys that its S^T accumulators belong to (4 g + r of each
//      block of 16), whole rows of 256 bytes per 16 lanes; pairs of keys are put together by v_perm.  Output tile i then
//      has dimension HD/16 c + i in row c, and no value of P changes its lane.
// P goes into the second product as two bf16 terms (value and remainder): one alone would add an error as large as the
// rounding of the output itself, and the matrix cores idle here anyway, the kernel is bound by reading K and V.
template <int HD, int T>
__global__ void __launch_bounds__(256, T >= 4 ? 1 : 2) cache_attention_kernel(CacheAttentionArgs a) {
  constexpr int KS = HD / 32;          // k-steps of the first product
  constexpr int NT = HD / 16;          // tiles of 16 output dimensions = dimensions a lane holds of a V row
  constexpr int VW = NT / 2;           // dwords of that
  constexpr int PITCH = HD + 4;
  extern __shared__ __attribute__((aligned(16))) float lds[];   // [WAVES][16 T][PITCH], then float2 [WAVES][16 T]
  float2* ml = (float2*)(lds + WAVES * 16 * T * PITCH);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int kvd = a.n_kv * HD;

  Item it;
  int b = 0;
  {
    int id = blockIdx.x;
    const int prefix_items = a.prefix_parts * a.n_kv * a.prefix_blocks;
    it.own = id >= prefix_items;
    if (!it.own) {
      it.part = id / (a.n_kv * a.prefix_blocks);
      id %= a.n_kv * a.prefix_blocks;
      it.kvh = id / a.prefix_blocks;
      it.row0 = id % a.prefix_blocks * 16 * T;
      it.n_rows = a.batch * a.q_len * a.group;
      it.tok0 = 0;
      it.stride = a.prefix_stride;
      it.k = a.prefix_k + it.kvh * HD;
      it.v = a.prefix_v + it.kvh * HD;
      it.n = a.prefix_len;
      it.n_tail = 1;
      it.k_tail = it.k + (a.prefix_len - 1) * it.stride;
      it.v_tail = it.v + (a.prefix_len - 1) * it.stride;
      it.tail_stride = 0;
      it.lo = it.part * a.prefix_range;
      it.hi = min(it.lo + a.prefix_range, a.prefix_len);
    } else {
      id -= prefix_items;
      const int part = id % a.own_parts;
      id /= a.own_parts;
      it.row0 = id % a.own_blocks * 16 * T;
      id /= a.own_blocks;
      it.kvh = id % a.n_kv;
      b = id / a.n_kv;
      it.part = a.prefix_parts + part;
      it.n_rows = a.q_len * a.group;
      it.tok0 = b * a.q_len;
      it.n = cached_tokens(a, b);
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
      if (part == 0 && it.kvh == 0 && it.row0 == 0 && threadIdx.x == 0 && a.status != nullptr && a.lengths[b] > a.max_len)
        atomicOr(a.status, ST_BAD_CU);
      it.stride = a.row_stride;
      it.k = a.k + b * a.batch_stride + it.kvh * HD;
      it.v = a.v + b * a.batch_stride + it.kvh * HD;
      it.n_tail = a.q_len;
      it.k_tail = a.k_new + ((size_t)it.tok0 * a.n_kv + it.kvh) * HD;
      it.v_tail = a.v_new + ((size_t)it.tok0 * a.n_kv + it.kvh) * HD;
      it.tail_stride = kvd;
      it.lo = part * a.own_range;
      it.hi = min(it.lo + a.own_range, it.n + a.q_len);
    }
  }
  if (it.lo >= it.hi) return;

  bf16x8_t qf[T][KS];
  int last[T];                          // the last key that a query row sees
  size_t out_row[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int r = min(it.row0 + 16 * t + c, it.n_rows - 1), tok = r / a.group;
    out_row[t] = (size_t)(it.tok0 + tok) * a.n_heads + it.kvh * a.group + r % a.group;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[t][s] = *(const bf16x8_t*)(a.q + out_row[t] * HD + 32 * s + 8 * g);
    last[t] = it.own ? it.n + tok : it.n - 1;
  }

  floatx4_t acc[T][NT];
  float m_run[T], l_run[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    m_run[t] = -INFINITY;
    l_run[t] = 0.f;
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[t][i] = {0.f, 0.f, 0.f, 0.f};
  }

  for (int k0 = it.lo + STEP * wave; k0 < it.hi; k0 += STEP * WAVES) {
    const bool tail = k0 + STEP > it.n;
    auto row = [&](const uint16_t* base, const uint16_t* behind, int key) {
      if (!tail || key < it.n) return base + key * it.stride;
      return behind + min(key - it.n, it.n_tail - 1) * it.tail_stride;
    };
    bf16x8_t kf[2][KS];
    uint32_t vf[8][VW];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      const uint16_t* kp = row(it.k, it.k_tail, k0 + 16 * sub + c) + 8 * g;
#pragma unroll
      for (int s = 0; s < KS; ++s) kf[sub][s] = *(const bf16x8_t*)(kp + 32 * s);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint16_t* vp = row(it.v, it.v_tail, k0 + 16 * (j >> 2) + 4 * g + (j & 3)) + NT * c;
      if (VW == 4) *(uint4*)vf[j] = *(const uint4*)vp;
      else *(uint2*)vf[j] = *(const uint2*)vp;
    }
    uint4 p_hi[T], p_lo[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      float z[8];                       // base-2 logits; z[4 sub + r] belongs to key k0 + 16 sub + 4 g + r
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        floatx4_t s4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[sub][s], qf[t][s], s4, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) z[4 * sub + r] = s4[r] * a.scale_log2e;
      }
      if (tail)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (k0 + 16 * (i >> 2) + 4 * g + (i & 3) > last[t]) z[i] = -INFINITY;
      if (a.z != nullptr && it.own && it.row0 + 16 * t + c < it.n_rows) {
        float* zp = a.z + out_row[t] * a.z_ld + k0 + 4 * g;
        *(float4*)zp = make_float4(z[0], z[1], z[2], z[3]);
        *(float4*)(zp + 16) = make_float4(z[4], z[5], z[6], z[7]);
      }
      float top = z[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, z[i]);
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
        p[i] = __builtin_amdgcn_exp2f(z[i] - m_use);
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
  }

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

// Merges the partial results and adds the weights.  The first workgroups take four output rows each, one a wave; the
// others 256 slots of a request each: every thread one slot, its rows added in order.
template <int HD>
__global__ void __launch_bounds__(256) cache_merge_kernel(CacheAttentionArgs a) {
  __shared__ float2 stats[256];
  const int all_rows = a.batch * a.q_len * a.n_heads;
  const int merge_groups = a.merge != 0 ? (all_rows + 3) / 4 : 0;
  const int lane = threadIdx.x & 63;
  if ((int)blockIdx.x < merge_groups) {
    const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= all_rows) return;
    const int n = cached_tokens(a, row / (a.q_len * a.n_heads));
    const int parts = n < 0 ? 0 : a.prefix_parts + (n + a.q_len + a.own_range - 1) / a.own_range;
    float m = -INFINITY, l = 0.f, x[2] = {0.f, 0.f};
    for (int s = 0; s < parts; ++s) m = fmaxf(m, a.stat[(size_t)s * all_rows + row].x);
    for (int s = 0; s < parts; ++s) {
      const float2 st = a.stat[(size_t)s * all_rows + row];
      const float w = st.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.x - m);
      l += w * st.y;
      const float* src = a.part + ((size_t)s * all_rows + row) * HD;
      if (HD == 128) {
        const float2 v = *(const float2*)(src + 2 * lane);
        x[0] += w * v.x;
        x[1] += w * v.y;
      } else {
        x[0] += w * src[lane];
      }
    }
    const float inv = parts == 0 ? 0.f : 1.0f / l;
    if (HD == 128) ((uint32_t*)(a.o + (size_t)row * HD))[lane] = pack_bf16(x[0] * inv, x[1] * inv);
    else a.o[(size_t)row * HD + lane] = to_bf16(x[0] * inv);
    return;
  }
  const int id = blockIdx.x - merge_groups;
  const int chunks = (a.max_len + a.q_len + 255) / 256;
  const int b = id / chunks, slot = id % chunks * 256 + threadIdx.x;
  const int n = cached_tokens(a, b);
  if (n < 0 || id % chunks * 256 >= n + a.q_len) return;
  const int rows = a.q_len * a.n_heads, row0 = b * rows;
  const int parts = a.prefix_parts + (n + a.q_len + a.own_range - 1) / a.own_range;
  float sum = 0.f;
  for (int base = 0; base < rows; base += 256) {
    const int count = min(256, rows - base);
    __syncthreads();
    if ((int)threadIdx.x < count) {
      const float2* st = a.stat + row0 + base + threadIdx.x;
      float m = -INFINITY, l = 0.f;
      for (int s = 0; s < parts; ++s) m = fmaxf(m, st[(size_t)s * all_rows].x);
      for (int s = 0; s < parts; ++s) {
        const float2 v = st[(size_t)s * all_rows];
        l += v.x == -INFINITY ? 0.f : v.y * __builtin_amdgcn_exp2f(v.x - m);
      }
      stats[threadIdx.x] = make_float2(m, 1.0f / l);
    }
    __syncthreads();
    if (slot < n + a.q_len) {
      const float* zp = a.z + (size_t)(row0 + base) * a.z_ld + slot;
      for (int r = 0; r < count; ++r) sum += __builtin_amdgcn_exp2f(zp[(size_t)r * a.z_ld] - stats[r].x) * stats[r].y;
    }
  }
  if (slot < n + a.q_len) {
    const size_t at = (size_t)b * a.capacity + slot;
    a.weight_out[at] = (slot < n ? a.weight[at] : 0.f) + sum / (float)a.n_heads;
  }
}

// How a call is cut: rows of an item, key ranges and the workspace.
CacheAttentionPlan cache_attention_plan(int batch, int n_heads, int n_kv, int head_dim, int q_len, int max_len,
                                        int prefix_len, bool weights) {
  CacheAttentionPlan p{};
  const int group = n_heads / n_kv;
  const long long own_rows = (long long)q_len * group, prefix_rows = prefix_len > 0 ? own_rows * batch : 0;
  const long long rows = prefix_rows > own_rows ? prefix_rows : own_rows;
  p.tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  p.own_blocks = (int)((own_rows + 16 * p.tiles - 1) / (16 * p.tiles));
  p.prefix_blocks = (int)((prefix_rows + 16 * p.tiles - 1) / (16 * p.tiles));
  auto cut = [](long long keys, long long items, int& range, int& parts) {
    long long want = 1024 / items;
    if (want < 1) want = 1;
    long long r = (keys + want - 1) / want;
    r = (r + 127) / 128 * 128;
    if (r < 256) r = 256;
    range = (int)r;
    parts = (int)((keys + r - 1) / r);
  };
  cut((long long)max_len + q_len, (long long)batch * n_kv * p.own_blocks, p.own_range, p.own_parts);
  if (prefix_len > 0) cut(prefix_len, (long long)n_kv * p.prefix_blocks, p.prefix_range, p.prefix_parts);
  const size_t all_rows = (size_t)batch * q_len * n_heads;
  const int parts = p.own_parts + p.prefix_parts;
  p.merge = parts > 1;
  p.z_ld = (max_len + q_len + STEP - 1) / STEP * STEP;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  p.part_bytes = p.merge ? up(all_rows * parts * head_dim * 4) : 0;
  p.stat_bytes = p.merge || weights ? up(all_rows * parts * 8) : 0;
  p.z_bytes = weights ? up(all_rows * p.z_ld * 4) : 0;
  return p;
}

hipError_t launch_cache_attention(CacheAttentionArgs a, const CacheAttentionPlan& p, int head_dim, void* workspace, hipStream_t st) {
  a.group = a.n_heads / a.n_kv;
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)head_dim);
  a.own_blocks = p.own_blocks; a.own_range = p.own_range; a.own_parts = p.own_parts;
  a.prefix_blocks = p.prefix_blocks; a.prefix_range = p.prefix_range; a.prefix_parts = p.prefix_parts;
  a.merge = p.merge;
  a.z_ld = p.z_ld;
  char* ws = (char*)workspace;
  a.part = p.part_bytes ? (float*)ws : nullptr;
  a.stat = p.stat_bytes ? (float2*)(ws + p.part_bytes) : nullptr;
  a.z = p.z_bytes ? (float*)(ws + p.part_bytes + p.stat_bytes) : nullptr;
  const long long items = (long long)p.prefix_parts * a.n_kv * p.prefix_blocks + (long long)a.batch * a.n_kv * p.own_blocks * p.own_parts;
  if (items > 0x7fffffff) return hipErrorInvalidValue;
#define LZ_CATT(HD, T)                                                                                             \
  do {                                                                                                             \
    constexpr int LDS_BYTES = WAVES * 16 * T * (HD + 4) * 4 + WAVES * 16 * T * 8;                                  \
    auto kern = cache_attention_kernel<HD, T>;                                                                     \
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, LDS_BYTES);  \
    if (e != hipSuccess) return e;                                                                                 \
    hipLaunchKernelGGL(kern, dim3((unsigned)items), dim3(64 * WAVES), LDS_BYTES, st, a);                           \
  } while (0)
  if (head_dim == 128) {
    if (p.tiles == 1) LZ_CATT(128, 1);
    else if (p.tiles == 2) LZ_CATT(128, 2);
    else LZ_CATT(128, 4);
  } else {
    if (p.tiles == 1) LZ_CATT(64, 1);
    else if (p.tiles == 2) LZ_CATT(64, 2);
    else LZ_CATT(64, 4);
  }
#undef LZ_CATT
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (a.merge == 0 && a.z == nullptr)) return e;
  const long long all_rows = (long long)a.batch * a.q_len * a.n_heads;
  const long long groups = (a.merge != 0 ? (all_rows + 3) / 4 : 0) +
                           (a.z != nullptr ? (long long)a.batch * ((a.max_len + a.q_len + 255) / 256) : 0);
  if (all_rows > 0x7fffffff || groups > 0x7fffffff) return hipErrorInvalidValue;
  if (head_dim == 128) hipLaunchKernelGGL(cache_merge_kernel<128>, dim3((unsigned)groups), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(cache_merge_kernel<64>, dim3((unsigned)groups), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace lz
