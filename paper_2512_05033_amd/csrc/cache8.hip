// The 8-bit paged KV cache: what writes it (head norms + rotary embedding + append in one launch) and what converts it
// from and to the bf16 cache.
//
// Format.  A row (one position's key or value of one kv head, hd elements) is hd e4m3 elements and one power-of-two scale:
// e = the least integer with max|x| <= 448 * 2^e, not below -100; element = e4m3(x * 2^-e) to nearest even, scale byte =
// e + 127.  A power of two costs no precision that a finer scale would keep (e4m3 has an exponent of its own: only elements
// below 2^-6 * 2^e, 1/28672 of the row's largest or less, lose bits), its product with an element is exact in bf16, and
// the conversion instruction applies it for nothing.
// A position whose key or value row holds a NaN, an infinity or a magnitude of 2^120 or more has no such form: its key
// is stored as NaN throughout and its value as zeros.  Whoever attends to it gets NaN; whoever does not see it (a row
// before it in the step) is not touched by it, as the product of a zero probability with a NaN value would be.
#include "common.h"

#include <math.h>

namespace {

constexpr uint32_t kTooLarge = 0x7B800000u;      // the bits of 2^120
constexpr int kMinScaleByte = 27;                // e = -100

// Scale byte of a row whose largest magnitude has these bits (below kTooLarge).  448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_byte(uint32_t max_bits) {
  return max((int)(max_bits >> 23) - 8 + ((max_bits & 0x7fffffu) > 0x600000u ? 1 : 0), kMinScaleByte);
}

__device__ __forceinline__ uint32_t e4m3_four(const float *x, float inv_scale) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv_scale, x[1] * inv_scale, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv_scale, x[3] * inv_scale, w, true);
}

__device__ __forceinline__ uint32_t abs_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// Over the LANES neighbouring lanes that share a row: the largest, or the sum.
template <int LANES>
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}
template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int o = 1; o < LANES; o *= 2) v += __shfl_xor(v, o, 64);
  return v;
}

// A key row and a value row (N elements each per lane, the row over LANES lanes) in the 8-bit format.
template <int LANES, int N>
__device__ __forceinline__ void quantize_rows(const float (&k)[N], const float (&v)[N], uint32_t (&k8)[N / 4], uint32_t (&v8)[N / 4],
                                              int &k_byte, int &v_byte) {
  uint32_t km = 0, vm = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    km = max(km, abs_bits(k[e]));                          // as integers: a NaN is larger than an infinity
    vm = max(vm, abs_bits(v[e]));
  }
  km = row_max<LANES>(km);
  vm = row_max<LANES>(vm);
  if (max(km, vm) >= kTooLarge) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) { k8[i] = 0x7f7f7f7fu; v8[i] = 0; }
    k_byte = v_byte = 127;
    return;
  }
  k_byte = scale_byte(km);
  v_byte = scale_byte(vm);
  const float ki = __builtin_bit_cast(float, (254 - k_byte) << 23), vi = __builtin_bit_cast(float, (254 - v_byte) << 23);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) { k8[i] = e4m3_four(k + 4 * i, ki); v8[i] = e4m3_four(v + 4 * i, vi); }
}

// ------------------------------------------------------- head norms + rotary embedding + append

// Sequence of step token j: the largest b with cu[b] <= j, by one round of loads per factor of 64 in the batch (a binary search is
// a chain of six dependent loads for 64 sequences, and this launch is little more than such chains when tokens are few).
__device__ __forceinline__ int sequence_of(const int32_t *__restrict__ cu, int batch, int j, int lane) {
  int lo = 0, hi = batch;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    const bool in = at < hi && cu[at] <= j;
    const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(in));
    lo += max(n - 1, 0) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

struct AppendArgs {
  bf16 *qkv;                     // PARTS: where q goes, row_heads = Hq; otherwise the projection's rows
  bf16 *q_out;                   // not PARTS: where q goes (rows of q_row elements; qkv itself for in place)
  int q_row;
  const float *parts;            // PARTS: fp32 partial products [*, T, (Hq + 2 Hkv) hd], added in a fixed order
  RowParts row_parts;
  size_t part_stride;
  const float *g_q, *g_k;        // null: no norm
  float eps, q_scale;
  const f32x2 *cs;               // TABLE: rotary table and pool slots of the tokens; otherwise found here
  const int32_t *tok_slot;
  const int32_t *prefix_lens, *cu, *tables;
  int batch, max_blocks;
  double log2_base;
  void *k_pool, *v_pool;
  uint8_t *k_scale, *v_scale;    // null: bf16 pools
  int T, Hq, Hkv, tokens;        // tokens: of a workgroup
};

// A unit is one query head, or one kv head's key and value, of one token: HD/2/PAIRS lanes, each with the pairs (t..t+PAIRS-1,
// t+HD/2..).  The sum of squares and the largest magnitude are shuffles among them, and everything of a row happens
// between one load and one store.  Bound: the projection's rows in, queries and cache rows out; with few tokens one chain of
// memory round trips.  Without a table (a call of its own) a workgroup first finds its tokens' slots and angles, a wave a
// token, while its first unit's loads are in flight.
template <int HD, int PAIRS, bool PARTS, bool TABLE, bool KV8>
__global__ __launch_bounds__(256) void norm_rope_append_kernel(AppendArgs a) {
  constexpr int HALF = HD / 2, LANES = HALF / PAIRS, UNITS = 256 / LANES, N = 2 * PAIRS;
  typedef bf16 vec_b __attribute__((ext_vector_type(PAIRS)));
  typedef uint32_t vec_w __attribute__((ext_vector_type(PAIRS / 4)));
  __shared__ __attribute__((aligned(16))) f32x2 s_cs[TABLE ? 1 : 4 * HALF];
  __shared__ int s_slot[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tok0 = blockIdx.x * a.tokens, n_tok = min(a.tokens, a.T - tok0);
  const int per_tok = a.Hq + a.Hkv, n_units = n_tok * per_tok, stride = gridDim.y * UNITS;
  const int t = (tid % LANES) * PAIRS;
  const int heads = a.Hq + 2 * a.Hkv;
  float x[N], v[N];
  auto load_head = [&](int j, int head, float (&to)[N]) {
    if (PARTS) {
      const float *p0 = a.parts + ((size_t)j * heads + head) * HD + t;
      const int n_parts = j < a.row_parts.row ? a.row_parts.head : a.row_parts.tail;
      constexpr int Q = PAIRS / 4, AHEAD = 16 / PAIRS;     // 16-byte pieces; partial products asked for together
#pragma unroll
      for (int e = 0; e < N; ++e) to[e] = 0.f;
      for (int p = 0; p < n_parts; p += AHEAD) {
        f32x4 pa[AHEAD][Q], pb[AHEAD][Q];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          if (p + i < n_parts)
#pragma unroll
            for (int w = 0; w < Q; ++w) {
              pa[i][w] = *(const f32x4 *)(p0 + (p + i) * a.part_stride + 4 * w);
              pb[i][w] = *(const f32x4 *)(p0 + (p + i) * a.part_stride + HALF + 4 * w);
            }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          if (p + i < n_parts)
#pragma unroll
            for (int e = 0; e < PAIRS; ++e) {
              to[e] += pa[i][e / 4][e % 4];
              to[PAIRS + e] += pb[i][e / 4][e % 4];
            }
      }
    } else {
      const bf16 *src = a.qkv + ((size_t)j * heads + head) * HD + t;
      const vec_b lo = *(const vec_b *)src, hi = *(const vec_b *)(src + HALF);
#pragma unroll
      for (int e = 0; e < PAIRS; ++e) { to[e] = (float)lo[e]; to[PAIRS + e] = (float)hi[e]; }
    }
  };
  auto load = [&](int u) {
    const int i = u / per_tok, h = u - i * per_tok;
    load_head(tok0 + i, h, x);                             // query heads, then key heads: unit h is head h
    if (h >= a.Hq) load_head(tok0 + i, h + a.Hkv, v);
  };
  auto store_b = [&](bf16 *dst, const float (&from)[N], float f) {
    vec_b lo, hi;
#pragma unroll
    for (int e = 0; e < PAIRS; ++e) { lo[e] = (bf16)(from[e] * f); hi[e] = (bf16)(from[PAIRS + e] * f); }
    *(vec_b *)dst = lo;
    *(vec_b *)(dst + HALF) = hi;
  };
  auto store_w = [&](uint8_t *dst, const uint32_t (&from)[N / 4]) {
    vec_w lo, hi;
#pragma unroll
    for (int w = 0; w < PAIRS / 4; ++w) { lo[w] = from[w]; hi[w] = from[PAIRS / 4 + w]; }
    *(vec_w *)dst = lo;
    *(vec_w *)(dst + HALF) = hi;
  };
  int u = blockIdx.y * UNITS + tid / LANES;
  if (u < n_units) load(u);
  if (!TABLE) {
    if (wave < n_tok) {
      const int j = tok0 + wave, b = sequence_of(a.cu, a.batch, j, lane), pos = a.prefix_lens[b] + (j - a.cu[b]);
      if (lane == 0) s_slot[wave] = a.tables[(size_t)b * a.max_blocks + pos / ARB_KV_BLOCK] * ARB_KV_BLOCK + pos % ARB_KV_BLOCK;
      if (lane < HALF) {                                   // 64 bits: positions reach tens of thousands
        double sn, cn;
        sincos((double)pos * exp2(-(double)lane / (double)HALF * a.log2_base), &sn, &cn);
        s_cs[wave * HALF + lane] = f32x2{(float)cn, (float)sn};
      }
    }
    __syncthreads();
  }
  while (u < n_units) {
    const int i = u / per_tok, h = u - i * per_tok, j = tok0 + i;
    const bool is_q = h < a.Hq;
    const float *g = is_q ? a.g_q : a.g_k;
    if (g) {
      float f = 1.0f;
      auto mean_square = [&] {                             // of f x
        float sum[PAIRS / 4];                              // of every four pairs by itself, neighbours joined first: the same order for both widths
#pragma unroll
        for (int w = 0; w < PAIRS / 4; ++w) {
          sum[w] = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[w] += (f * x[4 * w + e]) * (f * x[4 * w + e]);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[w] += (f * x[PAIRS + 4 * w + e]) * (f * x[PAIRS + 4 * w + e]);
        }
        return row_sum<LANES>(PAIRS == 8 ? sum[0] + sum[PAIRS / 4 - 1] : sum[0]) * (1.0f / HD);
      };
      float mean = mean_square();
      if (mean == INFINITY) {                              // squares beyond fp32: those of 2^-64 x, and eps is nothing beside them
        f = 0x1p-64f;
        mean = mean_square();
      }
      const float r = f / sqrtf(mean + a.eps);
#pragma unroll
      for (int w = 0; w < PAIRS / 4; ++w) {
        const f32x4 g0 = *(const f32x4 *)(g + t + 4 * w), g1 = *(const f32x4 *)(g + t + HALF + 4 * w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[4 * w + e] *= r * g0[e];
          x[PAIRS + 4 * w + e] *= r * g1[e];
        }
      }
    }
    const f32x2 *cs = TABLE ? a.cs + (size_t)j * HALF + t : s_cs + i * HALF + t;
#pragma unroll
    for (int w = 0; w < PAIRS / 2; ++w) {
      const f32x4 two = *(const f32x4 *)(cs + 2 * w);      // (cos, sin) of two pairs
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float c = two[2 * e], s = two[2 * e + 1], p = x[2 * w + e], q = x[PAIRS + 2 * w + e];
        x[2 * w + e] = p * c - q * s;
        x[PAIRS + 2 * w + e] = q * c + p * s;
      }
    }
    if (is_q) {
      store_b(PARTS ? a.qkv + ((size_t)j * a.Hq + h) * HD + t : a.q_out + (size_t)j * a.q_row + h * HD + t, x, a.q_scale);
    } else {
      const int slot = TABLE ? a.tok_slot[j] : s_slot[i];
      const size_t row = ((size_t)(slot / ARB_KV_BLOCK) * a.Hkv + (h - a.Hq)) * ARB_KV_BLOCK + slot % ARB_KV_BLOCK;
      if (KV8) {
        uint32_t k8[N / 4], v8[N / 4];
        int kb, vb;
        quantize_rows<LANES>(x, v, k8, v8, kb, vb);
        store_w((uint8_t *)a.k_pool + row * HD + t, k8);
        store_w((uint8_t *)a.v_pool + row * HD + t, v8);
        if (t == 0) {
          a.k_scale[row] = (uint8_t)kb;
          a.v_scale[row] = (uint8_t)vb;
        }
      } else {
        store_b((bf16 *)a.k_pool + row * HD + t, x, 1.0f);
        store_b((bf16 *)a.v_pool + row * HD + t, v, 1.0f);
      }
    }
    u += stride;
    if (u < n_units) load(u);
  }
}

// ------------------------------------------------------------------------ conversion of blocks

// Eight elements of a key row and of the value row of the same position per thread; a block of one kv head is 16 rows.
// Bound: memory, 4 HD bytes in and 2 HD + 2 out per position and kv head, or the other way round.  8192 blocks of 8 heads of 128
// packed in 134 us (6.0 TB/s), 9000 unpacked in 177 (5.0; two thirds of it is written, a large copy moves 4.8); with stores that
// are kept in the caches 138 and 180.
template <int HD>
__global__ __launch_bounds__(256) void pack_kernel(const bf16 *__restrict__ k, const bf16 *__restrict__ v,
                                                   const int32_t *__restrict__ src_blocks, uint8_t *__restrict__ k8,
                                                   uint8_t *__restrict__ v8, uint8_t *__restrict__ k_scale,
                                                   uint8_t *__restrict__ v_scale, const int32_t *__restrict__ dst_blocks,
                                                   int Hkv, long long rows) {
  constexpr int LANES = HD / 8;
  const long long r = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (r >= rows) return;                                   // whole rows: the lanes of a row stay together
  const int t = threadIdx.x % LANES * 8, per = Hkv * ARB_KV_BLOCK, n = (int)(r / per), in = (int)(r - (long long)n * per);
  const size_t from = ((size_t)(src_blocks ? src_blocks[n] : n) * per + in), to = ((size_t)(dst_blocks ? dst_blocks[n] : n) * per + in);
  const bf16x8 kx = *(const bf16x8 *)(k + from * HD + t), vx = *(const bf16x8 *)(v + from * HD + t);
  float kf[8], vf[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { kf[e] = (float)kx[e]; vf[e] = (float)vx[e]; }
  uint32_t kw[2], vw[2];
  int kb, vb;
  quantize_rows<LANES>(kf, vf, kw, vw, kb, vb);
  __builtin_nontemporal_store(u32x2{kw[0], kw[1]}, (u32x2 *)(k8 + to * HD + t));
  __builtin_nontemporal_store(u32x2{vw[0], vw[1]}, (u32x2 *)(v8 + to * HD + t));
  if (t == 0) {
    k_scale[to] = (uint8_t)kb;
    v_scale[to] = (uint8_t)vb;
  }
}

__device__ __forceinline__ bf16x8 eight_values(u32x2 w, uint32_t byte) {
  const float scale = __builtin_bit_cast(float, byte << 23);
  union { bf16x2 p[4]; bf16x8 v; } r;
  r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, false);
  r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, true);
  r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, false);
  r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, true);
  return r.v;
}

template <int HD>
__global__ __launch_bounds__(256) void unpack_kernel(const uint8_t *__restrict__ k8, const uint8_t *__restrict__ v8,
                                                     const uint8_t *__restrict__ k_scale, const uint8_t *__restrict__ v_scale,
                                                     const int32_t *__restrict__ src_blocks, bf16 *__restrict__ k,
                                                     bf16 *__restrict__ v, const int32_t *__restrict__ dst_blocks, int Hkv,
                                                     long long rows) {
  constexpr int LANES = HD / 8;
  const long long r = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (r >= rows) return;
  const int t = threadIdx.x % LANES * 8, per = Hkv * ARB_KV_BLOCK, n = (int)(r / per), in = (int)(r - (long long)n * per);
  const size_t from = ((size_t)(src_blocks ? src_blocks[n] : n) * per + in), to = ((size_t)(dst_blocks ? dst_blocks[n] : n) * per + in);
  const u32x2 kw = *(const u32x2 *)(k8 + from * HD + t), vw = *(const u32x2 *)(v8 + from * HD + t);
  const uint32_t kb = k_scale[from], vb = v_scale[from];
  __builtin_nontemporal_store(eight_values(kw, kb), (bf16x8 *)(k + to * HD + t));
  __builtin_nontemporal_store(eight_values(vw, vb), (bf16x8 *)(v + to * HD + t));
}

}  // namespace

// Few tokens: a workgroup per 256 lanes of units and four pairs a lane, so that a token is one round of loads.  Many: eight pairs a
// lane (16-byte accesses of bf16 rows) and, in a call of its own, two tokens per workgroup, whose angles two waves find at once.
// (32/8 heads into the 8-bit cache, few / many: 600 tokens 6.2 / 7.3 us, 900 9.1 / 8.4, 3001 17.7 / 14.6 (4.6 TB/s, nearly that of
// a large copy), 12000 61.8 / 56.2.  Of the 14.6 the angles are 0.5; with one token per workgroup 17.1, with four 14.6.)
constexpr int kAppendManyTokens = 768;

template <bool PARTS, bool TABLE>
static void launch_append(const AppendArgs &a, int head_dim, int pairs, dim3 grid, hipStream_t st) {
  grid.y = a.tokens > 1 ? 1 : ceil_div((a.Hq + a.Hkv) * (head_dim / 2 / pairs), 256);
#define ARB_APPEND(HD, PAIRS)                                                                                                  \
  if (a.k_scale) hipLaunchKernelGGL((norm_rope_append_kernel<HD, PAIRS, PARTS, TABLE, true>), grid, dim3(256), 0, st, a);      \
  else hipLaunchKernelGGL((norm_rope_append_kernel<HD, PAIRS, PARTS, TABLE, false>), grid, dim3(256), 0, st, a)
  if (head_dim == 128) { if (pairs == 8) { ARB_APPEND(128, 8); } else { ARB_APPEND(128, 4); } }
  else                 { if (pairs == 8) { ARB_APPEND(64, 8); } else { ARB_APPEND(64, 4); } }
#undef ARB_APPEND
}

arb_status launch_norm_rope_append(bf16 *qkv, const float *parts, RowParts n_parts, const f32x2 *cs, const int32_t *tok_slot,
                                   const arb_kv_layer &kv, const float *g_q, const float *g_k, float eps, int T, int n_q_heads,
                                   int n_kv_heads, int head_dim, float q_scale, hipStream_t st) {
  if (T == 0) return ARB_OK;
  AppendArgs a{};
  a.qkv = qkv;
  a.parts = parts;
  a.row_parts = n_parts;
  a.part_stride = (size_t)T * (n_q_heads + 2 * n_kv_heads) * head_dim;
  a.g_q = g_q, a.g_k = g_k, a.eps = eps, a.q_scale = q_scale;
  a.cs = cs, a.tok_slot = tok_slot;
  a.k_pool = kv.k_pool, a.v_pool = kv.v_pool, a.k_scale = kv.k_scale, a.v_scale = kv.v_scale;
  a.T = T, a.Hq = n_q_heads, a.Hkv = n_kv_heads, a.tokens = 1;
  launch_append<true, true>(a, head_dim, T >= kAppendManyTokens ? 8 : 4, dim3(T), st);
  ARB_CHECK_LAUNCH("norm_rope_append");
  return ARB_OK;
}

arb_status launch_norm_rope_append_rows(bf16 *qkv, bf16 *q_out, const arb_kv_layer &kv, const float *g_q, const float *g_k,
                                        float eps, float rope_base, const arb_batch &bt, int n_q_heads, int n_kv_heads,
                                        int head_dim, float q_scale, hipStream_t st) {
  const int T = bt.total_tokens;
  if (T == 0) return ARB_OK;
  AppendArgs a{};
  a.qkv = qkv;
  a.q_out = q_out ? q_out : qkv;
  a.q_row = (q_out ? n_q_heads : n_q_heads + 2 * n_kv_heads) * head_dim;
  a.g_q = g_q, a.g_k = g_k, a.eps = eps, a.q_scale = q_scale;
  a.prefix_lens = bt.prefix_lens, a.cu = bt.cu_step_lens, a.tables = bt.block_tables;
  a.batch = bt.batch, a.max_blocks = bt.max_blocks_per_seq;
  a.log2_base = log2((double)rope_base);
  a.k_pool = kv.k_pool, a.v_pool = kv.v_pool, a.k_scale = kv.k_scale, a.v_scale = kv.v_scale;
  a.T = T, a.Hq = n_q_heads, a.Hkv = n_kv_heads;
  const bool many = T >= kAppendManyTokens;
  a.tokens = many ? 2 : 1;
  launch_append<false, false>(a, head_dim, many ? 8 : 4, dim3(ceil_div(T, a.tokens)), st);
  ARB_CHECK_LAUNCH("norm_rope_append");
  return ARB_OK;
}

arb_status launch_kv8_convert(bool pack, const arb_kv_layer &src, const int32_t *src_blocks, const arb_kv_layer &dst,
                              const int32_t *dst_blocks, int n, int n_kv_heads, int head_dim, hipStream_t st) {
  if (n == 0) return ARB_OK;
  const long long rows = (long long)n * n_kv_heads * ARB_KV_BLOCK, groups = (rows * head_dim / 8 + 255) / 256;   // a launch has fewer than 2^32 threads
  if (groups >= 1 << 24) return arb_fail(ARB_EUNSUPPORTED, "kv8 conversion of %d blocks of %d heads in one call", n, n_kv_heads);
  const dim3 grid((unsigned)groups);
#define ARB_PACK(HD)                                                                                                           \
  if (pack) hipLaunchKernelGGL((pack_kernel<HD>), grid, dim3(256), 0, st, (const bf16 *)src.k_pool, (const bf16 *)src.v_pool,  \
                               src_blocks, (uint8_t *)dst.k_pool, (uint8_t *)dst.v_pool, dst.k_scale, dst.v_scale, dst_blocks, \
                               n_kv_heads, rows);                                                                              \
  else hipLaunchKernelGGL((unpack_kernel<HD>), grid, dim3(256), 0, st, (const uint8_t *)src.k_pool, (const uint8_t *)src.v_pool, \
                          src.k_scale, src.v_scale, src_blocks, (bf16 *)dst.k_pool, (bf16 *)dst.v_pool, dst_blocks, n_kv_heads, rows)
  if (head_dim == 128) { ARB_PACK(128); } else { ARB_PACK(64); }
#undef ARB_PACK
  ARB_CHECK_LAUNCH("kv8_convert");
  return ARB_OK;
}
