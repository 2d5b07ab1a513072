// Append-attention of few query rows over the 8-bit paged KV cache: decoding, and steps of a few tokens.
//
// With at most 32 rows per sequence and kv head the launch only streams the cache, and what bounds it is how many bytes the CUs
// keep in flight.  So nothing goes through LDS and no wave waits for another: a workgroup takes one chunk of the keys of one
// (sequence, kv head), its four waves take turns at 64-key tiles, each with an online softmax of its own, and meet once
// at the end.  A wave loads a tile straight into the registers of the matrix instructions (16x16x32: 16 query columns, where the
// 32x32 form would leave three quarters empty), and asks for the next tile's keys as soon as this one's are multiplied, for
// its values as soon as these are.
//
// A tile is four cache blocks.  Lane l = 16 g + c.  Scores S^T = K Q^T: score tile t (0..3) has row r = key 4 t + r % 4 of block
// r / 4, so that lane (g, c) receives rows 4 g .. 4 g + 3 of every score tile, i.e. all 16 keys of block g for query c.  The
// contraction index is free: lane (g, c) supplies elements 64 j + 16 g + 8 h + (0..7) in step 2 j + h, which are 16-byte
// pieces of a key's row, and the queries are loaded in the same order.
// O^T = V^T P^T: the lane's 16 probabilities are the two operands (keys 8 u + (0..7) of block g, u = 0, 1), so V^T wants the
// same eight keys of one column per lane.  Lane (g, c) loads HD/16 neighbouring columns of every key of block g, makes bf16 pairs of
// neighbouring columns of one key (v_cvt_scalef32_pk_bf16_fp8, which also applies the key's scale), and exchanges halves between
// two keys (v_perm): row c of tile mt is column c HD/16 + mt.
#include "attention_merge.h"
#include "common.h"

namespace {

constexpr int KT = ATTN_KT;
constexpr float kLazyLog2 = 8.0f;            // growth of a row maximum (log2 units) that forces a rescale

struct FewArgs {
  const bf16 *q;
  int q_row_stride;
  const uint8_t *k_pool, *v_pool, *k_scale, *v_scale;
  const int32_t *tables, *prefix_lens, *cu;
  int max_blocks, max_splits, kv_chunk, T, Hq, Hkv;
  float scale, cap_out;                      // scale: score -> logit in log2 units, or (CAP) -> the exponent of the tanh
  bf16 *out, *part_acc;
  float *part_ml;
};

// Two neighbouring elements of the four in `w`, times the scale of their row (its byte is the exponent): exact in bf16.
template <bool HIGH>
__device__ __forceinline__ uint32_t pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}
__device__ __forceinline__ float scale_of(uint32_t bytes, int i) { return __builtin_bit_cast(float, (bytes >> (8 * i) & 0xffu) << 23); }

template <int HD, int NQ, bool CAP>
__global__ __launch_bounds__(256, 2) void attention_few_kernel(FewArgs a) {
  constexpr int KK = HD / 32;                // contraction steps of the scores
  constexpr int KJ = HD / 64;                // 16-byte pieces of a key row per lane
  constexpr int MT = HD / 16;                // row tiles of O^T, and bytes of a value row per lane
  constexpr int VW = MT / 4;                 // ... in dwords
  constexpr int PITCH = HD + 4;
  __shared__ __attribute__((aligned(16))) float s_o[4][16 * NQ][PITCH];
  __shared__ float s_m[4][16 * NQ], s_l[4][16 * NQ];
  typedef uint32_t vword __attribute__((ext_vector_type(VW)));

  const int hk = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv, split = rest % a.max_splits, b = rest / a.max_splits;
  const int p = a.prefix_lens[b], tok0 = a.cu[b], s = a.cu[b + 1] - tok0, ctx = p + s;
  const int G = a.Hq / a.Hkv, rows = s * G;
  const int chunk = attn_seq_chunk(ctx, a.kv_chunk), begin = split * chunk, end = min(ctx, begin + chunk);
  if (begin >= ctx || rows > 16 * NQ) return;              // (more rows than the host's lengths said: not written)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;

  bf16x8 qf[NQ][KK];
  int limit[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = n * 16 + c, i = row < rows ? row / G : 0;
    limit[n] = p + i;
    const bf16 *src = a.q + (size_t)(tok0 + i) * a.q_row_stride + (hk * G + (row < rows ? row - i * G : 0)) * HD + g * 16;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      qf[n][kk] = *(const bf16x8 *)(src + (kk >> 1) * 64 + (kk & 1) * 8);
      if (row >= rows)
#pragma unroll
        for (int e = 0; e < 8; ++e) qf[n][kk][e] = (bf16)0.f;
    }
  }

  const int32_t *table = a.tables + (size_t)b * a.max_blocks;
  const int last_key = ctx - 1, last_blk = last_key / ARB_KV_BLOCK, last_row = last_key % ARB_KV_BLOCK;
  const int n_tiles = (end - begin + KT - 1) / KT;
  const int kb = c >> 2, krow = c & 3;                     // this lane's key block of a tile, and its row there for score tile 0
  u32x4 kd[4][KJ], ks, vs;
  vword vd[16];
  int k_id, v_id;                                          // pool blocks of the tile to be requested next
  auto ids = [&](int tile) {
    const int blk = (begin + tile * KT) / ARB_KV_BLOCK;
    k_id = table[min(blk + kb, last_blk)];
    v_id = table[min(blk + g, last_blk)];
  };
  // Blocks past the context's last one were looked up as that one; rows past its last key are read as that key.
  auto request_k = [&](int tile) {
    const size_t unit = (size_t)(unsigned)k_id * a.Hkv + hk;
    const uint8_t *src = a.k_pool + unit * (ARB_KV_BLOCK * HD) + g * 16;
    ks = *(const u32x4 *)(a.k_scale + unit * ARB_KV_BLOCK);
    if (begin + (tile + 1) * KT <= ctx) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < KJ; ++j) kd[t][j] = *(const u32x4 *)(src + krow * HD + t * 4 * HD + j * 64);
    } else {
      const int most = (begin + tile * KT) / ARB_KV_BLOCK + kb < last_blk ? 15 : last_row;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < KJ; ++j) kd[t][j] = *(const u32x4 *)(src + min(4 * t + krow, most) * HD + j * 64);
    }
  };
  auto request_v = [&](int tile) {
    const size_t unit = (size_t)(unsigned)v_id * a.Hkv + hk;
    const uint8_t *src = a.v_pool + unit * (ARB_KV_BLOCK * HD) + c * MT;
    vs = *(const u32x4 *)(a.v_scale + unit * ARB_KV_BLOCK);
    if (begin + (tile + 1) * KT <= ctx) {
#pragma unroll
      for (int k = 0; k < 16; ++k) vd[k] = *(const vword *)(src + k * HD);
    } else {
      const int most = (begin + tile * KT) / ARB_KV_BLOCK + g < last_blk ? 15 : last_row;
#pragma unroll
      for (int k = 0; k < 16; ++k) vd[k] = *(const vword *)(src + min(k, most) * HD);
    }
  };

  f32x4 o[NQ][MT];
  float m_run[NQ], l_run[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = -INFINITY;
    l_run[n] = 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[n][mt] = f32x4(0.f);
  }
  if (wave < n_tiles) {
    ids(wave);
    request_k(wave);
    request_v(wave);
    ids(min(wave + 4, n_tiles - 1));
  }
  for (int tile = wave; tile < n_tiles; tile += 4) {
    const int next = min(tile + 4, n_tiles - 1);           // past the end: the last tile again, unused
    const int key0 = begin + tile * KT;
    const bool whole = key0 + KT <= ctx;
    f32x4 st[4][NQ];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float sc = __builtin_bit_cast(float, (ks[t] >> (8 * krow) & 0xffu) << 23);
#pragma unroll
      for (int n = 0; n < NQ; ++n) st[t][n] = f32x4(0.f);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const uint32_t w0 = kd[t][kk >> 1][(kk & 1) * 2], w1 = kd[t][kk >> 1][(kk & 1) * 2 + 1];
        const u32x4 f = {pair<false>(w0, sc), pair<true>(w0, sc), pair<false>(w1, sc), pair<true>(w1, sc)};
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          st[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), qf[n][kk], st[t][n], 0, 0, 0);
      }
    }
    request_k(next);
    // Scale, cap, mask, and this lane's largest logit of each query (16 keys: those of block g).
    float mx[NQ];
    bool grows = false;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      mx[n] = -INFINITY;
      const int vis = limit[n] - key0 - 16 * g;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = st[t][n][e] * a.scale;
          if (CAP) x = fmaf(-2.f * a.cap_out, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x) + 1.f), a.cap_out);
          if (!whole || key0 + KT - 1 > p) x = 4 * t + e <= vis ? x : -INFINITY;
          st[t][n][e] = x;
          mx[n] = fmaxf(mx[n], x);
        }
      grows |= mx[n] > m_run[n] + kLazyLog2;               // m_run = -inf: any visible key
    }
    // The reference maximum moves only when a row has outgrown it by 2^8 (until then every weight is at most 2^8,
    // and the quotient is the same); the four lanes of a query share it, and so do its accumulators.
    if (__builtin_amdgcn_ballot_w64(grows) != 0) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        float m_new = fmaxf(mx[n], __shfl_xor(mx[n], 16, 64));
        m_new = fmaxf(m_run[n], fmaxf(m_new, __shfl_xor(m_new, 32, 64)));
        const float alpha = m_run[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[n] - m_new);
        l_run[n] *= alpha;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) o[n][mt] *= alpha;
        m_run[n] = m_new;
      }
    }
    // Probabilities in bf16, and their sum as the products will see them.
    u32x4 pf[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const float ref = m_run[n] == -INFINITY ? 0.f : m_run[n];
      const bf16x2 ones = {(bf16)1.0f, (bf16)1.0f};
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x2 pr = {(bf16)__builtin_amdgcn_exp2f(st[t][n][2 * h] - ref), (bf16)__builtin_amdgcn_exp2f(st[t][n][2 * h + 1] - ref)};
          l_run[n] = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, l_run[n], false);
          pf[n][t >> 1][(t & 1) * 2 + h] = __builtin_bit_cast(uint32_t, pr);
        }
    }
    if (!whole) {                                          // scale bytes of slots that were never written: their keys weigh nothing, but 0 * inf would
      const int valid = ctx - key0 - 16 * g;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const int n = min(max(valid - 4 * d, 0), 4);
        const uint32_t keep = n == 4 ? ~0u : (1u << (8 * n)) - 1;
        vs[d] = (vs[d] & keep) | (0x7f7f7f7fu & ~keep);
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32x4 vf[MT];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = 8 * u + 2 * i;
        const float s0 = scale_of(vs[k >> 2], k & 3), s1 = scale_of(vs[k >> 2], (k & 3) + 1);
#pragma unroll
        for (int w = 0; w < VW; ++w)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t lo = h ? pair<true>(vd[k][w], s0) : pair<false>(vd[k][w], s0);
            const uint32_t hi = h ? pair<true>(vd[k + 1][w], s1) : pair<false>(vd[k + 1][w], s1);
            vf[w * 4 + h * 2][i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
            vf[w * 4 + h * 2 + 1][i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
          }
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          o[n][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[mt]), __builtin_bit_cast(bf16x8, pf[n][u]), o[n][mt], 0, 0, 0);
    }
    request_v(next);
    ids(min(tile + 8, n_tiles - 1));
  }

  // The four waves' results under their common maximum.
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float l = l_run[n];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) {
      s_m[wave][n * 16 + c] = m_run[n];
      s_l[wave][n * 16 + c] = l;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int w = 0; w < VW; ++w) {
        const f32x4 four = {o[n][w * 4][e], o[n][w * 4 + 1][e], o[n][w * 4 + 2][e], o[n][w * 4 + 3][e]};
        *(f32x4 *)&s_o[wave][n * 16 + c][(4 * g + e) * MT + w * 4] = four;
      }
  }
  __syncthreads();
  for (int i = tid; i < rows * (HD / 8); i += 256) {
    const int row = i / (HD / 8), piece = i % (HD / 8), tok = row / G;
    const size_t idx = (size_t)(tok0 + tok) * a.Hq + hk * G + (row - tok * G);
    float m = -INFINITY, l = 0.f, acc[8];
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, s_m[w][row]);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      // a wave without visible keys has m = -inf, l = 0 and accumulators of 0
      const float f = s_m[w][row] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][row] - m);
      l += f * s_l[w][row];
      const f32x4 x0 = *(const f32x4 *)&s_o[w][row][piece * 8], x1 = *(const f32x4 *)&s_o[w][row][piece * 8 + 4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[e] += f * x0[e];
        acc[4 + e] += f * x1[e];
      }
    }
    const float inv = l != 0.f ? 1.0f / l : 0.f;           // NaN stays NaN; a row without visible keys in this split: 0
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (bf16)(acc[e] * inv);
    if (a.part_acc) {
      *(bf16x8 *)(a.part_acc + ((size_t)split * a.T * a.Hq + idx) * HD + piece * 8) = r;
      if (piece == 0) {
        float *ml = a.part_ml + ((size_t)split * a.T * a.Hq + idx) * 2;
        ml[0] = m;
        ml[1] = l;
      }
    } else {
      *(bf16x8 *)(a.out + idx * HD + piece * 8) = r;
    }
  }
}

// One workgroup per (sequence, kv head): its rows over all splits of the sequence.
template <int HD>
__global__ __launch_bounds__(256) void attention_few_merge_kernel(FewArgs a) {
  const int hk = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
  const int tok0 = a.cu[b], s = a.cu[b + 1] - tok0, ctx = a.prefix_lens[b] + s, G = a.Hq / a.Hkv;
  const int chunk = attn_seq_chunk(ctx, a.kv_chunk), n_splits = min((ctx + chunk - 1) / chunk, a.max_splits);
  for (int i = threadIdx.x; i < s * G * (HD / 8); i += 256) {
    const int row = i / (HD / 8), tok = row / G;
    merge_splits<HD>(a.part_acc, a.part_ml, (size_t)a.T * a.Hq, (size_t)(tok0 + tok) * a.Hq + hk * G + (row - tok * G),
                     i % (HD / 8), n_splits, a.out);
  }
}

}  // namespace

constexpr int kFewRows = 32;                 // most rows per sequence and kv head
static const int kPlaces = 512;              // workgroups that are resident at once: two per CU
static const int kMinFewChunk = 256, kMaxFewChunk = 2048, kMaxFewSplits = 64;

bool attention_few_takes(const AttnCache &cache, int max_rows) { return cache.k_scale && max_rows <= kFewRows; }

AttnPlan plan_attention_few(int batch, const int32_t *prefix_host, const int32_t *cu_host, int n_kv_heads) {
  long long keys = 0;
  int max_ctx = 0;
  for (int b = 0; b < batch; ++b) {
    const int ctx = prefix_host[b] + cu_host[b + 1] - cu_host[b];
    keys += (long long)ctx * n_kv_heads;
    max_ctx = ctx > max_ctx ? ctx : max_ctx;
  }
  long long chunk = (keys / kPlaces + KT - 1) / KT * KT;
  if (chunk > kMaxFewChunk) chunk = kMaxFewChunk;
  if (chunk < kMinFewChunk) chunk = kMinFewChunk;
  while (max_ctx > chunk * kMaxFewSplits) chunk += KT;
  return AttnPlan{(int)chunk, max_ctx > 0 ? ceil_div(max_ctx, (int)chunk) : 1, 1, 0};
}

arb_status launch_attention_few(const bf16 *q, int q_row_stride, const AttnCache &cache, const int32_t *block_tables,
                                int max_blocks_per_seq, int batch, int total_tokens, int max_rows, int n_q_heads, int n_kv_heads,
                                int head_dim, const AttnPlan &plan, bf16 *out, void *ws, size_t ws_bytes,
                                const int32_t *prefix_lens, const int32_t *cu_step_lens, hipStream_t st, bool q_prescaled) {
  if (batch == 0 || total_tokens == 0) return ARB_OK;
  const bool split = plan.max_splits > 1, capped = cache.softcap > 0.f;
  const size_t need = attention_ws_bytes(plan.max_splits, 0, total_tokens, n_q_heads, head_dim);
  if (split && (!ws || ws_bytes < need)) return arb_fail(ARB_ECAPACITY, "attention: workspace %zu < %zu bytes", ws_bytes, need);
  const float to_log2 = q_prescaled ? 1.0f : attention_q_scale(head_dim);
  FewArgs a{q, q_row_stride, (const uint8_t *)cache.k_pool, (const uint8_t *)cache.v_pool, cache.k_scale, cache.v_scale,
            block_tables, prefix_lens, cu_step_lens, max_blocks_per_seq, plan.max_splits, plan.kv_chunk, total_tokens, n_q_heads,
            n_kv_heads, capped ? 2.0f * to_log2 / cache.softcap : to_log2, capped ? 1.44269504f * cache.softcap : 0.f, out, nullptr, nullptr};
  if (split) {
    a.part_acc = (bf16 *)ws;
    a.part_ml = (float *)((char *)ws + attention_part_bytes(plan.max_splits, total_tokens, n_q_heads, head_dim));
  }
  const long long groups = (long long)batch * plan.max_splits * n_kv_heads;
  if (groups >= 1 << 24) return arb_fail(ARB_EUNSUPPORTED, "attention: %lld workgroups", groups);
  const dim3 grid((unsigned)groups), block(256);
#define ARB_FEW(HD, NQ)                                                                             \
  if (capped) hipLaunchKernelGGL((attention_few_kernel<HD, NQ, true>), grid, block, 0, st, a);      \
  else hipLaunchKernelGGL((attention_few_kernel<HD, NQ, false>), grid, block, 0, st, a)
  if (head_dim == 128) { if (max_rows <= 16) { ARB_FEW(128, 1); } else { ARB_FEW(128, 2); } }
  else                 { if (max_rows <= 16) { ARB_FEW(64, 1); } else { ARB_FEW(64, 2); } }
#undef ARB_FEW
  ARB_CHECK_LAUNCH("attention_few");
  if (split) {
    const dim3 mgrid(batch * n_kv_heads);
    if (head_dim == 128) hipLaunchKernelGGL((attention_few_merge_kernel<128>), mgrid, block, 0, st, a);
    else hipLaunchKernelGGL((attention_few_merge_kernel<64>), mgrid, block, 0, st, a);
    ARB_CHECK_LAUNCH("attention_few_merge");
  }
  return ARB_OK;
}
