// Append-attention of few query rows over the 8-bit paged KV cache, and over the bf16 one where scores are capped: decoding, and
// steps of a few tokens.
//
// With at most 32 rows per sequence and kv head the launch only streams the cache, and what bounds it is how many bytes the CUs
// keep in flight.  So nothing goes through LDS and no wave waits for another: the four waves of a workgroup take turns at
// 64-key tiles of one (sequence, kv head), each with an online softmax of its own, and meet once at the end.  A wave loads a tile
// straight into the registers of the matrix instructions (16x16x32: 16 query columns, where the 32x32 form would leave three
// quarters empty), and asks for the next tile's keys as soon as this one's are multiplied, for its values as soon as these are.
//
// Split.  As many workgroups as are resident at once, in one of two ways.  Even: every pair in parts of `per` tiles, a
// workgroup each.  In a row: the tiles of all pairs stand in one row, sequence by sequence, and every workgroup takes `per` of
// them; where they pass from one pair to the next it writes out the first one's result and goes on, with the next tile
// in flight already.  So all end together whatever the lengths are, at the price of a result more per workgroup.  A pair that was
// cut is merged by a second launch.
//
// Measured: 32 tokens of 32/8 heads of 128 against 4 K to 32 K keys 198 us (5.6 TB/s of cache) and 4.8 for the merge, 64 against 32 K
// 719 (6.0); one token of 12/2 heads against 1531 keys 6.1 and 2.7.  The bf16 cache's kernel, whose workgroup streams through
// LDS and lets one wave work, took 318 us for the first of these in its form for the 8-bit cache.
//
// A tile is four cache blocks.  Lane l = 16 g + c.  Scores S^T = K Q^T: score tile t (0..3) has row r = key 4 t + r % 4 of block
// r / 4, so that lane (g, c) receives rows 4 g .. 4 g + 3 of every score tile, i.e. all 16 keys of block g for query c.  The
// contraction index is free: lane (g, c) supplies elements 64 j + 16 g + 8 h + (0..7) in step 2 j + h, which are 16-byte
// pieces of a key's row, and the queries are loaded in the same order.
// O^T = V^T P^T: the lane's 16 probabilities are the two operands (keys 8 u + (0..7) of block g, u = 0, 1), so V^T wants the
// same eight keys of one column per lane.  Lane (g, c) loads HD/16 neighbouring columns of every key of block g, makes bf16 pairs of
// neighbouring columns of one key (v_cvt_scalef32_pk_bf16_fp8, which also applies the key's scale), and exchanges halves between
// two keys (v_perm): row c of tile mt is column c HD/16 + mt.  A bf16 cache needs no conversion: the lane's elements of step j are
// 32 j + 8 g + (0..7), and its pairs are there as they are loaded.
#include "attention_merge.h"
#include "common.h"

namespace {

constexpr int KT = ATTN_KT;
constexpr float kLazyLog2 = 8.0f;            // growth of a row maximum (log2 units) that forces a rescale

struct FewArgs {
  const bf16 *q;
  int q_row_stride;
  const uint8_t *k_pool, *v_pool, *k_scale, *v_scale;      // bf16: pools by bytes, no scales
  const int32_t *tables, *prefix_lens, *cu;
  int batch, max_blocks, max_splits, per, in_a_row, T, Hq, Hkv;
  float scale, cap_out;                      // scale: score -> logit in log2 units, or (CAP) -> the exponent of the tanh
  bf16 *out;
  float *part_acc, *part_ml;                 // fp32 throughout: few rows make little of it, and a rounding to bf16 would be as large as the result's own
};

// Word i of an array that no kernel of the launch writes, i the same for the wave: a scalar load.
__device__ __forceinline__ int uniform_word(const int32_t *p, int i) {
  return ((const __attribute__((address_space(4))) int32_t *)(uintptr_t)p)[i];
}

__device__ __forceinline__ int tiles_of(int ctx) { return (ctx + KT - 1) / KT; }

// Sum over the lanes up to this one.
__device__ __forceinline__ int wave_prefix_sum(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int other = __shfl_up(v, o, 64);
    if (lane >= o) v += other;
  }
  return v;
}

struct Sequence {
  int b, prefix, tok0, ctx, before;          // before: tiles of the row in front of it
};

// The sequence that holds tile `at` of the row; b = batch if the row is shorter.  64 sequences per round of loads.
__device__ __forceinline__ Sequence find_sequence(const FewArgs &a, int at, int lane) {
  Sequence r{a.batch, 0, 0, 0, 0};
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int i = min(b0 + lane, a.batch - 1), prefix = a.prefix_lens[i], tok0 = a.cu[i], ctx = prefix + a.cu[i + 1] - tok0;
    const int n = b0 + lane < a.batch ? tiles_of(ctx) * a.Hkv : 0, sum = wave_prefix_sum(n, lane);
    const uint64_t past = __builtin_amdgcn_ballot_w64(r.before + sum > at);
    if (past) {
      const int j = __builtin_ctzll(past);
      return Sequence{b0 + j, __builtin_amdgcn_readlane(prefix, j), __builtin_amdgcn_readlane(tok0, j), __builtin_amdgcn_readlane(ctx, j),
                      r.before + __builtin_amdgcn_readlane(sum - n, j)};
    }
    r.before += __builtin_amdgcn_readlane(sum, 63);
  }
  return r;
}

// Two neighbouring elements of the four in `w`, times the scale of their row (its byte is the exponent): exact in bf16.
template <bool HIGH>
__device__ __forceinline__ uint32_t pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}
__device__ __forceinline__ float scale_of(uint32_t bytes, int i) { return __builtin_bit_cast(float, (bytes >> (8 * i) & 0xffu) << 23); }

template <int HD, int NQ, bool KV8, bool CAP>
__global__ __launch_bounds__(256, HD == 64 && NQ == 1 && KV8 ? 4 : 2) void attention_few_kernel(FewArgs a) {
  constexpr int KK = HD / 32;                // contraction steps of the scores
  constexpr int EB = KV8 ? 1 : 2;            // bytes per element
  constexpr int KJ = HD * EB / 64;           // 16-byte pieces of a key row per lane
  constexpr int MT = HD / 16;                // row tiles of O^T, and elements of a value row per lane
  constexpr int VW = MT * EB / 4;            // ... in dwords
  constexpr int PITCH = HD + 4;
  __shared__ __attribute__((aligned(16))) float s_o[4][16 * NQ][PITCH];
  __shared__ float s_m[4][16 * NQ], s_l[4][16 * NQ];
  typedef uint32_t vword __attribute__((ext_vector_type(VW)));

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4, G = a.Hq / a.Hkv;

  // A stretch of tiles [tile, end) of one pair, and how many tiles of the workgroup come after it.
  struct Stretch {
    int b, hk, prefix, tok0, ctx, tile, end, left;
  };
  Stretch here;
  int split;                                               // which part of its pair the stretch is
  if (a.in_a_row) {
    const int at = blockIdx.x * a.per;
    const Sequence f = find_sequence(a, at, lane);
    if (f.b >= a.batch) return;                            // (a shorter row on the device than the host's lengths said)
    const int n = tiles_of(f.ctx), offset = at - f.before, hk = offset / n, tile = offset - hk * n, end = min(n, tile + a.per);
    here = Stretch{f.b, hk, f.prefix, f.tok0, f.ctx, tile, end, a.per - (end - tile)};
    split = (tile + a.per - 1) / a.per;                    // the pair's first stretch starts at its tile 0, the others `per` tiles apart
  } else {
    const int b = blockIdx.z, prefix = uniform_word(a.prefix_lens, b), tok0 = uniform_word(a.cu, b);
    const int ctx = prefix + uniform_word(a.cu, b + 1) - tok0;
    split = blockIdx.y;
    here = Stretch{b, (int)blockIdx.x, prefix, tok0, ctx, split * a.per, min(tiles_of(ctx), (split + 1) * a.per), 0};
  }
  // To the next pair's tiles; false: there are none.
  auto turn = [&](Stretch &x) {
    if (x.left <= 0) return false;
    if (x.hk + 1 < a.Hkv) {
      ++x.hk;
    } else {
      if (x.b + 1 == a.batch) return false;
      ++x.b;
      x.hk = 0;
      x.prefix = uniform_word(a.prefix_lens, x.b);
      x.tok0 = uniform_word(a.cu, x.b);
      x.ctx = x.prefix + uniform_word(a.cu, x.b + 1) - x.tok0;
    }
    const int n = tiles_of(x.ctx);
    x.tile = 0;
    x.end = min(n, x.left);
    x.left -= x.end;
    return true;
  };
  // This wave's tiles, one after the other over all stretches; `end` <= `tile` once there are no more.
  auto settle = [&](Stretch &x) {
    while (x.tile >= x.end) {
      if (!turn(x)) return;
      x.tile += wave;
    }
  };

  const int kb = c >> 2, krow = c & 3;                     // this lane's key block of a tile, and its row there for score tile 0
  u32x4 kd[4][KJ], ks, vs;
  vword vd[16];
  int k_id = 0, v_id = 0, lanes = 1;                       // pool blocks of the tile to be requested next
  // Rows past the last key are read as they are, whatever they hold: their scores are masked, their values and scales cleared.
  auto ids = [&](const Stretch &x) {
    const int32_t *table = a.tables + (size_t)x.b * a.max_blocks;
    const int blk = x.tile * (KT / ARB_KV_BLOCK);
    k_id = table[min(blk + kb, a.max_blocks - 1)];
    v_id = table[min(blk + g, a.max_blocks - 1)];
  };
  // Behind the context's last block the tile's first one, which lane 0 has, is read instead (the table need not hold anything there).
  // All lanes take part in the exchange: inside a condition it would read from the first lane that the condition leaves.
  auto unit_of = [&](const Stretch &x, int id, int i) {
    const int first = __builtin_amdgcn_readlane(id, 0);
    const bool within = x.tile * (KT / ARB_KV_BLOCK) + i <= (x.ctx - 1) / ARB_KV_BLOCK;
    return (size_t)(unsigned)(within ? id : first) * a.Hkv + x.hk;
  };
  auto request_k = [&](const Stretch &x) {
    const size_t unit = unit_of(x, k_id, kb);
    const uint8_t *src = a.k_pool + unit * (ARB_KV_BLOCK * HD * EB) + (krow * HD * EB + g * 16) * lanes;
    if (KV8) ks = *(const u32x4 *)(a.k_scale + unit * ARB_KV_BLOCK);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < KJ; ++j) kd[t][j] = *(const u32x4 *)(src + t * 4 * HD * EB + j * 64);
  };
  auto request_v = [&](const Stretch &x) {
    const size_t unit = unit_of(x, v_id, g);
    const uint8_t *src = a.v_pool + unit * (ARB_KV_BLOCK * HD * EB) + c * (MT * EB) * lanes;
    if (KV8) vs = *(const u32x4 *)(a.v_scale + unit * ARB_KV_BLOCK);
#pragma unroll
    for (int k = 0; k < 16; ++k) vd[k] = *(const vword *)(src + k * HD * EB);
  };

  bf16x8 qf[NQ][KK];
  int limit[NQ];
  auto load_q = [&](const Stretch &x) {
    const int rows = (x.ctx - x.prefix) * G;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const int row = n * 16 + c, i = row < rows ? row / G : 0;
      limit[n] = x.prefix + i;
      const bf16 *src = a.q + (size_t)(x.tok0 + i) * a.q_row_stride + (x.hk * G + (row < rows ? row - i * G : 0)) * HD + g * (KV8 ? 16 : 8);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) qf[n][kk] = *(const bf16x8 *)(src + (KV8 ? (kk >> 1) * 64 + (kk & 1) * 8 : kk * 32));
    }
  };

  // The tile behind the one in flight, its blocks looked up.  Requests under a condition would make the wait for the values wait for
  // the keys behind them too; so behind the last tile all lanes ask for the same few lines (lanes = 0), which cost nothing.
  Stretch later = here;
  auto advance = [&] {
    Stretch next = later;
    next.tile += 4;
    settle(next);
    if (next.tile < next.end) later = next;
    else lanes = 0;
    ids(later);
  };
  later.tile += wave;
  if (!a.in_a_row) ids(later);                             // does not wait for the lengths
  if (here.tile >= here.end) return;                       // an even part behind the end of a shorter context
  settle(later);
  if (later.tile < later.end) {
    if (a.in_a_row) ids(later);
    request_k(later);
    request_v(later);
    advance();
  }
  load_q(here);
  for (;;) {
    f32x4 o[NQ][MT];
    float m_run[NQ], l_run[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      m_run[n] = -INFINITY;
      l_run[n] = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) o[n][mt] = f32x4(0.f);
    }
    const int ctx = here.ctx, p = here.prefix;
    for (int tile = here.tile + wave; tile < here.end; tile += 4) {
      const int key0 = tile * KT;
      const bool whole = key0 + KT <= ctx;
      f32x4 st[4][NQ];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float sc = KV8 ? __builtin_bit_cast(float, (ks[t] >> (8 * krow) & 0xffu) << 23) : 0.f;
#pragma unroll
        for (int n = 0; n < NQ; ++n) st[t][n] = f32x4(0.f);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          u32x4 f;
          if (KV8) {
            const uint32_t w0 = kd[t][kk >> 1][(kk & 1) * 2], w1 = kd[t][kk >> 1][(kk & 1) * 2 + 1];
            f = u32x4{pair<false>(w0, sc), pair<true>(w0, sc), pair<false>(w1, sc), pair<true>(w1, sc)};
          } else {
            f = kd[t][kk % KJ];
          }
#pragma unroll
          for (int n = 0; n < NQ; ++n)
            st[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), qf[n][kk], st[t][n], 0, 0, 0);
        }
      }
      request_k(later);
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
        mx[n] += ATTN_HEADROOM;
        grows |= mx[n] > m_run[n] + kLazyLog2;               // m_run = -inf: any visible key
      }
      // The reference moves only when a row has outgrown it by 2^8, and is set 2^16 above the row's maximum (so every weight is at most
      // 2^-8 and sums of values near the largest of bf16 stay in fp32; the quotient is the same); the four lanes of a query share it, and so do its accumulators.
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
      if (!whole) {                                        // a probability of 0 does not silence a NaN
        const int valid = ctx - key0 - 16 * g;
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (k >= valid) vd[k] = vword(0u);
#pragma unroll
        for (int d = 0; d < 4 && KV8; ++d) {
          const int bytes = min(max(valid - 4 * d, 0), 4);
          const uint32_t keep = bytes == 4 ? ~0u : (1u << (8 * bytes)) - 1;
          vs[d] = (vs[d] & keep) | (0x7f7f7f7fu & ~keep);
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4 vf[MT];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 8 * u + 2 * i;
          const float s0 = KV8 ? scale_of(vs[k >> 2], k & 3) : 0.f, s1 = KV8 ? scale_of(vs[k >> 2], (k & 3) + 1) : 0.f;
#pragma unroll
          for (int w = 0; w < MT / 2; ++w) {               // columns 2 w and 2 w + 1
            uint32_t lo, hi;
            if (KV8) {
              lo = w & 1 ? pair<true>(vd[k][w / 2], s0) : pair<false>(vd[k][w / 2], s0);
              hi = w & 1 ? pair<true>(vd[k + 1][w / 2], s1) : pair<false>(vd[k + 1][w / 2], s1);
            } else {
              lo = vd[k][w % VW];
              hi = vd[k + 1][w % VW];
            }
            vf[w * 2][i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
            vf[w * 2 + 1][i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
          }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int n = 0; n < NQ; ++n)
            o[n][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[mt]), __builtin_bit_cast(bf16x8, pf[n][u]), o[n][mt], 0, 0, 0);
      }
      request_v(later);
      advance();
    }

    // The four waves' results under their common maximum.
    const int hk = here.hk, tok0 = here.tok0, rows = (ctx - p) * G, part = split;
    const bool entire = here.tile == 0 && here.end == tiles_of(ctx);
    split = 0;                                             // the next stretch starts its pair
    const bool more = turn(here);
    if (more) load_q(here);
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
        for (int w = 0; w < MT / 4; ++w) {
          const f32x4 four = {o[n][w * 4][e], o[n][w * 4 + 1][e], o[n][w * 4 + 2][e], o[n][w * 4 + 3][e]};
          *(f32x4 *)&s_o[wave][n * 16 + c][(4 * g + e) * MT + w * 4] = four;
        }
    }
    __syncthreads();
    // (more rows than the host's lengths said, or more parts than the partial results have room for: not written)
    for (int i = tid; i < min(rows, 16 * NQ) * (HD / 8) && (entire || (a.part_acc && part < a.max_splits)); i += 256) {
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
      const float inv = entire || l != 0.f ? 1.0f / l : 0.f;   // NaN stays NaN; a row without visible keys in this part: 0
      if (entire) {
        bf16x8 r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = (bf16)(acc[e] * inv);
        *(bf16x8 *)(a.out + idx * HD + piece * 8) = r;
      } else {
        float *dst = a.part_acc + ((size_t)part * a.T * a.Hq + idx) * HD + piece * 8;
        *(f32x4 *)dst = f32x4{acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
        *(f32x4 *)(dst + 4) = f32x4{acc[4] * inv, acc[5] * inv, acc[6] * inv, acc[7] * inv};
        if (piece == 0) {
          float *ml = a.part_ml + ((size_t)part * a.T * a.Hq + idx) * 2;
          ml[0] = m;
          ml[1] = l;
        }
      }
    }
    if (!more) return;
    __syncthreads();
  }
}

// One workgroup per (sequence, kv head) that was cut: its rows over the parts.  Threads beside those that the rows need take every
// n-th part, since many parts one after the other are a chain of memory round trips (57 parts of one token: 9.5 us).
template <int HD>
__global__ __launch_bounds__(256) void attention_few_merge_kernel(FewArgs a) {
  constexpr int LANES = HD / 8;
  __shared__ float s_part[256][11];                        // m, l and eight accumulators (odd pitch)
  const int hk = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv, tid = threadIdx.x, lane = tid & 63;
  const int tok0 = a.cu[b], s = a.cu[b + 1] - tok0, G = a.Hq / a.Hkv, n = tiles_of(a.prefix_lens[b] + s);
  int n_parts = (n + a.per - 1) / a.per;
  if (a.in_a_row) {
    int before = hk * n;
    for (int b0 = 0; b0 < b; b0 += 64) {
      const int i = min(b0 + lane, b - 1), all = tiles_of(a.prefix_lens[i] + a.cu[i + 1] - a.cu[i]) * a.Hkv;
      before += __builtin_amdgcn_readlane(wave_prefix_sum(b0 + lane < b ? all : 0, lane), 63);
    }
    n_parts = (before + n - 1) / a.per - before / a.per + 1;
  }
  n_parts = min(n_parts, a.max_splits);
  if (n_parts <= 1) return;                                // written by the workgroup that had all of it
  const int work = s * G * LANES;
  int teams = 1;
  while (teams * 2 * work <= 256 && teams * 8 < n_parts) teams *= 2;
  for (int i0 = 0; i0 < work; i0 += 256 / teams) {
    const int team = tid / (256 / teams), i = i0 + tid - team * (256 / teams);
    const int row = min(i / LANES, s * G - 1), piece = i % LANES, tok = row / G;
    const size_t stride = (size_t)a.T * a.Hq, idx = (size_t)(tok0 + tok) * a.Hq + hk * G + (row - tok * G);
    SplitSum sum;
    sum.clear();
    sum.add<HD>(a.part_acc, a.part_ml, stride, idx, piece, team, teams, n_parts);
    if (teams > 1) {
      float *mine = s_part[tid];
      mine[0] = sum.m;
      mine[1] = sum.l;
#pragma unroll
      for (int e = 0; e < 8; ++e) mine[2 + e] = sum.acc[e];
      __syncthreads();
      if (team == 0 && i < work)
        for (int t = 1; t < teams; ++t) sum.join(s_part[tid + t * (256 / teams)]);
    }
    if (team == 0 && i < work) sum.store(a.out + idx * HD + piece * 8);
  }
}

}  // namespace

constexpr int kLeastTiles = 4;               // of a workgroup: one per wave

// The uncapped launch over bf16 pools is the other kernel's, whose results it has always had.  A bf16 tile of 128 columns takes the
// registers of the second query tile.
bool attention_few_takes(const AttnCache &cache, int head_dim, int max_rows) {
  if (cache.k_scale) return max_rows <= kFewRows;
  return cache.softcap > 0.f && max_rows <= (head_dim == 64 ? kFewRows : 16);
}

constexpr int kUncutTiles = 12;              // contexts up to here are one part each: three tiles a wave cost less than a merge

// Most parts that a pair of n tiles is cut into, wherever in the row it begins.
static int most_parts(int n, int per) { return (n + per - 2) / per + 1; }

int attention_few_parts_cap(int max_ctx) { return attention_splits_cap(max_ctx) + 1; }

// Partial results [parts, T, Hq, hd] and their (m, l), fp32; none with one part.
static size_t few_acc_bytes(int parts, int T, int Hq, int hd) { return align_up((size_t)parts * T * Hq * hd * sizeof(float), 256); }
size_t attention_few_ws_bytes(int parts, int total_tokens, int n_q_heads, int head_dim) {
  if (parts <= 1) return 0;
  return few_acc_bytes(parts, total_tokens, n_q_heads, head_dim) + align_up((size_t)parts * total_tokens * n_q_heads * 2 * sizeof(float), 256);
}

FewPlan plan_attention_few(int batch, const int32_t *prefix_host, const int32_t *cu_host, int n_kv_heads, int head_dim, int max_rows, bool kv8) {
  auto tiles = [&](int b) { return ceil_div(prefix_host[b] + cu_host[b + 1] - cu_host[b], KT); };
  long long total = 0;
  int most = 0;
  for (int b = 0; b < batch; ++b) {
    const int n = tiles(b);
    total += n;
    most = n > most ? n : most;
  }
  total *= n_kv_heads;
  const int cap = attention_few_parts_cap(most * KT);      // of the parts: what arb_workspace_bytes counts on
  // As many workgroups as are resident at once: by their registers two on a CU, four of 64 columns in 8 bits and one query tile.
  const int places = 256 * (head_dim == 64 && max_rows <= 16 && kv8 ? 4 : 2);
  const long long pairs = (long long)batch * n_kv_heads;
  const bool grid_fits = batch <= 65535 && n_kv_heads <= 65535;
  if (most <= kUncutTiles && grid_fits) return FewPlan{kUncutTiles, 0, 1, pairs, total};
  // Even parts, if there are places for all of them with parts not much longer than the workgroups' fair shares.
  const long long share = (total + places - 1) / places, even = share > kLeastTiles ? share : kLeastTiles;
  // (64 contexts of 1 K to 16 K keys, 2 kv heads: 23 % longer parts 81.6 us, in a row 64.5; 16 of 2049, 8 kv heads: even parts of the
  // same length 19.5, in a row 21.2.)  Three lengths up to a sixteenth longer are tried, each evened out for the longest context.
  for (int i = 0; i <= 2 && grid_fits; ++i) {
    const long long longest = even + (i * even + 31) / 32;
    const int parts = ceil_div(most, longest < most ? (int)longest : most), per = ceil_div(most, parts);
    if (parts > cap) continue;
    long long n = 0;
    const double inverse = 1.0 / per;                      // (a division of integers takes five times as long)
    for (int b = 0; b < batch; ++b) n += 1 + (long long)((tiles(b) - 0.5) * inverse);
    if (n * n_kv_heads <= places) return FewPlan{per, 0, parts, pairs * parts, total};
  }
  // Otherwise in a row: a tile for every wave at least, but not several pairs one after the other where all are shorter than that.
  const long long mean = pairs > 0 ? (total + pairs - 1) / pairs : 1, least = mean < kLeastTiles ? mean : kLeastTiles;
  long long per = share > least ? share : least;
  while (most_parts(most, (int)per) > cap) ++per;
  return FewPlan{(int)per, 1, most_parts(most, (int)per), (total + per - 1) / per, total};
}

arb_status check_attention_few(const FewPlan &plan, int batch, int n_kv_heads) {
  const long long merges = plan.parts > 1 ? (long long)batch * n_kv_heads : 0;
  if (plan.tiles + plan.per <= 0x7fffffffLL && plan.groups < 1 << 24 && merges < 1 << 24) return ARB_OK;
  return arb_fail(ARB_EUNSUPPORTED, "attention: %lld tiles of keys in one call", plan.tiles);
}

arb_status launch_attention_few(const bf16 *q, int q_row_stride, const AttnCache &cache, const int32_t *block_tables,
                                int max_blocks_per_seq, int batch, int total_tokens, int max_rows, int n_q_heads, int n_kv_heads,
                                int head_dim, const FewPlan &plan, bf16 *out, void *ws, size_t ws_bytes,
                                const int32_t *prefix_lens, const int32_t *cu_step_lens, hipStream_t st, bool q_prescaled) {
  if (batch == 0 || total_tokens == 0) return ARB_OK;
  const bool split = plan.parts > 1, capped = cache.softcap > 0.f;
  const size_t need = attention_few_ws_bytes(plan.parts, total_tokens, n_q_heads, head_dim);
  if (split && (!ws || ws_bytes < need)) return arb_fail(ARB_ECAPACITY, "attention: workspace %zu < %zu bytes", ws_bytes, need);
  if (arb_status s = check_attention_few(plan, batch, n_kv_heads)) return s;
  const float to_log2 = q_prescaled ? 1.0f : attention_q_scale(head_dim);
  FewArgs a{q, q_row_stride, (const uint8_t *)cache.k_pool, (const uint8_t *)cache.v_pool, cache.k_scale, cache.v_scale,
            block_tables, prefix_lens, cu_step_lens, batch, max_blocks_per_seq, plan.parts, plan.per, plan.in_a_row, total_tokens, n_q_heads,
            n_kv_heads, capped ? 2.0f * to_log2 / cache.softcap : to_log2, capped ? 1.44269504f * cache.softcap : 0.f, out, nullptr, nullptr};
  if (split) {
    a.part_acc = (float *)ws;
    a.part_ml = (float *)((char *)ws + few_acc_bytes(plan.parts, total_tokens, n_q_heads, head_dim));
  }
  const dim3 grid = plan.in_a_row ? dim3((unsigned)plan.groups) : dim3(n_kv_heads, plan.parts, batch), block(256);
#define ARB_FEW(HD, NQ)                                                                                                     \
  if (!cache.k_scale) hipLaunchKernelGGL((attention_few_kernel<HD, NQ, false, true>), grid, block, 0, st, a);               \
  else if (capped) hipLaunchKernelGGL((attention_few_kernel<HD, NQ, true, true>), grid, block, 0, st, a);                   \
  else hipLaunchKernelGGL((attention_few_kernel<HD, NQ, true, false>), grid, block, 0, st, a)
  if (!attention_few_takes(cache, head_dim, max_rows)) return arb_fail(ARB_EUNSUPPORTED, "attention of few rows: %d rows", max_rows);
  if (head_dim == 64) {
    if (max_rows <= 16) { ARB_FEW(64, 1); } else { ARB_FEW(64, 2); }
  } else if (max_rows <= 16) {
    ARB_FEW(128, 1);
  } else if (capped) {
    hipLaunchKernelGGL((attention_few_kernel<128, 2, true, true>), grid, block, 0, st, a);
  } else {
    hipLaunchKernelGGL((attention_few_kernel<128, 2, true, false>), grid, block, 0, st, a);
  }
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
