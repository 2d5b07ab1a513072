// Ragged GQA append-attention over a block-paged KV cache, bf16 or 8-bit, scores optionally capped.
//
// Work decomposition.  For sequence b and kv head hk, the G = Hq/Hkv query heads
// that share hk and the s_b step tokens form s_b*G query rows (row = i*G + g,
// token-major).  A workgroup of 4 waves takes 128 rows (32 per wave) and one
// chunk of the key range ("split"); chunks of a sequence are merged afterwards
// from their online-softmax states (m, l) and normalised partial results (16 bits).  Every KV byte is
// streamed from HBM once per 128 rows that need it; rows of different query
// tiles of the same (b, hk) meet in L2.
//
// Per 64-key tile, K and V stream into LDS row-major [key][hd] (XOR-swizzled
// 16-byte chunks) by direct-to-LDS global loads, double-buffered: tile t+1 is in
// flight while tile t is multiplied out.  S^T = K Q^T (keys are MFMA rows, queries are columns), so a
// lane owns one query column: the row max / row sum are in-lane reductions plus
// one cross-half shuffle, and exp2(S^T - m) is already laid out as the B operand
// of O^T = V^T P^T.  The V^T fragments (a lane needs 8 keys of one hd column) come
// from the LDS transpose read ds_read_b64_tr_b16: within 16 lanes, source lane j
// points at 4 consecutive columns of one row and lane i receives element i%4 of
// source lanes i/4, 4+i/4, 8+i/4, 12+i/4; with source lane j addressing key j/4,
// columns 4*(j%4).., lane i gets column i of four consecutive keys.  The pairing of
// MFMA contraction slots with keys follows the 32x32 D layout (lane half h,
// registers 8u..8u+7 of tile t hold keys 32t+16u+4h+{0..3} and
// 32t+16u+8+4h+{0..3}); V^T is read with the same pairing.
//
// An 8-bit cache (e4m3 elements, a power-of-two scale per row) goes through registers: a thread loads 16 elements of a
// row and the row's scale, v_cvt_scalef32_pk_bf16_fp8 makes two bf16 of two elements and the scale, exactly, and the
// stages in LDS are those of the bf16 cache.  So a tile is converted once per workgroup, not once per wave, and the products are,
// bit for bit, those over the cache's bf16 values.
#include "attention_merge.h"
#include "common.h"

#include <math.h>

namespace {

constexpr int QROWS = ATTN_QROWS, KT = ATTN_KT;
constexpr float kLazyLog2 = 8.0f;   // growth of a row maximum (log2 units) that forces a rescale

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

#define GLOBAL_PTR(p) ((const __attribute__((address_space(1))) void *)(p))
#define LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))

// Chunk swizzles.  A key row of a stage is HD/8 chunks of 16 bytes; chunk c of key k sits in slot
// c ^ swizzle(k).  The LDS has 64 banks of 4 bytes and serves 256 bytes per clock:
//  - K is read with ds_read_b128, 16 lanes (16 consecutive keys, one chunk) per clock: the slots of
//    16 consecutive keys must cover 256 bytes, so with 256-byte rows the swizzle is k mod 16, with
//    128-byte rows (two keys per 256 bytes) it is (k/2) mod 8;
//  - V is read with ds_read_b64_tr_b16, 32 lanes (4 consecutive keys x 4 consecutive chunks) per
//    clock: the two low key bits must move the slot by multiples of 4, so the key bits are rotated
//    (measured on this access pattern: 171 bytes/clock/CU against 63 with the K swizzle).
template <int HD>
__device__ __forceinline__ int k_swizzle(int key) { return HD == 128 ? (key & 15) : ((key >> 1) & 7); }
template <int HD>
__device__ __forceinline__ int v_swizzle(int key) {
  if (HD == 128) return ((key & 3) << 2) | ((key >> 2) & 3);
  const int x = (key >> 1) & 7;                  // 128-byte rows: the row parity picks the 128-byte half
  return ((x & 1) << 2) | (x >> 1);
}
template <int HD>
__device__ __forceinline__ int k_off(int key, int chunk) { return key * HD + ((chunk ^ k_swizzle<HD>(key)) << 3); }   // elements
template <int HD>
__device__ __forceinline__ int v_off(int key, int chunk) { return key * HD + ((chunk ^ v_swizzle<HD>(key)) << 3); }

// One 64-key tile for one wave: scores, online softmax update, O^T accumulation.
//
// PRESCALED: the queries arrive multiplied by log2(e)/sqrt(hd) (the forward's rotary kernel stores them that
// way, in fp32 before their one rounding), so K Q^T is already the logit in log2 units, and the score MFMAs
// start from the accumulator tuple `negm` (every element = minus the lane's reference maximum): the matrix
// pipe delivers s - m, and the vector ALU, which is the busier pipe of this kernel, is left with one exp2,
// half a max3, half a dot2 (row sum over the rounded probabilities, the ones the PV product uses) and half a
// convert per score.  Otherwise (queries as given, exact) the scale and the reference are applied to the fp32
// scores by one FMA per score; negm[0] then holds minus the reference.
//
// CAP: the logit x becomes cap tanh(x / cap) = cap - 2 cap / (exp(2 x / cap) + 1), in log2 units: cap_out - 2 cap_out r with
// r = 1 / (exp2(cap_in s) + 1), which takes two more transcendentals per score.  It is no longer linear in the score, so the
// matrix pipe cannot start from the reference; but it is linear in r, so the maximum is a minimum of r, and cap and
// reference are one FMA in front of the exponential.  scale_log2 is then cap_in.
//
// NT: 32-key halves of the tile that the wave takes, from sk, sv and ts on.  HEAD: log2 of the room that the reference leaves above the
// maximum: weights may grow to 2^kLazyLog2 of it and sum up over the keys, and the accumulators are to hold values near the largest of
// bf16 all the same (0 for the uncapped bf16 form, whose results stay as they were).
template <int HD, bool PRESCALED, bool CAP, int NT, int HEAD>
__device__ __forceinline__ void attend_tile(const bf16 *sk, const bf16 *sv, const bf16x8 (&qf)[HD / 16], f32x16 (&o)[HD / 32],
                                            f32x16 &negm, float &m_run, float &l_run, int ts, int limit, float scale_log2,
                                            float cap_out, int col, int half, int lane) {
  static_assert(!(PRESCALED && CAP), "capped scores do not start from the reference maximum");
  constexpr int KSTEPS = HD / 16, MT = HD / 32;
  f32x16 st[NT];
  if (!PRESCALED) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) st[t][r] = 0.f;
  }
  {
    // K fragments are requested two steps ahead of the MFMAs that take them (an LDS read takes longer
    // than the two MFMAs of a step)
    bf16x8 kf[3][NT];
#pragma unroll
    for (int pre = 0; pre < 2; ++pre)
#pragma unroll
      for (int t = 0; t < NT; ++t) kf[pre][t] = *(const bf16x8 *)&sk[k_off<HD>(t * 32 + col, pre * 2 + half)];
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk) {
      if (kk + 2 < KSTEPS) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
          kf[(kk + 2) % 3][t] = *(const bf16x8 *)&sk[k_off<HD>(t * 32 + col, (kk + 2) * 2 + half)];
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
        st[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk % 3][t], qf[kk], PRESCALED && kk == 0 ? negm : st[t], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (CAP) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) st[t][r] = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(st[t][r] * scale_log2) + 1.f);
  }
  constexpr float kHidden = CAP ? INFINITY : -INFINITY;
  // Causal mask (it also hides keys past the context): only tiles that reach some row's limit pay
  // for it.  Register r of tile t holds key ts + 32t + 8(r/4) + 4*half + r%4.
  const int vis = limit - ts - 4 * half;
  if (__builtin_amdgcn_ballot_w64(vis < 32 * NT - 1) != 0) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) st[t][r] = (t * 32 + 8 * (r >> 2) + (r & 3)) <= vis ? st[t][r] : kHidden;
  }
  // largest logit this lane holds for its query (the positive scale commutes with max), relative to the
  // reference maximum.  A query's keys are split between lanes l and l ^ 32; the two are only combined
  // (a cross-lane exchange) on the rare path below.
  float mx = kHidden;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = CAP ? fminf(mx, st[t][r]) : fmaxf(mx, st[t][r]);
  if (CAP) mx = fmaf(-2.f * cap_out, mx, cap_out + negm[0]);
  else if (!PRESCALED) mx = fmaf(mx, scale_log2, negm[0]);
  // The reference maximum m_run is advanced only when some row's maximum has outgrown it by more
  // than kLazyLog2 (m_run is that maximum plus HEAD): until then exp2(s - m_run) <= 2^(kLazyLog2 - HEAD), inside the range of bf16 and
  // fp32, and o / l is unchanged because both carry the same factor.  Most tiles then skip the
  // rescaling of the accumulators.  A row without a visible key so far has m_run = -inf and the
  // reference 0; its first visible key always sets the reference.
  if (__builtin_amdgcn_ballot_w64(mx > kLazyLog2 - HEAD || (m_run == -INFINITY && mx > -INFINITY)) != 0) {
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    const float m_new = fmaxf(m_run, m_use + (mx + HEAD));           // -inf only while nothing is visible
    const float m_new_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_new_use);   // m_run = -inf -> 0
    l_run *= alpha;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[mt][r] *= alpha;
    if (PRESCALED) {
      const float shift = m_new_use - m_use;                         // the scores were taken against the old reference
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) st[t][r] -= shift;
#pragma unroll
      for (int r = 0; r < 16; ++r) negm[r] = -m_new_use;
    } else {
      negm[0] = -m_new_use;
    }
    m_run = m_new;
  }
  if (!PRESCALED) {
    const float factor = CAP ? -2.f * cap_out : scale_log2, shift = CAP ? cap_out + negm[0] : negm[0];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) st[t][r] = fmaf(st[t][r], factor, shift);
  }
  bf16x8 pf[NT][2];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) pf[t][r >> 3][r & 7] = (bf16)__builtin_amdgcn_exp2f(st[t][r]);   // raw v_exp_f32; -inf -> 0
  // row sum over the probabilities as the PV product sees them (bf16), two per instruction
  {
    bf16x2 ones;
    ones[0] = ones[1] = (bf16)1.0f;
    float l_add = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          bf16x2 pr;
          pr[0] = pf[t][u][e];
          pr[1] = pf[t][u][e + 1];
          l_add = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, l_add, false);
        }
    l_run += l_add;
  }
  // O^T += V^T P^T; V^T fragments by transpose reads (see the header comment)
  const int j16 = lane & 15;
  const int vcol = 16 * ((lane >> 4) & 1) + 4 * (j16 & 3);     // within a 32-column tile
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int key0 = t * 32 + u * 16 + 4 * half + (j16 >> 2);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const int c = mt * 32 + vcol;
        const bf16 *a0 = &sv[v_off<HD>(key0, c >> 3) + (c & 7)];
        const bf16 *a1 = &sv[v_off<HD>(key0 + 8, c >> 3) + (c & 7)];
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)a0);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)a1);
        union { s16x4 s[2]; bf16x8 b; } vf;
        vf.s[0] = lo;
        vf.s[1] = hi;
        o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.b, pf[t][u], o[mt], 0, 0, 0);
      }
    }
}

// Two neighbouring e4m3 elements times the scale of their row, as bf16: exact (four significant bits).
template <bool HIGH>
__device__ __forceinline__ bf16x2 e4m3_pair(uint32_t four, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, HIGH);
}

// 16 elements of a row into the two 16-byte chunks of the bf16 stage that they fill.
__device__ __forceinline__ void store_16_e4m3(const u32x4 &v, uint32_t scale_byte, bf16 *chunk0, bf16 *chunk1) {
  const float scale = __builtin_bit_cast(float, scale_byte << 23);
  union { bf16x2 p[4]; bf16x8 c; } a, b;
  a.p[0] = e4m3_pair<false>(v[0], scale); a.p[1] = e4m3_pair<true>(v[0], scale);
  a.p[2] = e4m3_pair<false>(v[1], scale); a.p[3] = e4m3_pair<true>(v[1], scale);
  b.p[0] = e4m3_pair<false>(v[2], scale); b.p[1] = e4m3_pair<true>(v[2], scale);
  b.p[2] = e4m3_pair<false>(v[3], scale); b.p[3] = e4m3_pair<true>(v[3], scale);
  *(bf16x8 *)chunk0 = a.c;
  *(bf16x8 *)chunk1 = b.c;
}

// ROWS: no step has more rows of a kv head.  32, the uncapped bf16 forms: one wave has them all, and its results go out straight from the accumulators
// (as they also do in the other forms where a tile has no more rows; a kernel without the detour through the LDS beside it
// holds fewer registers: 16 tokens of the 8B shape on 513 to 1024 keys 11.25 -> 11.05 us).
// 64, the 8-bit and the capped forms (PAIRED): waves w and w + 2 share 32 rows and take half a tile's keys each, with an online softmax
// of their own, and meet at the end; otherwise two of the four waves would only load.  (8B shape, 32 steps of 9 against 4 K to 32 K keys,
// 8 bits: 355 -> 274 us, capped 448 -> 324, capped over bf16 436 -> 398; 32 of 18 to 32 against 1 K to 16 K, 4/2 heads of 64: 49 -> 34; a few short
// contexts 0 to 7 % faster.)
// The arguments that only the 8-bit and the capped forms take are the last ones: the others fit two lines of 64 bytes, and one word of a third
// on the way to the first load of keys is a miss more (one token on 1531 keys 8.35 -> 8.72 us).
template <int HD, bool SPLIT, bool PRESCALED, bool KV8, bool CAP, int ROWS>
__global__ __launch_bounds__(256, 2) void attention_kernel(
    const bf16 *__restrict__ q, int q_row_stride, const void *__restrict__ k_pool, const void *__restrict__ v_pool,
    const int32_t *__restrict__ block_tables, int max_blocks, const int32_t *__restrict__ prefix_lens,
    const int32_t *__restrict__ cu, int max_qtiles, int max_splits, int kv_chunk, const AttnItem *__restrict__ items,
    int n_items, int run, int T,
    int Hq, int Hkv, float scale_log2, bf16 *__restrict__ out, bf16 *__restrict__ part_acc, float *__restrict__ part_ml,
    int32_t *__restrict__ tok_splits, const uint8_t *__restrict__ k_scale, const uint8_t *__restrict__ v_scale, float cap_out) {
  constexpr int CPK = KV8 ? HD / 16 : HD / 8;   // 16-byte chunks per key of the cache
  constexpr int LOADS = KT * CPK / 256;    // wave-wide 1 KB loads per wave, operand and tile
  constexpr int KPL = 64 / CPK;            // keys covered by one wave-wide load (4 or 8: inside one block)
  constexpr int KSTEPS = HD / 16;          // MFMA k-steps over the head dimension
  constexpr int MT = HD / 32;              // 32-row tiles of O^T
  constexpr int EPC = KV8 ? 16 : 8, EB = KV8 ? 1 : 2;      // elements per chunk, bytes per element
  constexpr bool PAIRED = ROWS == 64;
  // Two stages of K and V; one array per stage so that LDS reads of one stage are not ordered
  // behind the direct-to-LDS loads in flight into the other.
  __shared__ __attribute__((aligned(16))) bf16 K0[KT * HD], K1[KT * HD], V0[KT * HD], V1[KT * HD];

  // Work item of this workgroup.  The hardware deals workgroups round-robin to the 8 XCDs (blockIdx % 8), and
  // an XCD works through its share in order.  The query tiles of one group (sequence, split, kv head) stream the
  // same keys and are neighbours in the list: the list goes to the XCDs in runs of that length, so that most groups stay on
  // one XCD and meet in its L2 while every XCD gets the same share of every sequence.  (64 contexts of 1 K to 16 K on
  // the 1.5B shape, up to 6 query tiles: runs of 1, 2, 6 items 346, 313, 306 us; with a contiguous range of sequences per
  // XCD the one with the longest finished last.)
  const int xcd = blockIdx.x % 8, slot = blockIdx.x / 8;
  const int index = ((slot / run) * 8 + xcd) * run + slot % run;
  if (index >= n_items) return;                        // rounding of the grid
  const int G = Hq / Hkv;
  AttnItem item;
  if (items == nullptr) {
    // No list: the product of sequences, most splits, heads and most query tiles (the last ones, which see most keys, first);
    // a workgroup whose place holds no visible key returns.  The items, and with them the results, are the list's, bit for bit.
    const int hq = Hkv * max_qtiles, group = index / hq, rest = index - group * hq;
    const int seq = SPLIT ? group / max_splits : group, part = SPLIT ? group - seq * max_splits : 0;
    const int p0 = prefix_lens[seq], t0 = cu[seq], len = cu[seq + 1] - t0, r0 = (max_qtiles - 1 - rest % max_qtiles) * QROWS;
    if (r0 >= len * G) return;
    const int chunk = SPLIT ? attn_seq_chunk(p0 + len, kv_chunk) : p0 + len, begin = part * chunk;
    const int visible = p0 + (min(len * G, r0 + QROWS) - 1) / G + 1;          // keys any row of the tile may see
    if (begin >= visible) return;
    item = AttnItem{seq, t0, p0, len, r0, begin, min(visible, begin + chunk), part << 16 | rest / max_qtiles};
  } else {
    item = items[index];
  }
  const int hk = item.split_head & 0xffff, split = item.split_head >> 16, b = item.seq;
  const int p = item.prefix, tok0 = item.tok0, s = item.step;
  const int rows = s * G, row0 = item.row0;
  if (row0 >= rows) return;                            // an empty item
  const int kv_begin = item.kv_begin, kv_end = item.kv_end;
  const int ctx = p + s;

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const int row_wave = PAIRED ? wave & 1 : wave;
  const bool wave_active = row0 + row_wave * 32 < rows;   // waves past the last row only help with the loads

  // This lane's query row.  Lanes behind the last row repeat it (the wave that has them has it too, so that they change no decision
  // of the wave's): loads without conditions of their own, eight in a row, and none by waves without rows.  (With the assumption below: one token on 1531
  // keys 8.5 -> 7.9 us, 16 of the 8B shape on 2000 26.0 -> 25.5.)
  const int row = row0 + row_wave * 32 + col, row_in = min(row, rows - 1);
  const bool row_ok = row < rows;
  const int tok_i = row_in / G;
  const int head = hk * G + row_in - tok_i * G;
  const int limit = p + tok_i;                         // last visible key (inclusive)

  bf16x8 qf[KSTEPS];
  if (wave_active) {
    const bf16 *qrow = q + (size_t)(tok0 + tok_i) * q_row_stride + head * HD;
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk) qf[kk] = *(const bf16x8 *)(qrow + kk * 16 + half * 8);
  }

  f32x16 o[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[mt][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  f32x16 negm;                               // minus the reference maximum (PRESCALED: in every element, the score MFMAs' C operand)
#pragma unroll
  for (int r = 0; r < 16; ++r) negm[r] = 0.f;

  // Tile loads.  One wave-wide direct-to-LDS load moves KPL whole keys (1 KB) of one 16-key block:
  // the block id is wave-uniform (scalar), lane l lands in chunk slot l % CPK of key l / CPK and
  // fetches the logical chunk that the read-side swizzle expects there.  Keys past the context
  // re-read the last valid key (finite data; they are masked out of the softmax anyway), so every
  // address is in bounds and the loop body needs no branch.
  const int32_t *table = block_tables + (size_t)b * max_blocks;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int last_key = ctx - 1, last_blk = last_key / ARB_KV_BLOCK;
  const int n_tiles = (kv_end - kv_begin + KT - 1) / KT;
  // An item has a visible key.  Without knowing it the compiler moves the loads of the queries behind the first barrier, which costs (above)
  // but in the 8-bit form of more than 64 rows, where the first tile's conversion then does not wait for them (16 steps of 64 on 2048 keys
  // 33.1 -> 32.1 us).
  if (!KV8 || PAIRED) __builtin_assume(n_tiles > 0);
  const int lkey = lane / CPK, pchunk = lane % CPK;
  int blk_id[LOADS];                       // pool block of each load of the tile to be issued next
  const unsigned first_blk = (unsigned)kv_begin / ARB_KV_BLOCK + (unsigned)(wave_u * KPL) / ARB_KV_BLOCK;
  auto lookup = [&](int tile) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const unsigned blk = first_blk + (unsigned)(tile * KT + i * 4 * KPL) / ARB_KV_BLOCK;
      blk_id[i] = table[min(blk, (unsigned)last_blk)];
    }
  };
  // Lane-constant part of the addresses: load i of a tile covers keys [wave*KPL, wave*KPL + KPL) of the
  // tile's 16-key block i*KPL/4 + wave*KPL/16, so the key inside its block and the swizzled chunk do not
  // depend on i or on the tile; only the (scalar) pool block does.
  const int kib = (wave_u * KPL + lkey) % ARB_KV_BLOCK;
  const int tkey = wave_u * KPL + lkey;            // tile-local key of load 0 (the others differ by multiples of 16 or 32)
  // (8-bit rows are swizzled where they are stored into the stage)
  const unsigned koff = (unsigned)(kib * HD + (KV8 ? pchunk * EPC : (pchunk ^ k_swizzle<HD>(tkey)) << 3)) * EB;                  // bytes
  const unsigned voff = (unsigned)(kib * HD + (KV8 ? pchunk * EPC : (pchunk ^ v_swizzle<HD>(tkey)) << 3)) * EB;
  const int kib_tail = min(kib, last_key % ARB_KV_BLOCK);
  const unsigned koff_tail = koff - (unsigned)((kib - kib_tail) * HD) * EB, voff_tail = voff - (unsigned)((kib - kib_tail) * HD) * EB;
  const char *k_head = (const char *)k_pool + (size_t)hk * ARB_KV_BLOCK * HD * EB;
  const char *v_head = (const char *)v_pool + (size_t)hk * ARB_KV_BLOCK * HD * EB;
  const unsigned blk_bytes = (unsigned)Hkv * ARB_KV_BLOCK * HD * EB;
  auto dma = [&](bf16 *dk, bf16 *dv, int tile) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int g = i * 4 + wave_u;                                  // 1 KB slot of the tile
      const unsigned blk = first_blk + (unsigned)(tile * KT + i * 4 * KPL) / ARB_KV_BLOCK;
      const bool tail = blk >= (unsigned)last_blk;                    // scalar choice between two lane vectors
      const uint64_t base = (uint64_t)(unsigned)blk_id[i] * blk_bytes;
      __builtin_amdgcn_global_load_lds(GLOBAL_PTR(k_head + base + (tail ? koff_tail : koff)), LDS_PTR(dk + g * 512), 16, 0, 0);
      __builtin_amdgcn_global_load_lds(GLOBAL_PTR(v_head + base + (tail ? voff_tail : voff)), LDS_PTR(dv + g * 512), 16, 0, 0);
    }
  };

  auto attend = [&](const bf16 *sk, const bf16 *sv, int t) {
    const int key0 = PAIRED ? (wave_u >> 1) * 32 : 0;      // (a multiple of 32 keys changes no swizzle)
    if (wave_active)
      attend_tile<HD, PRESCALED, CAP, PAIRED ? 1 : 2, KV8 || CAP ? ATTN_HEADROOM : 0>(sk + key0 * HD, sv + key0 * HD, qf, o, negm, m_run, l_run, kv_begin + t * KT + key0, limit,
                                                      scale_log2, cap_out, col, half, lane);
  };
  const int last_tile = n_tiles - 1;
  if constexpr (KV8) {
    // Tile t is multiplied out of one stage; tile t+1, in registers since the last step, is converted into the other, and tile
    // t+2 is requested into the registers that this frees.
    u32x4 k8[LOADS], v8[LOADS];
    uint32_t ks8[LOADS], vs8[LOADS];
    const unsigned soff = kib, soff_tail = kib_tail;
    auto request = [&](int tile) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const unsigned blk = first_blk + (unsigned)(tile * KT + i * 4 * KPL) / ARB_KV_BLOCK;
        const bool tail = blk >= (unsigned)last_blk;
        const uint64_t base = (uint64_t)(unsigned)blk_id[i] * blk_bytes;
        const size_t srow = ((size_t)(unsigned)blk_id[i] * Hkv + hk) * ARB_KV_BLOCK;
        k8[i] = *(const u32x4 *)(k_head + base + (tail ? koff_tail : koff));
        v8[i] = *(const u32x4 *)(v_head + base + (tail ? voff_tail : voff));
        ks8[i] = k_scale[srow + (tail ? soff_tail : soff)];
        vs8[i] = v_scale[srow + (tail ? soff_tail : soff)];
      }
    };
    auto convert = [&](bf16 *dk, bf16 *dv) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int key = i * 4 * KPL + tkey;
        store_16_e4m3(k8[i], ks8[i], &dk[k_off<HD>(key, 2 * pchunk)], &dk[k_off<HD>(key, 2 * pchunk + 1)]);
        store_16_e4m3(v8[i], vs8[i], &dv[v_off<HD>(key, 2 * pchunk)], &dv[v_off<HD>(key, 2 * pchunk + 1)]);
      }
    };
    lookup(0);
    request(0);
    lookup(min(1, last_tile));
    convert(K0, V0);
    request(min(1, last_tile));
    lookup(min(2, last_tile));
    __syncthreads();
    for (int t = 0; t < n_tiles; t += 2) {
      convert(K1, V1);
      request(min(t + 2, last_tile));
      lookup(min(t + 3, last_tile));
      __builtin_amdgcn_sched_barrier(0);
      attend(K0, V0, t);
      __syncthreads();
      if (t + 1 < n_tiles) {
        convert(K0, V0);
        request(min(t + 3, last_tile));
        lookup(min(t + 4, last_tile));
        __builtin_amdgcn_sched_barrier(0);
        attend(K1, V1, t + 1);
        __syncthreads();
      }
    }
  } else {
    // Tile t is multiplied out of one stage while tile t+1 streams into the other and the block ids
    // of tile t+2 are looked up; the barrier that ends a step also waits for the loads.
    lookup(0);
    dma(K0, V0, 0);
    lookup(min(1, last_tile));
    __syncthreads();
    for (int t = 0; t < n_tiles; t += 2) {
      dma(K1, V1, min(t + 1, last_tile));
      lookup(min(t + 2, last_tile));
      __builtin_amdgcn_sched_barrier(0);
      attend(K0, V0, t);
      __syncthreads();
      if (t + 1 < n_tiles) {
        dma(K0, V0, min(t + 2, last_tile));
        lookup(min(t + 3, last_tile));
        __builtin_amdgcn_sched_barrier(0);
        attend(K1, V1, t + 1);
        __syncthreads();
      }
    }
  }

  if constexpr (PAIRED) {
    // Waves 2 and 3 leave theirs in the V stages and what follows the results of waves 0 and 1 in the K stages.
    float *acc = (float *)(wave_u & 1 ? V1 : V0) + lane, *ml = (float *)((wave_u & 1 ? K1 : K0) + 32 * HD) + lane;
    if (wave_u >= 2) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[(mt * 16 + r) * 64] = o[mt][r];
      ml[0] = m_run;
      ml[64] = l_run;
    }
    __syncthreads();
    if (wave_u >= 2) return;
    const float m1 = ml[0], l1 = ml[64], m = fmaxf(m_run, m1);
    const float f0 = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m), f1 = m1 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m1 - m);
    m_run = m;
    l_run = f0 * l_run + f1 * l1;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[mt][r] = f0 * o[mt][r] + f1 * acc[(mt * 16 + r) * 64];
  }

  // The wave's result, row-major through the LDS (the stages are free: every tile ends with a barrier), so that a store writes whole
  // rows; straight from the accumulators it is 16-byte pieces of 32 rows.  Chunks are swizzled by the row.  Where one wave has all the
  // rows of its tile they go straight: the detour is 0.5 us of a short chain and saves nothing (30 rows of 16 sequences on 2048 keys 13.4 -> 12.8
  // us, 32 of 8 on 2000 14.5 -> 14.0; with 48 and 60 rows no difference, with 64 rows on 8 sequences 19.35 -> 19.6).
  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  const size_t orow = (size_t)(tok0 + tok_i) * Hq + head;   // (token, head) index
  if (!wave_active) return;
  // With SPLIT this is the split's own normalised result (it lies in the hull of the values, like the output) in 16 bits plus its
  // (m, l) in fp32: half the partial traffic of fp32 accumulators.  bf16 over an uncapped bf16 cache, as ever; otherwise fp16
  // relative to a power of two that puts the row's largest at 2^14: three bits more (error against 64 bits, 16 steps of 64 in five
  // parts: 0.0023 of the result's norm in bf16, 0.0017 this way, 0.0016 with one rounding, the result's) down to 2^-28 of that
  // largest, and a multiple of 2^-39 of it below, where bf16 would keep the precision of each column.
  constexpr bool RELATIVE = SPLIT && (KV8 || CAP);
  const float inv = !SPLIT || l_tot > 0.f ? 1.0f / l_tot : 0.f;
  float scale = 1.f, rel = 1.f;
  if constexpr (RELATIVE) {
    float most = 0.f;                                       // of the finite ones: an infinity stays one in fp16
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = fabsf(o[mt][r]);
        most = fmaxf(most, x < INFINITY ? x : 0.f);
      }
    most = fmaxf(most, __shfl_xor(most, 32, 64)) * inv;
    const int e = min(max((int)(__builtin_bit_cast(uint32_t, most) >> 23), 27), 254);       // exponent + 127, from 2^-100 on
    scale = __builtin_bit_cast(float, (e - 14) << 23);
    rel = __builtin_bit_cast(float, (254 - (e - 14)) << 23);
  }
  constexpr int CPR = HD / 8, RPS = 64 / CPR;               // 16-byte chunks per row, rows per store
  bf16 *dst = SPLIT ? part_acc + (size_t)split * T * Hq * HD : out;
  const int rows_here = min(32, rows - row0 - row_wave * 32);
  auto piece = [&](int mt, int r4) {
    bf16x4 v;
    f16x4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = (bf16)(o[mt][r4 * 4 + e] * inv);
      h[e] = (_Float16)(o[mt][r4 * 4 + e] * inv * rel);
    }
    return RELATIVE ? __builtin_bit_cast(bf16x4, h) : v;
  };
  if (ROWS == 32 || rows - row0 <= 32) {
    if (row_ok) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) *(bf16x4 *)(dst + orow * HD + mt * 32 + 8 * r4 + 4 * half) = piece(mt, r4);
    }
  } else {
    bf16 *buf = wave_u == 0 ? K0 : wave_u == 1 ? K1 : wave_u == 2 ? V0 : V1;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) *(bf16x4 *)&buf[col * HD + (((mt * 4 + r4) ^ (col % CPR)) << 3) + half * 4] = piece(mt, r4);
    const int orow32 = (int)orow;
#pragma unroll
    for (int i = 0; i < 32 / RPS; ++i) {
      const int r = i * RPS + lane / CPR, chunk = lane % CPR;
      const size_t at = (size_t)(unsigned)__shfl(orow32, r, 64);
      const bf16x8 v = *(const bf16x8 *)&buf[r * HD + ((chunk ^ (r % CPR)) << 3)];
      if (r < rows_here) *(bf16x8 *)(dst + at * HD + chunk * 8) = v;
    }
  }
  if (SPLIT && half == 0 && row_ok) {
    float *ml = part_ml + ((size_t)split * T * Hq + orow) * 2;
    ml[0] = RELATIVE ? m_run + __builtin_amdgcn_logf(l_tot) : m_run;   // (v_log_f32: base 2)
    ml[1] = RELATIVE ? scale : l_tot;
    // the number of splits that the merge reads for a token, where no earlier launch has written it
    if (tok_splits && split == 0 && hk == 0) tok_splits[tok0 + tok_i] = min(limit / attn_seq_chunk(ctx, kv_chunk) + 1, max_splits);
  }
}

// Merge of the split partials.  A thread owns eight consecutive elements of one (token, head) row, so a workgroup of 256 merges
// 2048 / HD rows.
template <int HD, typename Part>
__global__ __launch_bounds__(256) void attention_merge_kernel(const Part *__restrict__ part_acc,
                                                              const float *__restrict__ part_ml,
                                                              const int32_t *__restrict__ tok_splits, int max_splits, int T,
                                                              int Hq, bf16 *__restrict__ out) {
  constexpr int TPR = HD / 8;                              // threads per row
  const size_t stride = (size_t)T * Hq;
  const size_t idx = (size_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;      // token * Hq + head
  if (idx >= stride) return;
  const int piece = threadIdx.x % TPR;
  // splits that start at or before this token's position (never more than there is memory for, whatever the word holds)
  const int n_splits = min(tok_splits[idx / Hq], max_splits);
  SplitSum sum;
  sum.clear();
  sum.add<HD>(part_acc, part_ml, stride, idx, piece, 0, 1, n_splits);
  sum.store(out + idx * HD + piece * 8);
}

}  // namespace

static const int kTargetWorkgroups = 512;    // two resident workgroups per CU on 256 CUs
static const int kMinChunk = 256, kMaxChunk = 4096, kMaxChunkDecode = 6144, kMaxSplits = 64;
static const double kReplanUs = 20;
static const int kFineSplits = 32;
static const long long kFineRows = 65536;    // most rows of partial results in a plan of finer parts: 128 each for twice the CUs
static const long long kMostGroups = 1 << 24;                // a launch has fewer than 2^32 threads
static const long long kMostRows = 0x7fffffff - 2 * QROWS;   // query rows are counted in 32 bits, in whole tiles
static const int kMaxRun = 16;                // longest run of work items on one XCD when there are few runs per XCD

float attention_q_scale(int head_dim) { return (float)(1.4426950408889634 / sqrt((double)head_dim)); }

int attention_splits_cap(int max_ctx) {
  if (max_ctx <= 0) return 1;
  const int n = ceil_div(max_ctx, kMinChunk);
  return n < kMaxSplits ? n : kMaxSplits;
}

// Estimated time of an attention launch and its merge with parts of at most `chunk` keys.  A 64-key tile of 128 rows takes `tile_alone` alone on
// a CU and `tile` of the CU's time when two workgroups share it, one of a few rows (one wave works) tile_alone_few and tile_few; an item costs
// `item` more, of which its neighbour leaves `shown`.  With more items than places the launch ends half an item after the average place.  Between three
// quarters and all of the places a launch takes up to a fifth longer than that: CUs that got two of the long items hold it up.
struct AttnCosts {
  double tile, tile_few, tile_alone, tile_alone_few;       // us
  double narrow;                                           // of these with heads of 64
  double item, shown;
  double second, second_few;                               // the tile of the items behind the first round; where all steps are of few rows
  double rounds;                                           // how far the launch goes by whole rounds of workgroups, beyond all places
  double element, rate;                                    // bytes per cache element, MB/s
  double merge, merge_round, merge_element;
};
// The uncapped launch over bf16 pools.  Fitted to 43 batches (1 to 64 sequences, 50 to 32 K keys, steps of 1 to 128, three shapes) x up to 17 chunks.
static const AttnCosts kPlainCosts = {1.15, 1.5, 1.4, 2.3, 0.6, 4.0, 0.5, 1.15, 1.5, 0.0, 4, 5.0e6, 5.0, 1.3, 4e-7};
// The 8-bit and the capped forms where some step has more than 64 rows.  They go by rounds, which the others do not: 20 % more workgroups than
// places are 10 to 30 % slower than 10 % fewer.  Fitted to 34 batches (2 to 64 sequences, 600 to 32 K keys, steps of 6 to 150, five head
// layouts) x 13 chunks; over 169 batches, 26 of them among those, the launches are 3.1 % faster than with the chunk that the other figures
// pick (geometric mean; at best 36 %, at worst 24 % slower).
static const AttnCosts kFineCosts = {1.24, 1.96, 1.75, 1.94, 0.53, 5.0, 0.2, 1.24, 1.24, 0.4, 2, 4.1e6, 7.2, 0.5, 4.7e-7};

static double plan_us(const AttnCosts &k, int batch, const int32_t *prefix_host, const int32_t *cu_host, int G, int n_kv_heads, int head_dim, int chunk) {
  const double f = head_dim == 128 ? 1.0 : k.narrow, places = kTargetWorkgroups, cus = kTargetWorkgroups / 2;
  double n = 0, work = 0, tiles_all = 0, parts = 0, bytes = 0, shortest = 1e30, alone = 0, shared = 0;
  const double per_chunk = 1.0 / chunk;
  int max_ctx = 0;
  bool decode = true;
  for (int b = 0; b < batch; ++b) {                        // without integer divisions: some hundred of these per call
    const int s = cu_host[b + 1] - cu_host[b], ctx = prefix_host[b] + s, ns = 1 + (int)((ctx - 1) * per_chunk);
    const bool few = (long long)s * G <= 32;
    const double count = (double)ns * ceil_div(s * G, QROWS) * n_kv_heads, tiles = 1 + (int)((ctx - 1) / (double)(ns * KT)), per = few ? k.tile_few : k.tile;
    n += count;
    work += count * (tiles * per * f + k.item * k.shown);
    tiles_all += count * tiles;
    parts += (double)ns * s * G * n_kv_heads;
    bytes += (double)ctx * n_kv_heads * head_dim * k.element;
    shortest = tiles < shortest ? tiles : shortest;
    alone = fmax(alone, tiles * (few ? k.tile_alone_few : k.tile_alone) * f);
    shared = fmax(shared, tiles * per * f);
    decode = decode && few;
    max_ctx = ctx > max_ctx ? ctx : max_ctx;
  }
  const double second = n <= cus ? 0 : (decode ? k.second_few : k.second) * f * (shortest + (tiles_all / n - shortest) * fmin(1.0, (n - cus) / cus));
  double us;
  if (n <= places) {
    us = k.item + fmax(alone, shared + second);
    if (n > 0.75 * places && n < 0.98 * places) us *= 1 + 0.22 * (n - 0.75 * places) / (0.25 * places);
  } else {
    us = fmax(k.item + alone, work / cus + 0.5 * work / n);
    if (k.rounds > 0) {
      const double round = k.item + 2 * work / n, last = k.item + k.tile_alone * f * tiles_all / n, full = floor(n / places), rest = n - full * places;
      const double step = k.item + full * round + (rest == 0 ? 0 : rest <= cus ? last : last + (round - last) * (rest - cus) / cus);
      us = (1 - k.rounds) * us + k.rounds * step;
    }
  }
  us = fmax(us, k.item + bytes / k.rate);
  const int splits = ceil_div(max_ctx, chunk);
  return splits > 1 ? us + k.merge + k.merge_round * ceil_div(splits, 8) + parts * head_dim * k.merge_element : us;
}

static AttnPlan plan_of_chunk(int batch, const int32_t *prefix_host, const int32_t *cu_host, int G, int n_kv_heads, int chunk,
                              int max_ctx, int max_step) {
  AttnPlan pl;
  pl.max_qtiles = ceil_div(max_step * G, QROWS);
  pl.kv_chunk = chunk;
  pl.max_splits = max_ctx > 0 ? ceil_div(max_ctx, pl.kv_chunk) : 1;
  long long items = 0;
  for (int b = 0; b < batch; ++b) {
    const int s = cu_host[b + 1] - cu_host[b], ctx = prefix_host[b] + s, c = attn_seq_chunk(ctx, pl.kv_chunk);
    for (int begin = 0; begin < ctx; begin += c)
      items += (long long)(ceil_div(s * G, QROWS) - attn_first_qtile(prefix_host[b], G, begin)) * n_kv_heads;
  }
  pl.n_items = items < 0x7fffffff ? (int)items : 0x7fffffff;
  return pl;
}

static long long first_chunk(long long keys_streamed, int max_ctx, int max_rows) {
  const int cap = max_rows <= 32 ? kMaxChunkDecode : kMaxChunk;
  long long chunk = (keys_streamed / kTargetWorkgroups + KT - 1) / KT * KT;
  if (chunk > cap) chunk = cap;
  if (chunk < kMinChunk) chunk = kMinChunk;
  while (max_ctx > chunk * kMaxSplits) chunk += KT;
  return chunk;
}

AttnPlan plan_attention(int batch, const int32_t *prefix_host, const int32_t *cu_host, int G, int n_kv_heads, int head_dim) {
  long long keys_streamed = 0;          // sum over (sequence, kv head, query tile) of the context length
  int max_ctx = 0, max_step = 0;
  for (int b = 0; b < batch; ++b) {
    const int s = cu_host[b + 1] - cu_host[b], ctx = prefix_host[b] + s;
    keys_streamed += (long long)ceil_div(s * G, QROWS) * n_kv_heads * ctx;
    max_ctx = ctx > max_ctx ? ctx : max_ctx;
    max_step = s > max_step ? s : max_step;
  }
  // Keys per split, a first choice: about kTargetWorkgroups workgroups, never more than kMaxChunk keys (a batch whose steps all fit one
  // wave only streams the cache: there a longer chunk wins).  A sequence is cut into equal parts of at most that many keys
  // (attn_seq_chunk).  It bounds the splits, and with them the scratch of a call.
  long long chunk = first_chunk(keys_streamed, max_ctx, max_step * G);
  // Then the chunk with the least estimated time among those that need no more splits, if it promises 3 %.  What the first choice does
  // not see: sequences of different lengths cut by one size make a quarter more items than there are places, or leave
  // a quarter of them empty, and a CU's two places share its pipes.  (Measured, first choice -> this, us of one layer: 1.5B shape,
  // 32 steps of 8 to 96 against 512 to 4 K 67 -> 57, one of 64 against 16 K 36 -> 28, 32 of 1 and 10
  // against 1 K to 32 K 156 -> 122; 8B shape, 12 of 16 to 64 against 512 to 2 K 43 -> 36, 16 of 1 against 2 K 42 -> 34.  Over 43 batches
  // the first choice is 9.4 % slower than the best chunk, this one 4.7 %.  Estimates miss: of 161 other batches that they move, 110 got faster by
  // more than 2 % and at best 32, 23 slower by more than 2 % and at worst 14, most of those many one-token steps on ragged contexts; 7 %
  // on the geometric mean.)
  // At most eight of the shortest parts (one round of the merge) stay: such a launch is the latency of one part.
  const int splits = max_ctx > 0 ? ceil_div(max_ctx, (int)chunk) : 1;
  // So does a choice of less than kReplanUs: the estimates themselves take some microseconds of the host, which a short pass waits for.
  const double first = chunk > kMinChunk || splits > 8 ? plan_us(kPlainCosts, batch, prefix_host, cu_host, G, n_kv_heads, head_dim, (int)chunk) : 0.0;
  if (first >= kReplanUs) {
    double best = 0.97 * first;
    long long pick = chunk;
    for (const int c : {256, 320, 384, 512, 640, 768, 1024, 1280, 1536, 2048, 2560, 3072, 4096, 6144, 8192}) {
      if (ceil_div(max_ctx, c) > splits || c >= 2 * max_ctx) continue;
      const double us = plan_us(kPlainCosts, batch, prefix_host, cu_host, G, n_kv_heads, head_dim, c);
      if (us < best) {
        best = us;
        pick = c;
      }
    }
    chunk = pick;
  }
  return plan_of_chunk(batch, prefix_host, cu_host, G, n_kv_heads, (int)chunk, max_ctx, max_step);
}

// Few workgroups, contexts of more than kMinChunk keys: the launch is the latency of one part, and a tile (1.4 us) costs more than
// another part does in the merge.  Parts of 64 keys where eight of them do (one round of the merge), otherwise of 128 or more, at most
// kFineSplits, and no more workgroups than there are CUs: two of them on a CU would share its pipes, and the merge grows.
// (e4m3, us of a call, parts of 256 keys -> these: 8B shape, 41 tokens on 360 15.1 -> 11.2, 16 on 1000 14.8 -> 11.9, 64 on 4000 20.4
// (128 keys: 23.6); 1.5B shape, 64 on 2000 16.4 -> 15.0 (64 keys: 17.4), 20 on 700 15.1 -> 12.0, 4 x 7 on 279 to 654 14.3 -> 11.3, 30 on 8000 20.1 (128
// keys in 63 parts: 22.7).)
// The uncapped launch over bf16 pools keeps the parts, and with them the results, that it has always had.
AttnPlan plan_attention_fine(int batch, const int32_t *prefix_host, const int32_t *cu_host, int G, int n_kv_heads, int head_dim) {
  long long keys_streamed = 0;
  int max_ctx = 0, max_step = 0;
  for (int b = 0; b < batch; ++b) {
    const int s = cu_host[b + 1] - cu_host[b], ctx = prefix_host[b] + s;
    keys_streamed += (long long)ceil_div(s * G, QROWS) * n_kv_heads * ctx;
    max_ctx = ctx > max_ctx ? ctx : max_ctx;
    max_step = s > max_step ? s : max_step;
  }
  const long long cus = kTargetWorkgroups / 2, least = max_ctx <= 8 * KT ? KT : 2 * KT;
  long long chunk = (keys_streamed / cus + KT - 1) / KT * KT;
  if (chunk < least) chunk = least;
  while (max_ctx > chunk * kFineSplits) chunk += KT;
  if (max_ctx <= kMinChunk || chunk >= kMinChunk ||
      (long long)cu_host[batch] * G * n_kv_heads * ceil_div(max_ctx, (int)chunk) > kFineRows) {
    if (max_step <= 64 / G) return plan_attention(batch, prefix_host, cu_host, G, n_kv_heads, head_dim);
    // Enough workgroups: of the first choice and these, the chunk with the least estimated time (as plan_attention, but with more parts
    // than the first choice if they pay: arb_workspace_bytes has room for parts of kMinChunk).
    chunk = first_chunk(keys_streamed, max_ctx, max_step * G);
    double best = chunk > kMinChunk || ceil_div(max_ctx, (int)chunk) > 8 ? plan_us(kFineCosts, batch, prefix_host, cu_host, G, n_kv_heads, head_dim, (int)chunk) : 0.0;
    if (best >= kReplanUs) {
      best *= 0.97;
      for (const int c : {256, 320, 384, 512, 640, 768, 1024, 1280, 1536, 2048, 2560, 4096, 6144, 8192}) {
        if (ceil_div(max_ctx, c) > kMaxSplits || c >= 2 * max_ctx) continue;
        const double us = plan_us(kFineCosts, batch, prefix_host, cu_host, G, n_kv_heads, head_dim, c);
        if (us < best) {
          best = us;
          chunk = c;
        }
      }
    }
  }
  return plan_of_chunk(batch, prefix_host, cu_host, G, n_kv_heads, (int)chunk, max_ctx, max_step);
}

// Workspace: partial results [splits, T, Hq, hd] in 16 bits and two fp32 beside each row (none with a single split), the splits of every
// token, the work list (none with n_items == 0).
static size_t part_acc_bytes(int max_splits, int T, int Hq, int hd) {
  return max_splits > 1 ? align_up((size_t)max_splits * T * Hq * hd * sizeof(bf16), 256) : 0;
}
static size_t part_ml_bytes(int max_splits, int T, int Hq) {
  return max_splits > 1 ? align_up((size_t)max_splits * T * Hq * 2 * sizeof(float), 256) : 0;
}

size_t attention_ws_bytes(int max_splits, size_t n_items, int total_tokens, int n_q_heads, int head_dim) {
  return part_acc_bytes(max_splits, total_tokens, n_q_heads, head_dim) + part_ml_bytes(max_splits, total_tokens, n_q_heads) +
         align_up((size_t)total_tokens * sizeof(int32_t), 256) + align_up(n_items * sizeof(AttnItem), 256);
}

size_t attention_fine_ws_bytes(int total_tokens, int max_ctx, int n_q_heads, int G, int head_dim) {
  if (max_ctx <= kMinChunk) return 0;
  const int splits = ceil_div(max_ctx, KT) < kFineSplits ? ceil_div(max_ctx, KT) : kFineSplits;
  long long rows = (long long)total_tokens * n_q_heads * splits;
  if (rows > kFineRows) rows = kFineRows;
  const size_t tokens = total_tokens < kFineRows ? total_tokens : kFineRows;
  // (an item is at least one token's rows against one part)
  return rows * (head_dim * sizeof(bf16) + 2 * sizeof(float)) + tokens * sizeof(int32_t) + rows / G * sizeof(AttnItem) + 4 * 256;
}

AttnLists attention_lists(void *ws, const AttnPlan &plan, int total_tokens, int n_q_heads, int head_dim) {
  char *p = (char *)ws + part_acc_bytes(plan.max_splits, total_tokens, n_q_heads, head_dim) +
            part_ml_bytes(plan.max_splits, total_tokens, n_q_heads);
  return AttnLists{plan.n_items > 0 ? (AttnItem *)(p + align_up((size_t)total_tokens * sizeof(int32_t), 256)) : nullptr, (int32_t *)p};
}

arb_status check_attention_rows(int total_tokens, int n_q_heads) {
  if ((long long)total_tokens * n_q_heads < kMostRows) return ARB_OK;
  return arb_fail(ARB_EUNSUPPORTED, "attention: %d tokens of %d query heads in one call", total_tokens, n_q_heads);
}

// The launch's places: items of the list, or the product that is searched without one.
static long long attention_places(const AttnPlan &plan, int batch, int n_kv_heads) {
  return plan.n_items > 0 ? plan.n_items : (long long)batch * plan.max_splits * n_kv_heads * plan.max_qtiles;
}
// A run is a group's query tiles, shortened where so few of them fit that some XCDs would get a whole run more.
static int attention_run(const AttnPlan &plan, long long places) {
  const int run = plan.max_qtiles;
  return run > kMaxRun && places % (8LL * run) != 0 && places < 4 * 8LL * run ? kMaxRun : run;
}
static long long attention_groups(long long places, int run) { return (places + 8LL * run - 1) / (8LL * run) * (8LL * run); }

arb_status check_attention_launch(const AttnPlan &plan, int batch, int total_tokens, int n_q_heads, int n_kv_heads, int head_dim) {
  const long long places = attention_places(plan, batch, n_kv_heads), groups = attention_groups(places, attention_run(plan, places));
  const long long merge = plan.max_splits > 1 ? (long long)total_tokens * n_q_heads / (2048 / head_dim) + 1 : 0;
  if (groups < kMostGroups && merge < kMostGroups) return ARB_OK;
  return arb_fail(ARB_EUNSUPPORTED, "attention: %lld workgroups in one call", groups > merge ? groups : merge);
}

arb_status launch_attention(const bf16 *q, int q_row_stride, const AttnCache &cache,
                            const int32_t *block_tables, int max_blocks_per_seq, int batch, int total_tokens, int n_q_heads,
                            int n_kv_heads, int head_dim, const AttnPlan &plan, bf16 *out, void *ws, size_t ws_bytes,
                            const int32_t *prefix_lens, const int32_t *cu_step_lens, hipStream_t st, bool q_prescaled, int max_rows, bool count_splits) {
  if (batch == 0 || total_tokens == 0) return ARB_OK;
  if (head_dim != 64 && head_dim != 128) return arb_fail(ARB_EUNSUPPORTED, "attention: head_dim %d", head_dim);
  const size_t need = attention_ws_bytes(plan.max_splits, plan.n_items, total_tokens, n_q_heads, head_dim);
  const bool split = plan.max_splits > 1, listed = plan.n_items > 0;
  if ((split || listed) && (!ws || ws_bytes < need))
    return arb_fail(ARB_ECAPACITY, "attention: workspace %zu < %zu bytes", ws_bytes, need);
  if (arb_status s = check_attention_launch(plan, batch, total_tokens, n_q_heads, n_kv_heads, head_dim)) return s;
  const int n_items = (int)attention_places(plan, batch, n_kv_heads), run = attention_run(plan, n_items);
  bf16 *part_acc = (bf16 *)ws;
  float *part_ml = (float *)((char *)ws + part_acc_bytes(plan.max_splits, total_tokens, n_q_heads, head_dim));
  const AttnLists lists = split || listed ? attention_lists(ws, plan, total_tokens, n_q_heads, head_dim) : AttnLists{};
  // Capped scores: the kernel's scale is what the exponential of the tanh takes, 2 log2(e) / cap per unit of the logit.
  const bool kv8 = cache.k_scale != nullptr, capped = cache.softcap > 0.f;
  const float to_log2 = q_prescaled ? 1.0f : attention_q_scale(head_dim);
  const float scale_log2 = capped ? 2.0f * to_log2 / cache.softcap : to_log2, cap_out = capped ? 1.44269504f * cache.softcap : 0.f;
  const dim3 grid((unsigned)attention_groups(n_items, run)), block(256);
  // (pairs of waves in the 8-bit and the capped forms only: the others keep the order of their sums)
  const bool paired = max_rows <= 64, one_wave = max_rows <= 32;
#define ARB_ATTN_LAUNCH(HD, SPLIT, PRE, KV8, CAP, ROWS)                                                            \
  hipLaunchKernelGGL((attention_kernel<HD, SPLIT, PRE, KV8, CAP, ROWS>), grid, block, 0, st, q, q_row_stride, cache.k_pool, \
                     cache.v_pool, block_tables, max_blocks_per_seq, prefix_lens, \
                     cu_step_lens, plan.max_qtiles, plan.max_splits, plan.kv_chunk, lists.items, n_items, run, total_tokens, \
                     n_q_heads, n_kv_heads, scale_log2, out, part_acc, part_ml, count_splits ? lists.tok_splits : nullptr, \
                     cache.k_scale, cache.v_scale, cap_out)
#define ARB_ATTN_FINE(HD, SPLIT, PRE, KV8, CAP)                                                                    \
  if (paired) ARB_ATTN_LAUNCH(HD, SPLIT, PRE, KV8, CAP, 64); else ARB_ATTN_LAUNCH(HD, SPLIT, PRE, KV8, CAP, 128)
#define ARB_ATTN_PLAIN(HD, SPLIT, PRE)                                                                             \
  if (one_wave) ARB_ATTN_LAUNCH(HD, SPLIT, PRE, false, false, 32); else ARB_ATTN_LAUNCH(HD, SPLIT, PRE, false, false, 128)
#define ARB_ATTN_FORM(HD, SPLIT)                                                                                   \
  if (kv8 && capped) { ARB_ATTN_FINE(HD, SPLIT, false, true, true); }                                              \
  else if (capped) { ARB_ATTN_FINE(HD, SPLIT, false, false, true); }                                               \
  else if (kv8 && q_prescaled) { ARB_ATTN_FINE(HD, SPLIT, true, true, false); }                                    \
  else if (kv8) { ARB_ATTN_FINE(HD, SPLIT, false, true, false); }                                                  \
  else if (q_prescaled) { ARB_ATTN_PLAIN(HD, SPLIT, true); }                                                       \
  else { ARB_ATTN_PLAIN(HD, SPLIT, false); }
  if (head_dim == 128) { if (split) { ARB_ATTN_FORM(128, true); } else { ARB_ATTN_FORM(128, false); } }
  else                 { if (split) { ARB_ATTN_FORM(64, true); } else { ARB_ATTN_FORM(64, false); } }
#undef ARB_ATTN_FORM
#undef ARB_ATTN_PLAIN
#undef ARB_ATTN_FINE
#undef ARB_ATTN_LAUNCH
  ARB_CHECK_LAUNCH("attention");
  if (split) {
    const dim3 mgrid(ceil_div(total_tokens * n_q_heads, 2048 / head_dim)), mblock(256);
#define ARB_ATTN_MERGE(HD, Part)                                                                                   \
  hipLaunchKernelGGL((attention_merge_kernel<HD, Part>), mgrid, mblock, 0, st, (const Part *)part_acc, part_ml, lists.tok_splits, \
                     plan.max_splits, total_tokens, n_q_heads, out)
    if (kv8 || capped) { if (head_dim == 128) ARB_ATTN_MERGE(128, _Float16); else ARB_ATTN_MERGE(64, _Float16); }
    else               { if (head_dim == 128) ARB_ATTN_MERGE(128, bf16); else ARB_ATTN_MERGE(64, bf16); }
#undef ARB_ATTN_MERGE
    ARB_CHECK_LAUNCH("attention_merge");
  }
  return ARB_OK;
}
