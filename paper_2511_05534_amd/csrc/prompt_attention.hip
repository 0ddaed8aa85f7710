// The prompt's attention: every token of every packed sequence as a query over the keys that it sees,
//   o_t = softmax_j(score(q_t k_j)) v_j,   j <= reach(t),
// reach(t) = t, or the last token of the prefix or of the image span that t lies in: one number per row, which never falls from row to
// row, is the whole mask.  The attention matrix is never stored: one pass over the keys with the running maximum and sum of each row.
//
// A wave holds 32 query rows of one head in registers, as the second operand: the accumulators of S = K Q^T hold keys in their registers and
// rows in their lanes, so that a row's statistics are a lane's own and P is, register for register, an operand of O^T = V^T P^T.  The eight
// waves of a workgroup take the heads of the kv group at the same rows first and walk over one stream of K and V tiles, which direct
// global->LDS loads fill, double buffered.  V comes out of LDS transposed (ds_read_b64_tr_b16; fp32: by ordinary reads).
// Where rows are few, two or four waves share them and split the keys.  32 rows and 128 keys at a time: 64 rows a wave would leave no registers for two waves on a SIMD,
// and one wave's matrix instructions do not cover its own softmax.
//
// What bounds it: matrix cores (512 cycles of 32 keys x 32 rows at 128 channels) and vector issue (about 400: per logit an exponential at a quarter of the rate, a multiply-add,
// half a maximum, half an addition, half a conversion) of the two waves of a SIMD, which overlap in part, and the power limit (2.0 GHz).  16384 tokens, 32/8 heads, bf16:
// 2030 us, 1.08 PFLOP/s of the 1.21 that a large product of the library reaches; matrix cores busy 52 % of the time.  8 sequences of up to 8192, capped, 28/4 heads: 1780 us,
// 0.82 PFLOP/s (two exponentials and a reciprocal per logit).  675 tokens, 32 heads: 17 us, 20 with a picture in them; the workgroup of a block of rows that only in part see
// the picture is the last one.  The loads cost nothing that shows (all from one tile: 3 % less).  Blocks that some rows see in part take the same path with a mask, two at
// a time as well (one by one, each of V's numbers filtered: 675 tokens with a picture 25.4 us).
//
// bf16: P is rounded to bf16 for the second product, as V is one (by 2^-8 of a weight at the most, each its own, so that it stays below the
// rounding of the result wherever many keys count); its sum is of the fp32 weights.  fp32: both products by the fp32 matrix instructions.
#include <cfloat>
#include <type_traits>

#include "attention_core.h"
#include "decode_core.h"
#include "kernels.h"
#include "profile.h"

namespace flowmm {

namespace {

constexpr int kPThreads = kPromptWaves * 64;
// Units of a group: as many as have a workgroup for every compute unit, so that the workgroups of a unit run together and its keys and values are fetched once (a unit stays
// on an XCD), in fours for every XCD, and those that are left over spread over the groups: with fewer units at a time rows as late as each other meet on an XCD's compute units
// less evenly.
// All units together / groups in eights, the rest behind them / these, us: 256 units x 2048 tokens 372 / 339 / 344, 512 x 1100 330 / 303 / 294, 1024 x 400 164 / 155 / 155, 112 x 675
// (28/4 heads) 188 / 178 / 183, 32 x 3000 93 / 119 / 92, 128 x 1100 79 / 89 / 76, 32 x 8 sequences of 1000 118 / 150 / 118, 32 x 4 of 2000 171 / 218 / 171; all together / in 32s, the rest
// behind them / these: 40 x 3000 111 / 156 / 111, 36 x 675 20 / 26 / 20, 72 x 2000 103 / 138 / 102, 128 x 675 40 / 43 / 40, 112 x 3000 (32/8) 1172 / 1131 / 1154; 8 units of 16384 tokens
// are one group.
constexpr int kPromptGroupWgs = 256;

// V rows in LDS: whole rows by direct loads as in KeyTile, the chunks of a row permuted so that the four rows that 16 lanes transpose, 32 bytes
// of each, lie in different banks
template <bool BF16, int D, int ROWS>
struct ValueTile {
  static constexpr int NCH = Cfg<BF16, D>::NCH, kChunks = ROWS * NCH, RPI = 64 / NCH;
  __device__ static __forceinline__ int permute(int r) { return BF16 ? (NCH == 16 ? (r & 3) << 2 : ((r >> 1) & 1) << 2) : ((r >> 2) & 1) << 3; }
  __device__ static __forceinline__ int slot(int r, int ch) { return r * NCH + (ch ^ permute(r)); }
  template <int WAVES>
  __device__ static __forceinline__ void request(const uint4 *src, long long row_stride, int r0, int last, uint4 *tile, int wave) {
    const int lane = lane_id_here(), j = lane / NCH;
    constexpr int kLoads = kChunks / 64;
    static_assert(kLoads % WAVES == 0, "every wave asks for as many rows");
    const uint4 *base = src + r0 * row_stride;
    const bool near = row_stride < (1ll << 32) / (16 * ROWS);
#pragma unroll
    for (int i = 0; i < kLoads / WAVES; ++i) {
      const int g = i * WAVES + wave, rt = g * RPI + j, r = min(rt, last - r0), ch = (lane % NCH) ^ permute(rt);
      if (near) load_to_lds<16>(base, ((unsigned)r * (unsigned)row_stride + (unsigned)ch) * 16u, tile + g * 64);
      else tile[g * 64 + lane] = base[r * row_stride + ch];
    }
  }
};

// The first of a sequence's spans (PromptWord) that ends behind row q, and the last key that row q, or this lane's of the rows p0 .. p0 + 31, sees.  All by scalar loads:
// a search of every lane's own was three dependent trips to memory at a workgroup's start.
struct PromptSeq { int L, prefix, n_spans; ScalarInts spans; };
__device__ __forceinline__ int span_of(const PromptSeq &s, int q) {
  int lo = 0, hi = s.n_spans - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (s.spans[2 * mid] > q) hi = mid; else lo = mid + 1;
  }
  return lo;
}
__device__ __forceinline__ int reach_of_rows(const PromptSeq &s, bool image_spans, int p0, int rows, int q) {
  int r = q < s.prefix ? max(q, s.prefix - 1) : q;
  if (image_spans) {
    int j = span_of(s, p0), begin = p0;
    for (;;) {
      const int end = s.spans[2 * j];
      if (s.spans[2 * j + 1] && q >= begin && q < end) r = max(r, end - 1);
      if (end >= p0 + rows || j + 1 >= s.n_spans) break;
      begin = end;
      ++j;
    }
  }
  return r;
}

// A wave's share of the call: the rows p0 .. p0 + 31 of query head h, and the keys that they see.
struct PromptWave {
  int l, gkv, h, tok, L, p0, ks;  // ks: of KS waves with the same rows, this one takes every KS-th block of 32 keys, from block ks on
  int limit;                      // last key of this lane's row
  int first, last, wg_last;       // last key of the first and of the last of the wave's rows (-1: no rows), and of the workgroup's last one
};

template <int KS>
__device__ __forceinline__ PromptWave prompt_wave(const PromptArgs &a, ScalarInts meta) {
  PromptWave w;
  // groups of units, a group's units in turn, late positions (long key streams) first
  const int units = a.n_layers * a.Hkv, u0 = blockIdx.x / (a.group * a.wgs_total) * a.group, n_group = min(a.group, units - u0);
  const int rest = blockIdx.x - u0 * a.wgs_total, turn = rest / n_group, unit = u0 + rest - turn * n_group, x = a.wgs_total - 1 - turn;
  w.l = unit / a.Hkv;
  w.gkv = unit - w.l * a.Hkv;
  int b = 0;
  for (int lo = 0, hi = meta[PW_BATCH]; hi - lo > 1;) {
    const int mid = (lo + hi) >> 1;
    if (meta[PW_HEADER + mid * PS_WORDS + PS_WG] <= x) b = lo = mid; else hi = mid;
  }
  const ScalarInts rec = meta + PW_HEADER + b * PS_WORDS;
  const PromptSeq seq = {rec[PS_L], rec[PS_PREFIX], rec[PS_N_SPANS], meta + meta[PW_SPANS] + 2 * rec[PS_SPAN]};
  w.L = seq.L;
  w.tok = rec[PS_TOK];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = threadIdx.x & 31;
  // item i of the sequence: head i % G of the kv group, query rows [32 * (i / G), + 32)
  const int items = (w.L + kPromptRows - 1) / kPromptRows * a.G;
  constexpr int kItems = kPromptWaves / KS;
  w.ks = wave / kItems;
  const int first = (x - rec[PS_WG]) * kItems, mine = first + wave - w.ks * kItems, item = min(mine, items - 1), pb = item / a.G;
  w.h = w.gkv * a.G + (item - pb * a.G);
  w.p0 = pb * kPromptRows;
  const int wg_row = min((min(first + kItems, items) - 1) / a.G * kPromptRows + kPromptRows, w.L) - 1;
  w.wg_last = __builtin_amdgcn_readfirstlane(reach_of_rows(seq, a.image_spans, wg_row, 1, wg_row));
  w.limit = reach_of_rows(seq, a.image_spans, w.p0, kPromptRows, min(w.p0 + n, w.L - 1));
  w.first = __builtin_amdgcn_readfirstlane(w.limit);
  w.last = mine < items ? __builtin_amdgcn_readlane(w.limit, 31) : -1;
  return w;
}

// The rows' outputs o [channel][row], maxima and sums (z: of either half-wave's keys) of the KS waves that share them, folded and stored by whole rows.
// Every wave of the workgroup calls.
template <bool BF16, int D, int KS>
__device__ __forceinline__ void store_rows(const PromptArgs &a, const PromptWave &w, const f32x16_t (&o)[D / 32], float m, float z, float *lds) {
  constexpr int NCH = Cfg<BF16, D>::NCH, EPC = Cfg<BF16, D>::kElemsPerChunk, kItems = kPromptWaves / KS;
  constexpr int SS = D + 4;  // row of a wave's output in LDS: D channels, m, z
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
  z += __shfl_xor(z, 32, 64);
  __syncthreads();  // nobody reads tiles any more
  float *st = lds + wave * 32 * SS;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *reinterpret_cast<float4 *>(st + n * SS + 32 * c + acc_row(i, half)) = make_float4(o[c][i], o[c][i + 1], o[c][i + 2], o[c][i + 3]);
  if (half == 0) { st[n * SS + D] = m; st[n * SS + D + 1] = z; }
  __syncthreads();
  if (w.last < 0) return;
  uint4 *out = reinterpret_cast<uint4 *>(a.out) + (long long)w.l * a.qs_layer + (long long)w.h * a.qs_head + (long long)(w.tok + w.p0) * a.qs_tok;
  const float *st0 = lds + (wave - w.ks * kItems) * 32 * SS;
  // the waves of the rows store a share of them each
#pragma unroll 1
  for (int r = w.ks * (32 / KS) + lane / NCH; r < (w.ks + 1) * (32 / KS); r += 64 / NCH) {
    if (w.p0 + r >= w.L) break;
    float M = -FLT_MAX, zz = 0.f, f[EPC];
#pragma unroll
    for (int i = 0; i < KS; ++i) M = fmaxf(M, st0[(i * kItems * 32 + r) * SS + D]);
#pragma unroll
    for (int e = 0; e < EPC; ++e) f[e] = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const float *row = st0 + (i * kItems * 32 + r) * SS;
      const float g = fast_exp2(row[D] - M);
      zz = fmaf(row[D + 1], g, zz);
#pragma unroll
      for (int e = 0; e < EPC; ++e) f[e] = fmaf(row[lane % NCH * EPC + e], g, f[e]);
    }
    const float inv = 1.f / zz;
#pragma unroll
    for (int e = 0; e < EPC; ++e) f[e] *= inv;
    out[r * a.qs_tok + lane % NCH] = floats_to_chunk<BF16>(f);
  }
}

// log2-domain scores of the products of row q with the keys key + acc_row(i, 0) (key: of this lane's half)
template <bool SCORED, bool FINE>
__device__ __forceinline__ void score(const PromptArgs &a, f32x16_t &s, float slope, int key, int q) {
#pragma clang fp contract(off)
  if (SCORED && a.score.cap > 0.f) {
    if (FINE || a.score.fine) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = capped<true>(a.score, s[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = capped<false>(a.score, s[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] *= a.score.cl;
  }
  if (SCORED && a.score.slopes) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = fmaf(-slope, fabsf((float)(key - q + acc_row(i, 0))), s[i]);
  }
}

// (an LDS address is 32 bits wide; the cast goes through uintptr_t for the host's pass over this file)
template <class T>
__device__ __forceinline__ const __attribute__((address_space(3))) T *lds_at(unsigned at) {
  return (const __attribute__((address_space(3))) T *)(uintptr_t)at;
}
__device__ __forceinline__ uint4 lds_chunk(unsigned at) {
  typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;
  const u32x4_t v = *lds_at<u32x4_t>(at);
  return make_uint4(v[0], v[1], v[2], v[3]);
}

template <bool BF16, int D, int KS, bool SCORED>
__global__ __launch_bounds__(kPThreads, 2) void prompt_attention_kernel(KernelArgs<PromptArgs> k) {
  const PromptArgs &a = k.a;
  using CF = Cfg<BF16, D>;
  using TL = KeyTile<BF16, D>;
  constexpr int NCH = CF::NCH, NF = CF::NF, KT = TL::kRows, CT = D / 32;
  using VT = ValueTile<BF16, D, KT>;
  constexpr int kBuffer = TL::kChunks + VT::kChunks;
  constexpr float kLazy = 8.f;  // the running maximum follows once it is 2^8 behind: exact all the same, z stays far below overflow
  extern __shared__ __align__(16) uint4 lds_kv[];  // [2] K tile, V tile; at the end the waves' outputs

  const ScalarInts meta = first_meta(k, a.meta);
  const PromptWave w = prompt_wave<KS>(a, meta);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
  const int L = w.L, p0 = w.p0, ks = w.ks, limit = w.limit, w_first = w.first, w_last = w.last;

  // ---- this wave's query rows (clamped past the end of the sequence), through its share of the LDS ----
  uint4 qf[NF];
  const uint4 *Q = reinterpret_cast<const uint4 *>(a.Q) + (long long)w.l * a.qs_layer + (long long)w.h * a.qs_head + (long long)(w.tok + p0) * a.qs_tok;
  static_assert(kPromptWaves * 32 * NCH <= 2 * kBuffer, "the waves' query rows");
  fetch_rows_staged<BF16, D>(Q, (unsigned)a.qs_tok, min(p0 + n, L - 1) - p0, lds_kv + wave * 32 * NCH, qf);
  __syncthreads();  // the tiles may overwrite the other waves' shares now

  const long long kv_at = (long long)w.l * a.ks_layer + (long long)w.gkv * a.ks_head + (long long)w.tok * a.ks_tok;
  const uint4 *K = reinterpret_cast<const uint4 *>(a.K) + kv_at, *V = reinterpret_cast<const uint4 *>(a.V) + kv_at;
  const float slope = SCORED && a.score.slopes ? a.score.slopes[w.h] * 1.4426950408889634f : 0.f;
  float m = -FLT_MAX, z = 0.f;  // of row n; z over the keys of this half-wave
  f32x16_t o[CT];               // [channel 32 c + ..][row n]
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[c][i] = 0.f;

  const int ntiles = w.wg_last / KT + 1;
  // Requests of a tile: this wave's share of its rows.  Whole tiles whose rows lie within 4 GiB (nearly all) by offsets from the tile's first row that stay the same.
  constexpr int kKLoads = KT / TL::kGroup / kPromptWaves, kVLoads = KT / VT::RPI / kPromptWaves;
  const bool near = a.ks_tok < (1ll << 32) / (16 * KT);
  unsigned k_off[kKLoads], v_off[kVLoads];
#pragma unroll
  for (int i = 0; i < kKLoads; ++i) {
    const int j = lane / NCH, r = (i * kPromptWaves + wave) * TL::kGroup + j;
    k_off[i] = ((unsigned)r * (unsigned)a.ks_tok + (unsigned)((lane % NCH) ^ TL::permute(j))) * 16u;
  }
#pragma unroll
  for (int i = 0; i < kVLoads; ++i) {
    const int r = (i * kPromptWaves + wave) * VT::RPI + lane / NCH;
    v_off[i] = ((unsigned)r * (unsigned)a.ks_tok + (unsigned)((lane % NCH) ^ VT::permute(r))) * 16u;
  }
  const unsigned lds0 = (unsigned)(uintptr_t)(lds_void *)lds_kv;
  auto request = [&](int t) {
    if (near && (t + 1) * KT <= L) {
      const long long skip = (long long)(t * KT) * a.ks_tok;
      const uint4 *kt = K + skip, *vt = V + skip;
      const unsigned to = lds0 + (t & 1) * kBuffer * 16;
#pragma unroll
      for (int i = 0; i < kKLoads; ++i) load_to_lds_at(kt, k_off[i], to + (i * kPromptWaves + wave) * TL::kGroupChunks * 16);
#pragma unroll
      for (int i = 0; i < kVLoads; ++i) load_to_lds_at(vt, v_off[i], to + (TL::kChunks + (i * kPromptWaves + wave) * 64) * 16);
    } else {
      uint4 *to = lds_kv + (t & 1) * kBuffer;
      TL::template request<kPromptWaves>(K, a.ks_tok, t * KT, L - 1, to, wave);
      VT::template request<kPromptWaves>(V, a.ks_tok, t * KT, L - 1, to + TL::kChunks, wave);
    }
  };
  const unsigned k_frag[2] = {(unsigned)TL::frag_offset(n, half, 0), (unsigned)TL::frag_offset(n, half, 1)};  // bytes from the start of a K tile
  unsigned v_frag[CT];  // .. of a V tile, to this lane's share of the four rows that 16 lanes transpose
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int i16 = lane & 15, g16 = (lane >> 4) & 1;
    v_frag[c] = BF16 ? (unsigned)(VT::slot(4 * half + (i16 >> 2), 4 * c + 2 * g16 + ((i16 & 3) >> 1)) * 16 + 8 * (i16 & 1)) : 0u;
  }
  // blocks kb, kb + KS, .. (NB of them) of tile t; MASKED: some row of the wave does not see all of their keys
  auto blocks = [&](auto nb, auto masked_t, int t, int kb) __attribute__((always_inline)) {
    constexpr int NB = decltype(nb)::value;
    constexpr bool MASKED = decltype(masked_t)::value;
    // LDS addresses of this lane's shares, one a register (opaque: the compiler would keep and advance one for every read)
    const unsigned tile = lds0 + (t & 1) * kBuffer * 16, values = tile + TL::kChunks * 16;
    unsigned k_at[2], v_at[BF16 ? CT : 1];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      k_at[i] = tile + k_frag[i] + kb * TL::block_bytes(1);
      asm volatile("" : "+v"(k_at[i]));
    }
#pragma unroll
    for (int c = 0; c < (BF16 ? CT : 1); ++c) {
      v_at[c] = values + v_frag[c] + kb * 32 * NCH * 16;
      asm volatile("" : "+v"(v_at[c]));
    }
    const int key0 = t * KT + 32 * kb;
    f32x16_t s[NB];  // [key][row]

    // K fragments asked for 3 steps ahead (pinned: left to itself the compiler reads each one right before its use)
    constexpr int kAhead = NF < 3 ? NF : 3;
    uint4 kf[NF][NB];
    auto read_k = [&](int f) {
#pragma unroll
      for (int u = 0; u < NB; ++u) kf[f][u] = lds_chunk(k_at[f & 1] + u * KS * TL::block_bytes(1) + 64 * (f >> 1));
    };
#pragma unroll
    for (int f = 0; f < kAhead; ++f) read_k(f);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < NF; ++f) {
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        if (f == 0) s[u] = f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        mma_chunk<BF16>(s[u], kf[f][u], qf[f]);
      }
      if (f + kAhead < NF) read_k(f + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
    // ---- scores ----
    auto most = [&]() {
      float x = fmaxf(s[0][0], s[0][1]);
#pragma unroll
      for (int u = 0; u < NB; ++u)
#pragma unroll
        for (int i = u ? 0 : 2; i < 16; i += 2) x = fmaxf(fmaxf(x, s[u][i]), s[u][i + 1]);
      return x;
    };
    auto mask = [&]() {
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        const int last = limit - key0 - 32 * u * KS - 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[u][i] = acc_row(i, 0) <= last ? s[u][i] : -INFINITY;
      }
    };
    // Weights are exp2(score - maximum), taken as exp2(fma(s, mul, add - maximum)) with whatever is left in s: the product, where it is neither capped nor
    // biased; -1 / (1 + e^(2 u)), where they are capped only (the cap's own rounding is larger); the score.  A product's fused multiply-add keeps what the maximum's
    // rounding lost, 2^-24 of it: nothing where scores are within 2^24, an overflow at 1e30.  Larger ones (or NaN) are rounded first.
    float mul = 1.f, add = 0.f, tm = 0.f;
    bool ready = false;
    if constexpr (!SCORED && (BF16 || !MASKED)) {
      if constexpr (MASKED) mask();
      tm = most();
      ready = !__any(!(fabsf(tm) * a.score.cl < 0x1p24f) && !(MASKED && tm == -INFINITY));
      if (ready) mul = a.score.cl;
    }
    if (!ready) {
      if (SCORED && BF16 && a.score.cap > 0.f && !a.score.slopes && !a.score.fine) {
        mul = 2.f * a.score.cap;
        add = a.score.cap;
        const float k = a.score.cap_in * 2.8853900817779268f;
#pragma unroll
        for (int u = 0; u < NB; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[u][i] = __builtin_amdgcn_rcpf(-1.f - fast_exp2(s[u][i] * k));
      } else {
#pragma unroll
        for (int u = 0; u < NB; ++u) score<SCORED, !BF16>(a, s[u], slope, key0 + 32 * u * KS + 4 * half, p0 + n);
      }
      if constexpr (MASKED && (SCORED || !BF16)) mask();
      tm = most();
    }
    tm = fmaf(tm, mul, add);
    if (__any(tm > m + kLazy)) {
      const float M = fmaxf(m, fmaxf(tm, __shfl_xor(tm, 32, 64))), f = fast_exp2(m - M);
      z *= f;
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[c][i] *= f;
      m = M;
    }
    const float base = add - m;
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      float za = 0.f, zb = 0.f;
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        s[u][i] = fast_exp2(fmaf(s[u][i], mul, base));
        s[u][i + 1] = fast_exp2(fmaf(s[u][i + 1], mul, base));
        za += s[u][i];
        zb += s[u][i + 1];
      }
      z += za + zb;
    }
    // ---- O += V^T P; a masked block's infinite or undefined values may only reach the rows that see them: taken out here, added with their weights below ----
    bool odd = false;
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      if constexpr (BF16) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const uint4 pf = make_uint4(pack_bf16(s[u][8 * kk], s[u][8 * kk + 1]), pack_bf16(s[u][8 * kk + 2], s[u][8 * kk + 3]), pack_bf16(s[u][8 * kk + 4], s[u][8 * kk + 5]),
                                      pack_bf16(s[u][8 * kk + 6], s[u][8 * kk + 7]));
          uint4 vf[CT];
#pragma unroll
          for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
              const s16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)lds_at<s16x4_t>(v_at[c] + (32 * u * KS + 16 * kk + 8 * jj) * NCH * 16));
              __builtin_memcpy(reinterpret_cast<char *>(&vf[c]) + 8 * jj, &v, 8);
            }
          if constexpr (MASKED) {
            typedef __attribute__((ext_vector_type(2))) unsigned short u16x2_t;
            u16x2_t most_v = {0, 0};  // magnitudes, as numbers of 15 bits
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const unsigned w = reinterpret_cast<const unsigned *>(&vf[c])[e] & 0x7fff7fffu;
                most_v = __builtin_elementwise_max(most_v, __builtin_bit_cast(u16x2_t, w));
              }
            if (__any(max(most_v.x, most_v.y) >= 0x7f80)) {
              odd = true;
#pragma unroll
              for (int c = 0; c < CT; ++c) {
                unsigned *w = reinterpret_cast<unsigned *>(&vf[c]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  w[e] = ((w[e] & 0x7f800000u) == 0x7f800000u ? 0u : w[e] & 0xffff0000u) | ((w[e] & 0x7f80u) == 0x7f80u ? 0u : w[e] & 0xffffu);
              }
            }
          }
#pragma unroll
          for (int c = 0; c < CT; ++c) mma_chunk<true>(o[c], vf[c], pf);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            float v = *lds_at<float>(values + VT::slot(32 * (kb + u * KS) + acc_row(i, half), 8 * c + (n >> 2)) * 16 + 4 * (n & 3));
            if constexpr (MASKED) {
              const bool bad = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u;
              odd |= bad;
              v = bad ? 0.f : v;
            }
            o[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[u][i], o[c], 0, 0, 0);
          }
      }
    }
    if constexpr (MASKED) {
      if (__any(odd)) {
        // (as in a whole block: infinite, and undefined where the weight is 0)
#pragma unroll 1
        for (int j = 0; j < 32 * NB; ++j) {
          const int row = 32 * kb + (j & 31) + 32 * KS * (j >> 5), key = t * KT + row;
          if (key >= L) break;
          float weight = 0.f;  // of key j, in the lanes of the half-wave that holds it
#pragma unroll
          for (int u = 0; u < NB; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) weight = 32 * u + acc_row(i, 0) == (j & ~4) ? s[u][i] : weight;
          weight = __shfl(weight, n + 8 * (j & 4), 64);
#pragma unroll
          for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int ch = 32 * c + acc_row(i, half);
              float v;
              if constexpr (BF16) v = bf16_bits_to_float(*lds_at<uint16_t>(values + VT::slot(row, ch >> 3) * 16 + 2 * (ch & 7)));
              else v = *lds_at<float>(values + VT::slot(row, ch >> 2) * 16 + 4 * (ch & 3));
              if (!(fabsf(v) < INFINITY) && key <= limit) o[c][i] += weight * v;
            }
        }
      }
    }
  };

  request(0);
  for (int t = 0; t < ntiles; ++t) {
    __builtin_amdgcn_s_waitcnt(0);  // this wave's part of tile t has landed
    __syncthreads();                // ... and everybody else's; tile t-1 is no longer read
    if (t + 1 < ntiles) request(t + 1);
    // blocks of 32 keys: those that all of the wave's rows see whole, then the others; two at a time
    const int full = min(max((w_first + 1 - t * KT) >> 5, 0), KT / 32), seen = min((w_last - t * KT + 32) >> 5, KT / 32);
    int kb = ks;
#pragma unroll 1
    for (; BF16 && kb + KS < full; kb += 2 * KS) blocks(std::integral_constant<int, 2>{}, std::false_type{}, t, kb);
    if constexpr (!BF16) {
#pragma unroll 1
      for (; kb < full; kb += KS) blocks(std::integral_constant<int, 1>{}, std::false_type{}, t, kb);
    }
#pragma unroll 1
    for (; BF16 && kb + KS < seen; kb += 2 * KS) blocks(std::integral_constant<int, 2>{}, std::true_type{}, t, kb);
#pragma unroll 1
    for (; kb < seen; kb += KS) blocks(std::integral_constant<int, 1>{}, std::true_type{}, t, kb);
  }

  store_rows<BF16, D, KS>(a, w, o, m, z, reinterpret_cast<float *>(lds_kv));
}

template <bool BF16, int D, int KS, bool SCORED>
hipError_t launch_prompt_t(const KernelArgs<PromptArgs> &k, unsigned grid, hipStream_t stream) {
  const size_t tiles = 2 * (size_t)(KeyTile<BF16, D>::kChunks + ValueTile<BF16, D, KeyTile<BF16, D>::kRows>::kChunks) * 16;
  const size_t outputs = (size_t)kPromptWaves * 32 * (D + 4) * sizeof(float);
  const size_t lds = tiles > outputs ? tiles : outputs;
  const hipError_t e = allow_full_lds<prompt_attention_kernel<BF16, D, KS, SCORED>>();
  if (e != hipSuccess) return e;
  ProfScope ps(stream, KID_PROMPT_ATTENTION);
  prompt_attention_kernel<BF16, D, KS, SCORED><<<dim3(grid), kPThreads, lds, stream>>>(k);
  return hipGetLastError();
}

template <bool BF16, int D>
hipError_t launch_prompt_d(const KernelArgs<PromptArgs> &k, unsigned grid, hipStream_t stream) {
  const bool scored = k.a.score.cap > 0.f || k.a.score.slopes;
  switch (k.a.ksplit) {
    case 4: return scored ? launch_prompt_t<BF16, D, 4, true>(k, grid, stream) : launch_prompt_t<BF16, D, 4, false>(k, grid, stream);
    case 2: return scored ? launch_prompt_t<BF16, D, 2, true>(k, grid, stream) : launch_prompt_t<BF16, D, 2, false>(k, grid, stream);
    default: return scored ? launch_prompt_t<BF16, D, 1, true>(k, grid, stream) : launch_prompt_t<BF16, D, 1, false>(k, grid, stream);
  }
}

}  // namespace

hipError_t launch_prompt_attention(const PromptArgs &args, const int *words, int n_words, hipStream_t stream) {
  PromptArgs a = args;
  const int units = a.n_layers * a.Hkv;
  const long long grid = (long long)units * a.wgs_total;
  if (grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  a.group = (kPromptGroupWgs / a.wgs_total + 31) / 32 * 32;
  if (a.group < 32) a.group = 32;
  const int groups = units / a.group;
  a.group = groups > 1 ? ((units + groups - 1) / groups + 7) / 8 * 8 : units;
  KernelArgs<PromptArgs> k;
  fill_kernel_args(k, a, words, n_words);
  if (a.bf16) return a.d == 128 ? launch_prompt_d<true, 128>(k, (unsigned)grid, stream) : launch_prompt_d<true, 64>(k, (unsigned)grid, stream);
  return a.d == 128 ? launch_prompt_d<false, 128>(k, (unsigned)grid, stream) : launch_prompt_d<false, 64>(k, (unsigned)grid, stream);
}

}  // namespace flowmm
