// One step of attention over a cache with head room, o = softmax(score(q K^T)) V over the valid rows of every sequence: rows as they are
// (bf16, fp32) or e4m3 codes with a scale per block of 32 (flowmm_cache_attention, flowmm_cache_attention_quantized).
//
// What bounds it is the stream of K and V rows: 2 * d bytes a row in 8 bits, two and four times that in bf16 and fp32; the products of
// up to 16 query heads with a row take a tenth of the time in which it arrives.  32 sequences of up to 16384 rows in 8 bits, 4 layers x 32/8 heads: 496 us,
// 5.7 TB/s of the 5.9 that plain reads reach here; 3688 bf16 rows of 32 x 32/8 heads: 89 us, 5.5 TB/s.  Small calls are trips to memory one after the other:
// 450 rows of 28 x 28/4, 13 MB, 8.1 us.  fp32 rows (4 sequences of up to 900, 8 layers x 16/4 heads, 64 channels: 16.5 us) also wait for their 32 products of 16x16x4 a tile.  Every wave works through tiles of 16 or 32 rows of its
// own, with one K and one V buffer in LDS that it refills by direct global->LDS loads (whole rows, no registers) as soon as the matrix
// operands have been read out of them, and no barrier until the end.
//   logits  : S[key][head] = K tile x queries.  Which channels share a k slot of the instruction is free as long as both operands agree:
//             lane (n, q4) takes the 16-byte chunks 4 j + q4 of row n, so that every LDS read is 16 bytes
//               codes: 16 of them, two v_mfma 16x16x32 after v_cvt_scalef32_pk_bf16_fp8 with the block's scale (exact); fp32 queries as three bf16 terms
//               bf16 : 8 channels, one 16x16x32;  fp32: 4 channels, four 16x16x4
//   scores  : scale, cap, bias by distance in fp32, log2 domain
//   output  : O[channel][head] += V^T x p, p at the accuracy of the result: the two leading bf16 terms (short of 2^-15) for bf16 results, three
//             for fp32 ones, fp32 itself beside fp32 rows.  V comes out of LDS transposed
//             (ds_read_b64_tr_b8, _tr_b16), in the order of keys in which the accumulators of S hold p.
// Rows past a sequence's end are read as its last one; their p is 0 and so are their V, whatever that row holds.
#include <cfloat>
#include <cmath>

#include "attention_core.h"
#include "decode_core.h"
#include "fp8_core.h"
#include "kernels.h"
#include "profile.h"

namespace flowmm {

namespace {

constexpr int kAHeads = 16;  // query heads of a kv group per launch

template <int R, int D>
struct RowCfg {
  static constexpr int kElemBytes = R == kRowFp8 ? 1 : R == kRowBF16 ? 2 : 4;
  static constexpr int NCH = D * kElemBytes / 16;        // chunks of a row
  static constexpr int kRows = R == kRowFp8 ? 32 : 16;   // of a tile (codes: a block)
  static constexpr int kSubs = kRows / 16;
  static constexpr int kLoads = kRows * NCH / 64;        // load instructions per tile
  static constexpr int kChunks = kRows * NCH;
};

typedef __attribute__((ext_vector_type(2))) int i32x2_t;
typedef __attribute__((address_space(3))) i32x2_t lds_i32x2_t;

// A block's scale as power * rest: the conversion of its codes takes the power of two along (exact, down to the smallest bf16 numbers), so that neither a
// product with the queries nor a weight leaves the range of its type where the rows themselves do not.  The rest goes into logits and weights: 1 for
// the powers of two that are written here, but 2 for the largest, 2^120, which would bring codes from 256 on (numbers that e4m3 rounded up, beyond the largest float) to infinity.
struct BlockScale { float power, rest; };
__device__ __forceinline__ BlockScale block_scale(int bits) {
  const int e = min(max(bits >> 23 & 255, 7), 246);  // 2^-120 .. 2^119
  return {__int_as_float(e << 23), __int_as_float(bits) * __int_as_float((254 - e) << 23)};
}

// eight e4m3 numbers times a power of two as bf16
__device__ __forceinline__ bf16x8_t fp8_to_bf16(unsigned w0, unsigned w1, float power) {
  const bf16x2_t p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, power, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, power, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, power, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, power, true)};
  bf16x8_t v;
  __builtin_memcpy(&v, p, 16);
  return v;
}

// the rows of a tile, n of them, the last one in the place of those behind it: chunk c of row r at slot c ^ (r % NCH)
template <int R, int D>
__device__ __forceinline__ void request_rows(const uint4 *src, long long stride, int n, uint4 *tile) {
  using RC = RowCfg<R, D>;
  constexpr int RPI = 64 / RC::NCH;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < RC::kLoads; ++j) {
    const int r = j * RPI + lane / RC::NCH, ch = (lane % RC::NCH) ^ (r % RC::NCH);
    load_to_lds<16>(src, ((unsigned)min(r, n - 1) * (unsigned)stride + (unsigned)ch) * 16u, tile + j * 64);
  }
}

// term k (the bf16 numbers in the upper halves) of four floats
__device__ __forceinline__ s16x4_t pack_upper(const unsigned (&v)[4]) {
  uint2 w = make_uint2(__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u));
  s16x4_t r;
  __builtin_memcpy(&r, &w, 8);
  return r;
}

// a task per workgroup (decode_task)
template <int R, bool QBF16, int D, int WAVES, bool POS, bool ORDERED>
__global__ __launch_bounds__(WAVES * 64, R == kRowF32 ? 2 : 4) void cache_attention_kernel(CacheAttnArgs a) {
  using RC = RowCfg<R, D>;
  constexpr int NCH = RC::NCH, TR = RC::kRows, SUBS = RC::kSubs, DT = D / 16;
  constexpr int kKLoads = RC::kLoads + (POS ? 1 : 0), kVLoads = RC::kLoads;
  constexpr int kTerms = QBF16 ? 2 : 3;  // of p
  constexpr int KJ = NCH / 4;  // chunks of a row in a lane
  extern __shared__ __align__(16) uint4 lds_rows[];  // [waves] K tile, V tile, positions; at the end the waves' states
  const DecodeTask task = decode_task<ORDERED>(a);
  const int b = task.b, x = task.x, gkv = task.gkv, l = task.l, len = task.B, s0 = task.s0, s1 = task.s1;
  const auto &s = a.cu[b];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, q4 = lane >> 4;
  const long long unit = (long long)l * a.Hkv + gkv;
  const long long seq_at = l * a.ks_layer + gkv * a.ks_head + (long long)s.row * a.ks_tok;
  const uint4 *Kc = reinterpret_cast<const uint4 *>(a.K_c) + seq_at, *Vc = reinterpret_cast<const uint4 *>(a.V_c) + seq_at;
  constexpr int kWaveChunks = 2 * RC::kChunks + (POS ? 16 : 0);
  uint4 *tk = lds_rows + wave * kWaveChunks, *tv = tk + RC::kChunks;
  int *tp = reinterpret_cast<int *>(tv + RC::kChunks);
  const int nh = min(kAHeads, a.G - a.g0);
  const int head0 = l * a.Hq + gkv * a.G + a.g0;  // first query head of this launch

  // ---- the queries, as the K rows' chunks want them ----
  constexpr int kQ = R == kRowFp8 ? 2 * KJ : KJ;  // fragments of a row
  bf16x8_t qb[R == kRowF32 ? 1 : kQ][QBF16 ? 1 : 3];
  float qf[R == kRowF32 ? kQ : 1][4];
  {
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const long long qrow = ((long long)(head0 + n) * a.batch + a.b0 + b) * D;
#pragma unroll
    for (int f = 0; f < kQ; ++f) {
      if constexpr (R == kRowF32) {
        const uint4 c = n < nh ? reinterpret_cast<const uint4 *>(reinterpret_cast<const float *>(a.q) + qrow)[4 * f + q4] : zero;
        chunk_to_floats<false>(c, qf[f]);
      } else {
        const int ch = R == kRowBF16 ? 8 * (4 * f + q4) : 16 * (4 * (f >> 1) + q4) + 8 * (f & 1);  // first of eight channels
        if constexpr (QBF16) {
          const uint4 c = n < nh ? *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(a.q) + qrow + ch) : zero;
          __builtin_memcpy(&qb[f][0], &c, 16);
        } else {
          const uint4 *c = reinterpret_cast<const uint4 *>(reinterpret_cast<const float *>(a.q) + qrow + ch);
          const Split8 t = split8(n < nh ? c[0] : zero, n < nh ? c[1] : zero);
#pragma unroll
          for (int k = 0; k < 3; ++k) qb[f][k] = t.t[k];
        }
      }
    }
  }
  const float slope = a.score.slopes && n < nh ? a.score.slopes[gkv * a.G + a.g0 + n] * 1.4426950408889634f : 0.f;
  __builtin_amdgcn_s_waitcnt(0);  // the counts below are of tile loads alone

  f32x4_t acc[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // of head n; z over this lane's keys only.  The maximum starts finite: rows whose logit is -inf weigh 0, not NaN, also where a wave sees no others (a query that sees no others gets 0 / 0)
  float m = -FLT_MAX, z = 0.f;
  const int step = WAVES * TR;
  int r0 = s0 + wave * TR;
  const int *pos = POS ? a.row_pos + unit * a.SB + s.slot : nullptr;
  auto request_k = [&](int r) {
    if constexpr (POS) {
      const int first = min(r, s.merged - 1);  // (offsets of 32 bits from the tile's first position)
      load_to_lds<4>(pos + first, (unsigned)min(lane & (TR - 1), s.merged - 1 - first) * 4u, tp);
    }
    request_rows<R, D>(Kc + (long long)r * a.ks_tok, a.ks_tok, s1 - r, tk);
  };
  auto request_v = [&](int r) { request_rows<R, D>(Vc + (long long)r * a.ks_tok, a.ks_tok, s1 - r, tv); };
  const long long scale_at = unit * a.NB + s.block;
  if (r0 < s1) {
    request_k(r0);
    request_v(r0);
  }
  for (; r0 < s1; r0 += step) {
    const bool more = r0 + step < s1;
    BlockScale kscale, vscale;
    if constexpr (R == kRowFp8) {
      kscale = block_scale(scalar_ints(reinterpret_cast<const int *>(a.k_scales))[scale_at + r0 / kQuantRows]);
      vscale = block_scale(scalar_ints(reinterpret_cast<const int *>(a.v_scales))[scale_at + r0 / kQuantRows]);
    }
    wait_loads<kVLoads>();  // the K tile is there, the V tile may still be on its way
    uint4 kf[SUBS][KJ];
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int j = 0; j < KJ; ++j) kf[u][j] = tk[(16 * u + n) * NCH + ((4 * j + q4) ^ (n % NCH))];
    int4 at[SUBS];
    if constexpr (POS) {
#pragma unroll
      for (int u = 0; u < SUBS; ++u) at[u] = *reinterpret_cast<const int4 *>(tp + 16 * u + 4 * q4);
    }
    wait_lds();
    if (more) request_k(r0 + step);
    f32x4_t p[SUBS];
#pragma unroll
    for (int u = 0; u < SUBS; ++u) {
      f32x4_t sc = {0.f, 0.f, 0.f, 0.f};  // [key 4 q4 + i][head n]
#pragma unroll
      for (int j = 0; j < KJ; ++j) {
        const uint4 c = kf[u][j];
        if constexpr (R == kRowF32) {
          sc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(c.x), qf[j][0], sc, 0, 0, 0);
          sc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(c.y), qf[j][1], sc, 0, 0, 0);
          sc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(c.z), qf[j][2], sc, 0, 0, 0);
          sc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(c.w), qf[j][3], sc, 0, 0, 0);
        } else if constexpr (R == kRowBF16) {
          bf16x8_t k;
          __builtin_memcpy(&k, &c, 16);
          sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qb[j][0], sc, 0, 0, 0);
        } else {
          const bf16x8_t k0 = fp8_to_bf16(c.x, c.y, kscale.power), k1 = fp8_to_bf16(c.z, c.w, kscale.power);
#pragma unroll
          for (int t = (QBF16 ? 1 : 3) - 1; t >= 0; --t) {
            sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qb[2 * j][t], sc, 0, 0, 0);
            sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qb[2 * j + 1][t], sc, 0, 0, 0);
          }
        }
      }
      p[u] = sc;
    }
#pragma unroll
    for (int u = 0; u < SUBS; ++u) {
      if constexpr (R == kRowFp8) p[u] *= kscale.rest;
      if (a.score.cap > 0.f) {
        if (!QBF16 || a.score.fine) {
#pragma unroll
          for (int i = 0; i < 4; ++i) p[u][i] = capped<true>(a.score, p[u][i]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) p[u][i] = capped<false>(a.score, p[u][i]);
        }
      } else {
        p[u] *= a.score.cl;
      }
      if (a.score.slopes) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = r0 + 16 * u + 4 * q4 + i;
          int far = len - 1 - r;
          if constexpr (POS) {
            const int pr[4] = {at[u].x, at[u].y, at[u].z, at[u].w};
            far = r < s.merged ? abs(s.q_pos - pr[i]) : far;
          }
          p[u][i] = fmaf(-slope, (float)far, p[u][i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) p[u][i] = r0 + 16 * u + 4 * q4 + i < s1 ? p[u][i] : -INFINITY;
    }
    float mt = fmaxf(fmaxf(p[0][0], p[0][1]), fmaxf(p[0][2], p[0][3]));
    if constexpr (SUBS == 2) mt = fmaxf(mt, fmaxf(fmaxf(p[1][0], p[1][1]), fmaxf(p[1][2], p[1][3])));
    mt = quad_max(mt);
    if (__any(mt > m)) {  // some head has a new maximum
      const float M = fmaxf(m, mt), f = fast_exp2(m - M);
      z *= f;
#pragma unroll
      for (int t = 0; t < DT; ++t) acc[t] *= f;
      m = M;
    }
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[u][i] = fast_exp2(p[u][i] - m);
        z += p[u][i];
        if constexpr (R == kRowFp8) p[u][i] *= vscale.rest;
      }
    if (more) wait_loads<kKLoads>(); else wait_loads<0>();  // the V tile is there
    const int left = s1 - r0 - 4 * q4;  // this lane's key i (of the second half: 16 + i) is a row while i < left

    if constexpr (R == kRowF32) {
      float vf[DT][4];
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * q4 + i;
          vf[t][i] = reinterpret_cast<const float *>(tv + r * NCH + ((4 * t + (n >> 2)) ^ (r % NCH)))[n & 3];
        }
      wait_lds();
      if (more) request_v(r0 + step);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < DT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(i < left ? vf[t][i] : 0.f, p[0][i], acc[t], 0, 0, 0);  // [channel 16 t + 4 q4 + i][head n]
      continue;
    }
    // p as bf16 terms, each the truncation of what the terms before it leave (the differences are exact)
    unsigned term[SUBS][kTerms][4];
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float rest = p[u][i];
#pragma unroll
        for (int k = 0; k < kTerms; ++k) {
          // (bf16 rows may be infinite: a term of 0 would make NaN of them where the weight is not 0)
          if (R == kRowBF16 && k > 0) rest = at_least_a_term(rest, term[u][0][i]);
          term[u][k][i] = __float_as_uint(rest) & (k + 1 < kTerms ? 0xffff0000u : 0xffffffffu);
          if (k + 1 < kTerms) rest -= __uint_as_float(term[u][k][i]);
        }
      }
    if constexpr (R == kRowBF16) {
      s16x4_t vf[DT];
      const int vr = 4 * q4 + (n >> 2);  // this lane's row of the 4 x 16 block that its 16 lanes transpose
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const char *from = reinterpret_cast<const char *>(tv + vr * NCH + ((2 * t + ((n & 3) >> 1)) ^ (vr % NCH))) + 8 * (n & 1);
        vf[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)from);
      }
      wait_lds();
      if (more) request_v(r0 + step);
      if (r0 + TR > s1) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) vf[t][i] = i < left ? vf[t][i] : (short)0;
      }
#pragma unroll
      for (int k = 0; k < kTerms; ++k) {
        const s16x4_t pk = pack_upper(term[0][k]);
#pragma unroll
        for (int t = 0; t < DT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vf[t], pk, acc[t], 0, 0, 0);
      }
    } else if constexpr (R == kRowFp8) {
      i32x2_t vf[DT];
      // this lane's row of the 8 x 16 block that its 16 lanes transpose: keys 4 q4 + 0..3 of either half of the tile
      const int vr = 4 * q4 + ((n >> 1) & 3) + 16 * (n >> 3);
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const char *from = reinterpret_cast<const char *>(tv + vr * NCH + (t ^ (vr % NCH))) + 8 * (n & 1);
        vf[t] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2_t *)from);
      }
      wait_lds();
      if (more) request_v(r0 + step);
      if (r0 + TR > s1) {  // bytes of rows that are not there: 0
        const unsigned m0 = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : 0xffffffffu >> (8 * (4 - left));
        const unsigned m1 = left >= 20 ? 0xffffffffu : left <= 16 ? 0u : 0xffffffffu >> (8 * (20 - left));
#pragma unroll
        for (int t = 0; t < DT; ++t) vf[t] = i32x2_t{(int)((unsigned)vf[t][0] & m0), (int)((unsigned)vf[t][1] & m1)};
      }
      bf16x8_t pk[kTerms];
#pragma unroll
      for (int k = 0; k < kTerms; ++k) {
        const s16x4_t lo = pack_upper(term[0][k]), hi = pack_upper(term[SUBS - 1][k]);
        __builtin_memcpy(&pk[k], &lo, 8);
        __builtin_memcpy(reinterpret_cast<char *>(&pk[k]) + 8, &hi, 8);
      }
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const bf16x8_t v = fp8_to_bf16((unsigned)vf[t][0], (unsigned)vf[t][1], vscale.power);
#pragma unroll
        for (int k = 0; k < kTerms; ++k) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pk[k], acc[t], 0, 0, 0);
      }
    }
  }
  z = quad_sum(z);

  // the waves' states, folded in wave order
  __syncthreads();  // nobody reads tiles any more
  float *st = reinterpret_cast<float *>(lds_rows);  // [waves][nh][D + 4]: O, then m, z
  constexpr int SS = D + 4;
  if (n < nh) {
    float *mine = st + (wave * nh + n) * SS;
#pragma unroll
    for (int t = 0; t < DT; ++t) *reinterpret_cast<float4 *>(mine + 16 * t + 4 * q4) = make_float4(acc[t][0], acc[t][1], acc[t][2], acc[t][3]);
    if (q4 == 0) { mine[D] = m; mine[D + 1] = z; }
  }
  __syncthreads();
  const bool whole = len <= a.chunk;
  for (int idx = threadIdx.x; idx < nh * D; idx += WAVES * 64) {
    const int h = idx / D, ci = idx - h * D;
    float M = -FLT_MAX;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) M = fmaxf(M, st[(w * nh + h) * SS + D]);
    float zz = 0.f, av = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float *o = st + (w * nh + h) * SS;
      const float f = fast_exp2(o[D] - M);  // 0 for a wave that had no tile
      zz = fmaf(o[D + 1], f, zz);
      av = fmaf(o[ci], f, av);
    }
    if (whole) {
      const float o = len > 0 ? av / zz : 0.f;
      const long long to = ((long long)(head0 + h) * a.batch + a.b0 + b) * D + ci;
      if constexpr (QBF16) reinterpret_cast<uint16_t *>(a.out)[to] = (uint16_t)float_to_bf16_bits(o);
      else reinterpret_cast<float *>(a.out)[to] = o;
    } else {
      float *part = a.part + ((long long)(head0 + h) * a.tasks + x) * (D + 2);
      part[ci] = av;
      if (ci == 0) { part[D] = M; part[D + 1] = zz; }
    }
  }
}

// out[l][h][b] of the sequences that several workgroups have worked on.  Lane i weighs part i (there are 64 at most); then the parts are added up in row order, eight
// loads at a time (one dependent fold after the other took 0.25 us a part).
template <bool QBF16, int D>
__global__ __launch_bounds__(D) void cache_attention_combine_kernel(CacheAttnArgs a) {
  static_assert(kCacheAttnMostParts <= 64, "a lane for every part");
  const int b = blockIdx.x;
  const int x0 = a.cu[b].task & 0xffff, n = (a.cu[b + 1].task & 0xffff) - x0;
  if (n < 2) return;
  const long long head = (long long)blockIdx.z * a.Hq + blockIdx.y;
  const int ci = threadIdx.x, lane = threadIdx.x & 63;
  const float *part = a.part + (head * a.tasks + x0) * (D + 2);
  const float m = lane < n ? part[lane * (D + 2) + D] : -INFINITY, z = lane < n ? part[lane * (D + 2) + D + 1] : 0.f;
  float M = m;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  const float w = fast_exp2(m - M), zz = wave_sum(z * w);  // (M is finite: no part's maximum is below the lowest float)
  float av = 0.f;
  for (int i = 0; i < n; i += 8) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = part[min(i + k, n - 1) * (D + 2) + ci];
#pragma unroll
    for (int k = 0; k < 8; ++k) av = i + k < n ? fmaf(v[k], __shfl(w, i + k, 64), av) : av;
  }
  const float o = av / zz;
  const long long at = (head * a.batch + a.b0 + b) * D + ci;
  if constexpr (QBF16) reinterpret_cast<uint16_t *>(a.out)[at] = (uint16_t)float_to_bf16_bits(o);
  else reinterpret_cast<float *>(a.out)[at] = o;
}

template <int R, bool QBF16, int D, int WAVES>
hipError_t launch_waves(const CacheAttnArgs &a, int n_layers, hipStream_t stream) {
  using RC = RowCfg<R, D>;
  const int nh = a.G - a.g0 < kAHeads ? a.G - a.g0 : kAHeads;
  size_t lds = (size_t)WAVES * (2 * RC::kChunks + (a.row_pos ? 16 : 0)) * 16;
  const size_t states = (size_t)WAVES * nh * (D + 4) * sizeof(float);
  if (states > lds) lds = states;
  const hipError_t e = allow_full_lds<cache_attention_kernel<R, QBF16, D, WAVES, false, false>, cache_attention_kernel<R, QBF16, D, WAVES, true, false>,
                                      cache_attention_kernel<R, QBF16, D, WAVES, false, true>, cache_attention_kernel<R, QBF16, D, WAVES, true, true>>();
  if (e != hipSuccess) return e;
  ProfScope ps(stream, KID_CACHE_ATTENTION);
  if (a.mixed < 0) {
    const dim3 grid(a.tasks, a.Hkv, n_layers);
    if (a.row_pos) cache_attention_kernel<R, QBF16, D, WAVES, true, false><<<grid, WAVES * 64, lds, stream>>>(a);
    else cache_attention_kernel<R, QBF16, D, WAVES, false, false><<<grid, WAVES * 64, lds, stream>>>(a);
  } else {
    const dim3 grid(a.Hkv, n_layers, a.tasks);
    if (a.row_pos) cache_attention_kernel<R, QBF16, D, WAVES, true, true><<<grid, WAVES * 64, lds, stream>>>(a);
    else cache_attention_kernel<R, QBF16, D, WAVES, false, true><<<grid, WAVES * 64, lds, stream>>>(a);
  }
  return hipGetLastError();
}

constexpr int kMostWaves = 8;

template <int R, bool QBF16, int D>
hipError_t launch_rows(CacheAttnArgs a, int n_layers, hipStream_t stream) {
  for (a.g0 = 0; a.g0 < a.G; a.g0 += kAHeads) {
    const hipError_t e = a.waves == 2 ? launch_waves<R, QBF16, D, 2>(a, n_layers, stream) : a.waves == 4 ? launch_waves<R, QBF16, D, 4>(a, n_layers, stream) : launch_waves<R, QBF16, D, kMostWaves>(a, n_layers, stream);
    if (e != hipSuccess) return e;
  }
  if (a.tasks > a.n_seqs) {
    ProfScope ps(stream, KID_CACHE_ATTENTION_COMBINE);
    cache_attention_combine_kernel<QBF16, D><<<dim3(a.n_seqs, a.Hq, n_layers), D, 0, stream>>>(a);
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_dim(const CacheAttnArgs &a, const CacheAttnCall &c, hipStream_t stream) {
  if (c.rows == kRowF32) return launch_rows<kRowF32, false, D>(a, c.n_layers, stream);
  if (c.rows == kRowBF16) return launch_rows<kRowBF16, true, D>(a, c.n_layers, stream);
  return c.bf16 ? launch_rows<kRowFp8, true, D>(a, c.n_layers, stream) : launch_rows<kRowFp8, false, D>(a, c.n_layers, stream);
}

// Rows of a task and waves of a workgroup for the sequences of a launch.
//
// A workgroup alone on its compute unit takes a trip of its eight waves over its rows in `trip` us (measured at 128 channels; 0.8 of it at 64); 224 of them (fp32 256)
// reach the memory's rate.  Fewer (counted as sequences of the longest one's length) are cut into about as many parts, if the trips saved are worth the second
// launch, 2.4 us and 0.25 a part, and into no more than the square root that balances the two.  Over 324 shapes of 1 to 512 units x 64 to 16000 equal rows this is
// 1 % from the best of all cuts on average, over 75 unequal batches 2 %.  us, whole / cut: codes 112 units x 16000 rows 97 / 85 in two, x 1800 16.4 / 17.2; 64 x 8000
// 46 / 30 in three; 16 x 3600 21.6 / 11.3 in six; 1 x 16000 80 / 16 in sixteen, x 450 6.5 / 7.7 in two; bf16 112 x 3600 47 / 42, 32 x 8000 77 / 31 in six, 256 x 900
// 25.1 / 30.1; fp32 112 x 450 18.9 / 16.7, 32 x 900 30 / 14 in six.
// Short sequences: where there are enough workgroups, fewer waves leave room for more of them (8 / 4 / 2 waves, codes 256 units x 64 rows 5.2 / - / 4.6, x 256 9.2 / 6.5 / -,
// 512 x 450 16.9 / 15.6 / -; bf16 512 x 256 17.5 / - / 16.1; fp32 512 x 256 30.4 / 27.5 / 31.3, 16 x 900 uncut 25.8 / 30.4 / 53.5).
void choose_tasks(CacheAttnArgs &a, const CacheAttnCall &c, const int *len) {
  long long sum = 0;
  int longest = 0;
  for (int i = 0; i < a.n_seqs; ++i) {
    sum += len[i];
    if (len[i] > longest) longest = len[i];
  }
  const long long units = (long long)c.n_layers * a.Hkv, wgs = units * a.n_seqs;
  const int tile = c.rows == kRowFp8 ? 32 : 16, rows = kMostWaves * tile;
  const float trip = (c.rows == kRowFp8 ? 1.25f : c.rows == kRowBF16 ? 0.7f : 1.8f) * (c.d == 64 ? 0.8f : 1.f);
  if (c.rows == kRowF32) a.waves = wgs >= 256 || longest <= 16 * tile ? 4 : kMostWaves;
  else a.waves = (wgs >= 64 && longest <= 2 * tile) || (wgs >= 256 && longest <= 4 * tile) ? 2 : wgs >= 256 && longest <= 28 * tile ? 4 : kMostWaves;
  long long chunk = longest;
  if (longest > kCacheAttnLeastPart) {
    const float room = c.rows == kRowF32 ? 256.f : 224.f;
    int parts = (int)(room * longest / ((float)units * sum) + 0.45f), balance = (int)std::sqrt((float)longest / rows * trip * 4.f);
    if (parts > balance) parts = balance;
    if (parts > kCacheAttnMostParts) parts = kCacheAttnMostParts;
    if (parts > 1) {
      const long long part = (longest + parts - 1) / parts;
      const int passes = (a.G + kAHeads - 1) / kAHeads;
      const long long saved = (longest + rows - 1) / rows - (part + rows - 1) / rows;
      if ((float)(saved * passes) * trip > 2.4f + 0.25f * parts) chunk = part;
    }
    // what the workspace has room for
    long long least = (sum * units + kCacheAttnTasks - 1) / kCacheAttnTasks;
    if (least < longest / kCacheAttnMostParts + 1) least = longest / kCacheAttnMostParts + 1;
    if (least < kCacheAttnLeastPart) least = kCacheAttnLeastPart;
    if (chunk < least) chunk = least;
  }
  if (chunk < kQuantRows) chunk = kQuantRows;
  a.chunk = (int)((chunk + kQuantRows - 1) / kQuantRows * kQuantRows);
}

}  // namespace

hipError_t launch_cache_attention(CacheAttnArgs a, const CacheAttnCall &c, hipStream_t stream) {
  int block = 0, slot = 0;
  for (a.b0 = 0; a.b0 < a.batch; a.b0 += kDecodeSeqs) {
    a.n_seqs = a.batch - a.b0 < kDecodeSeqs ? a.batch - a.b0 : kDecodeSeqs;
    const int *len = c.lengths + a.b0;
    choose_tasks(a, c, len);
    a.tasks = 0;
    long long sum = 0;
    int longest = 0;
    for (int i = 0; i < a.n_seqs; ++i) {
      const int b = a.b0 + i;
      const int merged = a.row_pos ? c.budgets[b] : 0;
      a.cu[i] = CacheAttnArgs::Seq{a.tasks, len[i], c.cu_capacity[b], block, merged, slot, a.row_pos ? c.q_pos[b] : 0, 0};
      a.tasks += len[i] <= a.chunk ? 1 : (len[i] - 1) / a.chunk + 1;  // (a length and a part's may add up to more than an int holds)
      block += (c.cu_capacity[b + 1] - c.cu_capacity[b] + kQuantRows - 1) / kQuantRows;
      slot += merged;
      sum += len[i];
      if (len[i] > longest) longest = len[i];
    }
    a.cu[a.n_seqs] = CacheAttnArgs::Seq{a.tasks, 0, 0, 0, 0, 0, 0, 0};
    // An order of their own for unequal sequences' tasks, where that can matter (as decode attention, in tiles of the most waves)
    const int units = a.Hkv * c.n_layers, tile = c.rows == kRowFp8 ? 32 : 16;
    const long long wgs = (long long)units * a.tasks, above = wgs <= 1024 ? kMostWaves * tile : tile;
    if (wgs > 256 && longest * (long long)a.n_seqs - sum >= above * a.n_seqs) order_tasks(a, len, units);
    else a.mixed = -1;
    const hipError_t e = c.d == 128 ? launch_dim<128>(a, c, stream) : launch_dim<64>(a, c, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace flowmm
