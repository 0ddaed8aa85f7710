// The compacted cache in 8 bits: rows to e4m3 codes with a power of two per block of 32 rows, back, and the append of one token's row.
//   k = the smallest integer >= -120 with max |x| <= 448 * 2^k over the block's finite numbers, code = e4m3(x * 2^-k), x ~ code * 2^k
// Powers of two: a floating code loses nothing by them (its steps are relative), x * 2^-k is exact, and a scale that an appended row
// raises takes the block's older codes along by a shift of their exponents, exact but for what falls below e4m3's smallest normal number.
// All three are bound by memory: every row is read once and every code written once.  A wave has a whole block in registers (8 to 32 KB of loads of 16 bytes in
// flight, no LDS, no barrier), so that it needs neither a second read for the rounding nor another wave for the maximum.  8 sequences of up to 4096 rows in 32 layers
// x 8 heads, bf16: 588 us, 5.3 TB/s (read and written; a copy reaches 4.83, plain reads 5.9).  410 rows of 28 layers x 4 heads: 10.2 us, as much as 35 MB take at that
// rate and the 2.5 us in which a grid starts and ends.  The way back, 1023 rows of 32 x 8: 41 us.  An append is one launch: 2.6 us on the GPU, 6.7 with the call.
#include "fp8_core.h"
#include "kernels.h"
#include "profile.h"

namespace flowmm {

namespace {

constexpr int kQuantWaves = 4;

__device__ __forceinline__ unsigned wave_max(unsigned v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, o, 64));
  return v;
}

// the sequence of the launch that block x belongs to (sequences without blocks have none)
__device__ __forceinline__ int seq_of_block(const QuantArgs &a, int x) {
  int lo = 0, hi = a.n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.seq[mid].first <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// grid (blocks of the launch, 4 a workgroup; 2 x kv heads; layers): a wave quantises one block of K or of V, its rows in registers between
// the maximum and the rounding
template <bool BF16, int D>
__global__ __launch_bounds__(kQuantWaves * 64) void cache_quantize_kernel(QuantArgs a) {
  constexpr int NCH = Cfg<BF16, D>::NCH, EPC = Cfg<BF16, D>::kElemsPerChunk, RPI = 64 / NCH, N = kQuantRows / RPI;
  const int x = blockIdx.x * kQuantWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (x >= a.blocks) return;
  const int lane = threadIdx.x & 63, tensor = blockIdx.y & 1, g = blockIdx.y >> 1, l = blockIdx.z;
  const int b = seq_of_block(a, x), blk = x - a.seq[b].first, r0 = blk * kQuantRows, n = min(kQuantRows, a.seq[b].len - r0);
  const uint4 *src = reinterpret_cast<const uint4 *>(tensor ? a.V_rows : a.K_rows) + l * a.ks_layer + g * a.ks_head + (a.seq[b].row + (long long)r0) * a.ks_tok + lane % NCH;
  uint4 c[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = i * RPI + lane / NCH;
    c[i] = r < n ? src[r * a.ks_tok] : make_uint4(0, 0, 0, 0);
  }
  unsigned most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float f[EPC];
    chunk_to_floats<BF16>(c[i], f);
#pragma unroll
    for (int e = 0; e < EPC; ++e) most = max(most, finite_magnitude(f[e]));
  }
  const int k = block_exponent(wave_max(most));
  if (lane == 0) (tensor ? a.v_scales : a.k_scales)[((long long)l * a.Hkv + g) * a.NB + a.seq[b].block + blk] = power_of_two(k);
  const float inv = power_of_two(-k);
  char *dst = reinterpret_cast<char *>(tensor ? a.v_codes : a.k_codes) + l * a.cs_layer + g * a.cs_head + (a.seq[b].code_row + (long long)r0) * a.cs_tok + lane % NCH * EPC;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = i * RPI + lane / NCH;
    float f[EPC];
    chunk_to_floats<BF16>(c[i], f);
#pragma unroll
    for (int e = 0; e < EPC; ++e) f[e] = fp8_range(f[e] * inv);
    if (r >= n) continue;
    if constexpr (BF16) *reinterpret_cast<uint2 *>(dst + r * a.cs_tok) = make_uint2(pack_fp8(f[0], f[1], f[2], f[3]), pack_fp8(f[4], f[5], f[6], f[7]));
    else *reinterpret_cast<unsigned *>(dst + r * a.cs_tok) = pack_fp8(f[0], f[1], f[2], f[3]);
  }
}

// the same grid: a wave brings one block back
template <bool BF16, int D>
__global__ __launch_bounds__(kQuantWaves * 64) void cache_dequantize_kernel(QuantArgs a) {
  constexpr int NCH = Cfg<BF16, D>::NCH, EPC = Cfg<BF16, D>::kElemsPerChunk, RPI = 64 / NCH, N = kQuantRows / RPI;
  const int x = blockIdx.x * kQuantWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (x >= a.blocks) return;
  const int lane = threadIdx.x & 63, tensor = blockIdx.y & 1, g = blockIdx.y >> 1, l = blockIdx.z;
  const int b = seq_of_block(a, x), blk = x - a.seq[b].first, r0 = blk * kQuantRows, n = min(kQuantRows, a.seq[b].len - r0);
  const float scale = (tensor ? a.v_scales : a.k_scales)[((long long)l * a.Hkv + g) * a.NB + a.seq[b].block + blk];
  const char *src = reinterpret_cast<const char *>(tensor ? a.v_codes : a.k_codes) + l * a.cs_layer + g * a.cs_head + (a.seq[b].code_row + (long long)r0) * a.cs_tok + lane % NCH * EPC;
  unsigned w[N][EPC / 4];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = min(i * RPI + lane / NCH, n - 1);
#pragma unroll
    for (int j = 0; j < EPC / 4; ++j) w[i][j] = reinterpret_cast<const unsigned *>(src + r * a.cs_tok)[j];
  }
  uint4 *dst = reinterpret_cast<uint4 *>(const_cast<void *>(tensor ? a.V_rows : a.K_rows)) + l * a.ks_layer + g * a.ks_head + (a.seq[b].row + (long long)r0) * a.ks_tok + lane % NCH;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = i * RPI + lane / NCH;
    float f[EPC];
#pragma unroll
    for (int j = 0; j < EPC / 4; ++j) unpack_fp8(w[i][j], f + 4 * j);
#pragma unroll
    for (int e = 0; e < EPC; ++e) f[e] *= scale;
    if (r < n) dst[r * a.ks_tok] = floats_to_chunk<BF16>(f);
  }
}

// grid (sequences of the launch, WAVES of them a workgroup; 2 x kv heads; layers): a wave places the new row of K or of V
template <bool BF16, int D, int N, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void cache_append_quantized_kernel(AppendQuantArgs<N> a, int n) {
  constexpr int EPL = D / 64;  // elements of the row in a lane
  const int b = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tensor = blockIdx.y & 1, g = blockIdx.y >> 1, l = blockIdx.z, lane = threadIdx.x & 63;
  if (b >= n) return;
  const long long unit = (long long)l * (gridDim.y >> 1) + g, at = (unit * a.batch + b) * D + lane * EPL;
  const unsigned where = a.where[b];
  const int inside = (int)(where % kQuantRows), row = a.row[b];
  float *scale = (tensor ? a.v_scales : a.k_scales) + unit * a.NB + where / kQuantRows;
  char *codes = reinterpret_cast<char *>(tensor ? a.v_codes : a.k_codes) + l * a.cs_layer + g * a.cs_head;
  float f[EPL];
  if constexpr (BF16) {
    const uint16_t *src = reinterpret_cast<const uint16_t *>(tensor ? a.v_new : a.k_new) + at;
#pragma unroll
    for (int e = 0; e < EPL; ++e) f[e] = bf16_bits_to_float(src[e]);
  } else {
    const float *src = reinterpret_cast<const float *>(tensor ? a.v_new : a.k_new) + at;
#pragma unroll
    for (int e = 0; e < EPL; ++e) f[e] = src[e];
  }
  const float had = inside ? *scale : 0.f;
  unsigned most = 0;
#pragma unroll
  for (int e = 0; e < EPL; ++e) most = max(most, finite_magnitude(f[e]));
  float sc = power_of_two(block_exponent(wave_max(most)));
  if (had >= sc) {
    sc = had;
  } else {
    if (lane == 0) *scale = sc;
    // the block's older codes to the new scale
    const float ratio = had / sc;
    for (int i = lane; i < inside * (D / 16); i += 64) {
      uint4 *p = reinterpret_cast<uint4 *>(codes + (long long)(row - inside + i / (D / 16)) * a.cs_tok) + i % (D / 16);
      uint4 v = *p;
      unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float o[4];
        unpack_fp8(w[j], o);
        w[j] = pack_fp8(o[0] * ratio, o[1] * ratio, o[2] * ratio, o[3] * ratio);
      }
      *p = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
#pragma unroll
  for (int e = 0; e < EPL; ++e) f[e] = fp8_range(f[e] / sc);
  char *dst = codes + (long long)row * a.cs_tok + lane * EPL;
  if constexpr (EPL == 2) *reinterpret_cast<uint16_t *>(dst) = (uint16_t)pack_fp8(f[0], f[1], 0.f, 0.f);
  else *dst = (char)pack_fp8(f[0], 0.f, 0.f, 0.f);
}

template <bool BF16, int D>
hipError_t launch_quant_t(const QuantArgs &a, bool back, int n_layers, hipStream_t stream) {
  const dim3 grid((a.blocks + kQuantWaves - 1) / kQuantWaves, 2 * a.Hkv, n_layers);
  ProfScope ps(stream, back ? KID_CACHE_DEQUANTIZE : KID_CACHE_QUANTIZE);
  if (back) cache_dequantize_kernel<BF16, D><<<grid, kQuantWaves * 64, 0, stream>>>(a);
  else cache_quantize_kernel<BF16, D><<<grid, kQuantWaves * 64, 0, stream>>>(a);
  return hipGetLastError();
}

template <bool BF16, int D, int N>
hipError_t launch_append_quantized_t(const AppendQuantCall &c, int b0, int n, hipStream_t stream) {
  AppendQuantArgs<N> a;
  a.k_codes = c.k_codes; a.v_codes = c.v_codes; a.k_scales = c.k_scales; a.v_scales = c.v_scales;
  const size_t skip = (size_t)b0 * D * (BF16 ? 2 : 4);
  a.k_new = reinterpret_cast<const char *>(c.k_new) + skip; a.v_new = reinterpret_cast<const char *>(c.v_new) + skip;
  a.cs_layer = c.cs_layer; a.cs_head = c.cs_head; a.cs_tok = c.cs_tok;
  a.NB = c.NB; a.batch = c.batch;
  int block = 0;
  for (int b = 0; b < b0 + n; ++b) {
    if (b >= b0) {
      a.row[b - b0] = c.cu_capacity[b] + c.lengths[b];
      a.where[b - b0] = (unsigned)block * kQuantRows + (unsigned)c.lengths[b];
    }
    block += (c.cu_capacity[b + 1] - c.cu_capacity[b] + kQuantRows - 1) / kQuantRows;
  }
  ProfScope ps(stream, KID_CACHE_APPEND_QUANTIZED);
  // (four rows a workgroup where there are many sequences, us: 64 x 256 units 9.5 -> 8.0)
  constexpr int kWaves = N > kAppendSeqsSmall ? 4 : 1;
  cache_append_quantized_kernel<BF16, D, N, kWaves><<<dim3((n + kWaves - 1) / kWaves, 2 * c.Hkv, c.n_layers), kWaves * 64, 0, stream>>>(a, n);
  return hipGetLastError();
}

template <int N>
hipError_t launch_append_quantized_n(const AppendQuantCall &c, int b0, int n, hipStream_t stream) {
  if (c.bf16) return c.d == 128 ? launch_append_quantized_t<true, 128, N>(c, b0, n, stream) : launch_append_quantized_t<true, 64, N>(c, b0, n, stream);
  return c.d == 128 ? launch_append_quantized_t<false, 128, N>(c, b0, n, stream) : launch_append_quantized_t<false, 64, N>(c, b0, n, stream);
}

}  // namespace

hipError_t launch_cache_quantize(QuantArgs a, const QuantCall &c, hipStream_t stream) {
  int block = 0;
  for (int b0 = 0; b0 < c.batch; b0 += kQuantSeqs) {
    a.n_seqs = c.batch - b0 < kQuantSeqs ? c.batch - b0 : kQuantSeqs;
    a.blocks = 0;
    for (int i = 0; i < a.n_seqs; ++i) {
      const int b = b0 + i;
      a.seq[i] = QuantArgs::Seq{a.blocks, c.lengths[b], c.cu_rows[b], c.cu_capacity[b], block};
      a.blocks += (c.lengths[b] + kQuantRows - 1) / kQuantRows;
      block += (c.cu_capacity[b + 1] - c.cu_capacity[b] + kQuantRows - 1) / kQuantRows;
    }
    if (a.blocks == 0) continue;
    const hipError_t e = c.bf16 ? (c.d == 128 ? launch_quant_t<true, 128>(a, c.back, c.n_layers, stream) : launch_quant_t<true, 64>(a, c.back, c.n_layers, stream))
                                : (c.d == 128 ? launch_quant_t<false, 128>(a, c.back, c.n_layers, stream) : launch_quant_t<false, 64>(a, c.back, c.n_layers, stream));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_cache_append_quantized(const AppendQuantCall &c, hipStream_t stream) {
  for (int b0 = 0; b0 < c.batch; b0 += kAppendSeqs) {
    const int n = c.batch - b0 < kAppendSeqs ? c.batch - b0 : kAppendSeqs;
    const hipError_t e = n <= kAppendSeqsSmall ? launch_append_quantized_n<kAppendSeqsSmall>(c, b0, n, stream) : launch_append_quantized_n<kAppendSeqs>(c, b0, n, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace flowmm
