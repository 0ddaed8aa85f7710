// What the decode-step attentions share: the order of their tasks, waits for a wave's own tiles, small reductions.
#pragma once
#include <algorithm>
#include <cstring>

#include "device_common.h"

namespace flowmm {

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// (m, z, acc) <- fold of two partial softmax states of the same query head
__device__ __forceinline__ void fold_state(float &m, float &z, float *acc, int n, float m2, float z2, const float *acc2) {
  const float M = fmaxf(m, m2);
  const float Ms = M == -INFINITY ? 0.f : M;
  const float s1 = fast_exp2(m - Ms), s2 = fast_exp2(m2 - Ms);
  z = z * s1 + z2 * s2;
  for (int e = 0; e < n; ++e) acc[e] = acc[e] * s1 + acc2[e] * s2;
  m = M;
}

template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// maximum over the lanes l, l^16, l^32, l^48
__device__ __forceinline__ float quad_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// A later bf16 term of a weight whose first one is `first` (bits): the smallest subnormal bf16, 2^-133, at the least, which the matrix cores
// keep and which times infinity is infinity; 0 where the weight is 0, whose product with the largest V has to be 0.
__device__ __forceinline__ float at_least_a_term(float rest, unsigned first) {
  return __uint_as_float(max(__float_as_uint(rest), min(first, 0x10000u)));
}

// ---- tasks: `chunk` slots of one (sequence, kv head, layer) for a workgroup ----
constexpr int kDecodeTail = 1024;  // four per compute unit (512: 0 to 3 us slower, 2048 to all: 0 to 9)

// The last sequence of the launch, lo .. hi - 1, whose task number from bit SHIFT on is not behind i.
template <int SHIFT, class A>
__device__ __forceinline__ int seq_of(const A &a, int i, int lo, int hi) {
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.cu[mid].task >> SHIFT <= i) lo = mid; else hi = mid;
  }
  return lo;
}

struct DecodeTask {
  int b, x, s0, s1, B;  // sequence of the launch, its task's number among all, the task's slots, the sequence's slots
  int gkv, l;
};

// Workgroups are handed out in the order of the linear index, to the eight XCDs in turn.  The last units' tasks (kDecodeTail of them) go
// from the longest to the shortest over all of these units: compute units that are done early take short ones, and what
// starts last is shortest.  Before, units go one after the other, so that long streams cover the starts of short ones (all tasks from the
// longest to the shortest: 1024 units x {72 .. 487} slots 184 us, 176 so), each one task further on: with eight tasks to a unit one
// sequence would stay on one XCD.
// Tasks of a unit in a row throughout -> this, us: 112 units x {160 .. 982} 57 -> 50 (58 with the fold that parts of 512 need), 224 x {529 ..
// 2856} 332 -> 274, 1024 x 8 x {103 .. 291} 155 -> 119, x {99 .. 506} 276 -> 232, 896 x 5 x {127 .. 551} 146 -> 144.
// ORDERED: all this.  It costs a workgroup two more dependent scalar loads than the plain grid (0.3 us), which calls keep that gain
// nothing from it.
template <bool ORDERED, class A>
__device__ __forceinline__ DecodeTask decode_task(const A &a) {
  DecodeTask t;
  int part;
  if constexpr (!ORDERED) {  // grid (tasks, kv heads, layers)
    t.x = blockIdx.x; t.gkv = blockIdx.y; t.l = blockIdx.z;
    t.b = seq_of<0>(a, t.x, max(0, t.x - (a.tasks - a.n_seqs)), min(a.n_seqs, t.x + 1));  // (every sequence has a task: whole ones need no search)
    part = t.x - a.cu[t.b].task;
  } else {  // grid (kv heads, layers, tasks), read by its linear index
    const unsigned lin = (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x, units = gridDim.x * gridDim.y;
    const unsigned tasks = (unsigned)a.tasks, first = (unsigned)a.mixed * tasks;
    unsigned unit, i;
    if (lin < first) {
      unsigned turn;
      unit = quotient(lin, tasks, a.inv_tasks, i);
      quotient(unit, tasks, a.inv_tasks, turn);
      i = i + turn < tasks ? i + turn : i + turn - tasks;
    } else {
      i = quotient(lin - first, units - (unsigned)a.mixed, a.inv_last, unit);
      unit += (unsigned)a.mixed;
    }
    unsigned gkv;
    t.l = (int)quotient(unit, gridDim.x, a.inv_heads, gkv);
    t.gkv = (int)gkv;
    if ((int)i < a.full) {
      t.b = seq_of<16>(a, (int)i, 0, a.n_seqs);  // (sequences without a full task share their successor's number)
      part = (int)i - (a.cu[t.b].task >> 16);
    } else {
      const int r = (int)i - a.full;
      t.b = a.rest[r >> 2] >> (8 * (r & 3)) & 255;
      part = (a.cu[t.b + 1].task >> 16) - (a.cu[t.b].task >> 16);
    }
    t.x = (a.cu[t.b].task & 0xffff) + part;
  }
  t.B = a.rows(t.b);
  t.s0 = part * a.chunk;
  t.s1 = min(t.B, t.s0 + a.chunk);
  return t;
}

// What decode_task<true> reads of the order.  (Only where the order counts: the smallest calls are bound by host time.)
template <class A>
inline void order_tasks(A &a, const int *budgets, int units) {
  int n_rest = 0;
  long long rest[kDecodeSeqs];  // slots << 8 | sequence
  a.full = 0;
  for (int i = 0; i < a.n_seqs; ++i) {
    a.cu[i].task |= a.full << 16;
    a.full += budgets[i] / a.chunk;
    if (budgets[i] % a.chunk || budgets[i] == 0) rest[n_rest++] = (long long)(budgets[i] % a.chunk) << 8 | i;  // (an empty one is a task, too)
  }
  a.cu[a.n_seqs].task |= a.full << 16;
  std::sort(rest, rest + n_rest, [](long long x, long long y) { return x > y; });
  std::memset(a.rest, 0, sizeof(a.rest));
  for (int i = 0; i < n_rest; ++i) a.rest[i >> 2] |= (int)(rest[i] & 255) << (8 * (i & 3));
  const int last = (kDecodeTail + a.tasks - 1) / a.tasks;
  a.mixed = units > last ? units - last : 0;
  a.inv_tasks = 0xffffffffu / (unsigned)a.tasks;
  a.inv_last = 0xffffffffu / (unsigned)(units > last ? last : units);
  a.inv_heads = 0xffffffffu / (unsigned)a.Hkv;
}

}  // namespace flowmm
