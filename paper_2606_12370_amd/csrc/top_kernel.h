// top_kernel.h — the M largest logits of every row, largest first with ties to
// the lowest index, and the row's log partition function, each logit read once.
//
// A workgroup streams its part of a row with a threshold below which no logit
// can be among the part's M largest, and collects what exceeds it in LDS:
//
//   - every candidate is one 64-bit key, the logit's order in the high half and
//     the reversed index in the low half, so that keys are distinct and "the M
//     largest keys" settles ties;
//   - the first load step bounds the threshold by the M-th largest of the 256
//     threads' own maxima (at least M logits are as large).  Later logits have
//     larger indices, so they must exceed it;
//   - where the candidates outgrow the buffer, a radix selection keeps the M
//     largest keys and raises the threshold to the least of them.
//
// A row of random order passes a few hundred candidates; a row in ascending
// order selects once per tile of 256 vectors and stays right.  Calls of few
// rows split each row over several workgroups, whose lists a second launch
// merges with the same buffer.  The pass is bound by its one read of the
// logits and, close behind, by the vector instructions of the log partition
// (an exponential, a fused multiply-add and an add per logit).
#pragma once

#include "sv_device.h"

namespace sv {

constexpr int kTopMax = 256;  // longest list
// tiles per load step
constexpr int kTopStep = 4;
// Candidates held: the list and one tile of 256 16-byte bfloat16 vectors, so
// that a selection always makes room for a tile.
constexpr int kTopCap = kTopMax + 2048;
// Candidates up to which the list is sorted without a selection before
// (each thread ranks two keys).
constexpr int kTopRank = 512;

struct TopArgs {
  RowsDesc rows;      // tgt rows only
  int64_t R;          // rows
  int M, P;           // list length, parts per row
  int part;           // elements per part (a multiple of a load step)
  int32_t* ids;       // [R, M]
  float* values;      // [R, M]
  float* logz;        // [R] or nullptr
  uint64_t* cand;     // [R, P, M] lists of the parts (P > 1)
  RowStat* stats;     // [R, P] (P > 1): largest logit m and sum of exp((z - m) / T); D is NaN for a part with a data error
};

// A float's place in the order of all floats as an unsigned integer (both
// zeros alike; NaN beyond the infinities), and back.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t top_key(float x, int v) {
  return (static_cast<uint64_t>(order_key(x)) << 32) | static_cast<uint32_t>(~v);
}

struct TopLds {
  uint64_t buf[kTopCap];
  uint32_t hist[kThreads];
  uint32_t maxima[kThreads];
  uint32_t slot[3];     // candidates appended in a step, three steps' counters in turn
  uint32_t wsum[kWaves];
  uint32_t sel_digit, sel_need, sel_count;
  uint32_t least;       // order of the least key kept
  uint32_t kept;
  uint32_t bad;
  RedLds<1> red;
};

// Keep the M largest of the n > M keys in s.buf (in any order); every thread
// receives the order of the least one kept.  Called by the whole workgroup
// with the keys visible to it; ends with a barrier.
__device__ __forceinline__ uint32_t top_select(TopLds& s, int n, int M) {
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  uint64_t prefix = 0, mask = 0;
  uint32_t need = static_cast<uint32_t>(M);
  for (int shift = 56;; shift -= 8) {
    s.hist[t] = 0;
    __syncthreads();
    for (int i = t; i < n; i += kThreads) {
      const uint64_t k = s.buf[i];
      if ((k & mask) == prefix) atomicAdd(&s.hist[static_cast<int>(k >> shift) & 255], 1u);
    }
    __syncthreads();
    // keys with a digit above 255 - t
    const uint32_t own = s.hist[255 - t];
    uint32_t inc = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t up = __shfl_up(inc, o, 64);
      if (lane >= o) inc += up;
    }
    if (lane == 63) s.wsum[wave] = inc;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w)
      if (w < wave) inc += s.wsum[w];
    if (inc >= need && inc - own < need) {
      s.sel_digit = 255u - t;
      s.sel_need = need - (inc - own);
      s.sel_count = own;
    }
    __syncthreads();
    prefix |= static_cast<uint64_t>(s.sel_digit) << shift;
    mask |= uint64_t{255} << shift;
    need = s.sel_need;
    if (s.sel_count == need || shift == 0) break;  // all keys of the prefix are kept
  }
  // move the kept keys to the front
  constexpr int PER = (kTopCap + kThreads - 1) / kThreads;
  uint64_t own[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = t + u * kThreads;
    own[u] = i < n ? s.buf[i] : 0;
  }
  if (t == 0) {
    s.kept = 0;
    s.least = 0xffffffffu;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    if (t + u * kThreads < n && own[u] >= prefix) {
      s.buf[atomicAdd(&s.kept, 1u)] = own[u];
      atomicMin(&s.least, static_cast<uint32_t>(own[u] >> 32));
    }
  }
  __syncthreads();
  return s.least;
}

// Rank of each of this thread's keys t and t + 256 among the n <= kTopRank
// keys of s.buf (keys are distinct); rank n for a slot beyond them.
__device__ __forceinline__ void top_rank(const TopLds& s, int n, uint64_t (&k)[2], int (&rank)[2]) {
  const int t = threadIdx.x;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = t + u * kThreads;
    k[u] = i < n ? s.buf[i] : 0;
    rank[u] = i < n ? 0 : n;
  }
  if (t >= n) return;
  for (int j = 0; j < n; ++j) {
    const uint64_t o = s.buf[j];
    rank[0] += o > k[0] ? 1 : 0;
    if (n > kThreads && k[1]) rank[1] += o > k[1] ? 1 : 0;
  }
}

// The sorted list of the n candidates in s.buf: row r of the outputs.
__device__ __forceinline__ void top_write(TopLds& s, int n, const TopArgs& a, int64_t r, bool bad) {
  const int t = threadIdx.x;
  int32_t* ids = a.ids + r * a.M;
  float* values = a.values + r * a.M;
  const float none = bad ? __builtin_nanf("") : -INFINITY;
  if (bad) n = 0;
  if (n > kTopRank) {
    top_select(s, n, a.M);
    n = a.M;
  }
  uint64_t k[2];
  int rank[2];
  top_rank(s, n, k, rank);
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (t + u * kThreads < n && rank[u] < a.M) {
      ids[rank[u]] = static_cast<int32_t>(~static_cast<uint32_t>(k[u]));
      values[rank[u]] = order_value(static_cast<uint32_t>(k[u] >> 32));
    }
  if (t >= n && t < a.M) {
    ids[t] = -1;
    values[t] = none;
  }
}

// log sum exp(z / T) from the largest logit and the sum relative to it.
__device__ __forceinline__ float top_logz(float M, float T, double D) {
  return M == -INFINITY ? -INFINITY
                        : static_cast<float>(static_cast<double>(M) / static_cast<double>(T) + log(D));
}

// One part of one row.  LZ: the log partition function is asked for.
template <class E, bool LZ>
__global__ __launch_bounds__(kThreads) void top_part_kernel(TopArgs a) {
  constexpr int EPV = E::EPV, S = kTopStep, TILE = kThreads * EPV;
  static_assert(TILE + kTopMax <= kTopCap, "a selection makes room for a tile");
  __shared__ TopLds s;
  const int t = threadIdx.x;
  const int64_t r = static_cast<int64_t>(blockIdx.x) / a.P;
  const int part = static_cast<int>(static_cast<int64_t>(blockIdx.x) % a.P);
  int b;
  const typename E::raw* row = row_of<E>(a.rows, static_cast<int>(r), &b);
  const float T = temperature_of(a.rows, b);
  const float sc = temperature_ok(T) ? scale_of(T) : 1.0f;
  const int lo = part * a.part;
  const int hi = a.rows.V - lo < a.part ? a.rows.V : lo + a.part;
  if (t < 3) s.slot[t] = 0;
  if (t == 0) s.bad = 0;
  float thr = -INFINITY;
  bool equal = false;  // logits equal to the threshold are candidates too
  int n = 0;           // candidates in s.buf
  float top = -INFINITY, ref = -INFINITY;
  double D = 0.0;
  __syncthreads();
  for (int e = lo, step = 0; e < hi; e += S * TILE, ++step) {
    float x[S][EPV];
    load_span<E, S, kThreads>(row, e, t, hi, x);
    float vmax[S];
    float tmax = -INFINITY;
#pragma unroll
    for (int j = 0; j < S; ++j) {
      vmax[j] = x[j][0];
#pragma unroll
      for (int k = 1; k < EPV; ++k) vmax[j] = max_nan(vmax[j], x[j][k]);
      tmax = max_nan(tmax, vmax[j]);
    }
    top = max_nan(top, tmax);
    if (LZ) {
      const float nr = max_nan(ref, tmax);
      if (nr != -INFINITY) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < S; ++j)
#pragma unroll
          for (int k = 0; k < EPV; ++k) sum += __builtin_amdgcn_exp2f((x[j][k] - nr) * sc);
        if (ref != -INFINITY && nr != ref) D *= static_cast<double>(__builtin_amdgcn_exp2f((ref - nr) * sc));
        D += static_cast<double>(sum);
        ref = nr;
      }
    }
    if (step == 0) {
      // the M-th largest of the threads' maxima, ties by thread
      const uint32_t mine = order_key(tmax);
      s.maxima[t] = mine;
      __syncthreads();
      int rank = 0;
      for (int j = 0; j < kThreads; ++j) {
        const uint32_t o = s.maxima[j];
        rank += (o > mine || (o == mine && j < t)) ? 1 : 0;
      }
      if (rank == a.M - 1) s.least = mine;
      __syncthreads();
      thr = order_value(s.least);
      equal = thr > -INFINITY;
    }
    const int at = step % 3;
#pragma unroll
    for (int j = 0; j < S; ++j) {
      if (vmax[j] > thr || (equal && vmax[j] == thr)) {
        const int v0 = e + (j * kThreads + t) * EPV;
#pragma unroll
        for (int k = 0; k < EPV; ++k)
          if (x[j][k] > thr || (equal && x[j][k] == thr)) {
            const uint32_t pos = n + atomicAdd(&s.slot[at], 1u);
            if (pos < kTopCap) s.buf[pos] = top_key(x[j][k], v0 + k);
          }
      }
    }
    if (t == 0) s.slot[(step + 1) % 3] = 0;
    __syncthreads();
    const int added = static_cast<int>(s.slot[at]);
    if (n + added <= kTopCap) {
      n += added;
    } else {
      // again tile by tile, each with room for all of its logits
      for (int j = 0; j < S; ++j) {
        if (n > a.M) {
          thr = order_value(top_select(s, n, a.M));
          equal = false;
          n = a.M;
        }
        __syncthreads();
        if (t == 0) s.kept = 0;
        __syncthreads();
        const int v0 = e + (j * kThreads + t) * EPV;
#pragma unroll
        for (int jj = 0; jj < S; ++jj)
          if (jj == j) {
#pragma unroll
            for (int k = 0; k < EPV; ++k)
              if (x[jj][k] > thr || (equal && x[jj][k] == thr))
                s.buf[n + atomicAdd(&s.kept, 1u)] = top_key(x[jj][k], v0 + k);
          }
        __syncthreads();
        n += static_cast<int>(s.kept);
      }
    }
    equal = false;
  }
  // a data error: NaN or +inf, a temperature that is none
  if (!(top < INFINITY) || !temperature_ok(T)) atomicOr(&s.bad, 1u);
  float M = 0.f;
  double sum = 0.0;
  if (LZ) {
    float m[1] = {ref};
    wg_max(m, s.red);  // (ends with a barrier, as wg_sum does)
    M = m[0];
    double d[1] = {0.0};
    if (ref != -INFINITY) d[0] = D * static_cast<double>(__builtin_amdgcn_exp2f((ref - M) * sc));
    wg_sum(d, s.red);
    sum = d[0];
  }
  __syncthreads();
  const bool bad = s.bad != 0;
  if (a.P == 1) {
    if (LZ && t == 0) {
      a.logz[r] = bad ? __builtin_nanf("") : top_logz(M, T, sum);
    }
    top_write(s, n, a, r, bad);
    return;
  }
  if (t == 0) {
    RowStat st;
    st.m = M;
    st.pad = 0.f;
    st.D = bad ? __builtin_nan("") : sum;
    a.stats[r * a.P + part] = st;
  }
  if (bad) n = 0;
  if (n > kTopRank) {
    top_select(s, n, a.M);
    n = a.M;
  }
  uint64_t k[2];
  int rank[2];
  top_rank(s, n, k, rank);
  uint64_t* out = a.cand + (r * a.P + part) * a.M;
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (t + u * kThreads < n && rank[u] < a.M) out[rank[u]] = k[u];
  if (t >= n && t < a.M) out[t] = 0;
}

// The lists of a row's P parts merged.  No key below both bounds can be among
// the M largest: the largest of the parts' M-th keys, and the least of the
// parts' ceil(M / P)-th keys (P ceil(M / P) >= M keys are as large).
template <bool LZ>
__global__ __launch_bounds__(kThreads) void top_merge_kernel(TopArgs a) {
  __shared__ TopLds s;
  __shared__ uint64_t bound[2];
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x;
  const uint64_t* cand = a.cand + r * a.P * a.M;
  const RowStat* st = a.stats + r * a.P;
  if (t == 0) {
    s.bad = 0;
    bound[0] = 0;
    bound[1] = ~uint64_t{0};
  }
  __syncthreads();
  const int j0 = (a.M + a.P - 1) / a.P - 1;
  for (int p = t; p < a.P; p += kThreads) {
    atomicMax(reinterpret_cast<unsigned long long*>(&bound[0]),
              static_cast<unsigned long long>(cand[static_cast<int64_t>(p) * a.M + a.M - 1]));
    atomicMin(reinterpret_cast<unsigned long long*>(&bound[1]),
              static_cast<unsigned long long>(cand[static_cast<int64_t>(p) * a.M + j0]));
    if (st[p].D != st[p].D) atomicOr(&s.bad, 1u);
  }
  __syncthreads();
  uint64_t least = bound[0] > bound[1] ? bound[0] : bound[1];
  if (least == 0) least = 1;  // empty places
  const bool bad = s.bad != 0;
  const int64_t total = bad ? 0 : static_cast<int64_t>(a.P) * a.M;
  int n = 0;
  for (int64_t i0 = 0; i0 < total; i0 += 8 * kThreads) {
    if (n + 8 * kThreads > kTopCap) {
      // (keys are distinct: one that ties the least kept is that key itself)
      if (n > a.M) {
        least = static_cast<uint64_t>(top_select(s, n, a.M)) << 32;
        n = a.M;
      }
    }
    __syncthreads();
    if (t == 0) s.kept = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t i = i0 + u * kThreads + t;
      const uint64_t k = i < total ? cand[i] : 0;
      if (k >= least) s.buf[n + atomicAdd(&s.kept, 1u)] = k;
    }
    __syncthreads();
    n += static_cast<int>(s.kept);
  }
  if (LZ && t < 64) {
    int b;
    (void)row_of<BF16>(a.rows, static_cast<int>(r), &b);
    const float T = temperature_of(a.rows, b);
    const float sc = scale_of(T);
    float M = -INFINITY;
    for (int p = t; p < a.P; p += 64) M = fmaxf(M, st[p].m);
    M = wave_max(M);
    double D = 0.0;
    for (int p = t; p < a.P; p += 64)
      if (st[p].m != -INFINITY) D += st[p].D * static_cast<double>(__builtin_amdgcn_exp2f((st[p].m - M) * sc));
    D = wave_sum(D);
    if (t == 0) {
      a.logz[r] = bad ? __builtin_nanf("") : top_logz(M, T, D);
    }
  }
  top_write(s, n, a, r, bad);
}

}  // namespace sv
