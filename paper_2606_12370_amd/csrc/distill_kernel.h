// distill_kernel.h — distillation of a draft head from a teacher's top logits:
// cross entropy or forward KL against the listed tokens, and the gradient
// w.r.t. the draft logits.
//
// Position (n, k), temperature T, list (id_j, t_j), j < M, entries with
// id_j < 0 unused; student logits z, q = softmax(z / T):
//   p_j = exp(t_j / T - lse),  lse = log sum_j exp(t_j / T) without a teacher
//         log Z, else lse = log Z and r = 1 - sum_j p_j is the mass outside the
//         list (0 where it is at most 2^-18, which a float32 log Z of the usual
//         size does not resolve); W = sum_j p_j
//   L = sum_j p_j (log p_j - log q_id_j) + r (log r - log q_out),
//         q_out = sum of q outside the list; cross entropy drops log p_j, log r
//   dL/dz_v = (1/T) [ (W + r) q_v - sum_{j: id_j = v} p_j - 1[v unlisted] r q_v / q_out ]
//
// With a teacher log Z the row's sums are kept apart: the unlisted logits'
// relative to their own largest one, in the pass over the row, and the listed
// logits' with the list.  q_out is therefore never a difference, nor does it
// underflow where the student's mass sits on the list, and neither does the
// gradient outside it.  The list's own quantities (M terms) are float64,
// exponentials of the row float32, their sums float32 over at most 128 elements
// and float64 beyond.
//
// Launches: 1 distill_stats (a wave per list, and a wave per sub-chunk of the
// student's row), 2 distill_grad (a workgroup per chunk), or distill_norm
// without a gradient, 3 distill_loss.
#pragma once

#include "sv_device.h"

namespace sv {

constexpr int kListMax = 256;
constexpr double kTailMin = 1.0 / 262144.0;
enum { kDistillForward = 0, kDistillCe = 1 };

struct DistillStat {
  float m;     // largest logit of the sub-chunk (-inf: empty), unlisted ones only with a teacher log Z
  float pad;
  double D;    // sum of exp((z - m) / T) over the same
};

struct ListInfo {
  double lse;    // natural log of the teacher's partition function
  double W;      // sum of p_j
  double r;      // mass outside the list
  double c;      // sum p_j (log p_j - (z_id_j - ref) / T) + r log r (logarithms of p and r only for forward KL);
                 // ref = ml, 0 if that is -inf
  double Dl;     // sum of exp((z - ml) / T) over the listed tokens (with a teacher log Z, else 0)
  float ml;      // the largest listed logit of the student (-inf: none)
  int state;     // 0: an empty list, 1: ordinary, 2: a data error
};

// A row's normalisers.
struct DistillNorm {
  double logD;   // log sum exp(z / T) - M / T
  double logDo;  // log of the unlisted sum, - M / T too
  double D;      // sum relative to M
  double Do;     // unlisted sum relative to mo
  float M, mo;   // the row's largest logit and the largest unlisted one (mo = M without a teacher log Z)
};

struct DistillArgs {
  const void* z; int64_t zsn, zsk;
  const int32_t* ids; const float* vals; int64_t lsn, lsk;
  const float* logz; int64_t osn, osk;   // logz nullptr: the list is renormalised
  int N, K, V, M;
  int C;             // sub-chunks per row
  int kind;
  float s_hi, s_lo;  // log2(e) / T as the sum of two positive floats
  double inv_t;      // 1 / T
  double f;          // scale / (K T), the gradient's factor
  double loss_scale; // scale / K
  float* loss; float* per_step; void* grad;
  ListInfo* info;         // [N K]
  DistillStat* stats;     // [N K][C]
  double* part;           // [N K] per-step losses
};

// exp((z - ref) / T) for z <= ref.  The difference comes first, so that a row
// of the type's lowest values is a flat one and not one of infinities; the
// scale's second part leaves the exponent with the roundings of the difference
// and of the fused multiply-add alone.  Both parts are positive: z = -inf gives 0.
__device__ __forceinline__ float scaled_exp(float z, float s_hi, float s_lo, float ref) {
  const float d = z - ref;
  return __builtin_amdgcn_exp2f(fmaf(d, s_hi, d * s_lo));
}

__device__ __forceinline__ void unit_of(const DistillArgs& a, int64_t u, int* n, int* k) {
  *n = static_cast<int>(u / a.K);
  *k = static_cast<int>(u - static_cast<int64_t>(*n) * a.K);
}
template <class E>
__device__ __forceinline__ const typename E::raw* student_row(const DistillArgs& a, int n, int k) {
  return static_cast<const typename E::raw*>(a.z) + n * a.zsn + k * a.zsk;
}
__device__ __forceinline__ int64_t list_of(const DistillArgs& a, int n, int k) { return n * a.lsn + k * a.lsk; }

__device__ __forceinline__ double wave_max_d(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, 64));
  return v;
}

// The teacher's side of one position, by one wave (64 entries at a time).
template <class E>
__device__ __forceinline__ ListInfo list_info(const DistillArgs& a, int n, int k) {
  const int lane = threadIdx.x & 63;
  const int32_t* ids = a.ids + list_of(a, n, k);
  const float* vals = a.vals + list_of(a, n, k);
  const typename E::raw* row = student_row<E>(a, n, k);
  constexpr int PER = kListMax / 64;
  int id[PER];
  double t[PER], z[PER];
  bool used = false, bad = false;
  double mx = -INFINITY;
  ListInfo o;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int j = u * 64 + lane;
    id[u] = -1;
    t[u] = -INFINITY;
    if (j < a.M) {
      id[u] = ids[j];
      const float v = vals[j];
      bad = bad || v != v || id[u] >= a.V;
      if (id[u] >= 0) {
        used = true;
        bad = bad || v == INFINITY;
        t[u] = static_cast<double>(v) * a.inv_t;
      }
    }
    mx = fmax(mx, t[u]);
  }
  float zmax = -INFINITY;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const float v = (id[u] >= 0 && id[u] < a.V) ? E::one(row + id[u]) : -INFINITY;
    bad = bad || !(v < INFINITY);
    zmax = fmaxf(zmax, v);
    z[u] = static_cast<double>(v);
  }
  o.ml = wave_max(zmax);
  const double ref = o.ml > -INFINITY ? static_cast<double>(o.ml) : 0.0;
#pragma unroll
  for (int u = 0; u < PER; ++u) z[u] = (z[u] - ref) * a.inv_t;
  o.r = 0.0;
  const float lz = a.logz ? a.logz[n * a.osn + k * a.osk] : 0.f;
  mx = wave_max_d(mx);
  // (with a teacher log Z, tokens listed at -inf leave all mass outside the list)
  const bool any = __ballot(used) != 0 && (a.logz || mx > -INFINITY);
  bad = __ballot(bad) != 0 || lz != lz;
  if (a.logz) {
    bad = bad || (any && !(lz > -INFINITY && lz < INFINITY));
    o.lse = static_cast<double>(lz);
  } else {
    double e = 0.0;
#pragma unroll
    for (int u = 0; u < PER; ++u)
      if (t[u] > -INFINITY) e += exp(t[u] - mx);
    o.lse = mx + log(wave_sum(e));
  }
  double W = 0.0, c = 0.0;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    if (t[u] > -INFINITY) {
      const double lp = t[u] - o.lse;
      const double p = exp(lp);
      W += p;
      // a p that underflows adds nothing, whatever its logarithms
      if (p > 0.0) c += p * ((a.kind == kDistillForward ? lp : 0.0) - z[u]);
    }
  }
  o.W = wave_sum(W);
  o.c = wave_sum(c);
  if (a.logz) {
    const double r = 1.0 - o.W;
    if (r > kTailMin) {
      o.r = r;
      if (a.kind == kDistillForward) o.c += r * log(r);
    }
  }
  o.state = bad ? 2 : (any ? 1 : 0);
  o.Dl = 0.0;
  if (a.logz) {
    // each listed token once: an entry with the id of an earlier one is left out
    bool again[PER] = {};
    for (int j = 0; j < a.M; ++j) {
      int other = id[0];
#pragma unroll
      for (int u = 1; u < PER; ++u) other = (j >> 6) == u ? id[u] : other;
      other = __builtin_amdgcn_readlane(other, j & 63);
#pragma unroll
      for (int u = 0; u < PER; ++u) again[u] = again[u] || (other == id[u] && j < u * 64 + lane);
    }
    double d = 0.0;
#pragma unroll
    for (int u = 0; u < PER; ++u)
      if (!again[u] && z[u] > -INFINITY) d += exp(z[u]);
    o.Dl = wave_sum(d);
  }
  return o;
}

// A row's normalisers from its sub-chunks' sums (m, D) and its list.
__device__ __forceinline__ DistillNorm distill_norm(const DistillArgs& a, const ListInfo& li, float m, double D) {
  DistillNorm n;
  n.mo = m;
  n.Do = D;
  n.M = fmaxf(m, li.ml);
  const double wo = m == -INFINITY ? 0.0 : exp((static_cast<double>(m) - static_cast<double>(n.M)) * a.inv_t);
  const double wl = li.Dl > 0.0 ? exp((static_cast<double>(li.ml) - static_cast<double>(n.M)) * a.inv_t) : 0.0;
  n.D = (D != D ? D : D * wo) + li.Dl * wl;
  n.logD = log(n.D);
  n.logDo = m == -INFINITY ? -INFINITY
                           : log(D) + (static_cast<double>(m) - static_cast<double>(n.M)) * a.inv_t;
  return n;
}
__device__ __forceinline__ bool norm_ok(const DistillNorm& n) { return n.D > 0.0 && n.D < INFINITY && n.M < INFINITY; }

// A row's loss: L = c + W (log Z - ref / T) - r (log of the unlisted sum / Z).
__device__ __forceinline__ double distill_loss_of(const DistillArgs& a, const ListInfo& li, const DistillNorm& n) {
  if (li.state == 0) return 0.0;
  if (li.state == 2 || !norm_ok(n)) return __builtin_nan("");
  const double ref = li.ml > -INFINITY ? static_cast<double>(li.ml) : 0.0;
  double L = li.c + li.W * ((static_cast<double>(n.M) - ref) * a.inv_t + n.logD);
  if (li.r > 0.0) L += li.r * (n.logD - n.logDo);
  return L;
}

// Combine a row's C sub-chunk statistics (one wave; every lane receives the
// result; the order of the sum is fixed).
__device__ __forceinline__ DistillNorm combine_distill(const DistillArgs& a, const ListInfo& li, int64_t u) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY;
  double d = 0.0;
  if (li.state == 1) {
    const DistillStat* st = a.stats + u * a.C;
    for (int c = lane; c < a.C; c += 64) m = fmaxf(m, st[c].m);
    m = wave_max(m);
    for (int c = lane; c < a.C; c += 64) {
      const float mc = st[c].m;
      const double dc = st[c].D;
      if (dc != dc) d += dc;
      else if (mc != -INFINITY) d += dc * static_cast<double>(scaled_exp(mc, a.s_hi, a.s_lo, m));
    }
    d = wave_sum(d);
  }
  return distill_norm(a, li, m, d);
}

// The entries of a list whose ids lie in [lo, hi), in list order, by one wave:
// ids into `out` (LDS of the wave, kListMax places; nullptr: none wanted) and
// their count, -1 for a list without entries.
__device__ __forceinline__ int list_in_range(const DistillArgs& a, int64_t at, int lo, int hi, int* out) {
  const int lane = threadIdx.x & 63;
  int cnt = 0;
  bool used = false;
  for (int base = 0; base < a.M; base += 64) {
    const int j = base + lane;
    const int id = j < a.M ? a.ids[at + j] : -1;
    used = used || __ballot(id >= 0) != 0;
    if (!out) continue;
    const bool in = id >= lo && id < hi;
    const uint64_t m = __ballot(in);
    if (in) out[cnt + __popcll(m & ((uint64_t{1} << lane) - 1))] = id;
    cnt += __popcll(m);
  }
  return used ? cnt : -1;
}

constexpr int kDistillVec = 16;  // vectors per lane of a sub-chunk
template <class E>
constexpr int distill_sub() { return kDistillVec * 64 * E::EPV; }

// Workgroups below `lists` hold a wave per list, the others a wave per
// sub-chunk.  TAIL: the listed tokens are left out of the sums.
template <class E, bool TAIL>
__global__ __launch_bounds__(kThreads) void distill_stats_kernel(DistillArgs a, int lists, int64_t nsub) {
  constexpr int EPV = E::EPV, S = 4, W = 64 * EPV, SUB = distill_sub<E>();
  __shared__ int in_list[TAIL ? kWaves : 1][TAIL ? kListMax : 1];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int n, k;
  if (static_cast<int>(blockIdx.x) < lists) {
    const int64_t u = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
    if (u >= static_cast<int64_t>(a.N) * a.K) return;
    unit_of(a, u, &n, &k);
    const ListInfo li = list_info<E>(a, n, k);
    if (lane == 0) a.info[u] = li;
    return;
  }
  const int64_t g = (static_cast<int64_t>(blockIdx.x) - lists) * kWaves + wave;
  if (g >= nsub) return;
  const int64_t u = g / a.C;
  const int c = static_cast<int>(g - u * a.C);
  unit_of(a, u, &n, &k);
  const typename E::raw* row = student_row<E>(a, n, k);
  const int e0 = c * SUB;
  uint32_t tiles = 0;  // tiles of vectors that hold a listed token
  const int cnt = list_in_range(a, list_of(a, n, k), e0, a.V - e0 < SUB ? a.V : e0 + SUB, TAIL ? in_list[wave] : nullptr);
  if (cnt < 0) return;  // (nothing reads the statistics of an empty list)
  if (TAIL) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (int j = lane; j < cnt; j += 64) tiles |= 1u << ((in_list[wave][j] - e0) / W);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) tiles |= __shfl_xor(tiles, o, 64);
    tiles = __builtin_amdgcn_readfirstlane(tiles);
  }
  float ref = -INFINITY;
  double D = 0.0;
#pragma unroll 1
  for (int st = 0; st < kDistillVec / S; ++st) {
    const int es = e0 + st * S * W;
    if (es >= a.V) break;
    float x[S][EPV];
    load_span<E, S, 64>(row, es, lane, a.V, x);
    if (TAIL) {
#pragma unroll
      for (int j = 0; j < S; ++j) {
        if ((tiles >> (st * S + j)) & 1u) {
          const int v0 = es + j * W + lane * EPV;
          for (int q = 0; q < cnt; ++q) {
            const int o = in_list[wave][q] - v0;
#pragma unroll
            for (int i = 0; i < EPV; ++i)
              if (o == i) x[j][i] = -INFINITY;
          }
        }
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < S; ++j)
#pragma unroll
      for (int i = 0; i < EPV; ++i) mx = max_nan(mx, x[j][i]);
    const float nr = max_nan(ref, mx);
    if (nr != -INFINITY) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < S; ++j)
#pragma unroll
        for (int i = 0; i < EPV; ++i) sum += scaled_exp(x[j][i], a.s_hi, a.s_lo, nr);
      if (ref != -INFINITY && nr != ref) D *= static_cast<double>(scaled_exp(ref, a.s_hi, a.s_lo, nr));
      D += static_cast<double>(sum);
      ref = nr;
    }
  }
  const float m = wave_max(ref);
  if (D == D && ref != -INFINITY) D *= static_cast<double>(scaled_exp(ref, a.s_hi, a.s_lo, m));
  D = wave_sum(D);
  if (lane == 0) {
    DistillStat o;
    o.m = m;
    o.pad = 0.f;
    o.D = D;
    a.stats[g] = o;
  }
}

// The loss of every position without a gradient (one wave each).
__global__ __launch_bounds__(kThreads) void distill_norm_kernel(DistillArgs a) {
  const int64_t u = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (u >= static_cast<int64_t>(a.N) * a.K) return;
  const ListInfo li = a.info[u];
  const DistillNorm nm = combine_distill(a, li, u);
  if ((threadIdx.x & 63) == 0) {
    const double L = distill_loss_of(a, li, nm);
    a.part[u] = L;
    if (a.per_step) a.per_step[u] = static_cast<float>(L);
  }
}

// Gradient elements: float32, or bfloat16 rounded to nearest even.
struct GradF32 {
  using raw = float;
  static __device__ __forceinline__ void store4(raw* p, const float (&g)[4]) {
    f32x4 v;
    v.x = g[0]; v.y = g[1]; v.z = g[2]; v.w = g[3];
    *reinterpret_cast<f32x4_any*>(p) = v;
  }
  static __device__ __forceinline__ void store1(raw* p, float g) { *p = g; }
};
struct GradBF16 {
  using raw = uint16_t;
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ uint32_t round2(float lo, float hi) {
    const f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
  }
  static __device__ __forceinline__ void store4(raw* p, const float (&g)[4]) {
    u32x2 v;
    v.x = round2(g[0], g[1]);
    v.y = round2(g[2], g[3]);
    *reinterpret_cast<u32x2_any*>(p) = v;
  }
  static __device__ __forceinline__ void store1(raw* p, float g) { *p = static_cast<uint16_t>(round2(g, 0.f)); }
};

// The gradient's coefficients: listed tokens get cl exp((z - M) / T) - f sum p,
// unlisted ones cu exp((z - ru) / T), ru = mo (0 where every one of them is -inf).
struct DistillCoef {
  float cl, cu, ru;
  bool nan;
};
__device__ __forceinline__ DistillCoef distill_coef(const DistillArgs& a, const ListInfo& li, const DistillNorm& n) {
  DistillCoef c;
  c.nan = li.state == 2 || (li.state == 1 && !norm_ok(n));
  const double all = a.f * (li.W + li.r) / n.D;
  c.cl = static_cast<float>(all);
  // where no unlisted token has mass, none has a gradient either
  c.cu = 0.f;
  c.ru = n.mo > -INFINITY ? n.mo : 0.f;
  if (n.mo > -INFINITY) {
    const double w = exp((static_cast<double>(n.mo) - static_cast<double>(n.M)) * a.inv_t);
    c.cu = static_cast<float>(all * w - (li.r > 0.0 ? a.f * li.r / n.Do : 0.0));
  }
  return c;
}

constexpr int kDistillChunk = 16384;

// One chunk of one row's gradient; the workgroup of chunk 0 also writes the
// position's loss.  E reads four elements per lane (one 16-byte store each).
template <class E, class G>
__global__ __launch_bounds__(kThreads) void distill_grad_kernel(DistillArgs a, int CH) {
  static_assert(E::EPV == 4, "one gradient vector per lane");
  constexpr int S = 4, TILE = kThreads * 4, NT = kDistillChunk / TILE;
  __shared__ int in_list[kListMax];
  __shared__ float in_p[kListMax];
  __shared__ int count;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int64_t u = static_cast<int64_t>(blockIdx.x) / CH;
  const int c = static_cast<int>(static_cast<int64_t>(blockIdx.x) - u * CH);
  int n, k;
  unit_of(a, u, &n, &k);
  const ListInfo li = a.info[u];
  const DistillNorm nm = combine_distill(a, li, u);
  const DistillCoef co = distill_coef(a, li, nm);
  if (c == 0 && t == 0) {
    const double L = distill_loss_of(a, li, nm);
    a.part[u] = L;
    if (a.per_step) a.per_step[u] = static_cast<float>(L);
  }
  const int e0 = c * kDistillChunk;
  const int e1 = a.V - e0 < kDistillChunk ? a.V : e0 + kDistillChunk;
  typename G::raw* out = static_cast<typename G::raw*>(a.grad) + u * a.V;
  const bool plain = li.state == 1 && !co.nan;
  if (wave == 0) {
    int cnt = 0;
    if (plain) {
      const int64_t at = list_of(a, n, k);
      for (int base = 0; base < a.M; base += 64) {
        const int j = base + lane;
        const int id = j < a.M ? a.ids[at + j] : -1;
        const bool in = id >= e0 && id < e1;
        const uint64_t m = __ballot(in);
        if (in) {
          const int pos = cnt + __popcll(m & ((uint64_t{1} << lane) - 1));
          in_list[pos] = id;
          in_p[pos] = static_cast<float>(a.f * exp(static_cast<double>(a.vals[at + j]) * a.inv_t - li.lse));
        }
        cnt += __popcll(m);
      }
    }
    if (lane == 0) count = cnt;
  }
  __syncthreads();
  const int cnt = count;
  // tiles of this wave that hold a listed token
  uint32_t tiles = 0;
  for (int j = lane; j < cnt; j += 64) {
    const int o = in_list[j] - e0;
    if ((o % TILE) / 256 == wave) tiles |= 1u << (o / TILE);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) tiles |= __shfl_xor(tiles, o, 64);
  tiles = __builtin_amdgcn_readfirstlane(tiles);
  const typename E::raw* row = student_row<E>(a, n, k);
  const float fill = co.nan ? __builtin_nanf("") : 0.f;
#pragma unroll 1
  for (int st = 0; st < NT / S; ++st) {
    const int es = e0 + st * S * TILE;
    if (es >= e1) break;
    float x[S][4];
    if (plain) load_span<E, S, kThreads>(row, es, t, a.V, x);
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const int v0 = es + (j * kThreads + t) * 4;
      float g[4];
      if (plain) {
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = co.cu * scaled_exp(x[j][i], a.s_hi, a.s_lo, co.ru);
        if ((tiles >> (st * S + j)) & 1u) {
          float p[4] = {0.f, 0.f, 0.f, 0.f};
          uint32_t hit = 0;
          for (int q = 0; q < cnt; ++q) {
            const int o = in_list[q] - v0;
            if (o >= 0 && o < 4) {
              hit |= 1u << o;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (i == o) p[i] += in_p[q];
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if ((hit >> i) & 1u) g[i] = co.cl * scaled_exp(x[j][i], a.s_hi, a.s_lo, nm.M) - p[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = fill;
      }
      if (v0 + 4 <= a.V) {
        G::store4(out + v0, g);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (v0 + i < a.V) G::store1(out + v0 + i, g[i]);
      }
    }
  }
}

// loss = scale / K times the sum of the per-step losses, in a fixed order.
__global__ __launch_bounds__(kThreads) void distill_loss_kernel(const double* __restrict__ part, int64_t units,
                                                                double scale, float* loss) {
  __shared__ RedLds<1> s;
  double v[1] = {0.0};
  for (int64_t i = threadIdx.x; i < units; i += kThreads) v[0] += part[i];
  wg_sum(v, s);
  if (threadIdx.x == 0) *loss = static_cast<float>(v[0] * scale);
}

}  // namespace sv
