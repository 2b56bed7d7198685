// The draw of a decode step's next tokens, and the embedding rows they start with.
//
//   k_sample       temperature, top-k, top-p, min-p and the draw from a given uniform
//   k_embed_rows   X[t] = E[tokens[t]] (+ E_pos[pos[t]]), positions advanced
//
// Sampling without a sort.  With the order "logit descending, index ascending" all three filters keep a prefix of a
// row's tokens, so what has to be found is the prefix's last token, never the order itself.  Weights are w = 2^-d,
// d = (M - z) log2(e) / T >= 0 in double; a token falls into bin floor(8 d), and a histogram of counts and weights over the
// bins tells in which bin the prefix ends.  Sums of weights are sums of 64-bit integers wherever threads add in any order, so
// they do not depend on it.  The bin where the prefix ends is cut again by the bits of its logits until one value is left,
// and equal logits are kept by ascending index.  The draw is a search in the kept tokens' running sum by index.
//
// One workgroup of 16 waves per row.  A row is read once for its maximum, once for the histogram (counts alone take no
// exponential: a top-k row needs none for the tokens it drops), and once to gather the tokens that matter into LDS, where
// the rest happens; only a row that keeps more than kList tokens reads them a third time, for its running sum.
#include "zo_device.hpp"
#include "zo_internal.hpp"

namespace zo {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = kThreads;      // eighths of d up to 128; the last bin holds the rest (weights below 2^-127: none)
constexpr int kLast = kBins - 1;
constexpr int kPieces = 4;           // loads of a wave under way, four neighbouring tokens a lane each
constexpr int kStrip = kPieces * 4 * kWave;
constexpr int kMaxVocab = 1 << 19;
constexpr int kMaxStrips = kMaxVocab / kStrip;
constexpr int kList = 4096;          // tokens that fit in LDS

typedef unsigned long long u64;

__device__ __forceinline__ float ld_logit(const float* p, int i) { return p[i]; }
__device__ __forceinline__ float ld_logit(const bf16_t* p, int i) { return bf16_to_f32(p[i]); }
// Neither NaN nor -infinity.  (Compared with the least number, not with -infinity: "above -infinity" is compiled into a
// comparison that NaN passes.)
constexpr float kLeast = -3.402823466e38f;
__device__ __forceinline__ bool is_token(float z) { return z >= kLeast; }
// Unsigned integers in the order of the floats, and back; -0 is 0.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// Four neighbouring logits as they lie in memory.
template <typename Tio> struct Raw;
template <> struct Raw<float> { typedef float4 type; };
template <> struct Raw<bf16_t> { typedef uint2 type; };
__device__ __forceinline__ void unpack(const float4& v, float (&x)[4]) {
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void unpack(const uint2& v, float (&x)[4]) {
  x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
  x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
}
// Four from `at` of a row of any alignment and end: -infinity behind it.
template <typename Tio>
__device__ __forceinline__ void four(const Tio* z, int at, int V, float (&x)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = at + j < V ? ld_logit(z, at + j) : -INFINITY;
}

// 2^(-y/8) for y in [0, 1): the Taylor polynomial about 0; its first omitted term is below 8e-14.
__device__ __forceinline__ double exp2_neg8(double y) {
  constexpr double kLn = -0.6931471805599453094 / 8;
  double p = kLn * kLn * kLn * kLn * kLn * kLn * kLn / 5040;
  p = p * y + kLn * kLn * kLn * kLn * kLn * kLn / 720;
  p = p * y + kLn * kLn * kLn * kLn * kLn / 120;
  p = p * y + kLn * kLn * kLn * kLn / 24;
  p = p * y + kLn * kLn * kLn / 6;
  p = p * y + kLn * kLn / 2;
  p = p * y + kLn;
  return p * y + 1.0;
}
// 2^-d for d >= 0 (NaN and beyond 2^-1074: 0): 2^-n times the Taylor polynomial of the rest, |rest| <= 1/2; its first omitted term
// is below 3e-13.  Exactly 1 at 0: rows of equal logits have weights whose sums are exact, and so is u * Z between two of them.
__device__ __forceinline__ double exp2_neg(double d) {
  d = __builtin_fmin(d, 1100.0);
  const double n = __builtin_rint(d), y = n - d;
  constexpr double k1 = 0.6931471805599453094, k2 = k1 * k1 / 2, k3 = k2 * k1 / 3, k4 = k3 * k1 / 4, k5 = k4 * k1 / 5, k6 = k5 * k1 / 6,
                   k7 = k6 * k1 / 7, k8 = k7 * k1 / 8, k9 = k8 * k1 / 9, k10 = k9 * k1 / 10;
  double p = k10;
  p = p * y + k9;
  p = p * y + k8;
  p = p * y + k7;
  p = p * y + k6;
  p = p * y + k5;
  p = p * y + k4;
  p = p * y + k3;
  p = p * y + k2;
  p = p * y + k1;
  p = p * y + 1.0;
  return __builtin_ldexp(p, -(int)n);
}

// How far a logit lies below the row's maximum, and its weight.
struct Scale {
  float zmax;
  double c;   // log2(e) / T
  // in octaves of its weight
  __device__ __forceinline__ double dist(float z) const {
    if (zmax == INFINITY) return z == zmax ? 0.0 : INFINITY;
    return ((double)zmax - (double)z) * c;
  }
  __device__ __forceinline__ int bin(float z) const {
    const double d = dist(z) * 8.0;
    return d < (double)kLast ? (int)d : kLast;
  }
  __device__ __forceinline__ double weight(float z) const { return exp2_neg(dist(z)); }
  // the weight in units of 2^-50 of the maximum's (sums of kList of them fit)
  __device__ __forceinline__ u64 units(float z) const { return (u64)(weight(z) * 0x1p50 + 0.5); }
};
// A weight is mant * bin_unit(bin) with mant in units of 2^-44: sums of kMaxVocab mantissas fit into 64 bits.
__device__ __forceinline__ u64 mant8(double frac) {   // (adding 2^8 leaves units of 2^-44 in the last bits)
  return (u64)__double_as_longlong(exp2_neg8(frac) + 256.0) - 0x4070000000000000ull;
}
__device__ __forceinline__ double bin_unit(int bin) { return bin >= kLast ? 0.0 : exp2_neg((double)bin * 0.125 + 44.0); }

template <class T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
template <class T>
__device__ __forceinline__ T wave_scan(T v, int lane) {   // inclusive
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const T x = __shfl_up(v, o);
    if (lane >= o) v += x;
  }
  return v;
}

struct Shared {
  uint32_t cnt[kBins];
  u64 mass[kBins];
  union {
    struct { float z[kList]; int32_t i[kList]; } list;
    double strip[kMaxStrips];
  };
  u64 wave_n[kWaves];
  double wave_m[kWaves];
  float wave_z[kWaves];
  // results of one thread, for all
  uint32_t lo, hi, n_list;
  int bin, index;
  u64 n_before, n_at;
  double m_before, m_at, total;
};

// What a row's threads share and know.
template <typename Tio>
struct Row {
  Shared& s;
  const Tio* z;
  int V, tid, lane, wave;
  bool vec;

  // f(x, first index) for every four tokens of a strip of kStrip tokens, strip by strip of this wave's share, then
  // done(strip).  A whole strip's loads are under way together; they are not conditional, or the next would wait for the last.
  template <class F, class Done>
  __device__ __forceinline__ void strips(F f, Done done) const {
    const int n = (V + kStrip - 1) / kStrip, whole = vec ? V / kStrip : 0;
    typedef typename Raw<Tio>::type R;
    int st = wave;
    for (; st < whole; st += kWaves) {
      R raw[kPieces];
#pragma unroll
      for (int u = 0; u < kPieces; ++u) raw[u] = *reinterpret_cast<const R*>(z + st * kStrip + u * (4 * kWave) + lane * 4);
#pragma unroll
      for (int u = 0; u < kPieces; ++u) {
        float x[4];
        unpack(raw[u], x);
        f(x, st * kStrip + u * (4 * kWave) + lane * 4);
      }
      done(st);
    }
    for (; st < n; st += kWaves) {
      for (int u = 0; u < kPieces; ++u) {
        float x[4];
        const int at = st * kStrip + u * (4 * kWave) + lane * 4;
        four(z, at, V, x);
        f(x, at);
      }
      done(st);
    }
  }
  template <class F>
  __device__ __forceinline__ void strips(F f) const {
    strips(f, [](int) {});
  }
};

// Inclusive running sums over the threads of the workgroup, in a fixed order.  `before` is the sum of the threads before.
// (Begins and ends with a barrier: the buffers may be in use on either side.)
__device__ __forceinline__ void block_scan(Shared& s, int lane, int wave, u64 n, double m, u64& n_before, double& m_before) {
  const u64 ni = wave_scan(n, lane);
  const double mi = wave_scan(m, lane);
  __syncthreads();
  if (lane == kWave - 1) { s.wave_n[wave] = ni; s.wave_m[wave] = mi; }
  __syncthreads();
  u64 nb = 0;
  double mb = 0.0;
  for (int w = 0; w < wave; ++w) { nb += s.wave_n[w]; mb += s.wave_m[w]; }
  n_before = nb + ni - n;
  const double up = __shfl_up(mi, 1);   // (every lane takes part)
  m_before = lane > 0 ? mb + up : mb;
  __syncthreads();
}

// What the search for a cut counts: tokens up to `n`, or weight up to `mass`, whichever ends first.
struct Goal {
  u64 n;
  double mass;
};

// The first of the workgroup's bins (one a thread: cnt and mass of it) at which the running count reaches goal.n or the running
// weight goal.mass, the last one in use if a rounding leaves none: s.bin, and what lies before it and in it.
__device__ __forceinline__ void find_bin(Shared& s, int tid, int lane, int wave, u64 n0, double m0, u64 cnt, double mass,
                                         const Goal& goal) {
  u64 nb;
  double mb;
  block_scan(s, lane, wave, cnt, mass, nb, mb);
  nb += n0;
  mb += m0;
  const bool used = cnt > 0, hit = used && (nb + cnt >= goal.n || mb + mass >= goal.mass);
  if (tid == 0) { s.bin = 0x7FFFFFFF; s.index = -1; }
  __syncthreads();
  if (hit) atomicMin(&s.bin, tid);
  if (used) atomicMax(&s.index, tid);
  __syncthreads();
  const int at = s.bin != 0x7FFFFFFF ? s.bin : s.index;
  __syncthreads();
  if (tid == at) {
    s.bin = at;
    s.n_before = nb; s.n_at = cnt;
    s.m_before = mb; s.m_at = mass;
  }
  __syncthreads();
}

// Where the prefix ends: tokens whose logit has a larger key are kept, and of those with this very key the ones up to an index.
struct Cut {
  uint32_t key;
  int limit;
};

// Cuts the tokens of bin `bin` by the bits of their logits.  each(f): f(z, index) for every token of a set that holds the whole
// bin.  n0, m0: what lies before the bin.  Leaves the key in s.lo, the number of equals to keep in s.n_at, the kept tokens'
// count in s.n_before + s.n_at and their weight in s.total.
template <class Each>
__device__ void refine(Shared& s, const Scale& sc, int tid, int lane, int wave, int bin, u64 n0, double m0, const Goal& goal, Each each) {
  const double unit = bin_unit(bin);
  __syncthreads();
  if (tid == 0) { s.lo = 0xFFFFFFFFu; s.hi = 0; }
  __syncthreads();
  uint32_t klo = 0xFFFFFFFFu, khi = 0;
  each([&](float x, int) {
    if (sc.bin(x) != bin) return;
    klo = min(klo, key_of(x));
    khi = max(khi, key_of(x));
  });
  atomicMin(&s.lo, klo);
  atomicMax(&s.hi, khi);
  __syncthreads();
  uint32_t lo = s.lo, hi = s.hi;
  for (;;) {   // (a round leaves at most a 512th of the keys: four rounds)
    int shift = 0;
    while (((hi - lo) >> shift) >= (uint32_t)kBins) ++shift;
    __syncthreads();
    s.cnt[tid] = 0;
    s.mass[tid] = 0;
    __syncthreads();
    each([&](float x, int) {
      const uint32_t key = key_of(x);
      if (key < lo || key > hi || sc.bin(x) != bin) return;
      const int b = (int)((hi - key) >> shift);
      const double d = 8.0 * sc.dist(x);
      atomicAdd(&s.cnt[b], 1u);
      if (bin < kLast) atomicAdd(&s.mass[b], mant8(d - bin));
    });
    __syncthreads();
    find_bin(s, tid, lane, wave, n0, m0, s.cnt[tid], (double)s.mass[tid] * unit, goal);
    const uint32_t top = hi - ((uint32_t)s.bin << shift);
    n0 = s.n_before;
    m0 = s.m_before;
    if (shift == 0) {
      if (tid == s.bin) {   // one key: how many of its equals
        const double w = (double)(s.mass[tid] / s.cnt[tid]) * unit;
        u64 ties = goal.n > n0 ? goal.n - n0 : 0;
        if (w > 0.0 && goal.mass < INFINITY) {
          const double t = ceil((goal.mass - m0) / w);
          if (t < (double)ties) ties = t > 0.0 ? (u64)t : 0;
        }
        if (ties > s.cnt[tid]) ties = s.cnt[tid];
        if (ties < 1) ties = 1;
        s.lo = top;
        s.n_at = ties;
        s.total = m0 + (double)ties * w;
      }
      __syncthreads();
      return;
    }
    const uint32_t width = (1u << shift) - 1;
    lo = top - lo > width ? top - width : lo;
    hi = top;
  }
}

// The lowest index at which the running sum by index of val(z, index) over a list exceeds `target` (below the whole sum): s.index.
template <class Val>
__device__ void list_index(Shared& s, int tid, int lane, int wave, int n, int V, u64 target, Val val) {
  int shift = 0;
  while (((V - 1) >> shift) >= kBins) ++shift;   // (at most 9)
  int first = 0;
  u64 base = 0;
#pragma unroll 1
  for (int level = 0; level < 2; ++level) {   // blocks of indexes, then the indexes of one
    __syncthreads();
    s.mass[tid] = 0;
    __syncthreads();
    for (int e = tid; e < n; e += kThreads) {
      const int i = s.list.i[e];
      const int b = level == 0 ? i >> shift : i - first;
      if (level == 1 && (b < 0 || b >> shift)) continue;
      const u64 v = val(s.list.z[e], i);
      if (v) atomicAdd(&s.mass[b], v);
    }
    __syncthreads();
    u64 nb;
    double mb;
    block_scan(s, lane, wave, s.mass[tid], 0.0, nb, mb);
    if (nb + base <= target && nb + base + s.mass[tid] > target) { s.bin = tid; s.n_before = nb + base; }
    __syncthreads();
    first = level == 0 ? s.bin << shift : first + s.bin;
    base = s.n_before;
  }
  if (tid == 0) s.index = first;
  __syncthreads();
}

template <typename Tio>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  Shared& s = *reinterpret_cast<Shared*>(lds);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x, V = a.V;
  Row<Tio> rw{s, (const Tio*)a.z + (int64_t)row * a.ld, V, tid, lane, wave, false};
  rw.vec = ((uintptr_t)rw.z & (4 * sizeof(Tio) - 1)) == 0;   // (a row whose four tokens do not start on their size goes one by one)
  const float temp = a.temperature[row];
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const float mp = a.min_p ? a.min_p[row] : 0.f;
  const bool greedy = !(temp > 0.f);

  // ---- maximum, tokens above -infinity
  float best = -INFINITY;
  u64 valid = 0;
  rw.strips([&](const float (&x)[4], int) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      best = fmaxf(best, x[j]);
      valid += (unsigned)__popcll(__ballot(is_token(x[j])));   // (of the wave)
    }
  });
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) best = fmaxf(best, __shfl_xor(best, o));
  if (lane == 0) { s.wave_z[wave] = best; s.wave_n[wave] = valid; }
  if (tid == 0) { s.index = 0x7FFFFFFF; s.n_list = 0; }
  s.cnt[tid] = 0;
  s.mass[tid] = 0;
  __syncthreads();
  valid = 0;
  for (int w = 0; w < kWaves; ++w) { best = fmaxf(best, s.wave_z[w]); valid += s.wave_n[w]; }
  if (valid == 0 || greedy) {
    if (valid) {   // the lowest index with the maximum
      int at = 0x7FFFFFFF;
      rw.strips([&](const float (&x)[4], int i) {
#pragma unroll
        for (int j = 3; j >= 0; --j)
          if (x[j] == best) at = min(at, i + j);
      });
      atomicMin(&s.index, at);
      __syncthreads();
    }
    if (tid == 0) {
      a.tokens[row] = valid ? s.index : -1;
      if (a.prob) a.prob[row] = valid ? 1.f : 0.f;
      if (a.n_kept) a.n_kept[row] = valid ? 1 : 0;
    }
    return;
  }
  const Scale sc{best, 1.4426950408889634074 / (double)temp};
  const double min_w = mp > 0.f ? (double)mp : 0.0;
  const bool limit_k = k > 0 && (u64)k < valid, limit_p = p < 1.f;

  // ---- the bins at which the prefix may end.  Tokens of bins [from, to] are gathered; those before `from` are kept.
  int to = kLast, from = 0, bin_k = kLast;
  u64 n_k = valid, nb_k = 0;          // tokens that top-k leaves; tokens before its bin
  double mb_k = 0.0, z_all = 0.0;
  u64 n_to = valid;                   // tokens of bins [0, to]
  if (limit_k) {
    rw.strips([&](const float (&x)[4], int) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (is_token(x[j])) atomicAdd(&s.cnt[sc.bin(x[j])], 1u);
    });
    __syncthreads();
    find_bin(s, tid, lane, wave, 0, 0.0, s.cnt[tid], 0.0, Goal{(u64)k, INFINITY});
    bin_k = to = s.bin;
    nb_k = s.n_before;
    n_to = s.n_before + s.n_at;
    n_k = (u64)k;
    __syncthreads();
  }
  // the weights of the bins, where a limit on weight follows and the tokens do not all fit in LDS
  const bool weigh = limit_p && (!limit_k || n_to > kList);
  int bin_p = -1;
  u64 nb_p = 0;
  double mb_p = 0.0;
  if (weigh) {
    __syncthreads();
    s.cnt[tid] = 0;
    __syncthreads();
    rw.strips([&](const float (&x)[4], int) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!is_token(x[j])) continue;
        const double d = 8.0 * sc.dist(x[j]);
        const int b = d < (double)kLast ? (int)d : kLast;
        atomicAdd(&s.cnt[b], 1u);
        if (b < kLast) atomicAdd(&s.mass[b], mant8(d - b));
      }
    });
    __syncthreads();
    u64 nb;
    double mb;
    const u64 cnt = s.cnt[tid];
    const double mass = (double)s.mass[tid] * bin_unit(tid);
    block_scan(s, lane, wave, cnt, mass, nb, mb);
    if (tid == kLast) s.total = mb + mass;
    if (tid == bin_k) { s.m_before = mb; s.m_at = mass; }
    __syncthreads();
    z_all = s.total;
    mb_k = s.m_before;
    // Z_k lies between the weight before top-k's bin and the weight with it
    const double lo = limit_k ? s.m_before : z_all;
    __syncthreads();
    find_bin(s, tid, lane, wave, 0, 0.0, cnt, mass, Goal{~0ull, (double)p * lo});
    bin_p = s.bin;
    nb_p = s.n_before;
    mb_p = s.m_before;
    const u64 with = s.n_before + s.n_at;
    if (!limit_k) { to = bin_p; n_to = with; }
    __syncthreads();
  }
  if (min_w > 0.0 && !limit_k && !limit_p) {   // (one bin more than the logarithm says: its rounding must not matter)
    const double d = -log2(min_w) * 8.0;
    to = d < (double)(kLast - 2) ? (d > 0.0 ? (int)d + 1 : 1) : kLast;
    n_to = 0;   // (not known: the gathering tells)
  }

  // ---- the tokens of the prefix in LDS, if they fit
  const bool cut_needed = limit_k || limit_p;
  bool whole = (cut_needed || min_w > 0.0) && n_to <= kList;
  auto gather = [&](int a_bin, int b_bin) {
    const double d_a = a_bin, d_b = b_bin == kLast ? INFINITY : b_bin + 1.0;
    __syncthreads();
    if (tid == 0) s.n_list = 0;
    __syncthreads();
    rw.strips([&](const float (&x)[4], int at) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const double d = 8.0 * sc.dist(x[j]);
        if (!(is_token(x[j]) && d >= d_a && (d < d_b || d_b == INFINITY))) continue;
        const uint32_t e = atomicAdd(&s.n_list, 1u);
        if (e < kList) { s.list.z[e] = x[j]; s.list.i[e] = at + j; }
      }
    });
    __syncthreads();
  };
  if (whole) {
    gather(0, to);
    whole = s.n_list <= kList;
  }
  int n_list = whole ? (int)s.n_list : 0;
  auto each_listed = [&](auto f) {
    for (int e = tid; e < n_list; e += kThreads) f(s.list.z[e], s.list.i[e]);
  };
  auto each_token = [&](auto f) {
    rw.strips([&](const float (&x)[4], int at) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (is_token(x[j])) f(x[j], at + j);
    });
  };

  // ---- the cut: by count, then by weight among what that left
  Cut cut{0u, 0x7FFFFFFF};   // keeps everything
  u64 ties = 0;
  if (limit_k) {
    const Goal goal{n_k, INFINITY};
    if (whole && !weigh) {
      // (the weights before the bin are those of the list)
      u64 u = 0;
      each_listed([&](float x, int) { u += sc.bin(x) < bin_k ? sc.units(x) : 0; });
      u64 nb;
      double mb;
      block_scan(s, lane, wave, u, 0.0, nb, mb);
      if (tid == kThreads - 1) s.m_before = (double)(nb + u) * 0x1p-50;
      __syncthreads();
      mb_k = s.m_before;
      __syncthreads();
    }
    if (whole) refine(s, sc, tid, lane, wave, bin_k, nb_k, mb_k, goal, each_listed);
    else refine(s, sc, tid, lane, wave, bin_k, nb_k, mb_k, goal, each_token);
    cut.key = s.lo;
    ties = s.n_at;
    z_all = s.total;
    __syncthreads();
  }
  if (limit_p) {
    const Goal goal{n_k, (double)p * z_all};
    // the bin: among those of the list, or of the histogram (its counts and weights have been overwritten if top-k came before)
    if (limit_k) {
      s.cnt[tid] = 0;
      s.mass[tid] = 0;
      __syncthreads();
      auto add = [&](float x, int) {
        const double d = 8.0 * sc.dist(x);
        const int b = d < (double)kLast ? (int)d : kLast;
        if (b > bin_k) return;
        atomicAdd(&s.cnt[b], 1u);
        if (b < kLast) atomicAdd(&s.mass[b], mant8(d - b));
      };
      if (whole) each_listed(add);
      else each_token(add);
      __syncthreads();
      find_bin(s, tid, lane, wave, 0, 0.0, s.cnt[tid], (double)s.mass[tid] * bin_unit(tid), goal);
      bin_p = s.bin;
      nb_p = s.n_before;
      mb_p = s.m_before;
      __syncthreads();
    }
    if (whole) {
      refine(s, sc, tid, lane, wave, bin_p, nb_p, mb_p, goal, each_listed);
    } else {
      gather(bin_p, bin_p);
      if (s.n_list <= kList) {
        n_list = (int)s.n_list;
        refine(s, sc, tid, lane, wave, bin_p, nb_p, mb_p, goal, each_listed);
      } else {
        refine(s, sc, tid, lane, wave, bin_p, nb_p, mb_p, goal, each_token);
      }
    }
    cut.key = s.lo;
    ties = s.n_at;
    __syncthreads();
  }
  // ---- equal logits at the cut are kept by ascending index
  if (cut_needed) {
    if (whole) {
      list_index(s, tid, lane, wave, n_list, V, ties - 1, [&](float x, int) { return (u64)(key_of(x) == cut.key); });
      cut.limit = s.index;
      __syncthreads();
    } else {
      // four tokens of every thread at a time, in order
      u64 seen = 0;
      for (int first = 0; first < V; first += 4 * kThreads) {
        float x[4];
        const int at = first + tid * 4;
        four(rw.z, at, V, x);
        u64 mine = 0, nb;
        double mb;
#pragma unroll
        for (int j = 0; j < 4; ++j) mine += is_token(x[j]) && key_of(x[j]) == cut.key;
        block_scan(s, lane, wave, mine, 0.0, nb, mb);
        nb += seen;
        if (nb < ties && nb + mine >= ties) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (is_token(x[j]) && key_of(x[j]) == cut.key && ++nb == ties) s.index = at + j;
        }
        if (tid == kThreads - 1) s.n_at = nb < ties || mine == 0 ? nb + mine : ties;
        __syncthreads();
        seen = s.n_at;
        __syncthreads();
        if (seen >= ties) break;
      }
      cut.limit = s.index;
      __syncthreads();
    }
  }
  const float z_cut = cut_needed ? of_key(cut.key) : kLeast;   // (no cut: all of the least are kept too)
  const int limit = cut_needed ? cut.limit : 0x7FFFFFFF;
  auto kept = [&](float x, int i) { return x > z_cut || (x == z_cut && i <= limit); };   // (false for NaN)
  const float u0 = a.u[row];
  const double u1 = u0 > 0.f ? (u0 < 1.f ? (double)u0 : 1.0) : 0.0;

  // ---- the draw
  if (whole) {
    auto val = [&](float x, int i) -> u64 {
      if (!kept(x, i)) return 0;
      const double w = sc.weight(x);
      return w >= min_w || x == sc.zmax ? (u64)(w * 0x1p50 + 0.5) : 0;
    };
    u64 sum = 0, number = 0;
    each_listed([&](float x, int i) {
      if (!kept(x, i)) return;
      const double w = sc.weight(x);
      if (!(w >= min_w || x == sc.zmax)) return;
      ++number;
      sum += (u64)(w * 0x1p50 + 0.5);
    });
    sum = wave_sum(sum);
    number = wave_sum(number);
    __syncthreads();
    if (lane == 0) { s.wave_n[wave] = sum; s.mass[wave] = number; }
    __syncthreads();
    sum = number = 0;
    for (int w = 0; w < kWaves; ++w) { sum += s.wave_n[w]; number += s.mass[w]; }
    u64 target = (u64)(u1 * (double)sum);
    if (target >= sum) target = sum - 1;   // (the last token with a weight)
    list_index(s, tid, lane, wave, n_list, V, target, val);
    if (tid == 0) {
      const int i = min(s.index, V - 1);
      a.tokens[row] = i;
      if (a.prob) a.prob[row] = (float)(sc.weight(ld_logit(rw.z, i)) / ((double)sum * 0x1p-50));
      if (a.n_kept) a.n_kept[row] = (int32_t)number;
    }
    return;
  }
  // (a token that is not kept lies at the far end: its weight underflows)
  auto weight = [&](float x, int i) { return exp2_neg(kept(x, i) ? sc.dist(x) : 1100.0); };
  const int strips = (V + kStrip - 1) / kStrip;
  u64 number = 0;
  double part = 0.0;
  __syncthreads();   // (the strips' sums take the list's place)
  rw.strips(
      [&](const float (&x)[4], int at) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          double w = weight(x[j], at + j);
          bool in = kept(x[j], at + j);
          if (min_w > 0.0) {
            in = in && (w >= min_w || x[j] == sc.zmax);
            w = in ? w : 0.0;
          }
          number += (unsigned)__popcll(__ballot(in));
          part += w;
        }
      },
      [&](int st) {
        const double sum = wave_sum(part);
        if (lane == 0) s.strip[st] = sum;
        part = 0.0;
      });
  if (lane == 0) s.wave_n[wave] = number;
  __syncthreads();
  number = 0;
  for (int w = 0; w < kWaves; ++w) number += s.wave_n[w];
  // a strip a thread: the running sum passes the target in one of them
  const double sum = tid < strips ? s.strip[tid] : 0.0;
  double mb;
  u64 nb;
  block_scan(s, lane, wave, 0, sum, nb, mb);
  if (tid == kThreads - 1) s.total = mb + sum;
  if (tid == 0) { s.bin = 0x7FFFFFFF; s.index = -1; }
  __syncthreads();
  const double total = s.total, target = u1 * total;
  if (sum > 0.0) {
    if (mb + sum > target) atomicMin(&s.bin, tid);
    atomicMax(&s.index, tid);
  }
  __syncthreads();
  const bool passed = s.bin != 0x7FFFFFFF;
  const int at = passed ? s.bin : max(s.index, 0);   // (the last strip with a weight if rounding leaves none)
  if (tid == at) s.m_before = mb;
  __syncthreads();
  if (wave != 0) return;
  // and the token in the strip
  double before = s.m_before, w_token = 0.0;
  int token = -1;
  for (int u = 0; u < kPieces; ++u) {
    float x[4];
    double w[4], run = 0.0;
    const int first = at * kStrip + u * (4 * kWave) + lane * 4;
    four(rw.z, first, V, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = weight(x[j], first + j);
      if (!(w[j] >= min_w || x[j] == sc.zmax)) w[j] = 0.0;
      run += w[j];
    }
    const double inc = wave_scan(run, lane);
    double b = before + (inc - run);
    int mine = -1, last = -1;
    double w_mine = 0.0, w_last = 0.0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      b += w[j];
      if (w[j] > 0.0) {
        if (mine < 0 && b > target) { mine = first + j; w_mine = w[j]; }
        last = first + j;
        w_last = w[j];
      }
    }
    const u64 pass = __ballot(mine >= 0), has = __ballot(last >= 0);
    if (has) {
      const int src = pass ? __ffsll((long long)pass) - 1 : 63 - __clzll((long long)has);
      const int i = pass ? mine : last;
      const double wi = pass ? w_mine : w_last;
      token = __shfl(i, src);
      w_token = __shfl(wi, src);
      if (pass) break;
    }
    before += __shfl(inc, kWave - 1);
  }
  if (lane == 0) {
    a.tokens[row] = token;
    if (a.prob) a.prob[row] = (float)(w_token / total);
    if (a.n_kept) a.n_kept[row] = (int32_t)number;
  }
}

// ------------------------------------------------------------------ embedding rows

__device__ __forceinline__ void st_elem(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void st_elem(bf16_t* p, int64_t i, float v) { p[i] = f32_to_bf16(v); }

template <typename Tio>
__global__ __launch_bounds__(256) void k_embed_rows(EmbedArgs a) {
  const int t = blockIdx.x;
  const int tok = a.tokens[t], pos = a.pos ? a.pos[t] : 0;
  const Tio* e = (unsigned)tok < (unsigned)a.vocab ? (const Tio*)a.E + (int64_t)tok * a.lde : nullptr;
  const Tio* q = a.Epos && (unsigned)pos < (unsigned)a.n_pos ? (const Tio*)a.Epos + (int64_t)pos * a.ldp : nullptr;
  Tio* x = (Tio*)a.X + (int64_t)t * a.ldx;
  for (int i = threadIdx.x; i < a.d; i += 256) {
    if (!q) { x[i] = e ? e[i] : (Tio)0; continue; }
    st_elem(x, i, (e ? ld_logit(e, i) : 0.f) + ld_logit(q, i));
  }
  if (a.pos_next) {
    __syncthreads();   // (pos_next may be pos: every wave has read it)
    if (threadIdx.x == 0) a.pos_next[t] = (int32_t)((uint32_t)pos + 1u);
  }
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t st) {
  if (a.bf16) k_sample<bf16_t><<<dim3(a.T), kThreads, sizeof(Shared), st>>>(a);
  else k_sample<float><<<dim3(a.T), kThreads, sizeof(Shared), st>>>(a);
  return hipGetLastError();
}

hipError_t launch_embed_rows(const EmbedArgs& a, hipStream_t st) {
  if (a.bf16) k_embed_rows<bf16_t><<<dim3(a.T), 256, 0, st>>>(a);
  else k_embed_rows<float><<<dim3(a.T), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace zo
