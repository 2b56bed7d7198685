// The draw of a decode step's next tokens, and the embedding rows they start with.
//
//   k_sample       temperature, top-k, top-p, min-p and the draw from a given uniform
//   k_embed_rows   X[t] = E[tokens[t]] (+ E_pos[pos[t]]), positions advanced
//
// Sampling without a sort.  With the order "logit descending, index ascending" all three filters keep a prefix of a
// row's tokens, so what has to be found is the prefix's last token, never the order itself.  Weights are w = 2^-d,
// d = (M - z) log2(e) / T >= 0 in double; sums of weights are sums of 64-bit integers wherever threads add in any order, so
// they do not depend on it.
//   top-k    the k-th largest of the threads' own maxima bounds the k-th largest token from below: the tokens above it, a
//            few more than k, are gathered into LDS and no other needs an exponential.  (More than kList of them, or k beyond
//            the threads: a histogram of counts finds the bound.)
//   top-p    a histogram of weights over bins of an eighth of an octave finds the bin in which the prefix ends; inside a bin
//            the weights' mantissas add up as integers, and their sum tells the number of tokens within 5 %.
//   min-p    a comparison.
// Up to kShort gathered tokens are ranked by comparing each with each, and their weights summed in that order; the same again
// by index.  More of them, up to kList: the bin is cut again by the bits of its logits until one value is left, and equal logits
// are kept by ascending index.  A prefix of more than kList tokens stays in memory: only the last bin's tokens are gathered, and
// the draw reads the row again for its running sum.
//
// One workgroup of 16 waves per row; what bounds it is the double-precision arithmetic, 20 operations for a weight.
#include <atomic>

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
constexpr int kShort = 512;          // tokens that are ranked by comparing each with each (7 us; 1024 take 27, cutting a bin 18)

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

// Four neighbouring logits as they lie in memory, of no more than a logit's alignment: one load all the same, and a row's strips
// and the order of its sums do not depend on where it begins.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <typename Tio> struct Raw;
template <> struct Raw<float> { typedef f32x4 type; typedef f32x4 __attribute__((aligned(4))) in_memory; };
template <> struct Raw<bf16_t> { typedef u32x2 type; typedef u32x2 __attribute__((aligned(2))) in_memory; };
__device__ __forceinline__ void unpack(const f32x4& v, float (&x)[4]) {
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void unpack(const u32x2& v, float (&x)[4]) {
  x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
  x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
}
// Four from `at` of a row, one by one: -infinity behind its end.
template <typename Tio>
__device__ __forceinline__ void four(const Tio* z, int at, int V, float (&x)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = at + j < V ? ld_logit(z, at + j) : -INFINITY;
}

// Adding it leaves the nearest integer in the low word.
constexpr double kMagic = 6755399441055744.0;   // 1.5 * 2^52
// 2^(y/8) for |y| <= 1/2: the Taylor polynomial; its first omitted term is below 6e-14.
__device__ __forceinline__ double exp2_eighth(double y) {
  constexpr double kLn = 0.6931471805599453094 / 8;
  double p = kLn * kLn * kLn * kLn * kLn * kLn / 720;
  p = p * y + kLn * kLn * kLn * kLn * kLn / 120;
  p = p * y + kLn * kLn * kLn * kLn / 24;
  p = p * y + kLn * kLn * kLn / 6;
  p = p * y + kLn * kLn / 2;
  p = p * y + kLn;
  return p * y + 1.0;
}
// 2^(-diff c) for diff c in [0, 1000]: 2^-n times the Taylor polynomial of the rest, |rest| <= 1/2; its first omitted term is
// below 3e-13.  Exactly 1 at 0: rows of equal logits have weights whose sums are exact, and so is u * Z between two of them.
__device__ __forceinline__ double exp2_neg(double diff, double c) {
  const double t = __builtin_fma(diff, c, kMagic), y = __builtin_fma(-diff, c, t - kMagic);
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
  // (the exponent takes n off by itself: p is next to 1 and the result no smaller than 2^-1001)
  return __hiloint2double(__double2hiint(p) - (__double2loint(t) << 20), __double2loint(p));
}

// How far a logit lies below the row's maximum, and its weight.
struct Scale {
  float zmax;
  double c;        // log2(e) / T
  float far_bin;   // below it lies the last bin (2^-127.8 of the largest weight)
  float far;       // below it a weight is none (2^-1000)

  __device__ __forceinline__ Scale(float zmax, float temp) : zmax(zmax), c(1.4426950408889634074 / (double)temp) {
    far_bin = below(127.8, true);
    far = below(1000.0, true);
  }
  // The logit whose weight is 2^-octaves of the largest: the next one above that or the next below.
  __device__ __forceinline__ float below(double octaves, bool above) const {
    const double z = (double)zmax - octaves / c;
    if (!(z > (double)kLeast)) return kLeast;
    const float f = (float)z;
    return above ? ((double)f < z ? nextafterf(f, INFINITY) : f) : ((double)f > z ? nextafterf(f, -INFINITY) : f);
  }
  __device__ __forceinline__ double diff(float z) const { return (double)zmax - (double)z; }
  __device__ __forceinline__ int bin(float z) const {
    if (!(z >= far_bin)) return kLast;
    return (int)min((uint32_t)__double2loint(__builtin_fma(diff(z), 8.0 * c, kMagic)), (uint32_t)kLast - 1);
  }
  // bin and mantissa of a logit from far_bin on: its weight is mant * bin_unit(bin)
  __device__ __forceinline__ int bin(float z, u64& mant) const {
    const double d = diff(z), t = __builtin_fma(d, 8.0 * c, kMagic), y = __builtin_fma(-d, 8.0 * c, t - kMagic);
    // (adding 2^8 leaves units of 2^-44 in the last bits: sums of kMaxVocab of them fit into 64)
    mant = (u64)__double_as_longlong(exp2_eighth(y) + 256.0) - 0x4070000000000000ull;
    return (int)min((uint32_t)__double2loint(t), (uint32_t)kLast - 1);
  }
  __device__ __forceinline__ double weight(float z) const { return z >= far ? exp2_neg(diff(z), c) : 0.0; }
  // a weight in units of 2^-50 of the largest (sums of kList of them fit), at least one
  __device__ __forceinline__ static u64 units(double w) {
    const u64 n = (u64)(w * 0x1p50 + 0.5);
    return n ? n : (u64)(w > 0.0);
  }
};
__device__ __forceinline__ double bin_unit(int bin) { return bin >= kLast ? 0.0 : exp2_neg((double)bin, 0.125) * 0x1p-44; }

// A lane's value moved by DPP, zero where none arrives: the steps of a running sum over the wave (shifts by 1, 2, 4, 8 within rows
// of 16 lanes, then the rows' last values).
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, kRows, 0xf, false); }
template <int kCtrl, int kRows>
__device__ __forceinline__ int moved(int v) { return (int)moved<kCtrl, kRows>((uint32_t)v); }
template <int kCtrl, int kRows>
__device__ __forceinline__ u64 moved(u64 v) {
  return (u64)moved<kCtrl, kRows>((uint32_t)(v >> 32)) << 32 | moved<kCtrl, kRows>((uint32_t)v);
}
template <int kCtrl, int kRows>
__device__ __forceinline__ double moved(double v) { return __longlong_as_double((long long)moved<kCtrl, kRows>((u64)__double_as_longlong(v))); }
template <class T>
__device__ __forceinline__ T wave_scan(T v) {   // inclusive
  v += moved<0x111, 0xf>(v);
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);
  v += moved<0x143, 0xc>(v);
  return v;
}
template <class T>
__device__ __forceinline__ T of_lane(T v, int lane) { return __shfl(v, lane); }
template <class T>
__device__ __forceinline__ T wave_sum(T v) { return of_lane(wave_scan(v), kWave - 1); }

// Between LDS accesses of the wave's own lanes to each other's places: a wave's accesses are executed in order, and this keeps the
// compiler from exchanging them.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

struct Shared {
  uint32_t cnt[kBins];
  u64 mass[kBins];
  union {
    struct { float z[kList]; int32_t i[kList]; } list;
    double strip[kMaxStrips];
  };
  float packed[kWaves][kStrip / 2];
  u64 wave_n[kWaves];
  double wave_m[kWaves];
  float wave_z[kWaves];
  // results of one thread, for all
  uint32_t lo, n_list;
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

  __device__ __forceinline__ int n_strips() const { return (V + kStrip - 1) / kStrip; }
  // the lane's first token in piece u of a strip
  __device__ __forceinline__ int first(int st, int u) const { return st * kStrip + u * (4 * kWave) + lane * 4; }

  // f(x, first index) for every four tokens of a strip of kStrip tokens, strip by strip of this wave's share, then
  // done(strip).  A whole strip's loads are under way together, and those of the next one under its work.
  template <class F, class Done>
  __device__ __forceinline__ void strips(F f, Done done) const {
    const int n = n_strips(), whole = V / kStrip;
    typedef typename Raw<Tio>::type R;
    typedef typename Raw<Tio>::in_memory R_mem;
    int st = wave;
    R next[kPieces];
    auto load = [&](int at) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < kPieces; ++u) next[u] = *reinterpret_cast<const R_mem*>(z + first(at, u));
    };
    if (st < whole) load(st);
    for (; st < whole; st += kWaves) {
      R raw[kPieces];
#pragma unroll
      for (int u = 0; u < kPieces; ++u) raw[u] = next[u];
      load(min(st + kWaves, whole - 1));   // (not conditional; the last one is loaded again)
#pragma unroll
      for (int u = 0; u < kPieces; ++u) {
        float x[4];
        unpack(raw[u], x);
        f(x, first(st, u));
      }
      done(st);
    }
    if (st < n) {   // the row's end, not a whole strip
      for (int u = 0; u < kPieces; ++u) {
        float x[4];
        four(z, first(st, u), V, x);
        f(x, first(st, u));
      }
      done(st);
    }
  }
  template <class F>
  __device__ __forceinline__ void strips(F f) const {
    strips(f, [](int) {});
  }
  // f(x, first index, strip) for the lane's 4 * kPieces tokens of a strip at once
  template <class F>
  __device__ __forceinline__ void whole_strips(F f) const {
    float x[kPieces][4];
    int u = 0, begin = 0;
    strips(
        [&](const float (&y)[4], int at) {
          if (u == 0) begin = at;
#pragma unroll
          for (int j = 0; j < 4; ++j) x[u & (kPieces - 1)][j] = y[j];
          ++u;
        },
        [&](int st) {
          f(x, begin, st);
          u = 0;
        });
  }
};

// Inclusive running sums over the threads of the workgroup, in a fixed order.  `before` is the sum of the threads before.
// (Begins and ends with a barrier: the buffers may be in use on either side.)
__device__ __forceinline__ void block_scan(Shared& s, int lane, int wave, u64 n, double m, u64& n_before, double& m_before) {
  const u64 ni = wave_scan(n);
  const double mi = wave_scan(m);
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
__device__ __forceinline__ void refine(Shared& s, const Scale& sc, int tid, int lane, int wave, int bin, u64 n0, double m0, const Goal& goal, Each each) {
  const double unit = bin_unit(bin);
  // (the logits between the middles of the bins on either side; which of them are the bin's is looked at token by token)
  float z_lo = bin >= kLast ? kLeast : sc.below((bin + 1) * 0.125, false), z_hi = bin == 0 ? sc.zmax : sc.below((bin - 1) * 0.125, true);
  uint32_t lo = key_of(z_lo), hi = key_of(z_hi);
  for (;;) {   // (a round leaves at most a 512th of the keys: four rounds)
    int shift = 0;
    while (((hi - lo) >> shift) >= (uint32_t)kBins) ++shift;
    __syncthreads();
    s.cnt[tid] = 0;
    s.mass[tid] = 0;
    __syncthreads();
    each([&](float x, int) {
      if (!(x >= z_lo && x <= z_hi) || sc.bin(x) != bin) return;
      const int b = (int)((hi - key_of(x)) >> shift);
      atomicAdd(&s.cnt[b], 1u);
      if (bin < kLast) {
        u64 mant;
        sc.bin(x, mant);
        atomicAdd(&s.mass[b], mant);
      }
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
    z_lo = of_key(lo);
    z_hi = of_key(hi);
  }
}

// The lowest index at which the running sum by index of val(z, index) over a list exceeds `target` (below the whole sum): s.index.
template <class Val>
__device__ __forceinline__ void list_index(Shared& s, int tid, int lane, int wave, int n, int V, u64 target, Val val) {
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

// The index of the n-th (from 0) token of the row for which is(z), which there is: s.index.  Counts by strips, then the strip.
template <typename Tio, class Is>
__device__ __forceinline__ void nth_index(const Row<Tio>& rw, u64 n, Is is) {
  Shared& s = rw.s;
  const int strips = rw.n_strips();
  uint32_t c = 0;
  __syncthreads();
  rw.strips(
      [&](const float (&x)[4], int) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c += (unsigned)__popcll(__ballot(is(x[j])));
      },
      [&](int st) {
        if (rw.lane == 0) s.cnt[st] = c;
        c = 0;
      });
  __syncthreads();
  const u64 mine = rw.tid < strips ? s.cnt[rw.tid] : 0;
  u64 nb;
  double mb;
  block_scan(s, rw.lane, rw.wave, mine, 0.0, nb, mb);
  if (rw.tid == 0) { s.bin = 0; s.index = 0; s.n_before = 0; }
  __syncthreads();
  if (nb <= n && nb + mine > n) { s.bin = rw.tid; s.n_before = nb; }
  __syncthreads();
  if (rw.wave == 0) {
    u64 seen = s.n_before;
    for (int u = 0; u < kPieces; ++u) {
      float x[4];
      const int at = rw.first(s.bin, u);
      four(rw.z, at, rw.V, x);
      int here = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) here += is(x[j]);
      const int inc = wave_scan(here);
      u64 b = seen + (u64)(inc - here);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (is(x[j]) && b++ == n) s.index = at + j;
      seen += (u64)of_lane(inc, kWave - 1);
    }
  }
  __syncthreads();
}

// Sum over the workgroup, for every thread.
__device__ __forceinline__ u64 block_sum(Shared& s, int lane, int wave, u64 v) {
  v = wave_sum(v);
  __syncthreads();
  if (lane == 0) s.wave_n[wave] = v;
  __syncthreads();
  u64 n = 0;
  for (int w = 0; w < kWaves; ++w) n += s.wave_n[w];
  return n;
}

template <typename Tio>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  Shared& s = *reinterpret_cast<Shared*>(lds);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x, V = a.V;
  Row<Tio> rw{s, (const Tio*)a.z + (int64_t)row * a.ld, V, tid, lane, wave};
  const float temp = a.temperature[row];
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const float mp = a.min_p ? a.min_p[row] : 0.f;
  const float u0 = a.u[row];
  const double u1 = u0 > 0.f ? (u0 < 1.f ? (double)u0 : 1.0) : 0.0;
  // (no weight reaches a min_p above 1: the first of the order is kept, as without a temperature)
  const bool greedy = !(temp > 0.f) || mp > 1.f;
  auto answer = [&](int token, double prob, u64 number) __attribute__((always_inline)) {
    a.tokens[row] = token;
    if (a.prob) a.prob[row] = (float)prob;
    if (a.n_kept) a.n_kept[row] = (int32_t)number;
  };

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
  const float own = best;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) best = fmaxf(best, __shfl_xor(best, o));
  if (lane == 0) { s.wave_z[wave] = best; s.wave_n[wave] = valid; }
  if (tid == 0) { s.index = 0; s.n_list = 0; }
  s.cnt[tid] = 0;
  s.mass[tid] = 0;
  __syncthreads();
  valid = 0;
  for (int w = 0; w < kWaves; ++w) { best = fmaxf(best, s.wave_z[w]); valid += s.wave_n[w]; }
  if (valid == 0) {
    if (tid == 0) answer(-1, 0.0, 0);
    return;
  }
  const bool limit_k = k > 0 && (u64)k < valid, limit_p = p < 1.f, limit_m = mp > 0.f;
  const double min_w = limit_m ? (double)mp : 0.0;
  if (greedy || best == INFINITY) {
    // the first of the largest, or one of those at +infinity: of weight 1 each, the others have none
    u64 n = 0, number = 1;
    double prob = 1.0;
    __syncthreads();
    if (!greedy) {
      u64 mine = 0;
      rw.strips([&](const float (&x)[4], int) {
#pragma unroll
        for (int j = 0; j < 4; ++j) mine += x[j] == best;
      });
      const u64 at_top = block_sum(s, lane, wave, mine), first_k = limit_k ? (u64)k : valid;
      const u64 mass_k = first_k < at_top ? first_k : at_top;
      number = first_k;
      if (limit_p) {
        const double c = ceil((double)p * (double)mass_k);
        number = c < 1.0 ? 1 : c < (double)mass_k ? (u64)c : mass_k;
      }
      if (limit_m && number > at_top) number = at_top;
      const u64 drawn = number < at_top ? number : at_top;
      n = (u64)(u1 * (double)drawn);
      if (n >= drawn) n = drawn - 1;
      prob = 1.0 / (double)drawn;
      __syncthreads();
    }
    nth_index(rw, n, [&](float x) { return x == best; });
    if (tid == 0) answer(s.index, prob, number);
    return;
  }
  const Scale sc(best, temp);
  auto weight = [&](float x) { return sc.weight(x); };
  auto by_min = [&](double w) { return w >= min_w; };   // (the largest weight is exactly 1)

  // ---- the tokens of bins 0 .. `to` hold the prefix; n_to of them, about
  int to = kLast;
  double n_to = (double)valid;
  // bin of the k-th largest of what add(f) passes to f
  if (limit_k) {
    const bool few = k <= kThreads / 2;
    if (few) {
      if (is_token(own)) atomicAdd(&s.cnt[sc.bin(own)], 1u);
    } else {
      rw.strips([&](const float (&x)[4], int) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (is_token(x[j])) atomicAdd(&s.cnt[sc.bin(x[j])], 1u);
      });
    }
    __syncthreads();
    // (fewer than k threads with a token: the last bin in use, and then every bin)
    find_bin(s, tid, lane, wave, 0, 0.0, s.cnt[tid], 0.0, Goal{(u64)k, INFINITY});
    to = s.n_before + s.n_at >= (u64)k ? s.bin : kLast;
    n_to = few ? 0.0 : (double)(s.n_before + s.n_at);   // (0: not known, the gathering tells)
    __syncthreads();
  }
  // weights of all bins, for a limit on weight among more tokens than fit in LDS
  double z_all = 0.0, m_to = 0.0;
  int bin_p = -1;
  auto weigh = [&]() __attribute__((always_inline)) {
    __syncthreads();
    s.mass[tid] = 0;
    __syncthreads();
    rw.strips([&](const float (&x)[4], int) {
      u64 mant[4];
      int b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = sc.bin(x[j], mant[j]);
      asm volatile("" : "+v"(mant[0]), "+v"(mant[1]), "+v"(mant[2]), "+v"(mant[3]));   // (all four at once)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (x[j] >= sc.far_bin) atomicAdd(&s.mass[b[j]], mant[j]);
    });
    __syncthreads();
  };
  if (limit_p && !limit_k) {
    weigh();
    const u64 sum = s.mass[tid];
    const double mass = (double)sum * bin_unit(tid);
    u64 nb;
    double mb;
    block_scan(s, lane, wave, sum, mass, nb, mb);
    if (tid == kLast) s.total = mb + mass;
    __syncthreads();
    z_all = s.total;
    find_bin(s, tid, lane, wave, 0, 0.0, (uint32_t)(sum > 0), mass, Goal{~0ull, (double)p * z_all});
    bin_p = to = s.bin;
    m_to = s.m_before;
    if (tid == to) s.total = (double)(nb + sum) * (0x1p-44 * 1.05);
    __syncthreads();
    n_to = s.total;
    __syncthreads();
  }
  if (limit_m && !limit_k && !limit_p) {   // (a bin more than the logarithm says: roundings must not matter)
    const double d = -log2(min_w) * 8.0 + 2.0;
    to = d < (double)(kLast - 1) ? (d > 1.0 ? (int)d : 1) : kLast;
    n_to = 0.0;
  }

  // ---- the tokens of the prefix in LDS, if they fit
  const bool cut_needed = limit_k || limit_p;
  auto gather = [&](int a_bin, int b_bin) __attribute__((always_inline)) {
    // (a comparison keeps most tokens out, with a bin to spare for its rounding)
    const float least = b_bin >= kLast - 2 ? kLeast : sc.below((b_bin + 1.5) * 0.125, false);
    __syncthreads();
    if (tid == 0) s.n_list = 0;
    __syncthreads();
    rw.strips([&](const float (&x)[4], int at) {   // (tokens that come in are rare: a branch each)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!(x[j] >= least)) continue;
        const int b = sc.bin(x[j]);
        if (b < a_bin || b > b_bin) continue;
        const uint32_t e = atomicAdd(&s.n_list, 1u);
        if (e < kList) { s.list.z[e] = x[j]; s.list.i[e] = at + j; }
      }
    });
    __syncthreads();
  };
  bool whole = (cut_needed || limit_m) && n_to <= (double)kList;
  if (whole) {
    gather(0, to);
    whole = s.n_list <= kList;
  }
  int n_list = whole ? (int)s.n_list : 0;

  // ---- short lists: each with each
  u64* const keys = reinterpret_cast<u64*>(&s.list.z[kList / 2]);   // (behind kThreads tokens)
  float* const lz = s.list.z;
  int32_t* const li = s.list.i;
  // How many of the n <= kShort keys are larger than thread tid's: s.cnt[tid].  Where there are fewer keys than threads,
  // several threads share one's comparisons.
  auto ranks = [&](u64 key, int n) __attribute__((always_inline)) {
    int width = kWave;
    while (width < n) width <<= 1;
    keys[tid] = key;   // (0 behind the n-th)
    s.cnt[tid] = 0;
    __syncthreads();
    const int mine = tid & (width - 1), share = (n * (width / kWave) + kThreads / kWave * 8 - 1) / (kThreads / kWave * 8) * 8;
    const int from = tid / width * share, upto = min(from + share, (n + 7) & ~7);
    const u64 own = keys[mine];
    uint32_t r = 0;
    for (int e0 = from; e0 < upto; e0 += 8) {
      u64 y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = keys[e0 + e];
#pragma unroll
      for (int e = 0; e < 8; ++e) r += y[e] > own;
    }
    if (r) atomicAdd(&s.cnt[mine], r);
    __syncthreads();
  };
  // the n <= kShort tokens of the list in order
  auto sort_list = [&](int n) __attribute__((always_inline)) {
    const float x = tid < n ? lz[tid] : -INFINITY;
    const int i = tid < n ? li[tid] : 0;
    ranks(tid < n ? (u64)key_of(x) << 32 | (uint32_t)~i : 0, n);
    const int rank = s.cnt[tid];
    if (tid < n) { lz[rank] = x; li[rank] = i; }
    __syncthreads();
  };
  if (whole && n_list <= kShort) {
    int n = n_list;
    u64 nb;
    double mb;
    if (cut_needed) sort_list(n);
    if (limit_k && n > k) n = k;
    const float x = tid < n ? lz[tid] : -INFINITY;
    const int i = tid < n ? li[tid] : 0;
    bool in = tid < n;
    const double w = in ? weight(x) : 0.0;
    u64 un = Scale::units(w);
    if (limit_p) {
      const double z_k = limit_k ? (double)block_sum(s, lane, wave, un) * 0x1p-50 : z_all;
      block_scan(s, lane, wave, un, 0.0, nb, mb);
      in = in && (tid == 0 || (double)nb * 0x1p-50 < (double)p * z_k);
    }
    in = in && by_min(w);
    un = in ? un : 0;
    const u64 sum = block_sum(s, lane, wave, un);
    const u64 number = block_sum(s, lane, wave, (u64)in);
    u64 target = (u64)(u1 * (double)sum);
    if (target >= sum) target = sum - 1;   // (the last token with a weight)
    // by index: their running sum
    __syncthreads();
    ranks(in ? (u64)(uint32_t)~i : 0, n);
    s.mass[tid] = 0;
    __syncthreads();
    const int place = s.cnt[tid];
    if (in) s.mass[place] = un;
    __syncthreads();
    block_scan(s, lane, wave, s.mass[tid], 0.0, nb, mb);
    if (nb <= target && nb + s.mass[tid] > target) s.bin = tid;
    __syncthreads();
    if (in && place == s.bin) answer(i, w / ((double)sum * 0x1p-50), number);
    return;
  }

  auto each_listed = [&](auto f) __attribute__((always_inline)) {
    for (int e = tid; e < n_list; e += kThreads) f(s.list.z[e], s.list.i[e]);
  };
  auto each_token = [&](auto f) __attribute__((always_inline)) {
    rw.strips([&](const float (&x)[4], int at) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (is_token(x[j])) f(x[j], at + j);
    });
  };
  // counts and weights of the bins 0 .. `to`
  auto histogram = [&](auto each) __attribute__((always_inline)) {
    __syncthreads();
    s.cnt[tid] = 0;
    s.mass[tid] = 0;
    __syncthreads();
    each([&](float x, int) {
      const int b = sc.bin(x);
      if (b > to) return;
      atomicAdd(&s.cnt[b], 1u);
      if (b == kLast) return;
      u64 mant;
      sc.bin(x, mant);
      atomicAdd(&s.mass[b], mant);
    });
    __syncthreads();
  };

  // ---- the cut: by count, then by weight among what that left
  Cut cut{0u, 0x7FFFFFFF};
  u64 ties = 0;
  if (limit_k) {
    const Goal by_count{(u64)k, INFINITY};
    auto cut_k = [&](auto each) __attribute__((always_inline)) {
      histogram(each);
      const uint32_t cnt = s.cnt[tid];
      const double mass = (double)s.mass[tid] * bin_unit(tid);
      find_bin(s, tid, lane, wave, 0, 0.0, cnt, mass, by_count);
      const int bin_k = s.bin;
      const u64 nb = s.n_before;
      const double mb = s.m_before;
      refine(s, sc, tid, lane, wave, bin_k, nb, mb, by_count, each);
      cut.key = s.lo;
      ties = s.n_at;
      if (limit_p) {
        const Goal by_both{(u64)k, (double)p * s.total};
        histogram(each);
        find_bin(s, tid, lane, wave, 0, 0.0, s.cnt[tid], (double)s.mass[tid] * bin_unit(tid), by_both);
        const int b = s.bin;
        const u64 nb_p = s.n_before;
        const double mb_p = s.m_before;
        refine(s, sc, tid, lane, wave, b, nb_p, mb_p, by_both, each);
        cut.key = s.lo;
        ties = s.n_at;
      }
    };
    if (whole) cut_k(each_listed);
    else cut_k(each_token);
  } else if (limit_p) {
    const Goal by_mass{~0ull, (double)p * z_all};
    if (!whole) {
      gather(bin_p, bin_p);
      n_list = s.n_list <= kList ? (int)s.n_list : 0;
    }
    if (!whole && n_list > 0 && n_list <= kShort) {
      sort_list(n_list);
      const bool in = tid < n_list;
      const float x = in ? lz[tid] : -INFINITY;
      const u64 un = in ? Scale::units(weight(x)) : 0;
      u64 nb;
      double mb;
      block_scan(s, lane, wave, un, 0.0, nb, mb);
      // (the bin was chosen because the limit lies in it: its first token is kept)
      if (tid == 0) s.index = 0;
      __syncthreads();
      if (in && m_to + (double)nb * 0x1p-50 < by_mass.mass) atomicMax(&s.index, tid);
      __syncthreads();
      cut.key = key_of(lz[s.index]);
      cut.limit = li[s.index];
      ties = 0;   // (settled)
    } else if (whole || n_list > 0) refine(s, sc, tid, lane, wave, bin_p, 0, m_to, by_mass, each_listed);
    else refine(s, sc, tid, lane, wave, bin_p, 0, m_to, by_mass, each_token);
    if (whole || n_list == 0 || n_list > kShort) {
      cut.key = s.lo;
      ties = s.n_at;
    }
  }
  __syncthreads();
  // ---- equal logits at the cut are kept by ascending index
  if (cut_needed && ties > 0) {
    if (whole || (!limit_k && n_list > 0))
      list_index(s, tid, lane, wave, n_list, V, ties - 1, [&](float x, int) { return (u64)(key_of(x) == cut.key); });
    else
      nth_index(rw, ties - 1, [&](float x) { return is_token(x) && key_of(x) == cut.key; });
    cut.limit = s.index;
    __syncthreads();
  }
  const float z_cut = cut_needed ? of_key(cut.key) : kLeast;   // (no cut: all of the least are kept too)
  const int limit = cut.limit;
  auto kept = [&](float x, int i) { return x > z_cut || (x == z_cut && i <= limit); };   // (false for NaN)

  // ---- the draw
  if (whole) {
    auto val = [&](float x, int i) __attribute__((always_inline)) -> u64 {
      if (!kept(x, i)) return 0;
      const double w = weight(x);
      return by_min(w) ? Scale::units(w) : 0;
    };
    u64 sum = 0, number = 0;
    each_listed([&](float x, int i) {
      if (!kept(x, i)) return;
      const double w = weight(x);
      if (!by_min(w)) return;
      ++number;
      sum += Scale::units(w);
    });
    sum = block_sum(s, lane, wave, sum);
    number = block_sum(s, lane, wave, number);
    u64 target = (u64)(u1 * (double)sum);
    if (target >= sum) target = sum - 1;   // (the last token with a weight)
    list_index(s, tid, lane, wave, n_list, V, target, val);
    if (tid == 0) {
      const int i = min(s.index, V - 1);
      answer(i, weight(ld_logit(rw.z, i)) / ((double)sum * 0x1p-50), number);
    }
    return;
  }
  const int strips = rw.n_strips();
  u64 number = 0;
  __syncthreads();   // (the strips' sums take the list's place)
  float* const packed = s.packed[wave];
  rw.whole_strips([&](const float (&x)[kPieces][4], int first, int st) {
    bool in[kPieces][4], equal = false;
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        in[u][j] = x[u][j] >= z_cut;   // (false for NaN)
        equal = equal || x[u][j] == z_cut;
      }
    if (__any(equal)) {   // (equal logits at the cut: as far as the limit)
#pragma unroll
      for (int u = 0; u < kPieces; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) in[u][j] = kept(x[u][j], first + u * (4 * kWave) + j);
    }
    int n = 0;
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) n += __popcll(__ballot(in[u][j]));
    double part = 0.0;
    auto add = [&](float z, bool there, double w) __attribute__((always_inline)) {
      bool take = there && z >= sc.far;
      if (limit_m) {
        take = take && by_min(w);
        number += (unsigned)__popcll(__ballot(take));
      }
      part += take ? w : 0.0;
    };
    if (!limit_m) number += (unsigned)n;
    if (n > kStrip / 2) {
#pragma unroll
      for (int u = 0; u < kPieces; ++u)
        {
          // (four at once, of no use where a token is not kept or too far: a branch around each costs more)
          double w[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) w[c] = exp2_neg(sc.diff(x[u][c]), sc.c);
          asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
#pragma unroll
          for (int c = 0; c < 4; ++c) add(x[u][c], in[u][c], w[c]);
        }
    } else {   // the kept ones packed: an exponential costs more than moving them
      int at = 0;
#pragma unroll
      for (int u = 0; u < kPieces; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u64 m = __ballot(in[u][j]);
          if (in[u][j]) packed[at + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0))] = x[u][j];
          at += __popcll(m);
        }
      wave_lds_order();
      for (int e = 0; e < n; e += kWave) {
        const float z = e + lane < n ? packed[e + lane] : sc.zmax;
        add(z, e + lane < n, exp2_neg(sc.diff(z), sc.c));
      }
      wave_lds_order();   // (the next strip's come to the same place)
    }
    const double sum = wave_sum(part);
    if (lane == 0) s.strip[st] = sum;
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
    const int first = rw.first(at, u);
    four(rw.z, first, V, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = kept(x[j], first + j) ? weight(x[j]) : 0.0;
      if (!by_min(w[j])) w[j] = 0.0;
      run += w[j];
    }
    const double inc = wave_scan(run);
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
    before += of_lane(inc, kWave - 1);
  }
  if (lane == 0) answer(token, w_token / total, number);
}

// ------------------------------------------------------------------ embedding rows

__device__ __forceinline__ void st_elem(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void st_elem(bf16_t* p, int64_t i, float v) { p[i] = f32_to_bf16(v); }

// Rows of any width and alignment, element by element.
template <typename Tio>
__global__ __launch_bounds__(256) void k_embed_rows_any(EmbedArgs a) {
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

// Rows whose pieces of 16 bytes are aligned: 2^log_lanes threads per row, about as many as it has pieces, four pieces of a thread
// under way.  16384 rows of 5120 with positions: 75 us (4.8 TB/s), element by element 180; few rows: the latency of two loads
// that depend on each other.
template <typename Tio>
__global__ __launch_bounds__(256) void k_embed_rows(EmbedArgs a, int log_lanes) {
  constexpr int kDeep = 4, kPer = 16 / sizeof(Tio);
  const int lanes = 1 << log_lanes, lane = threadIdx.x & (lanes - 1);
  const int64_t row = (int64_t)blockIdx.x * (256 >> log_lanes) + (threadIdx.x >> log_lanes);
  const bool there = row < a.T;
  const int t = there ? (int)row : 0;
  const int tok = a.tokens[t], pos = a.pos ? a.pos[t] : 0;
  const u32x4* e = (unsigned)tok < (unsigned)a.vocab ? (const u32x4*)((const Tio*)a.E + (int64_t)tok * a.lde) : nullptr;
  const u32x4* q = a.Epos && (unsigned)pos < (unsigned)a.n_pos ? (const u32x4*)((const Tio*)a.Epos + (int64_t)pos * a.ldp) : nullptr;
  u32x4* x = (u32x4*)((Tio*)a.X + (int64_t)t * a.ldx);
  const int n = there ? a.d / kPer : 0;
  for (int i0 = lane; i0 < n; i0 += kDeep * lanes) {
    u32x4 v[kDeep], w[kDeep];
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      const int i = i0 + u * lanes;
      v[u] = e && i < n ? e[i] : u32x4{0u, 0u, 0u, 0u};
      w[u] = q && i < n ? q[i] : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      const int i = i0 + u * lanes;
      if (i >= n) break;
      if (q) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if constexpr (sizeof(Tio) == 2)
            v[u][c] = pack_bf16x2(__uint_as_float(v[u][c] << 16) + __uint_as_float(w[u][c] << 16),
                                  __uint_as_float(v[u][c] & 0xFFFF0000u) + __uint_as_float(w[u][c] & 0xFFFF0000u));
          else
            v[u][c] = __float_as_uint(__uint_as_float(v[u][c]) + __uint_as_float(w[u][c]));
        }
      }
      x[i] = v[u];
    }
  }
  if (a.pos_next) {
    __syncthreads();   // (pos_next may be pos: every thread has read it)
    if (there && lane == 0) a.pos_next[t] = (int32_t)((uint32_t)pos + 1u);
  }
}

}  // namespace

namespace {
template <typename Tio>
hipError_t launch_sample_of(const SampleArgs& a, hipStream_t st) {
  static std::atomic<bool> ready[kMaxDevices];
  const hipError_t e = once_per_device(ready, [] {
    return hipFuncSetAttribute((const void*)k_sample<Tio>, hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(Shared));
  });
  if (e != hipSuccess) return e;
  k_sample<Tio><<<dim3(a.T), kThreads, sizeof(Shared), st>>>(a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t st) {
  return a.bf16 ? launch_sample_of<bf16_t>(a, st) : launch_sample_of<float>(a, st);
}

hipError_t launch_embed_rows(const EmbedArgs& a, hipStream_t st) {
  const int size = a.bf16 ? 2 : 4;
  auto aligned = [&](const void* p, int64_t ld) { return ((uintptr_t)p & 15u) == 0 && ld * size % 16 == 0; };
  const bool wide = a.d * size % 16 == 0 && aligned(a.E, a.lde) && aligned(a.X, a.ldx) && (!a.Epos || aligned(a.Epos, a.ldp));
  int log_lanes = 3;
  while (log_lanes < 8 && (16 << log_lanes) < a.d * size) ++log_lanes;
  const dim3 grid(a.T), rows((unsigned)(((int64_t)a.T + (256 >> log_lanes) - 1) / (256 >> log_lanes)));
  if (wide && a.bf16) k_embed_rows<bf16_t><<<rows, 256, 0, st>>>(a, log_lanes);
  else if (wide) k_embed_rows<float><<<rows, 256, 0, st>>>(a, log_lanes);
  else if (a.bf16) k_embed_rows_any<bf16_t><<<grid, 256, 0, st>>>(a);
  else k_embed_rows_any<float><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace zo
