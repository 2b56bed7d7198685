// The draw of a decode step's next tokens, and the embedding rows they start with.
//
//   k_sample       temperature, top-k, top-p, min-p and the draw from a given uniform
//   k_embed_rows   X[t] = E[tokens[t]] (+ E_pos[pos[t]]), positions advanced
//
// Sampling without a sort.  With the order "logit descending, index ascending" all three filters keep a prefix of a
// row's tokens, so what has to be found is the prefix's last token, never the order itself.  Weights are
// w = 2^-d, d = (M - z) log2(e) / T >= 0 in double; a token falls into bin floor(8 d), and a histogram of counts and
// weights over the bins tells in which bin the prefix ends.  Inside a bin all weights share floor(d), so their
// mantissas add up as 64-bit integers: the sums are exact and do not depend on the order in which threads add.  The
// bin where the prefix ends is cut again by the bits of its logits until one value is left, and equal logits are kept by
// ascending index.  The draw is a prefix sum by index over the kept tokens: sums of 256 tokens, then of one.
#include "zo_device.hpp"
#include "zo_internal.hpp"

namespace zo {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 1024;          // eighths of d up to 128; the last bin holds the rest (weights below 2^-127: none)
constexpr int kStrip = 256;          // tokens per partial sum of the draw
constexpr int kMaxStrips = (1 << 19) / kStrip;

__device__ __forceinline__ float ld_logit(const float* p, int i) { return p[i]; }
__device__ __forceinline__ float ld_logit(const bf16_t* p, int i) { return bf16_to_f32(p[i]); }
// NaN counts as -infinity, -0 as 0
__device__ __forceinline__ float clean(float z) { return z != z ? -INFINITY : z + 0.0f; }
// Unsigned integers in the order of the floats.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// 2^-f for f in [0, 1): 2^-1/2 times the Taylor polynomial of exp((1/2 - f) ln 2); its first omitted term is below 2e-16.
__device__ __forceinline__ double exp2_neg(double f) {
  const double x = (0.5 - f) * 0.6931471805599453094;
  double p = 1.0 / 479001600.0;
  p = p * x + 1.0 / 39916800.0;
  p = p * x + 1.0 / 3628800.0;
  p = p * x + 1.0 / 362880.0;
  p = p * x + 1.0 / 40320.0;
  p = p * x + 1.0 / 5040.0;
  p = p * x + 1.0 / 720.0;
  p = p * x + 1.0 / 120.0;
  p = p * x + 1.0 / 24.0;
  p = p * x + 1.0 / 6.0;
  p = p * x + 0.5;
  p = p * x + 1.0;
  p = p * x + 1.0;
  return p * 0.70710678118654752440;
}

// How far a logit lies below the row's maximum, and its weight.
struct Scale {
  float zmax;
  double c;   // log2(e) / T
  __device__ __forceinline__ double dist(float z) const { return z == zmax ? 0.0 : ((double)zmax - (double)z) * c; }
};
__device__ __forceinline__ int bin_of(double d) { return d < 127.875 ? (int)(d * 8.0) : kBins - 1; }
// mantissa of a weight as an integer of 2^-44 ulps; the weight is mant * 2^(-44 - floor(d))
__device__ __forceinline__ uint64_t mant_of(double d) { return (uint64_t)(exp2_neg(d - floor(d)) * 0x1p44 + 0.5); }
__device__ __forceinline__ double weight_of(double d) { return d < 1000.0 ? ldexp(exp2_neg(d - floor(d)), -(int)d) : 0.0; }
__device__ __forceinline__ double bin_unit(int bin) { return bin == kBins - 1 ? 0.0 : ldexp(1.0, -44 - (bin >> 3)); }

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Where the prefix ends: tokens whose logit has a larger key are kept, and of those with this very key the first `ties`.
struct Cut {
  uint32_t key;
  uint32_t ties;
};

struct Shared {
  uint32_t cnt[kBins];
  unsigned long long mass[kBins];
  double strip[kMaxStrips];
  float red_z[kWaves];
  int red_i[kWaves];
  uint32_t red_n[kWaves];
  double red_d[kWaves];
  // results of one thread, for all
  uint32_t lo, hi, key, ties, n;
  int bin;
  double before, total;
};

// What the search for a cut counts: tokens up to `n`, or weight up to `mass` (whichever ends first).
struct Goal {
  uint64_t n;
  double mass;
};

// Finds the first bin at which the running count reaches goal.n or the running weight goal.mass; thread 0's job (the bins
// are few).  unit(b): weight of one mantissa unit in bin b.
template <class Unit>
__device__ int find_bin(const Shared& s, int nbins, const Goal& goal, Unit unit, uint64_t& n, double& mass) {
  int last = -1;
  for (int b = 0; b < nbins; ++b) {
    if (s.cnt[b] == 0) continue;
    last = b;
    const double w = (double)s.mass[b] * unit(b);
    if (n + s.cnt[b] >= goal.n || mass + w >= goal.mass) return b;
    n += s.cnt[b];
    mass += w;
  }
  if (last >= 0) {   // (the goal lies beyond the last token by a rounding: the last bin)
    n -= s.cnt[last];
    mass -= (double)s.mass[last] * unit(last);
  }
  return last;
}

// One workgroup per row.
template <typename Tio>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  Shared& s = *reinterpret_cast<Shared*>(lds);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x, V = a.V;
  const Tio* z = (const Tio*)a.z + (int64_t)row * a.ld;
  const float temp = a.temperature[row];
  const bool greedy = !(temp > 0.f);

  // ---- maximum, the lowest index that has it, tokens above -infinity
  float best = -INFINITY;
  int best_i = 0x7FFFFFFF;
  uint32_t valid = 0;
  for (int i = tid; i < V; i += kThreads) {
    const float x = clean(ld_logit(z, i));
    if (x > best) { best = x; best_i = i; }
    valid += x > -INFINITY;
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const float ob = __shfl_xor(best, o);
    const int oi = __shfl_xor(best_i, o);
    if (ob > best || (ob == best && oi < best_i)) { best = ob; best_i = oi; }
    valid += __shfl_xor(valid, o);
  }
  if (lane == 0) { s.red_z[wave] = best; s.red_i[wave] = best_i; s.red_n[wave] = valid; }
  __syncthreads();
  best = s.red_z[0]; best_i = s.red_i[0]; valid = s.red_n[0];
  for (int w = 1; w < kWaves; ++w) {
    if (s.red_z[w] > best || (s.red_z[w] == best && s.red_i[w] < best_i)) { best = s.red_z[w]; best_i = s.red_i[w]; }
    valid += s.red_n[w];
  }
  if (valid == 0 || greedy) {
    if (tid == 0) {
      a.tokens[row] = valid ? best_i : -1;
      if (a.prob) a.prob[row] = valid ? 1.f : 0.f;
      if (a.n_kept) a.n_kept[row] = valid ? 1 : 0;
    }
    return;
  }
  const Scale sc{best, 1.4426950408889634074 / (double)temp};
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const float mp = a.min_p ? a.min_p[row] : 0.f;
  const double min_w = mp > 0.f ? (double)mp : 0.0;

  // ---- histogram over the bins of d
  for (int b = tid; b < kBins; b += kThreads) { s.cnt[b] = 0; s.mass[b] = 0; }
  __syncthreads();
  for (int i = tid; i < V; i += kThreads) {
    const float x = clean(ld_logit(z, i));
    if (!(x > -INFINITY)) continue;
    const double d = sc.dist(x);
    const int b = bin_of(d);
    atomicAdd(&s.cnt[b], 1u);
    if (b < kBins - 1) atomicAdd(&s.mass[b], (unsigned long long)mant_of(d));
  }
  __syncthreads();

  // ---- the cut: by count, then by weight among what that left
  Cut cut{0u, 0xFFFFFFFFu};   // keeps everything
  uint64_t n_cut = valid;
  double z_k = 0.0;
  const bool limit_k = k > 0 && (uint32_t)k < valid, limit_p = p < 1.f;
  for (int pass = 0; pass < 2; ++pass) {
    if (pass == 0 ? !limit_k : !limit_p) {
      if (pass == 0 && limit_p) {   // Z_k is the weight of all tokens
        if (tid == 0) {
          double m = 0.0;
          for (int b = 0; b < kBins; ++b) m += (double)s.mass[b] * bin_unit(b);
          s.total = m;
        }
        __syncthreads();
        z_k = s.total;
        __syncthreads();
      }
      continue;
    }
    const Goal goal = pass == 0 ? Goal{(uint64_t)k, INFINITY} : Goal{n_cut, (double)p * z_k};
    // bins of d
    if (tid == 0) {
      uint64_t n = 0;
      double m = 0.0;
      s.bin = find_bin(s, kBins, goal, bin_unit, n, m);
      s.n = (uint32_t)n;
      s.before = m;
      s.lo = 0xFFFFFFFFu;
      s.hi = 0;
    }
    __syncthreads();
    const int bin = s.bin;
    const double unit = bin_unit(bin);
    // the range of its keys
    uint32_t klo = 0xFFFFFFFFu, khi = 0;
    for (int i = tid; i < V; i += kThreads) {
      const float x = clean(ld_logit(z, i));
      if (!(x > -INFINITY) || bin_of(sc.dist(x)) != bin) continue;
      klo = min(klo, key_of(x));
      khi = max(khi, key_of(x));
    }
    atomicMin(&s.lo, klo);
    atomicMax(&s.hi, khi);
    __syncthreads();
    uint32_t lo = s.lo, hi = s.hi;
    // cut by the keys, from the largest down, until one is left
    __shared__ uint32_t sub_cnt[kBins];
    __shared__ unsigned long long sub_mass[kBins];
    for (;;) {
      int shift = 0;
      while (((hi - lo) >> shift) >= (uint32_t)kBins) ++shift;
      __syncthreads();
      for (int b = tid; b < kBins; b += kThreads) { sub_cnt[b] = 0; sub_mass[b] = 0; }
      __syncthreads();
      for (int i = tid; i < V; i += kThreads) {
        const float x = clean(ld_logit(z, i));
        if (!(x > -INFINITY)) continue;
        const uint32_t key = key_of(x);
        if (key < lo || key > hi) continue;
        const double d = sc.dist(x);
        atomicAdd(&sub_cnt[(hi - key) >> shift], 1u);
        if (bin < kBins - 1) atomicAdd(&sub_mass[(hi - key) >> shift], (unsigned long long)mant_of(d));
      }
      __syncthreads();
      if (tid == 0) {
        uint64_t n = s.n;
        double m = s.before;
        int last = -1;
        uint64_t n_last = n;
        double m_last = m;
        for (int b = 0; b < kBins; ++b) {
          if (sub_cnt[b] == 0) continue;
          last = b; n_last = n; m_last = m;
          const double w = (double)sub_mass[b] * unit;
          if (n + sub_cnt[b] >= goal.n || m + w >= goal.mass) break;
          n += sub_cnt[b];
          m += w;
        }
        s.bin = last;
        s.n = (uint32_t)n_last;
        s.before = m_last;
        if (last >= 0 && shift == 0) {   // one key: how many of its equals
          const double w = (double)(sub_mass[last] / sub_cnt[last]) * unit;
          uint64_t ties = goal.n > n_last ? goal.n - n_last : 0;
          if (w > 0.0 && goal.mass < INFINITY) {
            const double t = ceil((goal.mass - m_last) / w);
            if (t < (double)ties) ties = t > 0.0 ? (uint64_t)t : 0;
          }
          if (ties > sub_cnt[last]) ties = sub_cnt[last];
          if (ties < 1) ties = 1;
          s.ties = (uint32_t)ties;
          s.total = m_last + (double)ties * w;
        }
      }
      __syncthreads();
      const uint32_t top = hi - ((uint32_t)s.bin << shift);
      hi = top;
      if (shift == 0) { cut.key = top; cut.ties = s.ties; break; }
      const uint32_t width = (1u << shift) - 1;
      lo = top - lo > width ? top - width : lo;
    }
    n_cut = (uint64_t)s.n + s.ties;
    z_k = s.total;
    __syncthreads();
  }

  // ---- the draw.  Equal logits at the cut are kept by ascending index: limit = index of the last one
  int limit = 0x7FFFFFFF;
  if (cut.ties != 0xFFFFFFFFu) {
    uint32_t seen = 0;
    for (int base = 0; base < V; base += kThreads) {
      const int i = base + tid;
      const bool hit = i < V && key_of(clean(ld_logit(z, i))) == cut.key;
      const unsigned long long mask = __ballot(hit);
      if (lane == 0) s.red_n[wave] = __popcll(mask);
      __syncthreads();
      uint32_t off = seen, all = seen;
      for (int w = 0; w < kWaves; ++w) { if (w < wave) off += s.red_n[w]; all += s.red_n[w]; }
      if (hit && off + __popcll(mask & ((1ull << lane) - 1)) == cut.ties - 1) s.key = (uint32_t)i;
      __syncthreads();
      seen = all;
      if (seen >= cut.ties) break;
    }
    limit = (int)s.key;
  }
  auto weight = [&](int i) -> double {   // of token i; negative: not kept
    const float x = clean(ld_logit(z, i));
    const uint32_t key = key_of(x);
    if (!(x > -INFINITY) || key < cut.key || (key == cut.key && i > limit)) return -1.0;
    const double w = weight_of(sc.dist(x));
    return (w >= min_w || x == sc.zmax) ? w : -1.0;
  };
  const int strips = (V + kStrip - 1) / kStrip;
  uint32_t kept = 0;
  for (int st = wave; st < strips; st += kWaves) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < kStrip / kWave; ++j) {
      const int i = st * kStrip + j * kWave + lane;
      const double w = i < V ? weight(i) : -1.0;
      if (w >= 0.0) { sum += w; ++kept; }
    }
    sum = wave_sum(sum);
    if (lane == 0) s.strip[st] = sum;
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) kept += __shfl_xor(kept, o);
  if (lane == 0) s.red_n[wave] = kept;
  __syncthreads();
  if (wave != 0) return;
  kept = 0;
  for (int w = 0; w < kWaves; ++w) kept += s.red_n[w];
  double total = 0.0;
  for (int st = 0; st < strips; ++st) total += s.strip[st];
  const float u0 = a.u[row];
  const double target = (u0 > 0.f ? (u0 < 1.f ? (double)u0 : 1.0) : 0.0) * total;
  // the strip in which the running sum passes the target; the last one with a weight if rounding leaves none
  int at = 0;
  double before = 0.0, run = 0.0;
  for (int st = 0; st < strips; ++st) {
    if (!(s.strip[st] > 0.0)) continue;
    at = st;
    before = run;
    run += s.strip[st];
    if (run > target) break;
  }
  // and the token in the strip
  int token = -1;
  double w_token = 0.0;
  for (int j = 0; j < kStrip / kWave; ++j) {
    const int i = at * kStrip + j * kWave + lane;
    const double w0 = i < V ? weight(i) : -1.0;
    const double w = w0 > 0.0 ? w0 : 0.0;
    double inc = w;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const double v = __shfl_up(inc, o);
      if (lane >= o) inc += v;
    }
    const unsigned long long has = __ballot(w > 0.0);
    const unsigned long long pass = __ballot(w > 0.0 && before + inc > target);
    if (has) {
      const int src = pass ? __ffsll((long long)pass) - 1 : 63 - __clzll((long long)has);
      token = at * kStrip + j * kWave + src;
      w_token = __shfl(w, src);
      if (pass) break;
    }
    before += __shfl(inc, kWave - 1);
  }
  if (lane == 0) {
    a.tokens[row] = token;
    if (a.prob) a.prob[row] = (float)(w_token / total);
    if (a.n_kept) a.n_kept[row] = (int32_t)kept;
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
