// Decoding from a paged key/value cache (Sec. 2.2: a query is a prompt that a candidate continues; the rows of a
// decode step are one token per sequence, each under its own candidate).
//
//   k_cache_append[_heads]  per-head RMS norm + rotary embedding of new rows, keys and values into their pages
//   k_attention_paged   attention of a new row over its sequence's pages, a range of them per workgroup
//   k_attention_join    joins the ranges of a long row
//
// A row's place: sequence i with cu[i] <= t < cu[i+1], position kv_len[i] - (cu[i+1] - t); position p lies in slot
// p % page_size of page page_table[i][p / page_size].  Rows behind the last sequence are left as they were.
#include <math.h>

#include <atomic>

#include "zo_device.hpp"
#include "zo_internal.hpp"

namespace zo {
namespace {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float ld_elem(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float ld_elem(const bf16_t* p, int64_t i) { return bf16_to_f32(p[i]); }
__device__ __forceinline__ void st_elem(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void st_elem(bf16_t* p, int64_t i, float v) { p[i] = f32_to_bf16(v); }

// Largest i with cu[i] <= t; S when t lies behind the last sequence.
__device__ __forceinline__ int seq_of_row(const int32_t* cu, int S, int t) {
  int lo = 0, hi = S;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cu[mid] <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Page that holds position pos of sequence seq; -1 when there is none in the pool.
__device__ __forceinline__ int page_of(const CacheDev& c, int seq, int pos) {
  if (pos < 0 || (pos >> c.page_shift) >= c.max_pages) return -1;
  const int pg = c.table[(int64_t)seq * c.max_pages + (pos >> c.page_shift)];
  return (unsigned)pg < (unsigned)c.n_pages ? pg : -1;
}
// First element of (page, head, slot) in a pool.
__device__ __forceinline__ int64_t slot_at(const CacheDev& c, int page, int head, int pos) {
  return ((((int64_t)page * c.n_kv_heads + head) << c.page_shift) + (pos & ((1 << c.page_shift) - 1))) * c.dh;
}

struct Place {
  int seq, pos;   // seq < 0: behind the last sequence
};

// Sequence and position of row t, wave-wide: 63 bounds at a time, and the lengths travel with the last of them.
__device__ __forceinline__ Place place_of_row(const int32_t* cu, const int32_t* kv_len, int S, int t, int lane) {
  int lo = 0, n = S + 1;   // candidates lo .. lo + n - 1; cu[lo] <= t
  while (n > 63) {
    const int step = (n + 62) / 63;
    const int i = lo + lane * step;
    const unsigned long long le = __ballot(lane < 63 && lane * step < n && cu[min(i, S)] <= t);
    const int k = max(__popcll(le) - 1, 0);
    n = min(step, n - k * step);
    lo += k * step;
  }
  const int i = min(lo + lane, S);
  const int c = cu[i];
  const int len = kv_len[min(i, S - 1)];
  const int k = __popcll(__ballot(lane < n && c <= t)) - 1;
  if (lo + k >= S) return Place{-1, 0};
  const int next = __builtin_amdgcn_readlane(c, k + 1);
  return Place{__builtin_amdgcn_readfirstlane(lo + k), __builtin_amdgcn_readlane(len, k) - (next - t)};
}

// ------------------------------------------------------------------ append

// A pair turned by an angle; which product is rounded is written out, so that a pair has the same bits in every kernel.
__device__ __forceinline__ void rotate(float& lo, float& hi, float sn, float cs) {
  const float p = lo, q = hi;
  lo = __builtin_fmaf(p, cs, -(q * sn));
  hi = __builtin_fmaf(q, cs, p * sn);
}

// Any even head dimension up to 256: one wave per (row, head), lane l holds the pairs l and l + 64.  Heads 0..H-1 are
// queries, the next Hkv keys, the last Hkv values.
template <typename Tio>
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a) {
  const int lane = threadIdx.x & 63;
  const int nkv = a.c.n_kv_heads, heads = a.n_heads + 2 * nkv;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= (int64_t)a.T * heads) return;
  const int t = (int)(item / heads), head = (int)(item % heads);
  const int seq = seq_of_row(a.cu, a.S, t);
  if (seq >= a.S) return;
  const int pos = a.c.kv_len[seq] - (a.cu[seq + 1] - t);
  const int dh = a.c.dh, half = dh >> 1;
  const bool is_q = head < a.n_heads, is_v = head >= a.n_heads + nkv;
  const Tio* in;
  Tio* out;
  if (is_q) {
    in = (const Tio*)a.Q + (int64_t)t * a.ldq + head * dh;
    out = (Tio*)a.Qout + (int64_t)t * a.ldqo + head * dh;
  } else {
    const int g = head - a.n_heads - (is_v ? nkv : 0);
    const int page = page_of(a.c, seq, pos);
    if (page < 0) return;
    in = is_v ? (const Tio*)a.V + (int64_t)t * a.ldv + g * dh : (const Tio*)a.K + (int64_t)t * a.ldk + g * dh;
    out = (Tio*)(is_v ? a.c.V : a.c.K) + slot_at(a.c, page, g, pos);
  }
  if (is_v) {
    for (int i = lane; i < dh; i += kWave) out[i] = in[i];
    return;
  }
  float lo[2], hi[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int i = lane + c * kWave;
    lo[c] = i < half ? ld_elem(in, i) : 0.f;
    hi[c] = i < half ? ld_elem(in, half + i) : 0.f;
  }
  if (a.gamma_q) {
    const float ss = wave_sum(lo[0] * lo[0] + hi[0] * hi[0] + lo[1] * lo[1] + hi[1] * hi[1]);
    const float rstd = 1.0f / sqrtf(ss / (float)dh + a.eps);
    const float* gam = is_q ? a.gamma_q : a.gamma_k;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int i = lane + c * kWave;
      if (i < half) { lo[c] *= rstd * gam[i]; hi[c] *= rstd * gam[half + i]; }
    }
  }
  if (a.theta > 0.f) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int i = lane + c * kWave;
      if (i >= half) continue;
      double dsn, dcs;
      sincos((double)pos * exp2(-(double)(2 * i) / (double)dh * log2((double)a.theta)), &dsn, &dcs);
      rotate(lo[c], hi[c], (float)dsn, (float)dcs);
    }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int i = lane + c * kWave;
    if (i < half) { st_elem(out, i, lo[c]); st_elem(out, half + i, hi[c]); }
  }
}

// Head dimension 64, 128 or 256, rows aligned: kDh / 8 lanes have a head, each the elements 4 j .. 4 j + 3 and their rotation
// partners kDh/2 + 4 j .., so that the sum of squares is a few exchanges between neighbours and the rotation stays in the lane.
// A wave takes rows (one after another where there are many) and `per_wave` groups of 512 / kDh heads of each, the next group's
// loads under way; angles are formed once per row, frequencies once per wave.  Queries, keys and values are one list of heads.
// Bound by memory: 17233 rows of 32 + 2 * 8 heads of 128, 93 us (4.5 TB/s; fp32 175, 4.8; a wave per row and head took 676), keys
// and values alone 37; 16 rows: the latency of a launch.
template <typename Tio> struct Four;
template <> struct Four<bf16_t> {
  typedef uint2 type;
  static __device__ __forceinline__ void unpack(const uint2& v, float* x) {
    x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
    x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
  }
  static __device__ __forceinline__ uint2 pack(const float* x) { return make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])); }
};
template <> struct Four<float> {
  typedef float4 type;
  static __device__ __forceinline__ void unpack(const float4& v, float* x) { x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
  static __device__ __forceinline__ float4 pack(const float* x) { return make_float4(x[0], x[1], x[2], x[3]); }
};

template <typename Tio, int kDh>
__global__ __launch_bounds__(256) void k_cache_append_heads(AppendArgs a, int per_wave, double log2_theta) {
  typedef Four<Tio> F;
  typedef typename F::type V4;
  constexpr int kLanes = kDh / 8, kHeads = kWave / kLanes;   // lanes of a head, heads at a time
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = lane % kLanes, hh = lane / kLanes;
  const int nkv = a.c.n_kv_heads, heads = a.n_heads + 2 * nkv;
  const int g_first = blockIdx.y * per_wave, g_last = min(g_first + per_wave, (heads + kHeads - 1) / kHeads);
  // bf16: the lane's four pairs, revolutions per position.  fp32: radians per position, formed as in the other kernels of this
  // rotation, a row's angles spread over the wave's lanes (a sine in double precision is dear): lane l has l kOwn .. l kOwn + kOwn - 1.
  constexpr bool kExact = sizeof(Tio) == 4;
  constexpr int kOwn = kDh > 128 ? kDh / 128 : 1, kFreqs = kExact ? kOwn : 4;
  double freq[kFreqs];
  if (a.theta > 0.f) {
#pragma unroll
    for (int e = 0; e < kFreqs; ++e) {
      if constexpr (kExact) freq[e] = exp2(-(double)(2 * ((lane * kOwn + e) % (kDh / 2))) / (double)kDh * log2((double)a.theta));
      else freq[e] = exp2(-(double)(2 * (4 * j + e)) / kDh * log2_theta) * 0.15915494309189533577;
    }
  }
  float4 gq0 = make_float4(1.f, 1.f, 1.f, 1.f), gq1 = gq0, gk0 = gq0, gk1 = gq0;
  if (a.gamma_q) {
    gq0 = *reinterpret_cast<const float4*>(a.gamma_q + 4 * j);
    gq1 = *reinterpret_cast<const float4*>(a.gamma_q + kDh / 2 + 4 * j);
    gk0 = *reinterpret_cast<const float4*>(a.gamma_k + 4 * j);
    gk1 = *reinterpret_cast<const float4*>(a.gamma_k + kDh / 2 + 4 * j);
  }
  for (int t = blockIdx.x * 4 + wave; t < a.T; t += gridDim.x * 4) {
    auto load = [&](int grp, V4& lo, V4& hi) {
      const int head = min(grp * kHeads + hh, heads - 1);
      const Tio* in = head < a.n_heads ? (const Tio*)a.Q + (int64_t)t * a.ldq + head * kDh
                      : head < a.n_heads + nkv ? (const Tio*)a.K + (int64_t)t * a.ldk + (head - a.n_heads) * kDh
                                               : (const Tio*)a.V + (int64_t)t * a.ldv + (head - a.n_heads - nkv) * kDh;
      lo = *reinterpret_cast<const V4*>(in + 4 * j);
      hi = *reinterpret_cast<const V4*>(in + kDh / 2 + 4 * j);
    };
    V4 lo, hi;
    load(g_first, lo, hi);
    const Place pl = place_of_row(a.cu, a.c.kv_len, a.S, t, lane);
    if (pl.seq < 0) continue;
    const int page = page_of(a.c, pl.seq, pl.pos);
    float cs[4], sn[4];
    if (a.theta > 0.f) {
      if constexpr (kExact) {
        float own_sn[kOwn], own_cs[kOwn];   // rounded once: 6e-8
#pragma unroll
        for (int e = 0; e < kOwn; ++e) {
          double dsn, dcs;
          sincos((double)pl.pos * freq[e], &dsn, &dcs);
          own_sn[e] = (float)dsn;
          own_cs[e] = (float)dcs;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sn[e] = __shfl(own_sn[e % kOwn], (4 * j + e) / kOwn);
          cs[e] = __shfl(own_cs[e % kOwn], (4 * j + e) / kOwn);
        }
      } else {   // the hardware's sine and cosine, which take revolutions: 3e-7, under bf16's 4e-3
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double turns = (double)pl.pos * freq[e];
          const float part = (float)(turns - floor(turns));
          cs[e] = __builtin_amdgcn_cosf(part);
          sn[e] = __builtin_amdgcn_sinf(part);
        }
      }
    }
    for (int grp = g_first; grp < g_last; ++grp) {
      V4 nlo = lo, nhi = hi;
      if (grp + 1 < g_last) load(grp + 1, nlo, nhi);
      const int head = grp * kHeads + hh;
      const bool is_q = head < a.n_heads, is_v = head >= a.n_heads + nkv;
      float x[8];   // [0..3] first half, [4..7] partners
      F::unpack(lo, x);
      F::unpack(hi, x + 4);
      if (a.gamma_q) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
#pragma unroll
        for (int o = kLanes / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o);
        const float rstd = 1.0f / sqrtf(ss * (1.0f / kDh) + a.eps);
        const float4 g0 = is_q ? gq0 : gk0, g1 = is_q ? gq1 : gk1;
        x[0] *= rstd * g0.x; x[1] *= rstd * g0.y; x[2] *= rstd * g0.z; x[3] *= rstd * g0.w;
        x[4] *= rstd * g1.x; x[5] *= rstd * g1.y; x[6] *= rstd * g1.z; x[7] *= rstd * g1.w;
      }
      if (a.theta > 0.f) {   // (not by an angle of zero: zero times infinity is NaN)
#pragma unroll
        for (int e = 0; e < 4; ++e) rotate(x[e], x[4 + e], sn[e], cs[e]);
      }
      if (head < heads && (is_q || page >= 0)) {
        Tio* out = is_q ? (Tio*)a.Qout + (int64_t)t * a.ldqo + head * kDh
                        : (Tio*)(is_v ? a.c.V : a.c.K) + slot_at(a.c, page, head - a.n_heads - (is_v ? nkv : 0), pl.pos);
        *reinterpret_cast<V4*>(out + 4 * j) = is_v ? lo : F::pack(x);
        *reinterpret_cast<V4*>(out + kDh / 2 + 4 * j) = is_v ? hi : F::pack(x + 4);
      }
      lo = nlo;
      hi = nhi;
    }
  }
}

// ------------------------------------------------------------------ attention

// A row's positions are cut into ranges of range_keys(n), a function of the row's own n alone; two waves take one (row,
// key/value head, range).  They take steps of keys in turn, each with a running maximum and sum of its own, and join in LDS;
// a row of several ranges leaves (maximum, sum, unnormalised output) of each in the workspace and k_attention_join joins
// them in order.  A call that would leave compute units empty takes the up to four ranges of its rows in one workgroup,
// which joins them itself with the same arithmetic: one launch instead of two.
//
// Both products run on the matrix cores with up to 16 query heads of the key/value head as columns, transposed as in the
// attention of packed rows: S^T = K Q^T and O^T = V^T P^T, so that everything that belongs to a query lies in one column
// of lanes.  Keys and values go from memory to the registers of the matrix instruction directly, 16 bytes a lane, without
// LDS: a cache is read once, there is nothing to share.
//   keys    A operand: lane (r, g) of 16 x 4 holds 8 values of key row r.  Row r of tile hf is key 8 (r/4) + r%4 + 4 hf of
//           the 32, so that a lane's scores are those of keys 8 g .. 8 g + 7: what it must supply to the second product.
//   values  lane (r, g) loads columns [r dh/16, (r+1) dh/16) of keys 8 g .. 8 g + 7 (whole rows per load) and transposes them in
//           its own registers, two bytes at a time (v_perm, one per two values).  Tile d of the output then is the columns
//           r dh/16 + d, and a lane ends with dh/4 neighbouring columns of its query.
// fp32 uses the 16x16x4 instruction on 16 keys per step: a lane's scores are those of keys 4 g .. 4 g + 3, and since its operands
// are one value per lane, the values need no transposition.
// Bound by memory where there are rows enough: 32 rows of 2048, 40 heads, 238 us (5.6 TB/s); 2 rows of 131072, 32 heads over 8, 193
// us (5.6); 80 rows of 64..1024, 46.5 us (41.5 and the join 5).  The second product of a bf16 weight costs 0.3 to 0.5 us of them.  Four waves per range 49 us, eight 58, one 49 and slower on few rows;
// ranges of 512: 256 rows of 1000..4000 7 % faster, one row of 8000 15 % slower; one step in registers 545 -> 559 us.

constexpr int kRangeWaves = 2;       // waves of a range
constexpr int kMaxRanges = 64;       // of a row: one lane each in the join
constexpr int kHere = 4;             // most ranges that one workgroup joins by itself
// Positions per range of a row of n positions: four steps of each wave (the same bytes in either type), more where that makes
// too many ranges.
__host__ __device__ constexpr int range_keys(bool bf16, int n) {
  const int base = bf16 ? 256 : 128;
  return base * (n <= kMaxRanges * base ? 1 : (n + kMaxRanges * base - 1) / (kMaxRanges * base));
}
// most ranges of a row of up to n positions
constexpr int most_ranges(bool bf16, int n) {
  const int base = bf16 ? 256 : 128;
  return n >= kMaxRanges * base ? kMaxRanges : (n + base - 1) / base;
}

// Workspace: [T][n_heads][ranges] of (maximum, sum), then [T][n_heads][ranges][dh] unnormalised outputs.
__device__ __forceinline__ int64_t part_at(const PagedAttnArgs& a, int t, int h, int range) {
  return ((int64_t)t * a.n_heads + h) * a.ranges + range;
}

__device__ __attribute__((aligned(16))) const uint32_t kZeros[256] = {};   // the value of a key that is not seen

// What differs between the two types: loading a step's keys and values and the two products.
// at(key), value_at(key): the first element of what is read for a key of the step and for its value, in the pools.
template <int kDh>
struct Bf16Step {
  static constexpr int kKeys = 32, kPad = kDh, kCols = kDh / 16;   // columns of a value row per lane
  static constexpr int kScores = 8;       // per lane: keys 8 g + i
  static constexpr bool kAhead = true, kWhole = true;   // kWhole: the head dimension is kPad
  bf16x8 k[2][kDh / 32];
  u32x4 v[8][kCols > 8 ? kCols / 8 : 1];  // (kCols 4: the lower half of each)
  __device__ static constexpr int key_of_score(int g, int i) { return 8 * g + i; }

  template <class At, class ValueAt>
  __device__ __forceinline__ void load(const PagedAttnArgs& a, int r, int g, At at, ValueAt value_at) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const bf16_t* p = (const bf16_t*)a.c.K + at(8 * (r >> 2) + (r & 3) + 4 * hf) + g * 8;
#pragma unroll
      for (int ks = 0; ks < kDh / 32; ++ks) k[hf][ks] = load_frag(p + ks * 32);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bf16_t* p = (const bf16_t*)a.c.V + value_at(8 * g + j) + r * kCols;
      if constexpr (kCols == 4) {
        const uint2 w = *reinterpret_cast<const uint2*>(p);
        v[j][0] = u32x4{w.x, w.y, 0u, 0u};
      } else {
#pragma unroll
        for (int c = 0; c < kCols / 8; ++c) v[j][c] = *reinterpret_cast<const u32x4*>(p + c * 8);
      }
    }
  }
  typedef bf16x8 Query[kDh / 32];
  __device__ static __forceinline__ void load_query(const PagedAttnArgs& a, const void* row, bool valid, int g, Query& q) {
#pragma unroll
    for (int ks = 0; ks < kDh / 32; ++ks) q[ks] = valid ? load_frag((const bf16_t*)row + ks * 32 + g * 8) : zero_frag();
  }
  __device__ __forceinline__ void scores(const Query& q, float (&s)[kScores]) const {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < kDh / 32; ++ks) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[hf][ks], q[ks], acc, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * hf + i] = acc[i];
    }
  }
  // A weight takes two products: its upper 16 bits, and the rest rounded to bf16, so that 2^-15 of it is lost at most (2^-8 with
  // one).  The rest counts 2^-20 of the weight more, so that it is none only where the weight is: zero times an infinite value
  // would be NaN.
  __device__ __forceinline__ void values(const float (&p)[kScores], f32x4 (&o)[kCols]) const {
    u32x4 upper, rest;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t a = __float_as_uint(p[2 * j]), b = __float_as_uint(p[2 * j + 1]);
      upper[j] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      rest[j] = pack_bf16x2(__builtin_fmaf(p[2 * j], 1.0f + 0x1p-20f, -__uint_as_float(a & 0xFFFF0000u)),
                            __builtin_fmaf(p[2 * j + 1], 1.0f + 0x1p-20f, -__uint_as_float(b & 0xFFFF0000u)));
    }
    const bf16x8 pu = __builtin_bit_cast(bf16x8, upper), pr = __builtin_bit_cast(bf16x8, rest);
#pragma unroll
    for (int d = 0; d < kCols; ++d) {
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j)   // column d of keys 2 j and 2 j + 1
        w[j] = __builtin_amdgcn_perm(v[2 * j + 1][d >> 3][(d & 7) >> 1], v[2 * j][d >> 3][(d & 7) >> 1], (d & 1) ? 0x07060302u : 0x05040100u);
      const bf16x8 wf = __builtin_bit_cast(bf16x8, w);
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, pr, o[d], 0, 0, 0);
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, pu, o[d], 0, 0, 0);
    }
  }
};

// Four values of a query or output row, which need no alignment beyond their type's: one access all the same.
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

// kMode 0: the head dimension is kDh; 1: smaller, a multiple of 4; 2: smaller, any.
template <int kDh, int kMode>
struct F32Step {
  static constexpr int kKeys = 16, kPad = kDh, kCols = kDh / 16;
  static constexpr int kScores = 4;       // per lane: keys 4 g + i
  static constexpr bool kWhole = kMode == 0;
  static constexpr bool kAhead = kDh <= 64;   // (a third wave per SIMD instead: 64 rows of 500..2000, 8 heads over 4 of 128: 82 -> 72 us)
  f32x4 k[kDh / 16];
  f32x4 v[4][kCols / 4];
  __device__ static constexpr int key_of_score(int g, int i) { return 4 * g + i; }

  // four values from column `col` of a row of dh; zeros behind its end.  F4: as the row is aligned (the pools on 16 bytes)
  template <class F4 = f32x4>
  __device__ static __forceinline__ f32x4 four(const float* row, int col, int dh) {
    if constexpr (kMode == 0) return *reinterpret_cast<const F4*>(row + col);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if constexpr (kMode == 1) {
      if (col < dh) x = *reinterpret_cast<const F4*>(row + col);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < dh) x[e] = row[col + e];
    }
    return x;
  }
  template <class At, class ValueAt>
  __device__ __forceinline__ void load(const PagedAttnArgs& a, int r, int g, At at, ValueAt value_at) {
    const float* p = (const float*)a.c.K + at(r);
#pragma unroll
    for (int ks = 0; ks < kDh / 16; ++ks) k[ks] = four(p, ks * 16 + g * 4, a.c.dh);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float* w = (const float*)a.c.V + value_at(4 * g + j);
#pragma unroll
      for (int c = 0; c < kCols / 4; ++c) v[j][c] = four(w, r * kCols + c * 4, a.c.dh);
    }
  }
  typedef f32x4 Query[kDh / 16];
  __device__ static __forceinline__ void load_query(const PagedAttnArgs& a, const void* row, bool valid, int g, Query& q) {
#pragma unroll
    for (int ks = 0; ks < kDh / 16; ++ks) {
      q[ks] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (valid) q[ks] = four<f32x4_any>((const float*)row, ks * 16 + g * 4, a.c.dh);
    }
  }
  __device__ __forceinline__ void scores(const Query& q, float (&s)[kScores]) const {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < kDh / 16; ++ks)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(k[ks][e], q[ks][e], acc, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = acc[i];
  }
  __device__ __forceinline__ void values(const float (&p)[kScores], f32x4 (&o)[kCols]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int d = 0; d < kCols; ++d) o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j][d >> 2][d & 3], p[j], o[d], 0, 0, 0);
  }
};

// Maximum, sum of weights and four columns of the unnormalised output of some of a row's keys.
struct Joined {
  float m, l;
  f32x4 o;
};

// The maximum of a query that has met keys, but none above -infinity: beside a larger one it has no weight, alone it has no softmax.
constexpr float kLeast = -3.402823466e38f;
// What the output is multiplied by: zeros stay zeros where no key was met.
__device__ __forceinline__ float inverse_sum(float m, float l) {
  return l > 0.f ? 1.0f / l : m == -INFINITY ? 0.f : __builtin_nanf("");
}

// kTiles: tiles of 16 query heads per workgroup (1 or 2); with one its waves share the keys.  kRanges: ranges of a row per
// workgroup, 1 or kHere (then the table has room for no more).
template <typename Tio, class Step, int kTiles, int kRanges>
__global__ __launch_bounds__(kRanges* kRangeWaves* kWave, Step::kPad > 128 ? 1 : 2) void k_attention_paged(PagedAttnArgs a) {
  constexpr int kDh = Step::kPad, kCols = Step::kCols, kKeys = Step::kKeys, kSharers = kRangeWaves / kTiles;
  constexpr int kAttnWaves = kRanges * kRangeWaves;
  constexpr int kRowLds = kDh + 4;   // (rows of the joining buffer on different banks)
  extern __shared__ __attribute__((aligned(16))) float s_o[];     // [wave][16][kRowLds]
  __shared__ float s_m[kAttnWaves][16], s_l[kAttnWaves][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int per_head = (a.group + 16 * kTiles - 1) / (16 * kTiles);   // workgroups that share a key/value head
  const int item = blockIdx.x;
  const int part = item % per_head, kvh = item / per_head % a.c.n_kv_heads, t = item / per_head / a.c.n_kv_heads;
  const Place pl = place_of_row(a.cu, a.c.kv_len, a.S, t, lane);
  if (pl.seq < 0) return;
  const int n = max(0, min(pl.pos + 1, a.c.max_pages << a.c.page_shift));
  const int len = range_keys(a.c.bf16, n);
  const int n_ranges = n > 0 ? (n + len - 1) / len : 1;   // (an empty row: one empty range writes its zeros)
  const int tile = wave % kTiles, share = wave % kRangeWaves / kTiles;
  const int head0 = (part * kTiles + tile) * 16;            // of the group
  const int cols = min(16, a.group - head0);                 // columns in use (may be <= 0)
  typename Step::Query q;
  Step::load_query(a, (const Tio*)a.Q + (int64_t)t * a.ldq + (int64_t)(kvh * a.group + head0 + r) * a.c.dh, r < cols, g, q);
  const float sl2 = a.scale * 1.4426950408889634f;           // scores are kept in base-2 units
  const int32_t* table = a.c.table + (int64_t)pl.seq * a.c.max_pages;
  // the zeros' place as an element of the pool of values (both lie on 16 bytes)
  const int64_t no_value = ((int64_t)(uintptr_t)kZeros - (int64_t)(uintptr_t)a.c.V) / (int64_t)sizeof(Tio);

  if ((int)blockIdx.y >= n_ranges) return;   // (the grid has the ranges of the longest row that the table has room for)
  const int range = kRanges == 1 ? (int)blockIdx.y : wave / kRangeWaves;
  const int j_a = range * len, j_b = min(j_a + len, n);   // the range's positions (none behind the row's last)
  f32x4 o[kCols];
#pragma unroll
  for (int d = 0; d < kCols; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;   // l: this lane's share
  bool met = false;               // a key that is seen

  // pages of the 64 blocks of 16 positions that begin at block `first`, one a lane; -1: no position, or no page of the pool
  auto pages_from = [&](int first) {
    const int j = (first + lane) * 16;
    if (j >= j_b) return -1;
    const int pg = table[j >> a.c.page_shift];
    return (unsigned)pg < (unsigned)a.c.n_pages ? pg : -1;
  };
  int first = j_a / 16;
  int pages = pages_from(first);
  // Loads step `j0`; false when it has no key that is seen.  A key that is not seen is stood in for by one that is (its score is
  // replaced below), its value by zeros: what a slot holds that is not seen, and an infinite value of the stand-in's, must not
  // meet even a weight of zero.
  auto load = [&](int j0, Step& st, int& last, int& dead) -> bool {
    if (j0 / 16 - first >= 64) {
      first += 64;
      pages = pages_from(first);
    }
    const int b = j0 / 16 - first;
    const int p0 = __builtin_amdgcn_readlane(pages, b);
    const int p1 = kKeys == 32 ? __builtin_amdgcn_readlane(pages, b + 1) : p0;
    dead = (p0 < 0 ? 1 : 0) | (p1 < 0 ? 2 : 0);
    if (p0 < 0 && p1 < 0) return false;
    last = j_b - 1 - j0;
    const int64_t b0 = slot_at(a.c, p0 < 0 ? p1 : p0, kvh, j0), b1 = slot_at(a.c, p1 < 0 ? p0 : p1, kvh, j0 + 16);
    const bool whole = dead == 0 && last >= kKeys - 1;
    auto seen = [&](int key) { return key <= last && !(dead >> (key >> 4) & 1); };
    auto at = [&](int key) -> int64_t {
      int e = key;
      if (!whole) {
        if (kKeys == 32 && (dead >> (key >> 4) & 1)) e ^= 16;
        e = min(e, last);
      }
      return (kKeys == 32 && e >= 16 ? b1 : b0) + (e & 15) * a.c.dh;
    };
    auto value_at = [&](int key) -> int64_t { return whole || seen(key) ? at(key) : no_value; };
    st.load(a, r, g, at, value_at);
    return true;
  };
  auto attend = [&](const Step& st, int last, int dead) {
    met = true;
    float s[Step::kScores];
    st.scores(q, s);
#pragma unroll
    for (int i = 0; i < Step::kScores; ++i) s[i] *= sl2;
    if (dead != 0 || last < kKeys - 1) {
#pragma unroll
      for (int i = 0; i < Step::kScores; ++i) {
        const int key = Step::key_of_score(g, i);
        if (key > last || (dead >> (key >> 4) & 1)) s[i] = -INFINITY;   // (not seen)
      }
    }
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < Step::kScores; ++i) mx = fmaxf(mx, s[i]);
    float f = 1.0f;
    if (__any(mx > m)) {   // (otherwise every factor is one)
      const float m2 = fmaxf(column_max(mx), m);
      f = m == m2 ? 1.0f : __builtin_amdgcn_exp2f(m - m2);   // (a query that has met nothing above -infinity yet stays as it is)
      m = m2;
#pragma unroll
      for (int d = 0; d < kCols; ++d) o[d] *= f;
    }
    float p[Step::kScores], sum = 0.f;
    const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < Step::kScores; ++i) {
      p[i] = __builtin_amdgcn_exp2f(s[i] - off);
      sum += p[i];
    }
    l = __builtin_fmaf(l, f, sum);
    st.values(p, o);
  };
  if (cols > 0) {
    constexpr int kStride = kSharers * kKeys;
    int j0 = j_a + share * kKeys;
    if constexpr (Step::kAhead) {   // two steps in registers: while one is worked on, the next is on its way
      Step s0, s1;
      int last0 = 0, dead0 = 0, last1 = 0, dead1 = 0;
      bool seen0 = j0 < j_b && load(j0, s0, last0, dead0);
      for (; j0 < j_b; j0 += 2 * kStride) {
        const bool seen1 = j0 + kStride < j_b && load(j0 + kStride, s1, last1, dead1);
        if (seen0) attend(s0, last0, dead0);
        seen0 = j0 + 2 * kStride < j_b && load(j0 + 2 * kStride, s0, last0, dead0);
        if (seen1) attend(s1, last1, dead1);
      }
    } else {
      for (; j0 < j_b; j0 += kStride) {
        Step st;
        int last, dead;
        if (load(j0, st, last, dead)) attend(st, last, dead);
      }
    }
  }

  // ---- the waves join
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (met) m = fmaxf(m, kLeast);
  if (r < cols) {
    float* row = s_o + (wave * 16 + r) * kRowLds + g * (kDh / 4);   // columns (4 g + i) kCols + d
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < kCols; d += 4)
        *reinterpret_cast<f32x4*>(row + i * kCols + d) = f32x4{o[d][i], o[d + 1][i], o[d + 2][i], o[d + 3][i]};
    if (g == 0) { s_m[wave][r] = m; s_l[wave][r] = l; }
  }
  __syncthreads();
  const int group_cols = min(16 * kTiles, a.group - part * 16 * kTiles);
  for (int e = threadIdx.x; e < group_cols * (kDh / 4); e += kAttnWaves * kWave) {
    const int c = e / (kDh / 4), col = c & 15, tl = c >> 4, d = e % (kDh / 4) * 4;
    auto waves_of = [&](int rg) {   // the waves of one range
      Joined x{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int w = 0; w < kSharers; ++w) x.m = fmaxf(x.m, s_m[rg * kRangeWaves + w * kTiles + tl][col]);
#pragma unroll
      for (int w = 0; w < kSharers; ++w) {
        const int wv = rg * kRangeWaves + w * kTiles + tl;
        const float mw = s_m[wv][col];
        const float f = mw == x.m ? 1.0f : __builtin_amdgcn_exp2f(mw - x.m);   // (no key at all: zeros stay zeros)
        const f32x4 ow = *reinterpret_cast<const f32x4*>(s_o + (wv * 16 + col) * kRowLds + d);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.o[i] = __builtin_fmaf(ow[i], f, x.o[i]);
        x.l = __builtin_fmaf(s_l[wv][col], f, x.l);
      }
      return x;
    };
    const int h = kvh * a.group + part * 16 * kTiles + c;
    Joined x;
    if (kRanges == 1 || n_ranges == 1) {
      x = waves_of(0);
    } else {   // what k_attention_join does, for four ranges
#pragma clang fp contract(off)
      Joined y[kHere];
      x = Joined{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int rg = 0; rg < kHere; ++rg) {
        y[rg] = Joined{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
        if (rg < n_ranges) y[rg] = waves_of(rg);
        x.m = fmaxf(x.m, y[rg].m);
      }
      float lf[kHere];
#pragma unroll
      for (int rg = 0; rg < kHere; ++rg) {
        const float f = y[rg].m == x.m ? 1.0f : __builtin_amdgcn_exp2f(y[rg].m - x.m);
        lf[rg] = y[rg].l * f;
#pragma unroll
        for (int i = 0; i < 4; ++i) x.o[i] = x.o[i] + y[rg].o[i] * f;
      }
      x.l = (lf[0] + lf[2]) + (lf[1] + lf[3]);   // (the order of the wave's sum)
    }
    if (kRanges > 1 || n_ranges == 1) {
      const float inv = inverse_sum(x.m, x.l);
      Tio* out = (Tio*)a.O + (int64_t)t * a.ldo + (int64_t)h * a.c.dh + d;
      if constexpr (sizeof(Tio) == 2) {
        *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(x.o[0] * inv, x.o[1] * inv), pack_bf16x2(x.o[2] * inv, x.o[3] * inv));
      } else if constexpr (Step::kWhole) {
        *reinterpret_cast<f32x4_any*>(out) = x.o * inv;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (d + i < a.c.dh) out[i] = x.o[i] * inv;
      }
    } else {
      const int64_t at = part_at(a, t, h, range);
      if (d == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(x.m, x.l);
      float* out = a.part_o + at * a.c.dh + d;
      if constexpr (Step::kWhole) {
        *reinterpret_cast<f32x4*>(out) = x.o;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (d + i < a.c.dh) out[i] = x.o[i];
      }
    }
  }
}

// Joins the ranges of a row: ranges c, c + 4, ... are added in order into sum c % 4, and the four sums in order, a row's lanes
// over its columns.  Lane c of a wave has range c's maximum and sum of weights.  Few rows and heads: a workgroup each, a wave
// per sum; many: a wave each with all four sums, four to a workgroup.  (One sum and one load after another: 64 ranges of 128
// columns, 64 rows and heads, 46.7 us, now 4; a workgroup each for 10240 rows and heads of 4 ranges: 18.8.)
// kPer: columns per lane.
constexpr int kJoinSums = 4;
template <typename Tio, int kPer, bool kWave1>
__global__ __launch_bounds__(kJoinSums* kWave) void k_attention_join(PagedAttnArgs a) {
#pragma clang fp contract(off)   // (the same bits in every form of the joining)
  __shared__ float s_acc[kJoinSums - 1][kPer * kWave];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t item = kWave1 ? (int64_t)blockIdx.x * kJoinSums + wave : blockIdx.x;
  if (item >= (int64_t)a.T * a.n_heads) return;
  const int t = (int)(item / a.n_heads), h = (int)(item % a.n_heads);
  const Place pl = place_of_row(a.cu, a.c.kv_len, a.S, t, lane);
  if (pl.seq < 0) return;
  const int n = min(pl.pos + 1, a.c.max_pages << a.c.page_shift);
  const int len = range_keys(a.c.bf16, n);
  const int n_ranges = n > 0 ? (n + len - 1) / len : 1;
  if (n_ranges == 1) return;
  const int dh = a.c.dh;
  const int64_t at = part_at(a, t, h, 0);
  float m = -INFINITY, l = 0.f;
  if (lane < n_ranges) { m = a.part_ml[2 * (at + lane)]; l = a.part_ml[2 * (at + lane) + 1]; }
  const float* o = a.part_o + at * dh;
  constexpr int kSums = kWave1 ? kJoinSums : 1, kDeep = 8 / kSums;   // eight ranges under way
  float acc[kSums][kPer];
#pragma unroll
  for (int v = 0; v < kSums; ++v)
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[v][i] = 0.f;
  const float mm = wave_max(m);
  const float f = m == mm ? 1.0f : __builtin_amdgcn_exp2f(m - mm);
  for (int c0 = kWave1 ? 0 : wave; c0 < n_ranges; c0 += kJoinSums * kDeep) {
    float x[kDeep][kSums][kPer];
#pragma unroll
    for (int u = 0; u < kDeep; ++u)
#pragma unroll
      for (int v = 0; v < kSums; ++v) {
        const int c = c0 + u * kJoinSums + v;
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[u][v][i] = c < n_ranges && lane + i * kWave < dh ? o[c * dh + lane + i * kWave] : 0.f;
      }
#pragma unroll
    for (int u = 0; u < kDeep; ++u)
#pragma unroll
      for (int v = 0; v < kSums; ++v) {
        const int c = c0 + u * kJoinSums + v;
        if (c >= n_ranges) break;
        const float fc = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), c));
#pragma unroll
        for (int i = 0; i < kPer; ++i) acc[v][i] += x[u][v][i] * fc;
      }
  }
  if constexpr (kWave1) {
#pragma unroll
    for (int v = 1; v < kSums; ++v)
#pragma unroll
      for (int i = 0; i < kPer; ++i) acc[0][i] += acc[v][i];
  } else {
    if (wave > 0) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) s_acc[wave - 1][i * kWave + lane] = acc[0][i];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int v = 1; v < kJoinSums; ++v)
#pragma unroll
      for (int i = 0; i < kPer; ++i) acc[0][i] += s_acc[v - 1][i * kWave + lane];
  }
  const float sum = wave_sum(l * f);
  const float inv = inverse_sum(mm, sum);
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (lane + i * kWave < dh) st_elem((Tio*)a.O + (int64_t)t * a.ldo + (int64_t)h * dh, lane + i * kWave, acc[0][i] * inv);
}

}  // namespace

namespace {
template <typename Tio, int kDh>
hipError_t launch_append_heads(const AppendArgs& a, hipStream_t st) {
  constexpr int kHeads = 512 / kDh;
  const int groups = (a.n_heads + 2 * a.c.n_kv_heads + kHeads - 1) / kHeads, cus = compute_units();
  // Few rows: their heads are spread over waves until there are sixteen waves per compute unit.
  int per_wave = groups;
  while (per_wave > 1 && (int64_t)a.T * ((groups + per_wave - 1) / per_wave) < 16 * cus) per_wave = (per_wave + 1) / 2;
  const int splits = (groups + per_wave - 1) / per_wave;
  const int wgs = (a.T + 3) / 4, most = 8 * cus;   // (one round of waves that stride through the rows)
  const dim3 grid((unsigned)(wgs < most ? wgs : most), (unsigned)splits);
  k_cache_append_heads<Tio, kDh><<<grid, 256, 0, st>>>(a, per_wave, a.theta > 0.f ? log2((double)a.theta) : 0.0);
  return hipGetLastError();
}
template <typename Tio>
hipError_t launch_append(const AppendArgs& a, hipStream_t st) {
  auto aligned = [](const void* p, int64_t ld) { return ((uintptr_t)p & (4 * sizeof(Tio) - 1)) == 0 && ld % 4 == 0; };
  if (aligned(a.Q, a.ldq) && aligned(a.K, a.ldk) && aligned(a.V, a.ldv) && aligned(a.Qout, a.ldqo) &&
      (((uintptr_t)a.gamma_q | (uintptr_t)a.gamma_k) & 15u) == 0) {
    if (a.c.dh == 64) return launch_append_heads<Tio, 64>(a, st);
    if (a.c.dh == 128) return launch_append_heads<Tio, 128>(a, st);
    if (a.c.dh == 256) return launch_append_heads<Tio, 256>(a, st);
  }
  const int64_t items = (int64_t)a.T * (a.n_heads + 2 * a.c.n_kv_heads);
  k_cache_append<Tio><<<dim3((unsigned)((items + 3) / 4)), 256, 0, st>>>(a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t st) {
  return a.c.bf16 ? launch_append<bf16_t>(a, st) : launch_append<float>(a, st);
}

int attention_paged_ranges(bool bf16, int max_len) { return max_len > 0 ? most_ranges(bf16, max_len) : 1; }

namespace {
template <typename Tio, class Step, int kTiles, int kRanges>
hipError_t launch_paged(const PagedAttnArgs& a, int64_t groups, hipStream_t st) {
  constexpr int kWaves = kRanges * kRangeWaves, kLds = kWaves * 16 * (Step::kPad + 4) * 4;
  static std::atomic<bool> ready[kMaxDevices];
  if (kLds > 60 * 1024) {
    const hipError_t e = once_per_device(ready, [] {
      return hipFuncSetAttribute((const void*)k_attention_paged<Tio, Step, kTiles, kRanges>, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    });
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)groups, kRanges == 1 ? (unsigned)a.ranges : 1u);
  k_attention_paged<Tio, Step, kTiles, kRanges><<<grid, kWaves * kWave, kLds, st>>>(a);
  return hipGetLastError();
}
// A call whose rows have up to four ranges and whose (row, key/value head) pairs do not fill the compute units gives each pair
// one workgroup and needs no join.
template <typename Tio, class Step, int kTiles>
hipError_t launch_paged_ranges(const PagedAttnArgs& a, bool& joined, hipStream_t st) {
  const int64_t groups = (int64_t)a.T * a.c.n_kv_heads * ((a.group + 16 * kTiles - 1) / (16 * kTiles));
  if constexpr (Step::kPad <= 128) {
    joined = a.ranges > 1 && a.ranges <= kHere && groups <= compute_units();
    if (joined) return launch_paged<Tio, Step, kTiles, kHere>(a, groups, st);
  }
  return launch_paged<Tio, Step, kTiles, 1>(a, groups, st);
}
template <typename Tio, class Step>
hipError_t launch_paged_tiles(const PagedAttnArgs& a, bool& joined, hipStream_t st) {
  return a.group <= 16 ? launch_paged_ranges<Tio, Step, 1>(a, joined, st) : launch_paged_ranges<Tio, Step, 2>(a, joined, st);
}
template <int kDh>
hipError_t launch_paged_f32(const PagedAttnArgs& a, bool& joined, hipStream_t st) {
  if (a.c.dh == kDh) return launch_paged_tiles<float, F32Step<kDh, 0>>(a, joined, st);
  // (rows of other widths: only those of a multiple of 4 start on 16 bytes)
  if (a.c.dh % 4 == 0) return launch_paged_tiles<float, F32Step<kDh, 1>>(a, joined, st);
  return launch_paged_tiles<float, F32Step<kDh, 2>>(a, joined, st);
}
template <typename Tio, int kPer>
hipError_t launch_join_of(const PagedAttnArgs& a, hipStream_t st) {
  const int64_t items = (int64_t)a.T * a.n_heads;
  // (same sums either way; four waves per compute unit keep a wave's loads company)
  if (items >= 4 * compute_units()) k_attention_join<Tio, kPer, true><<<dim3((unsigned)((items + kJoinSums - 1) / kJoinSums)), kJoinSums * kWave, 0, st>>>(a);
  else k_attention_join<Tio, kPer, false><<<dim3((unsigned)items), kJoinSums * kWave, 0, st>>>(a);
  return hipGetLastError();
}
template <typename Tio>
hipError_t launch_join(const PagedAttnArgs& a, hipStream_t st) {
  return a.c.dh <= 64 ? launch_join_of<Tio, 1>(a, st) : a.c.dh <= 128 ? launch_join_of<Tio, 2>(a, st) : launch_join_of<Tio, 4>(a, st);
}
}  // namespace

hipError_t launch_attention_paged(const PagedAttnArgs& a, hipStream_t st) {
  hipError_t e;
  bool joined = false;
  if (a.c.bf16) {
    switch (a.c.dh) {
      case 64: e = launch_paged_tiles<bf16_t, Bf16Step<64>>(a, joined, st); break;
      case 128: e = launch_paged_tiles<bf16_t, Bf16Step<128>>(a, joined, st); break;
      case 256: e = launch_paged_tiles<bf16_t, Bf16Step<256>>(a, joined, st); break;
      default: return hipErrorInvalidValue;
    }
  } else {
    e = a.c.dh <= 64 ? launch_paged_f32<64>(a, joined, st) : a.c.dh <= 128 ? launch_paged_f32<128>(a, joined, st) : launch_paged_f32<256>(a, joined, st);
  }
  if (e != hipSuccess || a.ranges == 1 || joined) return e;
  return a.c.bf16 ? launch_join<bf16_t>(a, st) : launch_join<float>(a, st);
}

}  // namespace zo
