// Decoding from a paged key/value cache (Sec. 2.2: a query is a prompt that a candidate continues; the rows of a
// decode step are one token per sequence, each under its own candidate).
//
//   k_cache_append      per-head RMS norm + rotary embedding of new rows, keys and values into their pages
//   k_attention_paged   attention of a new row over its sequence's pages, a range of them per workgroup
//   k_attention_join    joins the ranges of a long row
//
// A row's place: sequence i with cu[i] <= t < cu[i+1], position kv_len[i] - (cu[i+1] - t); position p lies in slot
// p % page_size of page page_table[i][p / page_size].  Rows behind the last sequence are left as they were.
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

// ------------------------------------------------------------------ append

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
      const float sn = (float)dsn, cs = (float)dcs;
      const float p = lo[c], q = hi[c];
      lo[c] = p * cs - q * sn;
      hi[c] = q * cs + p * sn;
    }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int i = lane + c * kWave;
    if (i < half) { st_elem(out, i, lo[c]); st_elem(out, half + i, hi[c]); }
  }
}

// ------------------------------------------------------------------ attention

// A row's positions are cut into ranges of range_keys(n), a function of the row's own n alone; a workgroup of four waves
// takes one (row, key/value head, range).  Its waves take steps of keys in turn, each with a running maximum and sum of
// its own, and join in LDS in the order of the waves; a row of several ranges leaves (maximum, sum, unnormalised output)
// of each in the workspace and k_attention_join joins them in order.
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
// fp32 uses the 16x16x4 instruction on 16 keys per step: a lane's scores are those of keys 4 g .. 4 g + 3, and that one value
// per lane is the operand needs no transposition.

constexpr int kAttnWaves = 4;
constexpr int kRange = 256;          // keys per workgroup of a row of up to kMaxRanges * kRange positions
constexpr int kMaxRanges = 64;       // one lane each in the join
__host__ __device__ constexpr int range_keys(int n) {
  return kRange * (n <= kMaxRanges * kRange ? 1 : (n + kMaxRanges * kRange - 1) / (kMaxRanges * kRange));
}
// most ranges of a row of up to n positions
constexpr int most_ranges(int n) { return n >= kMaxRanges * kRange ? kMaxRanges : (n + kRange - 1) / kRange; }

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

// Workspace: [T][n_heads][ranges] of (maximum, sum), then [T][n_heads][ranges][dh] unnormalised outputs.
__device__ __forceinline__ int64_t part_at(const PagedAttnArgs& a, int t, int h, int range) {
  return ((int64_t)t * a.n_heads + h) * a.ranges + range;
}

// What differs between the two types: loading a step's keys and values and the two products.
// eff(key): which of the step's keys stands in for `key`; at(key): its first element in the pools.
template <int kDh>
struct Bf16Step {
  static constexpr int kKeys = 32, kPad = kDh, kCols = kDh / 16;   // columns of a value row per lane
  static constexpr int kScores = 8;       // per lane: keys 8 g + i
  bf16x8 k[2][kDh / 32];
  u32x4 v[8][kCols > 8 ? kCols / 8 : 1];  // (kCols 4: the lower half of each)
  __device__ static constexpr int key_of_score(int g, int i) { return 8 * g + i; }

  template <class At>
  __device__ __forceinline__ void load(const PagedAttnArgs& a, int r, int g, At at) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const bf16_t* p = (const bf16_t*)a.c.K + at(8 * (r >> 2) + (r & 3) + 4 * hf) + g * 8;
#pragma unroll
      for (int ks = 0; ks < kDh / 32; ++ks) k[hf][ks] = load_frag(p + ks * 32);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bf16_t* p = (const bf16_t*)a.c.V + at(8 * g + j) + r * kCols;
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
  // (the weights are rounded to bf16 here: half a step of 2^-8 each, averaged over the keys of a row)
  __device__ __forceinline__ void values(const float (&p)[kScores], f32x4 (&o)[kCols]) const {
    const u32x4 packed = {pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
    const bf16x8 pf = __builtin_bit_cast(bf16x8, packed);
#pragma unroll
    for (int d = 0; d < kCols; ++d) {
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j)   // column d of keys 2 j and 2 j + 1
        w[j] = __builtin_amdgcn_perm(v[2 * j + 1][d >> 3][(d & 7) >> 1], v[2 * j][d >> 3][(d & 7) >> 1], (d & 1) ? 0x07060302u : 0x05040100u);
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), pf, o[d], 0, 0, 0);
    }
  }
};

// kMode 0: the head dimension is kDh; 1: smaller, a multiple of 4; 2: smaller, any.
template <int kDh, int kMode>
struct F32Step {
  static constexpr int kKeys = 16, kPad = kDh, kCols = kDh / 16;
  static constexpr int kScores = 4;       // per lane: keys 4 g + i
  f32x4 k[kDh / 16];
  f32x4 v[4][kCols / 4];
  __device__ static constexpr int key_of_score(int g, int i) { return 4 * g + i; }

  // four values from column `col` of a row of dh; zeros behind its end
  __device__ static __forceinline__ f32x4 four(const float* row, int col, int dh) {
    if constexpr (kMode == 0) return *reinterpret_cast<const f32x4*>(row + col);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if constexpr (kMode == 1) {
      if (col < dh) x = *reinterpret_cast<const f32x4*>(row + col);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < dh) x[e] = row[col + e];
    }
    return x;
  }
  template <class At>
  __device__ __forceinline__ void load(const PagedAttnArgs& a, int r, int g, At at) {
    const float* p = (const float*)a.c.K + at(r);
#pragma unroll
    for (int ks = 0; ks < kDh / 16; ++ks) k[ks] = four(p, ks * 16 + g * 4, a.c.dh);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float* w = (const float*)a.c.V + at(4 * g + j);
#pragma unroll
      for (int c = 0; c < kCols / 4; ++c) v[j][c] = four(w, r * kCols + c * 4, a.c.dh);
    }
  }
  typedef f32x4 Query[kDh / 16];
  __device__ static __forceinline__ void load_query(const PagedAttnArgs& a, const void* row, bool valid, int g, Query& q) {
#pragma unroll
    for (int ks = 0; ks < kDh / 16; ++ks) {
      q[ks] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (valid) q[ks] = kMode == 0 ? *reinterpret_cast<const f32x4*>((const float*)row + ks * 16 + g * 4) : four((const float*)row, ks * 16 + g * 4, a.c.dh);
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

// kTiles: tiles of 16 query heads per workgroup (1 or 4); its waves share the keys 4 / kTiles ways.
template <typename Tio, class Step, int kTiles>
__global__ __launch_bounds__(kAttnWaves* kWave, Step::kPad > 128 ? 1 : 2) void k_attention_paged(PagedAttnArgs a) {
  constexpr int kDh = Step::kPad, kCols = Step::kCols, kKeys = Step::kKeys, kSharers = kAttnWaves / kTiles;
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
  const int len = range_keys(n);
  const int n_ranges = n > 0 ? (n + len - 1) / len : 1;   // (an empty row: one empty range writes its zeros)
  const int tile = wave % kTiles, share = wave / kTiles;
  const int head0 = (part * kTiles + tile) * 16;            // of the group
  const int cols = min(16, a.group - head0);                 // columns in use (may be <= 0)
  typename Step::Query q;
  Step::load_query(a, (const Tio*)a.Q + (int64_t)t * a.ldq + (int64_t)(kvh * a.group + head0 + r) * a.c.dh, r < cols, g, q);
  const float sl2 = a.scale * 1.4426950408889634f;           // scores are kept in base-2 units
  const int32_t* table = a.c.table + (int64_t)pl.seq * a.c.max_pages;

  for (int range = blockIdx.y; range < n_ranges; range += gridDim.y) {
    const int j_a = range * len, j_b = min(j_a + len, n);   // the range's positions
    f32x4 o[kCols];
#pragma unroll
    for (int d = 0; d < kCols; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;   // l: this lane's share

    // pages of the 64 blocks of 16 positions that begin at block `first`, one a lane; -1: no position, or no page of the pool
    auto pages_from = [&](int first) {
      const int j = (first + lane) * 16;
      if (j >= j_b) return -1;
      const int pg = table[j >> a.c.page_shift];
      return (unsigned)pg < (unsigned)a.c.n_pages ? pg : -1;
    };
    int first = j_a / 16;
    int pages = pages_from(first);
    // Loads step `j0`; false when it has no key that is seen.  A key that is not seen is stood in for by one that is: what a
    // slot behind the last position holds must not meet even a weight of zero.
    auto load = [&](int j0, Step& st, int& last, int& dead) -> bool {
      const int b = j0 / 16 - first;
      const int p0 = __builtin_amdgcn_readlane(pages, b);
      const int p1 = kKeys == 32 ? __builtin_amdgcn_readlane(pages, b + 1) : p0;
      dead = (p0 < 0 ? 1 : 0) | (p1 < 0 ? 2 : 0);
      if (p0 < 0 && p1 < 0) return false;
      last = j_b - 1 - j0;
      const int64_t b0 = slot_at(a.c, p0 < 0 ? p1 : p0, kvh, j0), b1 = slot_at(a.c, p1 < 0 ? p0 : p1, kvh, j0 + 16);
      const bool whole = dead == 0 && last >= kKeys - 1;
      st.load(a, r, g, [&](int key) -> int64_t {
        int e = key;
        if (!whole) {
          if (kKeys == 32 && (dead >> (key >> 4) & 1)) e ^= 16;
          e = min(e, last);
        }
        return (kKeys == 32 && e >= 16 ? b1 : b0) + (e & 15) * a.c.dh;
      });
      return true;
    };
    auto attend = [&](const Step& st, int last, int dead) {
      float s[Step::kScores];
      st.scores(q, s);
#pragma unroll
      for (int i = 0; i < Step::kScores; ++i) s[i] *= sl2;
      if (dead != 0 || last < kKeys - 1) {
#pragma unroll
        for (int i = 0; i < Step::kScores; ++i) {
          const int key = Step::key_of_score(g, i);
          if (key > last || (dead >> (key >> 4) & 1)) s[i] = -INFINITY;
        }
      }
      float mx = s[0];
#pragma unroll
      for (int i = 1; i < Step::kScores; ++i) mx = fmaxf(mx, s[i]);
      float f = 1.0f;
      if (__any(mx > m)) {   // (otherwise every factor is one)
        const float m2 = fmaxf(column_max(mx), m);
        f = __builtin_amdgcn_exp2f(m - m2);
        m = m2;
#pragma unroll
        for (int d = 0; d < kCols; ++d) o[d] *= f;
      }
      float p[Step::kScores], sum = 0.f;
#pragma unroll
      for (int i = 0; i < Step::kScores; ++i) {
        p[i] = __builtin_amdgcn_exp2f(s[i] - m);
        sum += p[i];
      }
      l = __builtin_fmaf(l, f, sum);
      st.values(p, o);
    };
    if (cols > 0) {
      for (int j0 = j_a + share * kKeys; j0 < j_b; j0 += kSharers * kKeys) {
        if (j0 / 16 - first >= 64) {
          first += 64;
          pages = pages_from(first);
        }
        Step st;
        int last, dead;
        if (load(j0, st, last, dead)) attend(st, last, dead);
      }
    }

    // ---- the waves join
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
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
      float mm = -INFINITY;
#pragma unroll
      for (int w = 0; w < kSharers; ++w) mm = fmaxf(mm, s_m[w * kTiles + tl][col]);
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kSharers; ++w) {
        const int wv = w * kTiles + tl;
        const float mw = s_m[wv][col];
        const float f = mw == mm ? 1.0f : __builtin_amdgcn_exp2f(mw - mm);   // (no key at all: zeros stay zeros)
        acc += *reinterpret_cast<const f32x4*>(s_o + (wv * 16 + col) * kRowLds + d) * f;
        sum += s_l[wv][col] * f;
      }
      const int h = kvh * a.group + part * 16 * kTiles + c;
      if (n_ranges == 1) {
        const float inv = sum > 0.f ? 1.0f / sum : sum;   // (NaN stays NaN)
        Tio* out = (Tio*)a.O + (int64_t)t * a.ldo + (int64_t)h * a.c.dh + d;
        if constexpr (sizeof(Tio) == 2) {
          *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv));
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (d + i < a.c.dh) out[i] = acc[i] * inv;
        }
      } else {
        const int64_t at = part_at(a, t, h, range);
        if (d == 0) { a.part_ml[2 * at] = mm; a.part_ml[2 * at + 1] = sum; }
        float* out = a.part_o + at * a.c.dh + d;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (kDh == a.c.dh || d + i < a.c.dh) out[i] = acc[i];
      }
    }
    if (range + (int)gridDim.y < n_ranges) __syncthreads();   // (the buffer is written again)
  }
}

// Joins the ranges of a row, one wave per (row, head): lane c has range c's maximum and sum, then the lanes go over the
// columns and add the ranges in order.
template <typename Tio>
__global__ __launch_bounds__(256) void k_attention_join(PagedAttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= (int64_t)a.T * a.n_heads) return;
  const int t = (int)(item / a.n_heads), h = (int)(item % a.n_heads);
  const Place pl = place_of_row(a.cu, a.c.kv_len, a.S, t, lane);
  if (pl.seq < 0) return;
  const int n = min(pl.pos + 1, a.c.max_pages << a.c.page_shift);
  const int len = range_keys(n);
  const int n_ranges = n > 0 ? (n + len - 1) / len : 1;
  if (n_ranges == 1) return;
  const int64_t at = part_at(a, t, h, 0);
  float m = -INFINITY, l = 0.f;
  if (lane < n_ranges) { m = a.part_ml[2 * (at + lane)]; l = a.part_ml[2 * (at + lane) + 1]; }
  const float mm = wave_max(m);
  const float f = m == mm ? 1.0f : __builtin_amdgcn_exp2f(m - mm);
  const float sum = wave_sum(l * f);
  const float inv = sum > 0.f ? 1.0f / sum : sum;
  for (int d = lane; d < a.c.dh; d += kWave) {
    const float* o = a.part_o + at * a.c.dh + d;
    float acc = 0.f;
    for (int c = 0; c < n_ranges; ++c) acc += o[(int64_t)c * a.c.dh] * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), c));
    st_elem((Tio*)a.O + (int64_t)t * a.ldo + (int64_t)h * a.c.dh, d, acc * inv);
  }
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t st) {
  const int64_t items = (int64_t)a.T * (a.n_heads + 2 * a.c.n_kv_heads);
  const dim3 grid((unsigned)((items + 3) / 4));
  if (a.c.bf16) k_cache_append<bf16_t><<<grid, 256, 0, st>>>(a);
  else k_cache_append<float><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

int attention_paged_ranges(int max_len) { return max_len > 0 ? most_ranges(max_len) : 1; }

namespace {
template <typename Tio, class Step, int kTiles>
hipError_t launch_paged(const PagedAttnArgs& a, hipStream_t st) {
  constexpr int kLds = kAttnWaves * 16 * (Step::kPad + 4) * 4;
  static std::atomic<bool> ready[kMaxDevices];
  if (kLds > 64 * 1024 - 1024) {
    const hipError_t e = once_per_device(ready, [] {
      return hipFuncSetAttribute((const void*)k_attention_paged<Tio, Step, kTiles>, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    });
    if (e != hipSuccess) return e;
  }
  const int per_head = (a.group + 16 * kTiles - 1) / (16 * kTiles);
  const dim3 grid((unsigned)((int64_t)a.T * a.c.n_kv_heads * per_head), (unsigned)a.ranges);
  k_attention_paged<Tio, Step, kTiles><<<grid, kAttnWaves * kWave, kLds, st>>>(a);
  return hipGetLastError();
}
template <typename Tio, class Step>
hipError_t launch_paged_tiles(const PagedAttnArgs& a, hipStream_t st) {
  return a.group <= 16 ? launch_paged<Tio, Step, 1>(a, st) : launch_paged<Tio, Step, 4>(a, st);
}
template <int kDh>
hipError_t launch_paged_f32(const PagedAttnArgs& a, hipStream_t st) {
  if (a.c.dh == kDh) return launch_paged_tiles<float, F32Step<kDh, 0>>(a, st);
  // (rows of other widths: only those of a multiple of 4 start on 16 bytes)
  if (a.c.dh % 4 == 0) return launch_paged_tiles<float, F32Step<kDh, 1>>(a, st);
  return launch_paged_tiles<float, F32Step<kDh, 2>>(a, st);
}
}  // namespace

hipError_t launch_attention_paged(const PagedAttnArgs& a, hipStream_t st) {
  hipError_t e;
  if (a.c.bf16) {
    switch (a.c.dh) {
      case 64: e = launch_paged_tiles<bf16_t, Bf16Step<64>>(a, st); break;
      case 128: e = launch_paged_tiles<bf16_t, Bf16Step<128>>(a, st); break;
      case 256: e = launch_paged_tiles<bf16_t, Bf16Step<256>>(a, st); break;
      default: return hipErrorInvalidValue;
    }
  } else {
    e = a.c.dh <= 64 ? launch_paged_f32<64>(a, st) : a.c.dh <= 128 ? launch_paged_f32<128>(a, st) : launch_paged_f32<256>(a, st);
  }
  if (e != hipSuccess || a.ranges == 1) return e;
  const dim3 grid((unsigned)(((int64_t)a.T * a.n_heads + 3) / 4));
  if (a.c.bf16) k_attention_join<bf16_t><<<grid, 256, 0, st>>>(a);
  else k_attention_join<float><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace zo
