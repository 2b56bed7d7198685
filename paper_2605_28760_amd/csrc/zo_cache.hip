// Decoding from a paged key/value cache (Sec. 2.2: a query is a prompt that a candidate continues; the rows of a
// decode step are one token per sequence, each under its own candidate).
//
//   k_cache_append      per-head RMS norm + rotary embedding of new rows, keys and values into their pages
//   k_attention_paged   attention of a new row over its sequence's pages
//
// A row's place: sequence i with cu[i] <= t < cu[i+1], position kv_len[i] - (cu[i+1] - t); position p lies in slot
// p % page_size of page page_table[i][p / page_size].  Rows behind the last sequence are left as they were.
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

constexpr int kMaxDh = 256;

// One wave per (row, head): 64 keys at a time, a lane scores a key, then the lanes go over the head dimension; running
// maximum and sum.
template <typename Tio>
__global__ __launch_bounds__(kWave) void k_attention_paged(PagedAttnArgs a) {
  __shared__ float s_q[kMaxDh];
  __shared__ float s_p[kWave];
  __shared__ int64_t s_at[kWave];
  const int lane = threadIdx.x;
  const int t = blockIdx.x, h = blockIdx.y, g = h / a.group;
  const int dh = a.c.dh;
  const int seq = seq_of_row(a.cu, a.S, t);
  if (seq >= a.S) return;
  const int pos = a.c.kv_len[seq] - (a.cu[seq + 1] - t);
  const int n = min(pos + 1, a.c.max_pages << a.c.page_shift);
  const Tio* q = (const Tio*)a.Q + (int64_t)t * a.ldq + h * dh;
  for (int d = lane; d < dh; d += kWave) s_q[d] = ld_elem(q, d);
  __syncthreads();
  float acc[kMaxDh / kWave] = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  for (int base = 0; base < n; base += kWave) {
    const int j = base + lane;
    const int page = j < n ? page_of(a.c, seq, j) : -1;
    const int64_t at = page >= 0 ? slot_at(a.c, page, g, j) : -1;
    float s = -INFINITY;
    if (page >= 0) {
      const Tio* k = (const Tio*)a.c.K + at;
      s = 0.f;
      for (int d = 0; d < dh; ++d) s += s_q[d] * ld_elem(k, d);
      s *= a.scale;
    }
    const float m2 = fmaxf(m, wave_max(s));
    const float p = page >= 0 ? expf(s - m2) : 0.f;
    const float f = m == m2 ? 1.f : expf(m - m2);
    l = l * f + p;
    m = m2;
    s_p[lane] = p;
    s_at[lane] = at;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kMaxDh / kWave; ++c) acc[c] *= f;
    for (int jj = 0; jj < kWave; ++jj) {
      if (s_at[jj] < 0) continue;
      const Tio* v = (const Tio*)a.c.V + s_at[jj];
#pragma unroll
      for (int c = 0; c < kMaxDh / kWave; ++c)
        if (lane + c * kWave < dh) acc[c] += s_p[jj] * ld_elem(v, lane + c * kWave);
    }
    __syncthreads();
  }
  l = wave_sum(l);
  const float inv = l > 0.f ? 1.0f / l : l;   // (NaN stays NaN)
  Tio* o = (Tio*)a.O + (int64_t)t * a.ldo + h * dh;
#pragma unroll
  for (int c = 0; c < kMaxDh / kWave; ++c)
    if (lane + c * kWave < dh) st_elem(o, lane + c * kWave, acc[c] * inv);
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t st) {
  const int64_t items = (int64_t)a.T * (a.n_heads + 2 * a.c.n_kv_heads);
  const dim3 grid((unsigned)((items + 3) / 4));
  if (a.c.bf16) k_cache_append<bf16_t><<<grid, 256, 0, st>>>(a);
  else k_cache_append<float><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_attention_paged(const PagedAttnArgs& a, hipStream_t st) {
  const dim3 grid(a.T, a.n_heads);
  if (a.c.bf16) k_attention_paged<bf16_t><<<grid, kWave, 0, st>>>(a);
  else k_attention_paged<float><<<grid, kWave, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace zo
