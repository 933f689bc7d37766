// kvc_cache_fill and kvc_cache_append: rows of K and V into the 8-bit block cache.
//
// Both round each value once, code = rne(x / s) with s the power of two of its (block, head), see
// kvc_cache.h.  A block of the fill is one workgroup's work from first to last: the largest magnitude
// has to be known before the first code can be written, so the 64 rows stay in registers in between.
#include <algorithm>

#include "kvc_cache.h"

namespace kvc {

namespace {

constexpr int CS_THREADS = 256;

// Largest |x| over the workgroup, of two quantities at once.  red: LDS, 2 * waves floats.
__device__ __forceinline__ void block_max2(float& a, float& b, float* red) {
  a = wave_max(a);
  b = wave_max(b);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) { red[2 * wave] = a; red[2 * wave + 1] = b; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < CS_THREADS / 64; ++i) { a = fmaxf(a, red[2 * i]); b = fmaxf(b, red[2 * i + 1]); }
}

// Table row whose blocks the unit u lies among.  Row r is given the units from offsets[r] / 64 + r on:
// as many as it has blocks or more, since ceil(n / 64) <= floor((a + n) / 64) - floor(a / 64) + 1.
// The wave probes 64 borders at a time.
__device__ __forceinline__ int find_row(const int64_t* __restrict__ offsets, int rows, int64_t u) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = rows;
  while (hi - lo > 1) {                             // wave-uniform
    const int step = (hi - lo + 63) / 64, mid = lo + lane * step;
    const bool at_or_before = mid < hi && offsets[mid] / CB_TOKENS + mid <= u;
    const int last = 63 - __clzll((long long)(__ballot(at_or_before) | 1ull));
    lo += last * step;
    hi = min(lo + step, hi);
  }
  return lo;
}

// One workgroup = one block of one head (a grid-stride loop over them).  Thread units are 8 elements of
// a token; NU of them per thread cover 64 * d elements.  Bound by HBM: 4 * d bytes of bf16 rows in and
// 2 * d bytes of codes out per (token, head).
template <int FMT, typename T, int NU>
__global__ __launch_bounds__(CS_THREADS) void cache_fill(PtrTable k_tab, PtrTable v_tab,
                                                         const int32_t* __restrict__ idx,
                                                         const float* __restrict__ scores,
                                                         const int32_t* __restrict__ lengths,
                                                         const int64_t* __restrict__ offsets, SeqTable seq,
                                                         CacheView c, int total, int64_t units) {
  extern __shared__ __align__(16) uint8_t tile[];   // V codes [64][d + 8]
  __shared__ float red[2 * CS_THREADS / 64];
  const int d = c.d, pieces = d / 8, stride = d + 8, tid = threadIdx.x;
  const int per_layer = c.hkv / c.hb, rows = seq.batch * c.layers * per_layer;
  for (int64_t w = blockIdx.x; w < units * c.hb; w += gridDim.x) {
    const int64_t u = w / c.hb;
    const int hh = (int)(w - u * c.hb);
    const int row = find_row(offsets, rows, u);
    const int64_t j = u - (offsets[row] / CB_TOKENS + row);
    const int bl = row / per_layer, b = bl / c.layers, l = bl - b * c.layers;
    const int h = c.hb == 1 ? row - bl * per_layer : hh;
    const int n_b = seq.cu[b + 1] - seq.cu[b];
    const int len = cache_length(c, min(lengths[row], n_b));
    if (j < 0 || j * CB_TOKENS >= len) continue;    // uniform: a unit that no block needs
    const int id = c.table[(int64_t)row * c.width + j];
    if (id < 0 || id >= c.blocks) continue;
    const int here = min(len - (int)j * CB_TOKENS, CB_TOKENS);
    const size_t at = (size_t)id * c.hb + hh;
    const size_t head = (size_t)h * total + seq.cu[b];
    const int32_t* list = idx ? idx + ((size_t)l * c.hkv + h) * total + seq.cu[b] + j * CB_TOKENS : nullptr;
    const T* kl = static_cast<const T*>(k_tab.p[l]);
    const T* vl = static_cast<const T*>(v_tab.p[l]);

    Row8<T> kr[NU], vr[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int e = i * CS_THREADS + tid, token = e / pieces, piece = e - token * pieces;
      kr[i].clear();
      vr[i].clear();
      if (token < here) {
        const int p = list ? list[token] : (int)j * CB_TOKENS + token;
        if (p >= 0 && p < n_b) {                    // never read outside the cache
          const size_t src = (head + p) * d + piece * 8;
          kr[i].load(kl + src);
          vr[i].load(vl + src);
        }
      }
    }
    float wt = 0.f;
    if (c.weight && scores && tid < here) {
      const int p = list ? list[tid] : (int)j * CB_TOKENS + tid;
      if (p >= 0 && p < n_b) wt = scores[((size_t)l * c.hkv) * total + head + p];
    }
    float ka = 0.f, va = 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      float x[8];
      kr[i].get(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) ka = fmaxf(ka, fabsf(x[e]));
      vr[i].get(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) va = fmaxf(va, fabsf(x[e]));
    }
    block_max2(ka, va, red);
    const float ks = block_scale<FMT>(ka), vs = block_scale<FMT>(va);
    const float ki = inverse_scale(ks), vi = inverse_scale(vs);
    uint8_t* ko = c.k + at * CB_TOKENS * d;
    uint8_t* vo = c.v + at * CB_TOKENS * d;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int e = i * CS_THREADS + tid;
      if (e < CB_TOKENS * pieces) {
        float x[8];
        kr[i].opaque();                             // else the floats of the maximum are kept in registers until here
        vr[i].opaque();
        kr[i].get(x);
        u32x2_t w2{Code<FMT>::encode(x[0] * ki, x[1] * ki, x[2] * ki, x[3] * ki),
                   Code<FMT>::encode(x[4] * ki, x[5] * ki, x[6] * ki, x[7] * ki)};
        __builtin_nontemporal_store(w2, reinterpret_cast<u32x2_t*>(ko + (size_t)e * 8));
        vr[i].get(x);
        u32x2_t v2{Code<FMT>::encode(x[0] * vi, x[1] * vi, x[2] * vi, x[3] * vi),
                   Code<FMT>::encode(x[4] * vi, x[5] * vi, x[6] * vi, x[7] * vi)};
        const int token = e / pieces;
        *reinterpret_cast<u32x2_t*>(tile + token * stride + (e - token * pieces) * 8) = v2;
      }
    }
    if (tid == 0) { c.k_scale[at] = ks; c.v_scale[at] = vs; }
    if (c.weight && tid < CB_TOKENS) c.weight[at * CB_TOKENS + tid] = wt;
    __syncthreads();
    // 16 tokens of a dimension per lane, whole lines per store, with the streaming hint (128k tokens, a tenth kept,
    // 32 layers: 488 us; neighbouring lanes on neighbouring dimensions 527, and 930 with the hint)
    for (int e = tid; e < 4 * d; e += CS_THREADS) {
      const int dim = e >> 2, t0 = (e & 3) * 16;
      u32x4_t o;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t x = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) x |= (uint32_t)tile[(t0 + 4 * q + t) * stride + dim] << (8 * t);
        o[q] = x;
      }
      __builtin_nontemporal_store(o, reinterpret_cast<u32x4_t*>(vo + (size_t)dim * CB_TOKENS + t0));
    }
    __syncthreads();                                // the tile and red are free again
  }
}

template <typename T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_float<uint16_t>(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// grid: (blocks that M tokens can touch, hkv, batch).  The M new tokens are the last of the row's `len`.
// A block that already holds tokens keeps its scale unless a new row needs a larger one; then its old
// codes are rounded again to the larger steps (code * s / s' is exact before that rounding).
// Latency bound: one chain of length -> table -> scale, rows -> maximum -> codes.
template <int FMT, typename T>
__global__ __launch_bounds__(CS_THREADS) void cache_append(const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                           const int32_t* __restrict__ lengths, CacheView c, int layer,
                                                           int window) {
  __shared__ float red[2 * CS_THREADS / 64];
  const int b = blockIdx.z, h = blockIdx.y, d = c.d, tid = threadIdx.x;
  const int64_t row = cache_row(c, b, layer, h);
  const int len = lengths[row];
  if (len <= 0 || (int64_t)len > (int64_t)c.width * CB_TOKENS) return;   // uniform; a full row takes nothing
  const int start = len - window;                   // slot of the first new token; below 0 those rows are skipped
  const int block = max(start, 0) / CB_TOKENS + blockIdx.x;
  if ((int64_t)block * CB_TOKENS >= len) return;
  const int id = c.table[row * c.width + block];
  if (id < 0 || id >= c.blocks) return;
  const int lo = max(start - block * CB_TOKENS, 0), hi = min(len - block * CB_TOKENS, CB_TOKENS);
  const size_t at = (size_t)id * c.hb + cache_head(c, h);
  uint8_t* ko = c.k + at * CB_TOKENS * d;
  uint8_t* vo = c.v + at * CB_TOKENS * d;
  const size_t first = (((size_t)b * c.hkv + h) * window + (block * CB_TOKENS + lo - start)) * d;
  const int count = (hi - lo) * d;                  // new elements of this block
  const float ks_old = c.k_scale[at], vs_old = c.v_scale[at];

  float ka = 0.f, va = 0.f;
  for (int e = tid; e < count; e += CS_THREADS) {
    ka = fmaxf(ka, fabsf(to_float(k_new[first + e])));
    va = fmaxf(va, fabsf(to_float(v_new[first + e])));
  }
  block_max2(ka, va, red);
  float ks = block_scale<FMT>(ka), vs = block_scale<FMT>(va);
  if (lo > 0) {
    ks = fmaxf(ks, ks_old);
    vs = fmaxf(vs, vs_old);
    // old codes: the first lo rows of K, the first lo bytes of every row of V
    if (ks > ks_old) {
      const float f = ks_old * inverse_scale(ks);
      for (int e = tid; e < lo * d / 4; e += CS_THREADS) {
        float x[4];
        uint32_t* w = reinterpret_cast<uint32_t*>(ko) + e;
        Code<FMT>::decode(*w, x);
        *w = Code<FMT>::encode(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
      }
    }
    if (vs > vs_old) {
      const float f = vs_old * inverse_scale(vs);
      for (int e = tid; e < d * (CB_TOKENS / 4); e += CS_THREADS) {
        const int dim = e / (CB_TOKENS / 4), t = (e % (CB_TOKENS / 4)) * 4;
        if (t >= lo) continue;
        float x[4];
        uint32_t* w = reinterpret_cast<uint32_t*>(vo + dim * CB_TOKENS + t);
        const uint32_t was = *w;
        Code<FMT>::decode(was, x);
        const uint32_t old = lo - t >= 4 ? ~0u : (1u << (8 * (lo - t))) - 1;   // bytes of old tokens
        *w = (Code<FMT>::encode(x[0] * f, x[1] * f, x[2] * f, x[3] * f) & old) | (was & ~old);
      }
    }
    __syncthreads();                                // new bytes of the words that were just written come behind
  }
  const float ki = inverse_scale(ks), vi = inverse_scale(vs);
  for (int e = tid; e < count; e += CS_THREADS) {
    const int token = e / d, dim = e - token * d;
    const float x = to_float(k_new[first + e]) * ki, y = to_float(v_new[first + e]) * vi;
    ko[lo * d + e] = (uint8_t)Code<FMT>::encode(x, 0.f, 0.f, 0.f);
    vo[dim * CB_TOKENS + lo + token] = (uint8_t)Code<FMT>::encode(y, 0.f, 0.f, 0.f);
  }
  if (tid == 0) { c.k_scale[at] = ks; c.v_scale[at] = vs; }
  if (c.weight && tid < hi - lo) c.weight[at * CB_TOKENS + lo + tid] = 0.f;
}

template <int FMT, typename T>
kvc_status fill_form(const Problem& pb, const PtrTable& kt, const PtrTable& vt, const int32_t* idx, const float* scores,
                     const int32_t* lengths, const int64_t* offsets, const CacheView& c, int64_t units, unsigned grid,
                     hipStream_t stream) {
#define KVC_FILL(NU)                                                                                              \
  KVC_LAUNCH("cache_fill", stream, cache_fill<FMT, T, NU><<<grid, CS_THREADS, CB_TOKENS * (c.d + 8), stream>>>(          \
      kt, vt, idx, scores, lengths, offsets, pb.seq, c, int(pb.total), units))
  if (c.d <= 64) KVC_FILL(2);
  else if (c.d <= 128) KVC_FILL(4);
  else KVC_FILL(8);
#undef KVC_FILL
  return KVC_OK;
}

}  // namespace

kvc_status launch_cache_fill(const Problem& pb, const void* const* k, const void* const* v, const int32_t* idx,
                             const float* scores, const int32_t* lengths, const int64_t* offsets, int64_t total_budget,
                             int format, const CacheView& c, hipStream_t stream) {
  PtrTable kt{}, vt{};
  for (int l = 0; l < pb.layers; ++l) { kt.p[l] = k[l]; vt.p[l] = v[l]; }
  const int64_t rows = int64_t(pb.batch) * pb.sel_rows;
  const int64_t units = total_budget / CB_TOKENS + rows;
  const unsigned grid = (unsigned)std::min<int64_t>(units * c.hb, 1 << 20);
  const bool half = pb.dtype == KVC_BF16;
  if (format == KVC_E4M3)
    return half ? fill_form<KVC_E4M3, uint16_t>(pb, kt, vt, idx, scores, lengths, offsets, c, units, grid, stream)
                : fill_form<KVC_E4M3, float>(pb, kt, vt, idx, scores, lengths, offsets, c, units, grid, stream);
  return half ? fill_form<KVC_INT8, uint16_t>(pb, kt, vt, idx, scores, lengths, offsets, c, units, grid, stream)
              : fill_form<KVC_INT8, float>(pb, kt, vt, idx, scores, lengths, offsets, c, units, grid, stream);
}

kvc_status launch_cache_append(const Problem& pb, int layer, const void* k_new, const void* v_new, const int32_t* lengths,
                               int format, const CacheView& c, hipStream_t stream) {
  const dim3 grid((pb.window + CB_TOKENS - 2) / CB_TOKENS + 1, pb.hkv, pb.batch);
#define KVC_APPEND(FMT, T)                                                                              \
  KVC_LAUNCH("cache_append", stream, cache_append<FMT, T><<<grid, CS_THREADS, 0, stream>>>(             \
      static_cast<const T*>(k_new), static_cast<const T*>(v_new), lengths, c, layer, pb.window))
  const bool half = pb.dtype == KVC_BF16;
  if (format == KVC_E4M3) {
    if (half) KVC_APPEND(KVC_E4M3, uint16_t); else KVC_APPEND(KVC_E4M3, float);
  } else {
    if (half) KVC_APPEND(KVC_INT8, uint16_t); else KVC_APPEND(KVC_INT8, float);
  }
#undef KVC_APPEND
  return KVC_OK;
}

}  // namespace kvc
