// kvc_cache_evict: every head of every row keeps its forced tokens and those with the largest gathered
// weights, in ascending position, in the blocks of another table.
//
// evict_select, one workgroup per head: a radix select (11 + 11 + 10 bits) over the ordered bits of the
// weights finds the smallest kept weight and how many tokens of exactly that weight still fit (the
// lowest positions); an ordered pass then writes the kept positions, ascending, to a list.
// evict_move, one workgroup per block that is written: takes 64 kept tokens from wherever they lie,
// finds the new scale from the values they stand for and writes their codes.  A value keeps its bits
// unless the new block's scale is larger than its old one (kvc_cache.h).
#include <algorithm>

#include "kvc_cache.h"

namespace kvc {

namespace {

constexpr int EV_THREADS = 1024;
constexpr int EV_WAVES = EV_THREADS / 64;
constexpr int EV_BINS = 2048;
constexpr uint32_t EV_FORCED = 0xff800000u;         // +infinity: forced tokens rank first
constexpr uint32_t EV_ABSENT = 0x007fffffu;         // -infinity: a token of a block that is not there
constexpr int EM_THREADS = 256;
constexpr float EM_RATIO = 1048576.0f;

struct EvictArgs {
  CacheView c;
  const int32_t* table_out;
  const int32_t* lengths;
  const int32_t* keep;
  int32_t* lengths_out;
  int32_t* list;            // [rows * hb, lpad] kept positions, ascending
  int64_t heads;            // rows * hb
  int max_keep, lpad, keep_first, keep_last;
};

__device__ __forceinline__ int kept_tokens(const EvictArgs& a, int64_t row, int len) {
  return max(min(min(a.keep[row], a.max_keep), len), 0);
}

// KPT > 0: every key of the row lies in registers, token i * EV_THREADS + tid in key[i].  KPT = 0: longer rows
// read their weights again in every pass.
template <int KPT>
__global__ __launch_bounds__(EV_THREADS) void evict_select(EvictArgs a) {
  __shared__ uint32_t hist[EV_BINS];
  __shared__ uint32_t part[EV_WAVES], found[2];
  __shared__ uint32_t counts[2][2][EV_WAVES];
  const CacheView& c = a.c;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  for (int64_t head = blockIdx.x; head < a.heads; head += gridDim.x) {
    const int64_t row = head / c.hb;
    const int hh = (int)(head - row * c.hb);
    const int len = cache_length(c, a.lengths[row]);
    const int keep = kept_tokens(a, row, len);
    if (hh == 0 && tid == 0) a.lengths_out[row] = keep;
    int32_t* list = a.list + head * a.lpad;
    if (keep == len) {                              // nothing leaves
      for (int i = tid; i < len; i += EV_THREADS) list[i] = i;
      continue;
    }
    if (keep == 0) continue;
    const auto read = [&](int t) -> uint32_t {
      if (t < a.keep_first || t >= len - a.keep_last) return EV_FORCED;
      const int id = c.table[row * c.width + t / CB_TOKENS];
      if (id < 0 || id >= c.blocks) return EV_ABSENT;
      return float_to_ordered(c.weight[((size_t)id * c.hb + hh) * CB_TOKENS + t % CB_TOKENS]);
    };
    uint32_t key[KPT > 0 ? KPT : 1];
    if (KPT > 0)
#pragma unroll
      for (int i = 0; i < KPT; ++i) {
        const int t = i * EV_THREADS + tid;
        key[i] = t < len ? read(t) : 0u;
      }
    const int chunks = (len + EV_THREADS - 1) / EV_THREADS;

    // ---- the keep-th largest key, digit by digit ----
    uint32_t prefix = 0, mask = 0, left = keep;     // left: to be taken among the keys that match prefix
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
      for (int i = tid; i < EV_BINS; i += EV_THREADS) hist[i] = 0;
      __syncthreads();
      const auto count = [&](uint32_t k, int t) {
        if (t < len && (k & mask) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
      };
      if (KPT > 0) {
#pragma unroll
        for (int i = 0; i < KPT; ++i) count(key[i], i * EV_THREADS + tid);
      } else {
        for (int i = 0; i < chunks; ++i) {
          const int t = i * EV_THREADS + tid;
          if (t < len) count(read(t), t);
        }
      }
      __syncthreads();
      // thread tid holds the bins 2 tid and 2 tid + 1 counted from the top
      const uint32_t hi = 2 * tid < bins ? hist[bins - 1 - 2 * tid] : 0u, lo = 2 * tid < bins ? hist[bins - 2 - 2 * tid] : 0u;
      uint32_t incl = hi + lo;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const uint32_t o = __shfl_up(incl, off);
        if (lane >= off) incl += o;
      }
      if (lane == 63) part[wave] = incl;
      __syncthreads();
      for (int w = 0; w < wave; ++w) incl += part[w];
      const uint32_t before = incl - hi - lo;
      if (before < left && left <= incl) {          // one thread
        const bool first = left <= before + hi;
        found[0] = bins - 1 - 2 * tid - (first ? 0 : 1);
        found[1] = left - before - (first ? 0 : hi);
      }
      __syncthreads();
      prefix |= found[0] << shift;
      mask |= (uint32_t)(bins - 1) << shift;
      left = found[1];
    }

    // ---- kept positions, ascending ----
    uint32_t above = 0, equal = 0;                  // so far, of all earlier chunks
    const auto emit = [&](int i, uint32_t k) {
      const int t = i * EV_THREADS + tid;
      const bool gt = t < len && k > prefix, eq = t < len && k == prefix;
      const uint64_t bg = __ballot(gt), be = __ballot(eq);
      uint32_t (*cnt)[EV_WAVES] = counts[i & 1];
      if (lane == 0) { cnt[0][wave] = __popcll(bg); cnt[1][wave] = __popcll(be); }
      __syncthreads();
      uint32_t g0 = above, e0 = equal;
#pragma unroll
      for (int w = 0; w < EV_WAVES; ++w) {
        const uint32_t x = cnt[0][w], y = cnt[1][w];
        if (w < wave) { g0 += x; e0 += y; }
        above += x;
        equal += y;
      }
      const uint64_t below = (1ull << lane) - 1;
      g0 += __popcll(bg & below);
      e0 += __popcll(be & below);
      const uint32_t at = g0 + min(e0, left);
      if ((gt || (eq && e0 < left)) && at < (uint32_t)keep) list[at] = t;
    };
    if (KPT > 0) {
#pragma unroll
      for (int i = 0; i < KPT; ++i)
        if (i < chunks) emit(i, key[i]);
    } else {
      for (int i = 0; i < chunks; ++i) {
        const int t = i * EV_THREADS + tid;
        emit(i, t < len ? read(t) : 0u);
      }
    }
    __syncthreads();                                // shared memory is free for the next head
  }
}

// NU: 16-byte pieces of K per thread, 64 * d / 16 / 256 rounded up; ND: words of four dimensions of V per
// thread, d / 16 rounded up.  V lies dimension by dimension, so a token of it is a column of bytes: lane =
// token, and a wave reads the same dimension of its 64 tokens, neighbours in one or a few rows.
template <int FMT, int NU, int ND>
__global__ __launch_bounds__(EM_THREADS) void evict_move(EvictArgs a, int blocks, int64_t units) {
  extern __shared__ __align__(16) uint8_t tile[];   // V codes [64][d + 4]
  __shared__ float red[2 * EM_THREADS / 64];
  const CacheView& c = a.c;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, d = c.d, pieces = d / 16, stride = d + 4;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t head = u / blocks;
    const int j = (int)(u - head * blocks);
    const int64_t row = head / c.hb;
    const int hh = (int)(head - row * c.hb);
    const int keep = kept_tokens(a, row, cache_length(c, a.lengths[row]));
    if (j * CB_TOKENS >= keep) continue;            // uniform
    const int to = a.table_out[row * c.width + j];
    if (to < 0 || to >= c.blocks) continue;
    const int here = min(keep - j * CB_TOKENS, CB_TOKENS);
    const int32_t* list = a.list + head * a.lpad + j * CB_TOKENS;
    const int32_t* ids = c.table + row * c.width;

    u32x4_t kw[NU];
    float kf[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int e = i * EM_THREADS + tid, token = e / pieces, piece = e - token * pieces;
      kw[i] = u32x4_t{0, 0, 0, 0};
      kf[i] = 0.f;
      if (token < here) {
        const int p = list[token], id = ids[p / CB_TOKENS];
        if (id >= 0 && id < c.blocks) {
          const size_t at = (size_t)id * c.hb + hh;
          kf[i] = c.k_scale[at];
          kw[i] = *reinterpret_cast<const u32x4_t*>(c.k + (at * CB_TOKENS + p % CB_TOKENS) * d + piece * 16);
        }
      }
    }
    uint32_t vw[ND];
    float vf = 0.f, wt = 0.f;
    const uint8_t* from = nullptr;
    if (lane < here) {
      const int p = list[lane], id = ids[p / CB_TOKENS];
      if (id >= 0 && id < c.blocks) {
        const size_t at = (size_t)id * c.hb + hh;
        vf = c.v_scale[at];
        wt = c.weight[at * CB_TOKENS + p % CB_TOKENS];
        from = c.v + at * CB_TOKENS * d + p % CB_TOKENS;
      }
    }
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      const int dim = (i * 4 + wave) * 4;
      vw[i] = 0;
      if (from && dim < d)
#pragma unroll
        for (int q = 0; q < 4; ++q) vw[i] |= (uint32_t)from[(dim + q) * CB_TOKENS] << (8 * q);
    }
    float ka = 0.f, va = 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float x[4];
        Code<FMT>::decode(kw[i][w], x);
#pragma unroll
        for (int e = 0; e < 4; ++e) ka = fmaxf(ka, fabsf(x[e]) * kf[i]);
      }
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      float x[4];
      Code<FMT>::decode(vw[i], x);
#pragma unroll
      for (int e = 0; e < 4; ++e) va = fmaxf(va, fabsf(x[e]) * vf);
    }
    ka = wave_max(ka);
    va = wave_max(va);
    if (lane == 0) { red[2 * wave] = ka; red[2 * wave + 1] = va; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EM_THREADS / 64; ++i) { ka = fmaxf(ka, red[2 * i]); va = fmaxf(va, red[2 * i + 1]); }
    const float ks = block_scale<FMT>(ka), vs = block_scale<FMT>(va);
    // old over new scale: a code that is not 0 has at most 2^18 of it, a larger one belongs to a row of zeros
    const float ki = inverse_scale(ks), vi = fminf(vf * inverse_scale(vs), EM_RATIO);
    const size_t at = (size_t)to * c.hb + hh;
    uint8_t* ko = c.k + at * CB_TOKENS * d;
    uint8_t* vo = c.v + at * CB_TOKENS * d;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int e = i * EM_THREADS + tid;
      if (e < CB_TOKENS * pieces) {
        const float f = fminf(kf[i] * ki, EM_RATIO);
        u32x4_t w4;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float x[4];
          Code<FMT>::decode(kw[i][w], x);
          w4[w] = Code<FMT>::encode(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
        }
        *reinterpret_cast<u32x4_t*>(ko + (size_t)e * 16) = w4;
      }
    }
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      const int dim = (i * 4 + wave) * 4;
      if (dim < d) {
        float x[4];
        Code<FMT>::decode(vw[i], x);
        *reinterpret_cast<uint32_t*>(tile + lane * stride + dim) = Code<FMT>::encode(x[0] * vi, x[1] * vi, x[2] * vi, x[3] * vi);
      }
    }
    if (tid == 0) { c.k_scale[at] = ks; c.v_scale[at] = vs; }
    if (tid < CB_TOKENS) c.weight[at * CB_TOKENS + tid] = wt;      // wave 0: lane = token
    __syncthreads();
    for (int e = tid; e < 4 * d; e += EM_THREADS) {
      const int dim = e % d, t0 = e / d * 16;
      u32x4_t o;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t x = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) x |= (uint32_t)tile[(t0 + 4 * q + t) * stride + dim] << (8 * t);
        o[q] = x;
      }
      *reinterpret_cast<u32x4_t*>(vo + (size_t)dim * CB_TOKENS + t0) = o;
    }
    __syncthreads();
  }
}

int list_pad(int64_t max_keep) { return int((max_keep + CB_TOKENS - 1) / CB_TOKENS * CB_TOKENS); }

}  // namespace

size_t evict_workspace_bytes(const Problem& pb, int64_t max_keep) {
  return align_up(size_t(pb.batch) * pb.layers * pb.hkv * size_t(list_pad(max_keep)) * 4);
}

kvc_status launch_cache_evict(const Problem& pb, const int32_t* lengths, const int32_t* keep, int64_t max_keep, int format,
                              const CacheView& c, const int32_t* table_out, int32_t* lengths_out, void* ws,
                              hipStream_t stream) {
  EvictArgs a{};
  a.c = c;
  a.table_out = table_out; a.lengths = lengths; a.keep = keep; a.lengths_out = lengths_out;
  a.list = static_cast<int32_t*>(ws);
  a.heads = int64_t(pb.batch) * pb.layers * pb.hkv;
  a.max_keep = int(max_keep); a.lpad = list_pad(max_keep);
  a.keep_first = pb.keep_first; a.keep_last = pb.keep_last;
  const unsigned grid = (unsigned)std::min<int64_t>(a.heads, 1 << 16);
  const int64_t longest = int64_t(c.width) * CB_TOKENS;
#define KVC_SELECT(KPT) KVC_LAUNCH("evict_select", stream, evict_select<KPT><<<grid, EV_THREADS, 0, stream>>>(a))
  if (longest <= 4 * EV_THREADS) KVC_SELECT(4);
  else if (longest <= 16 * EV_THREADS) KVC_SELECT(16);
  else if (longest <= 32 * EV_THREADS) KVC_SELECT(32);
  else KVC_SELECT(0);
#undef KVC_SELECT
  if (max_keep == 0) return KVC_OK;
  const int blocks = a.lpad / CB_TOKENS;
  const int64_t units = a.heads * blocks;
  const unsigned move = (unsigned)std::min<int64_t>(units, 1 << 20);
  const size_t lds = size_t(CB_TOKENS) * (pb.d + 4);
#define KVC_MOVE(FMT, NU, ND) \
  KVC_LAUNCH("evict_move", stream, evict_move<FMT, NU, ND><<<move, EM_THREADS, lds, stream>>>(a, blocks, units))
#define KVC_MOVE_D(FMT)                       \
  do {                                        \
    if (pb.d <= 64) KVC_MOVE(FMT, 1, 4);      \
    else if (pb.d <= 128) KVC_MOVE(FMT, 2, 8); \
    else KVC_MOVE(FMT, 4, 16);                \
  } while (0)
  if (format == KVC_E4M3) KVC_MOVE_D(KVC_E4M3); else KVC_MOVE_D(KVC_INT8);
#undef KVC_MOVE_D
#undef KVC_MOVE
  return KVC_OK;
}

}  // namespace kvc
