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

// Rows are worked on EV_THREADS * KPT tokens at a time, token i * EV_THREADS + tid in key[i]: those of a row that is
// no longer stay in registers; longer ones (LOOP) are read again in every pass, KPT keys in flight per thread.  (256
// heads of 30517 tokens: 50 us in registers, 104 read again; 60000 tokens 201 us, of 1260 for the eviction.)
template <int KPT, bool LOOP>
__global__ __launch_bounds__(EV_THREADS, KPT <= 16 ? 8 : 4) void evict_select(EvictArgs a) {
  __shared__ uint32_t hist[EV_BINS];
  __shared__ uint32_t part[EV_WAVES], found[2];
  __shared__ uint32_t counts[KPT * EV_WAVES + 1];   // above | equal << 16 of a wave's 64 tokens; of all
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
    // key of token i * EV_THREADS + tid: a wave's 64 tokens are one block, whose id is a scalar
    const int wave_s = __builtin_amdgcn_readfirstlane(wave);
    const auto read = [&](int i) -> uint32_t {
      const int block = i * EV_WAVES + wave_s, t = block * CB_TOKENS + lane;
      if (block * CB_TOKENS >= len) return 0u;      // 0: no token; every token has a larger key
      const int id = c.table[row * c.width + block];
      const bool there = id >= 0 && id < c.blocks;
      const uint32_t k = float_to_ordered(c.weight[((size_t)(there ? id : 0) * c.hb + hh) * CB_TOKENS + lane]);
      const uint32_t key = t < a.keep_first || t >= len - a.keep_last ? EV_FORCED : there ? max(k, 1u) : EV_ABSENT;
      return t < len ? key : 0u;
    };
    uint32_t key[KPT];
    const auto load = [&](int part) {
#pragma unroll
      for (int i = 0; i < KPT; ++i) key[i] = read(part * KPT + i);
    };
    const int parts = LOOP ? (len + EV_THREADS * KPT - 1) / (EV_THREADS * KPT) : 1;
    if (!LOOP) load(0);

    // ---- the keep-th largest key, digit by digit ----
    uint32_t prefix = 0, mask = 0, left = keep;     // left: to be taken among the keys that match prefix
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
      for (int i = tid; i < EV_BINS; i += EV_THREADS) hist[i] = 0;
      __syncthreads();
      const auto count = [&](uint32_t k) {
        if (pass == 0 ? k != 0 : (k & mask) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
      };
      for (int s = 0; s < parts; ++s) {
        if (LOOP) load(s);
#pragma unroll
        for (int i = 0; i < KPT; ++i) count(key[i]);
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
    // base: keys above and equal to the threshold in front of the wave's 64 tokens
    const auto put = [&](int t, uint32_t k, uint32_t above, uint32_t equal) {
      const bool gt = k > prefix;
      const uint64_t bg = __ballot(gt), be = __ballot(k == prefix);
      above = __builtin_amdgcn_mbcnt_hi((uint32_t)(bg >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bg, above));
      bool take = gt;
      if (be) {                                     // uniform: the few waves that hold the threshold itself
        equal = __builtin_amdgcn_mbcnt_hi((uint32_t)(be >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)be, equal));
        take = gt || (k == prefix && equal < left);
      }
      const uint32_t at = above + min(equal, left);
      if (take && at < (uint32_t)keep) list[at] = t;
    };
    uint32_t above = 0, equal = 0;                  // of all earlier parts
    for (int s = 0; s < parts; ++s) {
      if (LOOP) load(s);
#pragma unroll
      for (int i = 0; i < KPT; ++i) {
        const uint64_t gt = __ballot(key[i] > prefix), eq = __ballot(key[i] == prefix);
        if (lane == 0) counts[i * EV_WAVES + wave] = __popcll(gt) | __popcll(eq) << 16;
      }
      __syncthreads();
      if (wave == 0) {                              // exclusive sums over KPT * 16 entries, KPT / 4 per lane
        constexpr int PER = KPT / 4;
        uint32_t mine[PER], incl = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) { mine[i] = counts[lane * PER + i]; incl += mine[i]; }
        uint32_t run = incl;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
          const uint32_t o = __shfl_up(incl, off);
          if (lane >= off) incl += o;
        }
        if (lane == 63) counts[KPT * EV_WAVES] = incl;
        run = incl - run;
#pragma unroll
        for (int i = 0; i < PER; ++i) { counts[lane * PER + i] = run; run += mine[i]; }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < KPT; ++i) {
        const uint32_t base = counts[i * EV_WAVES + wave];
        put((s * KPT + i) * EV_THREADS + tid, key[i], above + (base & 0xffff), equal + (base >> 16));
      }
      if (LOOP) {
        above += counts[KPT * EV_WAVES] & 0xffff;
        equal += counts[KPT * EV_WAVES] >> 16;
        __syncthreads();                            // counts are free for the next part
      }
    }
    __syncthreads();                                // shared memory is free for the next head
  }
}

// One workgroup per block that is written, of one wave per 64 dimensions; K and V in launches of their
// own (in one they share the registers of the larger: 1504 us instead of 367 + 601 for 105k blocks of
// 64 x 128 int8 at half of their rows).  Every lane = token of the block first finds out where its token lies and
// under which scale.
//
// K: a row of d bytes per token, moved as 16-byte pieces that stay in registers until the new scale is known.
// V lies dimension by dimension: a token of it is a column of bytes.  A source block comes in whole, in lines,
// and turns in LDS so that a lane holds the 64 bytes of one dimension.  Which of them stay is a scalar: two
// v_perm per word put its kept bytes behind those that wait for a full word, which goes to the lane's
// row in LDS.  (Measured on 105k blocks of 128 x 64, V alone: a byte at a time from source blocks in LDS
// 1858 us; a branch per token 1344; the 64 bytes of a lane loaded by the lane itself, in pieces 64 bytes apart
// over the wave, 1363.)  Rows whose scale the new block keeps are copied; only the others are decoded and rounded
// again.
constexpr int EM_STAGE = CB_TOKENS * 64;            // bytes of a wave's 64 dimensions of a source block
constexpr int EM_ROW = CB_TOKENS / 4 + 1;           // words of a row that is written: 64 lanes lie in 64 different banks
constexpr int EM_WAVE_LDS = EM_STAGE + 64 * EM_ROW * 4;

__device__ __forceinline__ float move_max(float x, float* red, int waves) {
  x = wave_max(x);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  for (int i = 0; i < waves; ++i) x = fmaxf(x, red[i]);
  return x;
}

// old over new scale: a code that is not 0 has at most 2^18 of it, a larger one belongs to a row of zeros
__device__ __forceinline__ float move_ratio(float old_scale, float inverse) { return fminf(old_scale * inverse, EM_RATIO); }

template <int FMT>
__device__ __forceinline__ float largest_code(uint32_t w, float most) {
  float x[4];
  Code<FMT>::decode(w, x);
  return fmaxf(fmaxf(fmaxf(fmaxf(most, fabsf(x[0])), fabsf(x[1])), fabsf(x[2])), fabsf(x[3]));
}
template <int FMT>
__device__ __forceinline__ uint32_t rescale(uint32_t w, float a, float b, float c, float d) {
  float x[4];
  asm("" : "+v"(w));                                // else the numbers of the maximum are kept in registers until here
  Code<FMT>::decode(w, x);
  return Code<FMT>::encode(x[0] * a, x[1] * b, x[2] * c, x[3] * d);
}
__device__ __forceinline__ float lane_float(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane));
}

// blockDim: 64 * waves, waves = d / 64 rounded up.  magic: 65536 / (d / 16) rounded up.  VALUES: V, else K.
// Bound by HBM: K 5.0 TB/s, V 4.8 TB/s of the bytes that it moves, which are those of every source block that
// a kept token lies in, and of no other: 64 tokens at the two ends of 131072 (32 rows of 8 heads) take 398 us, most of it the
// selection, and 2150 if every block between them is walked over.
template <int FMT, bool VALUES>
__global__ __launch_bounds__(EM_THREADS) void evict_move(EvictArgs a, int blocks, int64_t units, uint32_t magic) {
  extern __shared__ __align__(16) uint8_t smem[];   // EM_WAVE_LDS per wave
  __shared__ float red[EM_THREADS / 64];
  const CacheView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, d = c.d, pieces = d / 16, waves = blockDim.x / 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // workgroups go to the eight chiplets in turn: each is given EM_STRETCH neighbours, which share source blocks
  // of V, at a time
  constexpr int EM_STRETCH = 32;
  for (int64_t x = blockIdx.x; x < (units + 8 * EM_STRETCH - 1) / (8 * EM_STRETCH) * (8 * EM_STRETCH); x += gridDim.x) {
    const int in = (int)(x & (8 * EM_STRETCH - 1));
    const int64_t w = x - in + (in & 7) * EM_STRETCH + (in >> 3);
    if (w >= units) continue;
    const int64_t head = w / blocks;
    const int j = (int)(w - head * blocks);
    const int64_t row = head / c.hb;
    const int hh = (int)(head - row * c.hb);
    const int keep = kept_tokens(a, row, cache_length(c, a.lengths[row]));
    if (j * CB_TOKENS >= keep) continue;            // uniform
    const int to = a.table_out[row * c.width + j];
    if (to < 0 || to >= c.blocks) continue;
    const int here = min(keep - j * CB_TOKENS, CB_TOKENS);
    const int32_t* ids = c.table + row * c.width;
    const size_t at = (size_t)to * c.hb + hh;

    // lane = token, the same in every wave; scale 0: not there
    int page = 1 << 30, slot = 0, id = -1;
    float old_scale = 0.f, weight = 0.f;
    if (lane < here) {
      const int p = a.list[head * a.lpad + j * CB_TOKENS + lane];
      page = p / CB_TOKENS;
      slot = p % CB_TOKENS;
      id = ids[page];
      if (id >= c.blocks) id = -1;
      if (id >= 0) {
        const size_t from = (size_t)id * c.hb + hh;
        old_scale = (VALUES ? c.v_scale : c.k_scale)[from];
        if (VALUES && wave == 0) weight = c.weight[from * CB_TOKENS + slot];
      }
    }

    if constexpr (!VALUES) {
      u32x4_t kw[4];
      float kf[4], most = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = i * blockDim.x + tid;
        const int token = min((int)(e * magic >> 16), CB_TOKENS - 1), piece = e - token * pieces;
        const int from_id = __shfl(id, token), from_slot = __shfl(slot, token);
        kf[i] = __shfl(old_scale, token);
        kw[i] = u32x4_t{0, 0, 0, 0};
        if (e < CB_TOKENS * pieces && from_id >= 0)
          kw[i] = *reinterpret_cast<const u32x4_t*>(c.k + (((size_t)from_id * c.hb + hh) * CB_TOKENS + from_slot) * d + piece * 16);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float code = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) code = largest_code<FMT>(kw[i][q], code);
        most = fmaxf(most, code * kf[i]);
      }
      const float scale = block_scale<FMT>(move_max(most, red, waves)), inv = inverse_scale(scale);
      uint8_t* ko = c.k + at * CB_TOKENS * d;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = i * blockDim.x + tid;
        if (__ballot(kf[i] != scale)) {
          const float f = move_ratio(kf[i], inv);
#pragma unroll
          for (int q = 0; q < 4; ++q) kw[i][q] = rescale<FMT>(kw[i][q], f, f, f, f);
        }
        if (e < CB_TOKENS * pieces) __builtin_nontemporal_store(kw[i], reinterpret_cast<u32x4_t*>(ko + (size_t)e * 16));
      }
      if (tid == 0) c.k_scale[at] = scale;
    } else {
      if (wave == 0) c.weight[at * CB_TOKENS + lane] = weight;
      uint8_t* stage = smem + wave * EM_WAVE_LDS;
      uint32_t* rows = reinterpret_cast<uint32_t*>(stage + EM_STAGE);
      // in lines: lane = (dimension 16 n + r4, tokens 16 piece .. + 15); rows past d repeat the last one
      const int piece = lane & 3, r4 = lane >> 2;
      u32x4_t next[4];
      const auto load = [&](int page_of) {
        const int from_id = ids[page_of];
#pragma unroll
        for (int n = 0; n < 4; ++n) next[n] = u32x4_t{0, 0, 0, 0};
        if (from_id >= 0 && from_id < c.blocks)
#pragma unroll
          for (int n = 0; n < 4; ++n)
            next[n] = *reinterpret_cast<const u32x4_t*>(
                c.v + (((size_t)from_id * c.hb + hh) * d + min(64 * wave + 16 * n + r4, d - 1)) * CB_TOKENS + 16 * piece);
      };
      load(__builtin_amdgcn_readfirstlane(page));
      int done = 0;                                 // tokens of earlier source blocks; token `done` lies in the next one
      uint32_t acc = 0;                             // bytes that wait for a full word
      while (done < here) {                         // uniform; the next four source blocks that hold a kept token
        // which slots of a block stay: every kept token raises the flag of the lane of its slot
        uint64_t mine = 0;
        int before = done;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int now = done < here ? __builtin_amdgcn_readlane(page, done) : -1;
          const bool from_here = page == now;
          const int flag = __builtin_amdgcn_ds_permute((from_here ? slot : 0) * 4, from_here ? 1 : 0);
          // lanes without a token of this block push 0 to lane 0, which may win over a flag there
          const uint64_t stay = (__ballot(flag) & ~1ull) | (__ballot(from_here && slot == 0) ? 1ull : 0ull);
          if (lane >> 4 == g) { mine = stay; before = done; }
          done += __popcll(stay);
        }
        // lane 16 g + i: word i of block g of the four.  Its n kept bytes follow f that wait.
        const int word = lane & 15;
        const uint32_t m4 = (uint32_t)(mine >> (4 * word)) & 15u;
        uint32_t order = 0, n8 = 0;                 // the kept bytes' numbers, 8 n
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          order |= (m4 >> e & 1) ? (uint32_t)e << n8 : 0u;
          n8 += (m4 >> e & 1) * 8;
        }
        order += 0x04040404u;                       // as selectors: 4 + number, 0..3 are the waiting bytes
        const int place = before + __popcll(mine & ((1ull << (4 * word)) - 1));
        const uint32_t f8 = (place & 3) * 8;
        const uint32_t fill = (0x03020100u & ((1u << f8) - 1)) | order << f8;
        const uint32_t rest = f8 + n8 < 32 ? fill : f8 ? order >> (32 - f8) : 0u;
        const int at_word = place >> 2;
#pragma unroll 1
        for (int g = 0; g < 4; ++g) {
          if (__builtin_amdgcn_readlane(before, 16 * g) >= here) break;   // no such block
          const int next_token = g < 3 ? __builtin_amdgcn_readlane(before, 16 * g + 16) : done;
#pragma unroll
          for (int n = 0; n < 4; ++n)               // pieces change places so that the reads below meet no bank twice
            *reinterpret_cast<u32x4_t*>(stage + (16 * n + r4) * 64 + ((piece ^ (r4 >> 2 & 3)) << 4)) = next[n];
          if (next_token < here) load(__builtin_amdgcn_readlane(page, next_token));
          u32x4_t x[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) x[q] = *reinterpret_cast<const u32x4_t*>(stage + lane * 64 + ((q ^ (lane >> 2 & 3)) << 4));
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t s_fill = __builtin_amdgcn_readlane(fill, 16 * g + i);
            const uint32_t s_rest = __builtin_amdgcn_readlane(rest, 16 * g + i);
            const int s_word = __builtin_amdgcn_readlane(at_word, 16 * g + i);
            rows[lane * EM_ROW + s_word] = __builtin_amdgcn_perm(x[i / 4][i % 4], acc, s_fill);   // word 16 is padding
            acc = __builtin_amdgcn_perm(x[i / 4][i % 4], acc, s_rest);
          }
        }
      }
      // bytes that the last word of all left waiting
      if (done & 3) rows[lane * EM_ROW + (done >> 2)] = acc;
      u32x4_t out[4];                               // in lines again
      const int left = here - 16 * piece;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int of_word = left - 4 * q;
          out[n][q] = rows[(16 * n + r4) * EM_ROW + 4 * piece + q] &
                      (of_word >= 4 ? ~0u : of_word <= 0 ? 0u : (1u << (8 * of_word)) - 1);
        }
      const float first_scale = lane_float(old_scale, 0);
      const bool alike = __ballot(lane < here && old_scale != first_scale) == 0;
      float most = 0.f;
      if (alike) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int q = 0; q < 4; ++q) most = largest_code<FMT>(out[n][q], most);
        most *= first_scale;
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float s[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] = __shfl(old_scale, 16 * piece + 4 * q + e);
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            float y[4];
            Code<FMT>::decode(out[n][q], y);
#pragma unroll
            for (int e = 0; e < 4; ++e) most = fmaxf(most, fabsf(y[e]) * s[e]);
          }
        }
      }
      const float scale = block_scale<FMT>(move_max(most, red, waves));
      if (__ballot(lane < here && old_scale != scale)) {
        const float ratio = move_ratio(old_scale, inverse_scale(scale));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float s[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] = __shfl(ratio, 16 * piece + 4 * q + e);
#pragma unroll
          for (int n = 0; n < 4; ++n) out[n][q] = rescale<FMT>(out[n][q], s[0], s[1], s[2], s[3]);
        }
      }
      uint8_t* vo = c.v + at * d * CB_TOKENS;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int dim = 64 * wave + 16 * n + r4;
        if (dim < d) __builtin_nontemporal_store(out[n], reinterpret_cast<u32x4_t*>(vo + dim * CB_TOKENS + 16 * piece));
      }
      if (tid == 0) c.v_scale[at] = scale;
    }
    __syncthreads();                                // red is free for the next block
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
#define KVC_SELECT(KPT, LOOP) \
  KVC_LAUNCH("evict_select", stream, evict_select<KPT, LOOP><<<grid, EV_THREADS, 0, stream>>>(a))
  if (longest <= 4 * EV_THREADS) KVC_SELECT(4, false);
  else if (longest <= 16 * EV_THREADS) KVC_SELECT(16, false);
  else if (longest <= 32 * EV_THREADS) KVC_SELECT(32, false);
  else KVC_SELECT(16, true);
#undef KVC_SELECT
  if (max_keep == 0) return KVC_OK;
  const int blocks = a.lpad / CB_TOKENS;
  const int64_t units = a.heads * blocks;
  const unsigned move = (unsigned)std::min<int64_t>((units + 255) / 256 * 256, 1 << 20);
  const int threads = (pb.d + 63) / 64 * 64;
  const uint32_t magic = (65536 + pb.d / 16 - 1) / (pb.d / 16);   // e / (d / 16) = e * magic >> 16 for e < 1024 and d <= 256
#define KVC_MOVE(FMT)                                                                                                     \
  do {                                                                                                                    \
    KVC_LAUNCH("evict_move<k>", stream, evict_move<FMT, false><<<move, threads, 0, stream>>>(a, blocks, units, magic));   \
    KVC_LAUNCH("evict_move<v>", stream, evict_move<FMT, true><<<move, threads, threads / 64 * EM_WAVE_LDS, stream>>>(     \
        a, blocks, units, magic));                                                                                        \
  } while (0)
  if (format == KVC_E4M3) KVC_MOVE(KVC_E4M3); else KVC_MOVE(KVC_INT8);
#undef KVC_MOVE
  return KVC_OK;
}

}  // namespace kvc
