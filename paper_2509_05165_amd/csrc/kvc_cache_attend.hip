// kvc_cache_attend: attention of M query tokens over the 8-bit block cache.
//
// Mathematics, per (sequence, KV head), rows r = (g, m) of the G query heads that share it:
//   s[r,c] = scale * ks(block of c) * sum_d q[r,d] kc[c,d]        kc, vc: codes as numbers
//   p[r,c] = 2^(s log2e - ref)                                      one pass, running reference and sum
//   out[r,:] = sum_c p[r,c] vs(block) vc[c,:] / sum_c p[r,c]
// Codes of both formats are bf16 numbers exactly, so both products run on the bf16 matrix cores with
// fp32 accumulation; the scales are applied to the fp32 logits and to the fp32 probabilities
// (exactly, they are powers of two).  For the second product bf16 calls round the probabilities to two bf16
// terms, 16 bits, so that only the output's own rounding counts; float32 calls split queries and probabilities
// into three terms each, 24 bits.
//
// Layout: v_mfma_f32_16x16x32_bf16 with tokens on the rows and queries on the columns of the first
// product.  A wave takes a block of 64 tokens as four tiles; tile t holds the tokens 16*g + 4*t + i
// (g, i: the lane group and register of the result), so that a lane ends up with the probabilities
// of the 16 consecutive tokens of its group, in the order in which the second product wants them as
// its operand, and with one query: the softmax needs two cross-lane steps per block and the probabilities
// none.  The other operand, V transposed, is 16 consecutive bytes of a dimension's row of the block.
// Codes and probabilities never go through LDS: the queries of some forms do (Q_LDS), logits that a workgroup keeps for
// the weights of its row (kept), and what the four waves join.
//
// Work is split over the tokens: a workgroup takes `chunk` blocks of one head (its waves every fourth
// one); attend_join adds the splits of a row and, where weights are gathered, turns the stored
// logits into probabilities once the sum over all tokens is known.
#include <algorithm>
#include <cmath>

#include "kvc_cache.h"

namespace kvc {

namespace {

constexpr int CA_THREADS = 256;
constexpr int CA_WAVES = CA_THREADS / 64;
constexpr int CA_CHUNK_MOST = 64;                   // blocks of a workgroup, see attend_plan
// A reference further than this below the largest logit is moved up (log2 units): sums stay below
// 2^8 * 2^30 and rescaling is rare.
constexpr float CA_SLACK = 8.0f;
// The scale of V goes into the exponential of the probabilities, which costs nothing, as long as it lies between these:
// at 2^-60 numbers stay normal down to p = 2^-66, so that the sum of a row misses nothing whatever its values; a
// block of zeros has the scale 2^-100, where all p below 2^-26 would be missing.  What is left of a smaller or larger
// scale multiplies the operand of the product with V alone (always multiplying there: 64 x 8k..16k tokens, heads of 64,
// 8 query tokens 223 us instead of 204).
constexpr float CA_EXP_LEAST = 0x1p-60f, CA_EXP_MOST = 0x1p60f;

struct AttendArgs {
  const void* q;
  void* out;
  float* lse;               // may be null
  const int32_t* lengths;
  float* part_o;            // [batch * hkv * rows, splits, d]
  float2* part_ml;          // [batch * hkv * rows, splits]: reference, sum
  float* logits;            // [batch * hkv, lblocks, rows, 64] in log2 units, or null
  int kept, kept_blocks;    // where in LDS a workgroup that takes whole rows keeps those of its first blocks (0: nowhere)
  const float* weight_in;   // may be null
  float* weight_out;        // may be null
  CacheView c;
  int layer, group, window, rows, row_chunks, splits, chunk, max_length, lblocks, causal;
  float scale_log2;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Both halves / all four rows of 16 lanes see the combined value of lanes l, l^16, l^32, l^48.
__device__ __forceinline__ float across_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float across_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Eight floats as TERMS bf16 vectors whose sum they are (to 8 bits a term).
template <int TERMS>
__device__ __forceinline__ void split_terms(const float (&x)[8], bf16x8_t (&t)[TERMS]) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
  for (int n = 0; n < TERMS; ++n)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      t[n][i] = (__bf16)rest[i];
      if (n + 1 < TERMS) rest[i] -= (float)t[n][i];
    }
}

template <typename T> struct Store4;
template <> struct Store4<float> {
  static __device__ __forceinline__ void put(float* p, f32x4_t x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = x[i];
  }
};
template <> struct Store4<uint16_t> {
  static __device__ __forceinline__ void put(uint16_t* p, f32x4_t x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = __builtin_bit_cast(uint16_t, (__bf16)x[i]);
  }
};

// Waves per SIMD that the registers of a form are held to: one block of K and V (32 registers per 64
// dimensions), the queries and the output have to fit.  More waves would not help (they only spread the
// loads over more of the pool): 128 dimensions, bf16, 1 x 128k tokens of 8 heads 55.9 us with two, 67.8
// with three (and a few spilled registers).
constexpr int attend_waves(int nj, int qt, int esz) {
  return esz == 2 ? (nj == 1 && qt == 1 ? 3 : nj <= 3 ? 2 : 1) : (nj <= 2 && qt == 1 ? 2 : 1);
}

// 16 bytes of codes.  Codes that one workgroup alone reads carry the streaming hint (with whole lines,
// see PAIRED): 16 x 400..13000 tokens of 8 heads 47.6 us without, 39.2 with; 1 x 128k 55.9 / 48.2.
template <bool STREAM>
__device__ __forceinline__ u32x4_t load16(const uint8_t* p) {
  const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p);
  return STREAM ? __builtin_nontemporal_load(q) : *q;
}
constexpr int DPP_ROR8 = 0x128;                     // rotate rows of 16 lanes by eight

// Logits of the query rows 4 M .. 4 M + 3 of a tile, times ks.  Lane 4 M + i of 16 holds all 16 tokens of row i, so
// that storing them as they lie would be four stores by four lanes, in pieces of 16 bytes; turned among the
// 16 lanes they are one store, 64 bytes to a row: lane c stores tokens 4 (c / 4) .. + 3 of row c % 4.
// (64 x 8k..16k tokens of 8 heads with weights: 369 us as they lie, 355 turned.)
template <int M, int TILE>
__device__ __forceinline__ float turned(float old, float x) {   // x of lane c - 4 (TILE - M), where c / 4 == TILE
  constexpr int by = 4 * ((TILE - M) & 3);
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(old), (int)__float_as_uint(x),
                                                              by ? 0x120 + by : 0xe4, 0xf, 1 << TILE, false));
}
template <int M>
__device__ __forceinline__ void store_rows(float* to, const f32x4_t (&s)[4], float ks, int rows, int col) {
  if (4 * M >= rows) return;                        // uniform
  f32x4_t y;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float x = turned<M, 0>(0.f, s[0][e]);
    x = turned<M, 1>(x, s[1][e]);
    x = turned<M, 2>(x, s[2][e]);
    y[e] = turned<M, 3>(x, s[3][e]) * ks;
  }
  const int r = 4 * M + (col & 3);
  if (r < rows) *reinterpret_cast<f32x4_t*>(to + r * CB_TOKENS + 4 * (col >> 2)) = y;
}

// Tokens of the row that this call reads.
__device__ __forceinline__ int attend_length(const AttendArgs& a, int64_t row) {
  return min(cache_length(a.c, a.lengths[row]), a.max_length);
}

// weight_out = weight_in + gained for four tokens of a block; those of a block that is not there have no weight.
__device__ __forceinline__ void add_weights(const AttendArgs& a, int64_t row, int hh, int token, int len, f32x4_t gained) {
  const CacheView& c = a.c;
  const int id = c.table[row * c.width + token / CB_TOKENS];
  if (id < 0 || id >= c.blocks) return;
  const size_t at = ((size_t)id * c.hb + hh) * CB_TOKENS + token % CB_TOKENS;
  if (token + 4 <= len) {
    u32x4_word w{0, 0, 0, 0}, y;
    if (a.weight_in) w = *reinterpret_cast<const u32x4_word*>(a.weight_in + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = __float_as_uint(__uint_as_float(w[e]) + gained[e]);
    *reinterpret_cast<u32x4_word*>(a.weight_out + at) = y;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (token + e < len) a.weight_out[at + e] = (a.weight_in ? a.weight_in[at + e] : 0.f) + gained[e];
  }
}

// NJ: groups of 64 dimensions, d = 64 * NJ where EXACT; QT: tiles of 16 query rows per workgroup.
// grid: (splits * row_chunks * hkv, 1, batch), the head fastest: with 8 heads all row chunks of a head
// run on the same chiplet and share its L2.
//
// Bound by HBM: 2 * 64 * d bytes of codes per block and head.  A wave keeps one block of K and one of V
// in flight: the next block's K is asked for as soon as this block's logits are there, the next V as soon
// as this block's output is.
template <int FMT, typename T, int NJ, bool EXACT, int QT, bool STREAM>
__global__ __launch_bounds__(CA_THREADS, attend_waves(NJ, QT, sizeof(T))) void attend_split(AttendArgs a) {
  // Terms of the queries and of the probabilities.  bf16 calls: queries are one term, probabilities two whatever the
  // shape (16 bits; output error against float64 1.7e-3, its own rounding; 2.4e-3 with one).  That is free where the codes
  // bound the kernel (64 x 16k tokens, 32/8 heads 335.9 us with one, 338.7 with two) and costs where 32 rows share them:
  // 64 x 8k..16k tokens 357 / 372 with 8 query tokens, 16 x 8k..16k 395 / 469 with 64.
  constexpr int TERMS = sizeof(T) == 2 ? 1 : 3, PTERMS = sizeof(T) == 2 ? 2 : 3;
  constexpr int NT = 4 * NJ;                        // tiles of 16 dimensions
  // bf16 queries lie in LDS where they would make registers spill: two tiles of them (26 spilled; 8 query tokens, as above:
  // 416 us), where the waves join their results later (17 rows or more of d floats from every wave are room enough),
  // and those of d = 144 to 176 (12 spilled), in LDS of their own.
  constexpr bool Q_LDS = sizeof(T) == 2 && (QT == 2 || (NJ == 3 && !EXACT));
  extern __shared__ __align__(16) float lds[];      // [waves][nq][d], nq = query rows of this workgroup; at kept [kept_blocks][nq][64]
  __shared__ float sm[CA_WAVES][16 * QT], sl[CA_WAVES][16 * QT], lse2[16 * QT];
  const CacheView& c = a.c;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int d = EXACT ? 64 * NJ : c.d, b = blockIdx.z;
  const int x = blockIdx.x / c.hkv, h = blockIdx.x - x * c.hkv;
  const int split = x / a.row_chunks, rc = x - split * a.row_chunks;
  const int64_t row = cache_row(c, b, a.layer, h);
  const int hh = cache_head(c, h);
  const int lo = split * a.chunk, first_block = lo + __builtin_amdgcn_readfirstlane(wave);
  // The blocks of this wave, one per lane (asked for before the length is known): ids and scales.
  // (a chunk has at most 64 * CA_WAVES blocks)
  const int my_block = first_block + CA_WAVES * lane;
  int my_id = c.table[row * c.width + min(my_block, c.width - 1)];
  const int whole_len = cache_length(c, a.lengths[row]), len = min(whole_len, a.max_length);
  const int nb = (len + CB_TOKENS - 1) / CB_TOKENS;
  const int hi = min(lo + a.chunk, nb);
  if (split > 0 && lo >= nb) return;                // attend_join knows that this split is empty
  if (my_block >= hi || my_id >= c.blocks) my_id = -1;
  const size_t my_scale = (size_t)max(my_id, 0) * c.hb + hh;
  // (an entry that names no block: block 0 is loaded in its place, whatever it holds, and masked; 1 as its scales)
  const float my_ks = my_id < 0 ? 1.0f : c.k_scale[my_scale], my_vs = my_id < 0 ? 1.0f : c.v_scale[my_scale];
  const auto lane_of = [](float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); };
  const int r0 = rc * 16 * QT, nq = min(a.rows - r0, 16 * QT);
  const int64_t out_row = ((int64_t)b * c.hkv + h) * a.rows + r0;

  // Offsets inside a block: K row of tile 0, V row of tile 0.  Pieces past d repeat ones that are there
  // (their queries are zero, their results are not stored).
  // PAIRED: a load takes whole lines of 128 bytes of eight rows instead of half lines of sixteen, the second
  // one the other eight rows; exchanging the upper and lower lanes of the two gives the operands (operand()).
  constexpr bool PAIRED = EXACT && NJ % 2 == 0;
  uint32_t k_off[NJ], v_off[NT];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int piece = 64 * j + 16 * g;
    if (PAIRED) k_off[j] = (16 * (col >> 2 & 1) + (col & 3) + 32 * (j & 1)) * d + 128 * (j >> 1) + 64 * (col >> 3) + 16 * g;
    else k_off[j] = (16 * (col >> 2) + (col & 3)) * d + (EXACT || piece < d ? piece : 0);
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) v_off[n] = (EXACT ? 16 * n : min(16 * n, d - 16)) * CB_TOKENS + col * CB_TOKENS + 16 * g;
  const uint32_t block_bytes = CB_TOKENS * d;
  u32x4_t kw[4][NJ], vw[NT];
  const auto load_k = [&](int id) {                 // an entry that names no block: any block, masked below
    const uint8_t* kb = c.k + ((size_t)max(id, 0) * c.hb + hh) * block_bytes;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < NJ; ++j) kw[t][j] = load16<STREAM && (PAIRED || NJ == 1)>(kb + k_off[j] + uint32_t(4 * t * d));
  };
  const auto load_v = [&](int id) {
    const uint8_t* vb = c.v + ((size_t)max(id, 0) * c.hb + hh) * block_bytes;
#pragma unroll
    for (int n = 0; n < NT; ++n) vw[n] = load16<STREAM>(vb + v_off[n]);
  };
  // word w of the 16 bytes of tile t and dimensions 64 j + 16 g
  const auto operand = [&](int t, int j, int w) -> uint32_t {
    if (!PAIRED) return kw[t][j][w];
    const int even = (int)kw[t][j & ~1][w], odd = (int)kw[t][j | 1][w];
    return (uint32_t)(j & 1 ? __builtin_amdgcn_update_dpp(odd, even, DPP_ROR8, 0xf, 0x3, false)
                            : __builtin_amdgcn_update_dpp(even, odd, DPP_ROR8, 0xf, 0xc, false));
  };
  if (first_block < hi) {
    const int id = __builtin_amdgcn_readfirstlane(my_id);
    load_k(id);
    load_v(id);
  }

  // ---- queries: lane col holds row col, dimensions 64 j + 16 g + 8 half (q_lds: its own 16 bytes of every piece) ----
  bf16x8_t q[QT][NJ][2][TERMS];
  __shared__ u32x4_t q_own[Q_LDS && QT == 1 ? 2 * NJ * 64 : 1];
  u32x4_t* const q_lds = (QT == 1 ? q_own : reinterpret_cast<u32x4_t*>(lds)) + lane;
  int limit[QT];                                    // tokens that the lane's query sees (of them, those below len are read)
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = t * 16 + col;
    limit[t] = a.causal && r < nq ? whole_len - (a.window - 1 - (r0 + r) % a.window) : len;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int at = 64 * j + 16 * g + 8 * half;
        Row8<T> w;
        w.clear();
        if (r < nq && at < d) w.load(static_cast<const T*>(a.q) + (out_row + r) * d + at);
        float f[8];
        w.get(f);
        split_terms<TERMS>(f, q[t][j][half]);
        const int piece = (t * NJ + j) * 2 + half;  // the waves hold the same queries: each stores some
        if (Q_LDS && piece % CA_WAVES == wave) q_lds[piece * 64] = __builtin_bit_cast(u32x4_t, q[t][j][half][0]);
      }
  }
  if (Q_LDS) __syncthreads();

  f32x4_t o[QT][NT];
  float ref[QT], sum[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    ref[t] = -INFINITY;
    sum[t] = 0.f;
#pragma unroll
    for (int n = 0; n < NT; ++n) o[t][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  int it = 0;
  for (int p = first_block; p < hi; p += CA_WAVES, ++it) {
    const int id = __builtin_amdgcn_readlane(my_id, it);
    // (a scale that is too small for a normal number gives logits of 0, and -infinity stays what it is)
    const float ks = fmaxf(lane_of(my_ks, it) * a.scale_log2, 1.17549435e-38f), vs = lane_of(my_vs, it);
    const bool more = p + CA_WAVES < hi;
    const int next = __builtin_amdgcn_readlane(my_id, (it + 1) & 63);

    // ---- logits ----
    f32x4_t s[QT][4];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt)
#pragma unroll
      for (int t = 0; t < 4; ++t) s[qt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bf16x8_t qf[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
          if (Q_LDS) qf[qt] = __builtin_bit_cast(bf16x8_t, q_lds[((qt * NJ + j) * 2 + half) * 64]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const bf16x8_t kf = Code<FMT>::widen(operand(t, j, 2 * half), operand(t, j, 2 * half + 1));
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int n = TERMS - 1; n >= 0; --n)
              s[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, Q_LDS ? qf[qt] : q[qt][j][half][n], s[qt][t], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);          // no more than one step's widened codes in registers
      }
    if (more) load_k(next);
    const int here = id < 0 ? 0 : len;              // tokens of an absent block are masked like those past the end
    const int first = p * CB_TOKENS + 16 * g;       // the lane's 16 tokens
    const bool tail = (p + 1) * CB_TOKENS > here - (a.causal ? a.window - 1 : 0);   // wave-uniform
    const float in_exp = fminf(fmaxf(vs, CA_EXP_LEAST), CA_EXP_MOST);   // of vs, what the exponential takes
    const float shift = __builtin_amdgcn_logf(in_exp);   // whole: a power of two
    const float inv_exp = inverse_scale(in_exp);
    bf16x8_t pf[QT][2][PTERMS];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      if (tail) {
        const int seen = min(limit[qt], here);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[qt][t][i] = first + 4 * t + i < seen ? s[qt][t][i] : -INFINITY;
      }
      if (p < a.kept_blocks) {
        float* to = lds + a.kept + (size_t)((p - lo) * nq + qt * 16) * CB_TOKENS + 16 * g;
        store_rows<0>(to, s[qt], ks, nq - qt * 16, col);
        store_rows<1>(to, s[qt], ks, nq - qt * 16, col);
        store_rows<2>(to, s[qt], ks, nq - qt * 16, col);
        store_rows<3>(to, s[qt], ks, nq - qt * 16, col);
      } else if (a.logits) {
        float* to = a.logits + ((((size_t)b * c.hkv + h) * a.lblocks + p) * a.rows + r0 + qt * 16) * CB_TOKENS + 16 * g;
        store_rows<0>(to, s[qt], ks, nq - qt * 16, col);
        store_rows<1>(to, s[qt], ks, nq - qt * 16, col);
        store_rows<2>(to, s[qt], ks, nq - qt * 16, col);
        store_rows<3>(to, s[qt], ks, nq - qt * 16, col);
      }
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[qt][t][i]);
      top = across_max(top) * ks;                   // ks > 0
      if (__ballot(top > ref[qt] + CA_SLACK)) {
        const float to = fmaxf(ref[qt], top);
        const float f = ref[qt] == -INFINITY ? 0.f : exp2_fast(ref[qt] - to);   // 0: nothing summed yet
        ref[qt] = to;
        sum[qt] *= f;
#pragma unroll
        for (int n = 0; n < NT; ++n) o[qt][n] *= f;
      }
      // p * in_exp = 2^(s ks - ref + log2 in_exp); no token seen yet: 2^(-inf - 0) = 0
      const float base = shift - (ref[qt] == -INFINITY ? 0.f : ref[qt]);
      float pr[2][8], part = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = exp2_fast(fmaf(s[qt][t][i], ks, base));
          part += e;
          pr[t >> 1][4 * (t & 1) + i] = e;
        }
      sum[qt] = fmaf(part, inv_exp, sum[qt]);
      if (in_exp != vs)                             // uniform
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 8; ++i) pr[u][i] *= vs * inv_exp;
#pragma unroll
      for (int u = 0; u < 2; ++u) split_terms<PTERMS>(pr[u], pf[qt][u]);
    }
    // ---- values ----
    if ((p + 1) * CB_TOKENS > here) {               // slots behind the last token hold anything: no code 0 times NaN
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int left = here - first - 4 * w;      // tokens of this word that are there
        const uint32_t mask = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
        for (int n = 0; n < NT; ++n) vw[n][w] &= mask;
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const bf16x8_t vf = Code<FMT>::widen(vw[n][2 * u], vw[n][2 * u + 1]);
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int m = PTERMS - 1; m >= 0; --m)
            o[qt][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[qt][u][m], o[qt][n], 0, 0, 0);
        if (n % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
    if (more) load_v(next);
  }

  // ---- join the waves ----
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    sum[qt] = across_sum(sum[qt]);
    if (g == 0) { sm[wave][qt * 16 + col] = ref[qt]; sl[wave][qt * 16 + col] = sum[qt]; }
  }
  __syncthreads();
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int r = qt * 16 + col;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < CA_WAVES; ++w) top = fmaxf(top, sm[w][r]);
    const float f = ref[qt] == -INFINITY ? 0.f : exp2_fast(ref[qt] - top);
    if (r < nq)
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (16 * n < d) *reinterpret_cast<f32x4_t*>(lds + ((size_t)wave * nq + r) * d + 16 * n + 4 * g) = o[qt][n] * f;
  }
  __syncthreads();
  const bool whole = a.splits == 1;
  for (int e = tid; e < nq * d / 4; e += CA_THREADS) {
    const int r = e / (d / 4), at = (e - r * (d / 4)) * 4;
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < CA_WAVES; ++w) top = fmaxf(top, sm[w][r]);
#pragma unroll
    for (int w = 0; w < CA_WAVES; ++w) total += sm[w][r] == -INFINITY ? 0.f : sl[w][r] * exp2_fast(sm[w][r] - top);
    f32x4_t y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < CA_WAVES; ++w) y += *reinterpret_cast<const f32x4_t*>(lds + ((size_t)w * nq + r) * d + at);
    if (whole) {
      const float inv = total > 0.f ? 1.0f / total : 0.f;        // a query that sees no token: zeros
      Store4<T>::put(static_cast<T*>(a.out) + (out_row + r) * d + at, y * inv);
      if (at == 0 && a.lse) a.lse[out_row + r] = total > 0.f ? (top + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
    } else {
      *reinterpret_cast<f32x4_t*>(a.part_o + ((out_row + r) * a.splits + split) * d + at) = y;
    }
    if (at == 0) lse2[r] = total > 0.f ? top + __builtin_amdgcn_logf(total) : INFINITY;
    if (at == 0 && a.part_ml) a.part_ml[(out_row + r) * a.splits + split] = make_float2(top, total);
  }
  if (a.kept) {                                     // the logits of the whole row are this workgroup's: its weights too
    __syncthreads();
    for (int token = tid * 4; token < len; token += CA_THREADS * 4) {
      const int block = token / CB_TOKENS, in = token % CB_TOKENS;   // four tokens of one block
      f32x4_t gained{0.f, 0.f, 0.f, 0.f};
      // a query that sees no token adds nothing: 2^(-inf - inf)
      const auto add = [&](f32x4_t s, int r) {
        const float m = lse2[r];
#pragma unroll
        for (int e = 0; e < 4; ++e) gained[e] += exp2_fast(s[e] - m);
      };
      if (block < a.kept_blocks) {                  // wave-uniform but for the last wave that is in
        const float* from = lds + a.kept + block * nq * CB_TOKENS + in;
#pragma unroll 4
        for (int r = 0; r < nq; ++r) add(*reinterpret_cast<const f32x4_t*>(from + r * CB_TOKENS), r);
      } else {
        const float* from = a.logits + (((size_t)b * c.hkv + h) * a.lblocks + block) * a.rows * CB_TOKENS + in;
#pragma unroll 4
        for (int r = 0; r < nq; ++r) add(*reinterpret_cast<const f32x4_t*>(from + r * CB_TOKENS), r);
      }
      add_weights(a, row, hh, token, len, gained);
    }
  }
}

// Reference and sum of a row over its first n splits, by LANES neighbouring lanes.
template <int LANES>
__device__ __forceinline__ float2 join_sums(const float2* __restrict__ ml, int n, int lane) {
  float2 y = lane < n ? ml[lane] : make_float2(-INFINITY, 0.f);
  for (int s = lane + LANES; s < n; s += LANES) {
    const float2 x = ml[s];
    const float top = fmaxf(x.x, y.x);
    if (top > -INFINITY) y = make_float2(top, x.y * exp2_fast(x.x - top) + y.y * exp2_fast(y.x - top));
  }
  float top = y.x;
#pragma unroll
  for (int off = LANES / 2; off; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  float total = y.x == -INFINITY ? 0.f : y.y * exp2_fast(y.x - top);
#pragma unroll
  for (int off = LANES / 2; off; off >>= 1) total += __shfl_xor(total, off);
  return make_float2(top, total);
}

// The first `joins` workgroups add the splits of a query row each: groups of d / 4 lanes take every
// groups-th split, four dimensions a lane.  The others: CJ_TOKENS tokens of one head each, whose gathered
// weight grows by the probabilities of the head's rows; the logits of the next CJ_AHEAD rows are always
// in flight, the first ones while the log-sum-exps are worked out.
constexpr int CJ_ROWS = 64;                         // rows whose log-sum-exps are in LDS at a time
constexpr int CJ_TOKENS = CA_THREADS * 4;
constexpr int CJ_AHEAD = 4;
static_assert(CJ_ROWS % CJ_AHEAD == 0, "the rows ahead are those of the next turn");
template <typename T>
__global__ __launch_bounds__(CA_THREADS) void attend_join(AttendArgs a, int64_t joins, int weight_chunks) {
  __shared__ float lse2[CJ_ROWS];
  __shared__ __align__(16) float acc[CA_THREADS * 4];
  const CacheView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, d = c.d;
  if (blockIdx.x < joins) {
    const int64_t r = blockIdx.x;
    const int64_t bh = r / a.rows;
    const int b = (int)(bh / c.hkv), h = (int)(bh - (int64_t)b * c.hkv);
    const int nb = (attend_length(a, cache_row(c, b, a.layer, h)) + CB_TOKENS - 1) / CB_TOKENS;
    const int n = max((nb + a.chunk - 1) / a.chunk, 1);
    const float2* ml = a.part_ml + r * a.splits;
    const float2 all = join_sums<64>(ml, n, lane);
    const int wide = d / 4, groups = CA_THREADS / wide, group = tid / wide, at = (tid - group * wide) * 4;
    const float* from = a.part_o + r * a.splits * d + at;
    f32x4_t y{0.f, 0.f, 0.f, 0.f};
    if (group < groups)
#pragma unroll 4
      for (int s = group; s < n; s += groups) {
        const float m = ml[s].x;
        const f32x4_t o = *reinterpret_cast<const f32x4_t*>(from + (size_t)s * d);
        y += o * (m == -INFINITY ? 0.f : exp2_fast(m - all.x));
      }
    *reinterpret_cast<f32x4_t*>(acc + tid * 4) = y;
    __syncthreads();
    if (group == 0) {
      for (int i = 1; i < min(groups, n); ++i) y += *reinterpret_cast<const f32x4_t*>(acc + (i * wide + tid) * 4);
      const float inv = all.y > 0.f ? 1.0f / all.y : 0.f;
      Store4<T>::put(static_cast<T*>(a.out) + r * d + at, y * inv);
    }
    if (tid == 0 && a.lse) a.lse[r] = all.y > 0.f ? (all.x + __builtin_amdgcn_logf(all.y)) * 0.6931471805599453f : -INFINITY;
    return;
  }
  const int64_t w = blockIdx.x - joins;
  const int64_t bh = w / weight_chunks;
  const int chunk = (int)(w - bh * weight_chunks);
  const int b = (int)(bh / c.hkv), h = (int)(bh - (int64_t)b * c.hkv);
  const int64_t row = cache_row(c, b, a.layer, h);
  const int len = attend_length(a, row);
  if (chunk * CJ_TOKENS >= len) return;             // uniform
  const int token = chunk * CJ_TOKENS + tid * 4;    // four tokens of one block
  const int n = max(((len + CB_TOKENS - 1) / CB_TOKENS + a.chunk - 1) / a.chunk, 1);
  const int known = token < len ? token : 0;
  const float* from = a.logits + ((size_t)bh * a.lblocks + known / CB_TOKENS) * a.rows * CB_TOKENS + known % CB_TOKENS;
  f32x4_t s[CJ_AHEAD], gained{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < CJ_AHEAD; ++i) s[i] = *reinterpret_cast<const f32x4_t*>(from + min(i, a.rows - 1) * CB_TOKENS);
  for (int r0 = 0; r0 < a.rows; r0 += CJ_ROWS) {
    const int most = min(a.rows - r0, CJ_ROWS);
    for (int r = tid / 16; r < most; r += CA_THREADS / 16) {
      const float2 all = join_sums<16>(a.part_ml + (bh * a.rows + r0 + r) * a.splits, n, tid & 15);
      // a row that sees no token adds nothing: 2^(-inf - inf)
      if ((tid & 15) == 0) lse2[r] = all.y > 0.f ? all.x + __builtin_amdgcn_logf(all.y) : INFINITY;
    }
    __syncthreads();
    for (int r = 0; r < most; r += CJ_AHEAD) {
      f32x4_t now[CJ_AHEAD];
#pragma unroll
      for (int i = 0; i < CJ_AHEAD; ++i) now[i] = s[i];
      if (r0 + r + CJ_AHEAD < a.rows)
#pragma unroll
        for (int i = 0; i < CJ_AHEAD; ++i)
          s[i] = *reinterpret_cast<const f32x4_t*>(from + (size_t)min(r0 + r + CJ_AHEAD + i, a.rows - 1) * CB_TOKENS);
#pragma unroll
      for (int i = 0; i < CJ_AHEAD; ++i)
        if (r + i < most) {
          const float m = lse2[r + i];
#pragma unroll
          for (int e = 0; e < 4; ++e) gained[e] += exp2_fast(now[i][e] - m);
        }
    }
    __syncthreads();
  }
  if (token < len) add_weights(a, row, cache_head(c, h), token, len, gained);
}

// How a call is split.  Two workgroups run on a compute unit, 512 on the chip.  us per call, 32/8 heads of
// 128, e4m3, by blocks per workgroup (chunk):
//   one sequence: enough chunks to fill the chip once, at least a block per wave: 777 tokens 9.5 (4) 11.0 (8);
//     3000 10.3 (4) 11.9 (8); 8000 10.8 (4) 12.6 (8); 32000 19.0 (8) 21.4 (12); 128k, 64/8 heads 49.2 (32) 52.0 (16)
//   several: smaller ones, because lengths differ and nobody knows them here: 16 x 400..13000 46.5 (16) 52.3 (48);
//     8 x 2000 12.6 (8) 12.9 (4); 8 x 4000 17.8 (8) 19.1 (16); but from 128 heads on at least 16 blocks:
//     16 x 1000 13.3 (16) 14.3 (8)
//   512 heads and more: whole rows, up to 64 blocks, beyond which one long row among short ones would be
//     waited for: 64 x 1500 34.1 (24) 41.7 (12); 64 x 6000..12000 192 (whole) 196 (64); 256 x 400..800 59.4 (whole)
//     115 (4)
// With weights, a workgroup that has whole rows of a head gathers them too, from logits that it keeps in LDS beside
// what joins the waves, and where they do not fit, behind the first blocks', in the workspace, which it reads back while
// the next workgroup's codes come in; only rows that are split leave that to attend_join.  So from 256 heads on rows
// of up to 256 blocks stay whole (whole / split, us): 64 x 4000 tokens of 32/8 heads 91 / 115, of 64/8 heads (126 KB of
// logits, one workgroup to a compute unit) 116 / 131; 32 x 1500 26 / 33; 64 x 8000 218 / 231; 64 x 8192..16384 323 / 360
// (16 KB of LDS 364, 64 KB 342); 256 x 2800..14000 900 / 1135; 32 x 16384 206 / 229; but short rows only if all
// their logits fit: 256 x 100..1000 with 32 query rows to a head 203 / 158; and with 128 heads it does not pay: 16 x 4000
// 46 / 36.
// The workspace is that of the most splits that any shorter max_length asks for, with its logits.
constexpr int64_t CA_LDS = 152 << 10;               // of 160 KB
struct AttendPlan {
  int rows, qt, row_chunks, chunk, splits, lblocks;
  bool kept;                                        // a workgroup gathers the weights of its whole row
  int kept_blocks;                                  // of it, blocks whose logits stay in LDS
  size_t off_o, off_ml, off_logits, total;
};

AttendPlan attend_plan(const Problem& pb, int64_t max_length, bool weights) {
  AttendPlan P{};
  P.rows = pb.group * pb.window;
  P.qt = P.rows > 16 && pb.d <= 128 ? 2 : 1;
  P.row_chunks = (P.rows + 16 * P.qt - 1) / (16 * P.qt);
  const int64_t nb = std::max<int64_t>((max_length + CB_TOKENS - 1) / CB_TOKENS, 1);
  const int64_t heads = int64_t(pb.batch) * pb.hkv * P.row_chunks;
  const int64_t target = pb.batch == 1 ? 512 : 2048;             // workgroups
  const int64_t least = heads >= 512 ? int64_t(CA_CHUNK_MOST) : heads >= 128 ? 16 : CA_WAVES;
  int64_t chunk = std::min(std::max((nb * heads + target - 1) / target, least), int64_t(CA_CHUNK_MOST));
  if (pb.batch > 1 && chunk < 8 && heads * ((nb + 7) / 8) >= 256) chunk = 8;
  const auto room = [&](int64_t lds) { return (lds / (P.rows * 4) - CA_WAVES * pb.d) / CB_TOKENS; };   // blocks
  const bool alone = weights && P.row_chunks == 1 && nb <= 64 * CA_WAVES;   // a workgroup could take a whole row
  const bool fits = alone && nb <= room(CA_LDS);
  if (alone && heads >= 256 && (fits || nb >= 32)) chunk = std::max(chunk, nb);
  P.chunk = int((chunk + CA_WAVES - 1) / CA_WAVES * CA_WAVES);
  P.splits = int((nb + P.chunk - 1) / P.chunk);
  P.lblocks = int(nb);
  P.kept = alone && P.splits == 1 && (fits || nb >= 32);
  P.kept_blocks = P.kept ? int(std::min(nb, room(CA_LDS))) : 0;
  const size_t all = size_t(pb.batch) * pb.hkv * P.rows;
  // no fewer than splits, whatever nb, and never falling with nb
  const size_t most = size_t(std::min((nb + least - 1) / least,
                                      std::max((target + heads - 1) / heads, (nb + CA_CHUNK_MOST - 1) / CA_CHUNK_MOST)));
  size_t cur = 0;
  P.off_o = cur;
  if (most > 1) cur += align_up(all * most * pb.d * 4);
  P.off_ml = cur;
  if (most > 1 || weights) cur += align_up(all * most * 8);
  P.off_logits = cur;
  if (weights) cur += align_up(all * size_t(P.lblocks) * CB_TOKENS * 4);
  P.total = cur;
  return P;
}

template <int FMT, typename T>
kvc_status attend_form(const Problem& pb, const AttendPlan& P, const AttendArgs& a, unsigned grid, hipStream_t stream) {
  const dim3 g(grid, 1, pb.batch);
  const size_t lds = size_t(CA_WAVES) * std::min(P.rows, 16 * P.qt) * pb.d * 4 +
                     size_t(P.kept_blocks) * P.rows * CB_TOKENS * 4;
#define KVC_ATTEND(NJ, QT, STREAM)                                                                                        \
  do {                                                                                                                    \
    if (pb.d == 64 * NJ)                                                                                                  \
      KVC_LAUNCH("attend_split", stream, attend_split<FMT, T, NJ, true, QT, STREAM><<<g, CA_THREADS, lds, stream>>>(a));  \
    else                                                                                                                  \
      KVC_LAUNCH("attend_split", stream, attend_split<FMT, T, NJ, false, QT, STREAM><<<g, CA_THREADS, lds, stream>>>(a)); \
  } while (0)
  const int nj = (pb.d + 63) / 64;
  if (P.qt == 2) {
    if (nj == 1) KVC_ATTEND(1, 2, false); else KVC_ATTEND(2, 2, false);
  } else if (P.row_chunks == 1) {
    if (nj == 1) KVC_ATTEND(1, 1, true);
    else if (nj == 2) KVC_ATTEND(2, 1, true);
    else if (nj == 3) KVC_ATTEND(3, 1, true);
    else KVC_ATTEND(4, 1, true);
  } else {                                          // d > 128: row chunks read the same codes
    if (nj == 3) KVC_ATTEND(3, 1, false); else KVC_ATTEND(4, 1, false);
  }
#undef KVC_ATTEND
  return KVC_OK;
}

}  // namespace

size_t attend_workspace_bytes(const Problem& pb, int64_t max_length, bool weights) {
  return attend_plan(pb, max_length, weights).total;
}

// Workgroups of the two launches; a launch holds fewer than 2^24 of them.
bool attend_fits(const Problem& pb, int64_t max_length, bool weights) {
  const AttendPlan P = attend_plan(pb, max_length, weights);
  const int64_t split = int64_t(P.splits) * P.row_chunks * pb.hkv;
  const int64_t heads = int64_t(pb.batch) * pb.hkv;
  const int64_t join = heads * P.rows + (weights ? heads * ((max_length + CJ_TOKENS - 1) / CJ_TOKENS) : 0);
  return split < (1 << 24) && join < (1 << 24);
}

kvc_status launch_cache_attend(const Problem& pb, int layer, const void* q, const int32_t* lengths, int64_t max_length,
                               int format, const CacheView& c, void* out, float* lse, const float* weight_in,
                               float* weight_out, void* ws, hipStream_t stream) {
  const bool weights = weight_out != nullptr;
  const AttendPlan P = attend_plan(pb, max_length, weights);
  char* base = static_cast<char*>(ws);
  AttendArgs a{};
  a.q = q; a.out = out; a.lse = lse; a.lengths = lengths;
  a.part_o = reinterpret_cast<float*>(base + P.off_o);
  a.part_ml = P.splits > 1 || weights ? reinterpret_cast<float2*>(base + P.off_ml) : nullptr;
  a.kept = P.kept ? CA_WAVES * P.rows * pb.d : 0;
  a.kept_blocks = P.kept_blocks;
  a.logits = weights && P.kept_blocks < P.lblocks ? reinterpret_cast<float*>(base + P.off_logits) : nullptr;
  a.weight_in = weight_in; a.weight_out = weight_out;
  a.c = c;
  a.layer = layer; a.group = pb.group; a.window = pb.window; a.rows = P.rows; a.row_chunks = P.row_chunks;
  a.splits = P.splits; a.chunk = P.chunk; a.max_length = int(max_length); a.lblocks = P.lblocks; a.causal = pb.causal_tail;
  a.scale_log2 = pb.scale * 1.4426950408889634f;
  const unsigned grid = unsigned(P.splits) * P.row_chunks * pb.hkv;
  const bool half = pb.dtype == KVC_BF16;
  kvc_status st;
  if (format == KVC_E4M3)
    st = half ? attend_form<KVC_E4M3, uint16_t>(pb, P, a, grid, stream) : attend_form<KVC_E4M3, float>(pb, P, a, grid, stream);
  else
    st = half ? attend_form<KVC_INT8, uint16_t>(pb, P, a, grid, stream) : attend_form<KVC_INT8, float>(pb, P, a, grid, stream);
  if (st != KVC_OK) return st;
  const int64_t heads = int64_t(pb.batch) * pb.hkv;
  const int64_t joins = P.splits > 1 ? heads * P.rows : 0;
  const int chunks = int((max_length + CJ_TOKENS - 1) / CJ_TOKENS);
  const int64_t total = joins + (weights && !P.kept ? heads * chunks : 0);
  if (total == 0) return KVC_OK;
#define KVC_JOIN(T) \
  KVC_LAUNCH("attend_join", stream, attend_join<T><<<(unsigned)total, CA_THREADS, 0, stream>>>(a, joins, std::max(chunks, 1)))
  if (half) KVC_JOIN(uint16_t); else KVC_JOIN(float);
#undef KVC_JOIN
  return KVC_OK;
}

}  // namespace kvc
