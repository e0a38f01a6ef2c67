// Causal attention over the 8-bit key/value cache, and the attention weight that
// each cached token receives.
//
// A column is one query: row i of a sequence and head j of a group, numbered
// i * nq + j (the heads share the group's keys and values).  Two forms:
// - few columns (at most 16: decode steps): a tile of 16 walks the pages with 16x16x32
//   MFMAs fed from registers; reading the pages is all the work;
// - many (chunks): tiles of up to 256 columns share each page through LDS.
// A call whose sequences may have more than 16 columns takes the second form, for short
// sequences too, unless most of them look short (see attn_plan): then each form takes
// its sequences.
// In both, S^T = K Q^T and O^T += V^T P^T with an online softmax in base 2, and the
// work is dealt out alike: the (sequence, group, tile, page) units of the batch,
// numbered in that order, are cut into equal ranges, one for each workgroup of a
// grid that fills the chip, whatever the lengths are.  A workgroup walks the tiles in
// its range; a tile that lies in one range is written at once, the others leave their
// unnormalised parts, which the next launch joins in page order.  (One workgroup per
// tile of 16 columns: 1151 us instead of 188 for four sequences of 131072 tokens, 8 groups.)
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "kv_cache.hpp"
#include "lds_dma.hpp"

namespace foe {
namespace {

constexpr int kAttThr = 256;          // few columns: four waves, each taking every fourth page
constexpr int kAttWaves = kAttThr / kWave;
constexpr int kFewCols = 16;
constexpr int kShapedCols = 128;      // up to which that form takes shaped calls
constexpr int kTileThr = 512;         // many columns: eight waves of 32 columns
constexpr int kTileCols = 256;
constexpr int kCus = 256;             // compute units of the card; a multiple of the XCDs
// The running maximum starts below any finite score (times log2 e / sqrt(hd) < 0.15), and is
// at least the next value once the column has seen a token: where the sum stays 0, that
// tells a row whose scores are all -inf (NaN) from one that sees no token (zeros).
constexpr float kMFloor = -0x1.000002p126f;
constexpr float kMSeen = -0x1p126f;

// 1 / sum
__device__ __forceinline__ float inv_sum(float m, float l) {
  return l == 0.f ? (m > kMFloor ? __builtin_nanf("") : 0.f) : 1.f / l;
}
// A probability is 2^(s c - m), s c not rounded before the subtraction, where m is a rounded
// product: its rounding is a factor of all of a column's probabilities, and of their sum.
// From 2^24 on that factor leaves [1/2, 2] and would soon leave fp32, so there s c is rounded
// too, which makes the largest probability 1 again.
__device__ __forceinline__ bool far_max(float m) {
  return fabsf(m) >= 0x1p24f && fabsf(m) < 0x1p126f;
}
__device__ __forceinline__ float far_exponent(float s, float c, float m) {
#pragma clang fp contract(off)
  const float t = s * c;
  return t - m;
}
// What the mass needs of a column: its maximum and 1 / sum, negative for a far maximum.
__device__ __forceinline__ float2 column_stat(float m, float inv) {
  return float2{m, far_max(m) ? -inv : inv};
}

// ---- scores and masks of other shapes ----------------------------------------------
// foe_cache_attention_ex: a score may be capped, cap * tanh(s / cap), and get a bias of
// -slope * |distance|; a row may see the new rows that its bits name, and the first tokens
// whatever its own place.  A lane holds scores of one column at several keys; the scores are
// transformed where the matrix instructions leave them, before the maximum, so that what
// follows is the same as without.  With a cap or a bias they are then in units of log2 e (and
// c_log2 is 1), else as they were.
// (TRANSFORMS: with a cap or a bias; masks alone leave the kernels more registers.)
template <bool TRANSFORMS>
struct Shape {
  static constexpr bool kTransforms = TRANSFORMS;
  CacheScores a;
  float scale;            // log2 e / sqrt(hd)
  float cap, x_of;        // cap * log2 e; 1 / (cap * sqrt(hd))
  float bound, poly[5];   // |s| <= bound: the capped score is s * (poly in s^2)
  float near, low[3];     // and the same for |s| <= near
};

struct NoShape {  // causal, scores as they are
  static constexpr bool kTransforms = false;
};
template <typename S>
constexpr bool is_shaped = !std::is_same<S, NoShape>::value;
// what the mass needs of a column (see put_stat)
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <typename S>
using Stat = typename std::conditional<is_shaped<S>, f32x4, f32x2>::type;

// Tokens from the first on that row i and those behind it see, whose distances are place - key
// and not negative.
template <bool T>
__device__ __forceinline__ int plain_tokens(const Shape<T>& sh, int ctx, int i) {
  return sh.a.tree != nullptr || (T && sh.a.depth != nullptr) ? ctx : ctx + i + 1;
}
__device__ __forceinline__ int plain_tokens(const NoShape&, int ctx, int i) {
  return ctx + i + 1;
}

// tanh(x) / x for |x| <= kTanhBound as a polynomial in x^2, fitted here for a small largest
// relative error: 8.2e-8 (at 0.6), and 8.9e-8 with the coefficients in fp32.
constexpr float kTanhBound = 0.6f;
constexpr double kTanhPoly[5] = {0.99999993, -0.33332308, 0.13310172, -0.052101476, 0.015475425};
// And for |x| <= kTanhNear, 7.4e-8, in fp32 8.4e-8.
constexpr float kTanhNear = 0.1875f;
constexpr double kTanhLow[3] = {0.99999993, -0.33329659, 0.13053289};

// What a lane keeps of its column.
struct Column {
  float slope;  // times log2 e
  int place;    // in its sequence
};

// Column c (of ncol; row c / nq, head c % nq) of sequence b, group h.
template <bool T>
__device__ __forceinline__ Column column_of(const Shape<T>& sh, const CacheBatch& bt, int b, int h,
                                            int ctx, int c, int ncol) {
  Column k{0.f, ctx};
  if (!T || c >= ncol) return k;
  const int row = c / bt.nq;
  k.place = ctx + (sh.a.depth != nullptr ? sh.a.depth_of(bt.first_row(b) + row) : row);
  if (sh.a.slope != nullptr)
    k.slope = sh.a.slope[h * bt.nq + c - row * bt.nq] * 1.4426950408889634f;
  return k;
}

// The keys of page blk that the column sees, a bit each.
template <bool T>
__device__ __forceinline__ uint64_t keys_seen(const Shape<T>& sh, const CacheBatch& bt, int b,
                                              int row, int ctx, int len, int blk) {
  auto first = [](int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; };
  const int key0 = blk * kPage;
  int seen = min(sh.a.tree != nullptr ? ctx : ctx + row + 1, len);
  if (sh.a.prefix != nullptr) seen = max(seen, min(sh.a.prefix[b], len));
  uint64_t m = first(seen - key0);
  if (sh.a.tree != nullptr && key0 + kPage > ctx && key0 < len) {
    // the new row at the page's first key, in bit k of word w, or the first row in bit `up`
    const int i0 = max(key0 - ctx, 0), up = max(ctx - key0, 0), w = i0 >> 5, k = i0 & 31;
    const uint32_t* bits = sh.a.tree + (size_t)(bt.first_row(b) + row) * sh.a.words;
    const int last = sh.a.words - 1;
    uint32_t lo = bits[min(w, last)], mid = bits[min(w + 1, last)], hi = bits[min(w + 2, last)];
    asm volatile("" : "+v"(lo), "+v"(mid), "+v"(hi));  // (on their way together)
    if (w > last) lo = 0;
    if (w + 1 > last) mid = 0;
    if (w + 2 > last) hi = 0;
    lo = __builtin_amdgcn_alignbit(mid, lo, k);
    mid = __builtin_amdgcn_alignbit(hi, mid, k);
    const uint64_t x = (lo | (uint64_t)mid << 32) << up;
    m |= x & first(len - key0);
  }
  return m;
}

// NE scores of a lane (get, set) at keys key0 + off(i), in place.  `all`: the column sees them
// all, at distances place - key >= 0, and none is a new row of a depth of its own.  `masked`: some
// column does not, and those outside `sees` (bit of key key0 + off(i): off(i)) are taken out.
template <int NE, bool T, typename Get, typename Set, typename Off>
__device__ __forceinline__ void shape_scores(const Shape<T>& sh, const CacheBatch& bt, int b,
                                             int ctx, int rows, const Column& c, int key0, bool all,
                                             bool masked, uint64_t sees, Get get, Set set,
                                             Off off) {
  if constexpr (T) {
    const bool biased = sh.a.slope != nullptr;
    const float d = (float)(c.place - key0);
    // the bias of a page that is seen whole, linear in the key, joins the score's last product:
    // slope * key - slope * place (of the page's start: what is rounded is small where it counts)
    const bool linear = biased && all;
    const float base = -c.slope * d;
    auto each = [&](auto with, auto factor) {
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        const float s = get(i), y = factor(s);
        set(i, decltype(with)::value ? fmaf(s, y, fmaf(c.slope, (float)off(i), base)) : s * y);
      }
    };
    auto scaled = [&](auto factor) {
      if (linear) each(std::true_type{}, factor);
      else each(std::false_type{}, factor);
    };
    if (sh.cap != 0.f) {
      float big = 0.f;
#pragma unroll
      for (int i = 0; i < NE; ++i) big = fmaxf(big, fabsf(get(i)));
      // Scores are mostly well below the cap, where the polynomial is 6 operations; the
      // exponential, which loses the small ones' last digits besides, is taken where a lane
      // needs it.  us for 2048 rows over 6144 tokens, 8 groups of two heads, keys of unit scale:
      // queries of 1.5 under a cap of 50 (three coefficients mostly) 192, of 20 (five) 201, queries
      // of 10 under a cap of 30 (the exponential) 292.
      if (__builtin_amdgcn_ballot_w64(big > sh.near) == 0) {
        scaled([&](float s) {
          const float u = s * s;
          return fmaf(fmaf(sh.low[2], u, sh.low[1]), u, sh.low[0]);
        });
      } else if (__builtin_amdgcn_ballot_w64(big > sh.bound) == 0) {
        scaled([&](float s) {
          const float u = s * s;
          float y = fmaf(sh.poly[4], u, sh.poly[3]);
          y = fmaf(y, u, sh.poly[2]);
          y = fmaf(y, u, sh.poly[1]);
          return fmaf(y, u, sh.poly[0]);
        });
      } else {
#pragma unroll
        for (int i = 0; i < NE; ++i) {
          if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
          const float x = get(i) * sh.x_of, u = x * x;
          float y = (float)kTanhPoly[4];
#pragma unroll
          for (int k = 3; k >= 0; --k) y = fmaf(y, u, (float)kTanhPoly[k]);
          const float e = __builtin_amdgcn_exp2f(fabsf(x) * 2.885390081777927f);
          const float far = copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f), x);
          const float add = linear ? fmaf(c.slope, (float)off(i), base) : 0.f;
          set(i, fmaf(sh.cap, fabsf(x) > kTanhBound ? far : x * y, add));
        }
      }
    } else {
      scaled([&](float) { return sh.scale; });
    }
    if (biased && !all) {
      if (sh.a.depth != nullptr) {
        const int row0 = bt.first_row(b);
#pragma unroll
        for (int i = 0; i < NE; ++i) {
          if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);  // (few loads' addresses at a time)
          const int key = key0 + off(i), r = key - ctx;
          const int at = r >= 0 && r < rows ? ctx + sh.a.depth_of(row0 + r) : key;
          set(i, fmaf(-c.slope, fabsf((float)(c.place - at)), get(i)));
        }
      } else {
#pragma unroll
        for (int i = 0; i < NE; ++i) set(i, fmaf(-c.slope, fabsf(d - (float)off(i)), get(i)));
      }
    }
  }
  if (masked) {
    const uint32_t lo = (uint32_t)sees, hi = (uint32_t)(sees >> 32);
    // (through the bit spread over a word: a comparison each would hold a scalar pair each)
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const uint32_t keep =
          (uint32_t)__builtin_amdgcn_sbfe((int)(off(i) < 32 ? lo : hi), off(i) & 31, 1);
      set(i, __uint_as_float((keep & __float_as_uint(get(i))) | (~keep & 0xff800000u)));
    }
  }
}

// ---- dealing out the work -------------------------------------------------------

// What a call's tiles reach beyond their own rows: the prefix, and with a tree every new row.
struct Reach {
  const int32_t* prefix;
  bool tree;
  __device__ __forceinline__ int pages(const CacheBatch& bt, int b, int ctx, int n) const {
    if (tree) return (ctx + n + kPage - 1) / kPage;
    if (prefix == nullptr) return 0;
    return (min(max(prefix[b], 0), min(ctx + n, bt.cap())) + kPage - 1) / kPage;
  }
};

// The units of a batch in a form, numbered by sequence, group, tile and page.  A tile of
// many columns has 2^log2r rows, tile t reaches page ceil((ctx + last row + 1) / 64), and
// the sums over tiles are closed forms (which count pages past the table's end too).
// (WIDE: shaped calls.  Rows may see past themselves, see Reach; and with few columns each
// (sequence, group) has kStartPages units before its pages', for what starting on it costs.  us
// with 2, 5, 7 and 12, calls of 48 trees of 25 rows (hd 96, 100 to 4096 tokens, mass) 87 84 82 85,
// of 64 trees of 16 (256 to 8192) 142 135 134 133, of 64 capped and biased rows 121 122 124 128.)
constexpr int kStartPages = 7;

template <bool FEW, bool WIDE = false>
struct Units {
  CacheBatch bt;
  int max_rows;
  int log2r;   // (many)
  int lo, hi;  // columns that a sequence of this form has: lo < columns <= hi
  Reach reach;
  long long* prefix;  // [B + 1]: units before each sequence, and in all (for the launches after)

  // rows of sequence b in this form
  __device__ __forceinline__ int rows(int b) const {
    const int n = min(bt.rows(b), max_rows);
    return n * bt.nq > lo && n * bt.nq <= hi ? n : 0;
  }
  __device__ __forceinline__ int tiles(int n) const { return (n + (1 << log2r) - 1) >> log2r; }
  // pages that every tile of sequence b reaches, if its rows are not causal alone
  __device__ __forceinline__ int least(int b, int ctx, int n) const {
    return WIDE && !FEW ? reach.pages(bt, b, ctx, n) : 0;
  }
  // pages of the tiles before tile t (t < tiles), all of them at least `least`
  __device__ __forceinline__ long long before(int ctx, int t, int least) const {
    if (!WIDE || least == 0) return causal_before(ctx, t);
    // the tiles whose own pages are no more than that
    const long long j = max(((long long)least * kPage - ctx) >> log2r, 0LL);
    if (t <= j) return (long long)t * least;
    return j * least + causal_before(ctx, t) - causal_before(ctx, (int)j);
  }
  // the same for causal rows
  __device__ __forceinline__ long long causal_before(int ctx, int t) const {
    const long long c = ctx + kPage - 1;
    if (log2r >= 6) return t * (c / kPage) + ((long long)t * (t + 1) / 2 << (log2r - 6));
    const int m = kPage >> log2r;  // tiles per page
    auto sum = [&](long long x) {  // sum over j < x of j / m
      const long long q = x / m;
      return m * (q * (q - 1) / 2) + q * (x - q * m);
    };
    const long long a = c >> log2r;
    return sum(a + t + 1) - sum(a + 1);
  }
  // pages of tile t of a sequence with n rows
  __device__ __forceinline__ int pages(int ctx, int n, int t, int least) const {
    if (FEW) return min((ctx + n + kPage - 1) / kPage, bt.max_blocks);
    const int np = (ctx + min((t + 1) << log2r, n) + kPage - 1) / kPage;
    return WIDE ? max(np, least) : np;
  }
  // units of one group of sequence b
  __device__ __forceinline__ long long group(int b) const {
    const int n = rows(b);
    if (n <= 0) return 0;
    const int ctx = bt.context(b), t = FEW ? 0 : tiles(n) - 1, more = least(b, ctx, n);
    return (FEW ? (WIDE ? kStartPages : 0) : before(ctx, t, more)) + pages(ctx, n, t, more);
  }
};

// How a batch's units are dealt out: to `ranges` workgroups, at least `least` units each;
// where `round` workgroups would have few enough (see kOneRound in rules.hpp), to those.
struct Deal {
  int ranges, least, round;
  // units of a range
  __device__ __forceinline__ long long per(long long total) const {
    return range_units(total, ranges, least, round);
  }
};

// Total of the units, count(b) of sequence b, and the sequence that unit range * per falls
// in (b, or -1 past the end) with its offset there.  Every thread of the workgroup calls
// it; range 0 writes the prefix, if any: the units before each sequence, and in all.
template <int NT, typename Count>
__device__ __forceinline__ void locate(int B, Count count, const Deal& deal, int range,
                                       long long* prefix, long long& total, int& b,
                                       long long& off) {
  constexpr int NW = NT / kWave;
  __shared__ long long wave_sum[NW];
  __shared__ long long found[2];
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  auto scan = [&](long long c, long long& all) {  // inclusive sum over the threads
    long long incl = c;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const long long up = __shfl_up(incl, o);
      if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == kWave - 1) wave_sum[wave] = incl;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      if (v < wave) incl += wave_sum[v];
      all += wave_sum[v];
    }
    return incl;
  };
  const long long first = (int)threadIdx.x < B ? count(threadIdx.x) : 0;
  long long mine = first;
  for (int i = threadIdx.x + NT; i < B; i += NT) mine += count(i);
  long long incl = scan(mine, total);
  const long long u0 = range * deal.per(total);
  const bool writes = prefix != nullptr && range == 0;
  if (threadIdx.x == 0) found[0] = -1;
  if (B > NT && (u0 < total || writes)) {  // (uniform) again, a row of threads at a time
    long long run = 0, all;
    for (int base = 0; base < B; base += NT) {
      const int i = base + (int)threadIdx.x;
      const long long c = base == 0 ? first : i < B ? count(i) : 0;
      incl = run + scan(c, all);
      if (u0 >= incl - c && u0 < incl) found[0] = i, found[1] = u0 - (incl - c);
      if (writes && i < B) prefix[i] = incl - c;
      run += all;
    }
  } else if (B <= NT) {
    __syncthreads();
    const int i = threadIdx.x;
    if (u0 >= incl - first && u0 < incl) found[0] = i, found[1] = u0 - (incl - first);
    if (writes && i < B) prefix[i] = incl - first;
  }
  if (writes && threadIdx.x == 0) prefix[B] = total;
  __syncthreads();
  b = (int)found[0];
  off = found[1];
}

// ---- few columns ------------------------------------------------------------------
// The page layouts feed both products from registers, without LDS.  With lane (n, g) =
// (lane % 16, lane / 16):
// - score tile t (0..3) of a page takes as row r key 16 (r / 4) + 4 t + r % 4, so
//   that a lane ends with the scores of the 16 consecutive keys 16 g .. 16 g + 15 of
//   column n, the four tiles one after another;
// - those are, eight at a time, the B operand of the second product, whose A operand
//   is then 8 consecutive tokens of one dim: the value layout's 16-byte pieces (16
//   tokens of one dim) hold them for both k-steps.

template <int HD>
struct PageFrags {
  static constexpr int NST = HD / 32;  // score k-steps
  static constexpr int NDT = HD / 16;  // output tiles
  // tile t: 16 bytes at 64 h + 16 g (8 at 64 + 8 g for HD = 96)
  u32x4 k[4][(HD + 63) / 64];
  u32x4 v[NDT];                        // dims 16 dt + n, tokens 16 g .. +15

  __device__ __forceinline__ void load_k(const uint8_t* kp, int lane) {
    const int n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint8_t* row = kp + (16 * (n >> 2) + 4 * t + (n & 3)) * HD;
      k[t][0] = *reinterpret_cast<const u32x4*>(row + 16 * g);
      if constexpr (HD == 128) {
        k[t][1] = *reinterpret_cast<const u32x4*>(row + 64 + 16 * g);
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(row + 64 + 8 * g);
        k[t][1] = u32x4{x[0], x[1], 0u, 0u};
      }
    }
  }
  __device__ __forceinline__ void load_v(const uint8_t* vp, int lane) {
    const int n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
      v[dt] = *reinterpret_cast<const u32x4*>(vp + g * (HD * kSub) + (16 * dt + n) * kSub);
  }
  // key fragment of score tile t and k-step st
  __device__ __forceinline__ bf16x8 key(int t, int st, float ks) const {
    const u32x4 w = k[t][st / 2];
    return codes_to_bf16(w[2 * (st % 2)], w[2 * (st % 2) + 1], ks);
  }
  // scores of the page: s[t][v] = key 16 g + 4 t + v of column n
  __device__ __forceinline__ void scores(const bf16x8* qf, float ks, f32x4* s) const {
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < NST; ++st)
#pragma unroll
      for (int t = 0; t < 4; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key(t, st, ks), qf[st], s[t], 0, 0, 0);
  }
};

// dims of lane group g in score step st (see PageFrags::load_k)
template <int HD>
__device__ __forceinline__ int frag_dim(int st, int g) {
  if (HD == 96 && st == 2) return 64 + 8 * g;
  return 64 * (st / 2) + 16 * g + 8 * (st % 2);
}

// The queries of columns c0 .. c0+15 (of ncol) of a sequence, as B operand.
template <int HD>
__device__ __forceinline__ void load_q(const bf16* q, int col, int ncol, int g, bf16x8* qf) {
#pragma unroll
  for (int st = 0; st < HD / 32; ++st) {
    qf[st] = bf16x8{};
    if (col < ncol)
      qf[st] = *reinterpret_cast<const bf16x8*>(q + (size_t)col * HD + frag_dim<HD>(st, g));
  }
}

// A part of a tile that several workgroups share: unnormalised sums ([columns][HD] with
// few columns; [HD / 4][columns][4] with many, as the lanes hold them, a column each),
// then [columns] (maximum, sum).  Workgroup r leaves at most two: of its first tile
// (slot 2 r), and of its last one if another (2 r + 1).
__host__ __device__ inline size_t part_floats(int cols, int hd) { return (size_t)cols * (hd + 2); }

struct AttnOut {
  bf16* out;
  void* stat;        // of each column (see put_stat), or null
  float* part;
  int part_cols;
};

// A column's entry for the mass: its maximum and 1 / sum (see column_stat); with a Shape its
// slope and place besides.  Column c of sequence b, group h is number `at` of the batch.
__device__ __forceinline__ void put_stat(const NoShape&, const CacheBatch&, int, int, int, int,
                                         int, size_t at, const AttnOut& o, float m, float inv) {
  const float2 z = column_stat(m, inv);
  static_cast<f32x2*>(o.stat)[at] = f32x2{z.x, z.y};
}
template <bool T>
__device__ __forceinline__ void put_stat(const Shape<T>& sh, const CacheBatch& bt, int b, int h,
                                         int ctx, int rows, int c, size_t at, const AttnOut& o,
                                         float m, float inv) {
  const Column k = column_of(sh, bt, b, h, ctx, c, rows * bt.nq);
  const float2 z = column_stat(m, inv);
  static_cast<f32x4*>(o.stat)[at] = f32x4{z.x, z.y, k.slope, __int_as_float(k.place)};
}

template <int HD>
struct FewLds {
  float mm[kAttWaves][16], ll[kAttWaves][16];
  float oo[kAttWaves][16][HD + 4];  // (rows of other bank groups)
};

// Pages blk0 .. blk1-1 of the columns (at most 16) of sequence b, group h, dealt to the
// waves of the workgroup; `slot` is where a part goes, `score` the scores of page blk0 or
// null.
template <int HD>
__device__ __forceinline__ void few_columns(
    const bf16* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
    const float* __restrict__ kv_scale, const CacheBatch& bt, int b, int h, int rows, int ctx,
    int np, int blk0, int blk1, float c_log2, const AttnOut& o, size_t slot,
    float* __restrict__ score, FewLds<HD>& lds) {
  using F = PageFrags<HD>;
  constexpr int NW = kAttWaves;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const int n = lane & 15, g = lane >> 4;
  const int ncol = rows * bt.nq;
  const size_t qrow = ((size_t)h * bt.N + bt.first_row(b)) * bt.nq;
  bf16x8 qf[F::NST];
  load_q<HD>(q + qrow * HD, n, ncol, g, qf);
  const int len = min(ctx + rows, bt.cap());  // tokens the cache holds now
  const int seen = n < ncol ? min(ctx + n / bt.nq + 1, bt.cap()) : 0;
  const int fewest = min(ctx + 1, bt.cap());  // that a column sees
  f32x4 oacc[F::NDT];
#pragma unroll
  for (int dt = 0; dt < F::NDT; ++dt) oacc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kMFloor, l_run = 0.f;
  // page numbers and scales of the wave's next 64 pages, one a lane
  int pid = -1;
  float2 psc{0.f, 0.f};
  F fn;
  auto fetch = [&](int i) {  // the wave's i-th page; an absent one loads page 0
    if ((i & 63) == 0) {
      const int blk = blk0 + wave + NW * (i + lane);
      pid = blk < blk1 ? bt.page(b, blk) : -1;
      if (pid >= 0)
        psc = *reinterpret_cast<const float2*>(kv_scale + ((size_t)pid * bt.H + h) * 2);
    }
    const int page = __builtin_amdgcn_readlane(pid, i & 63);
    const size_t pg = ((size_t)max(page, 0) * bt.H + h) * (kPage * HD);
    fn.load_k(kc + pg, lane);
    fn.load_v(vc + pg, lane);
  };
  const int mine = (blk1 - blk0 - wave + NW - 1) / NW;  // pages of this wave
  int first = -1;    // the first that is there
  bool far = false;  // (uniform) a column's maximum is far from 0
  if (mine > 0) fetch(0);
  for (int i = 0; i < mine; ++i) {
    const int blk = blk0 + wave + NW * i;
    const int page = __builtin_amdgcn_readlane(pid, i & 63);
    const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(psc.x), i & 63));
    const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(psc.y), i & 63));
    F f = fn;
    if (i + 1 < mine) fetch(i + 1);
    if (page < 0) continue;
    if (first < 0) first = blk;
    f32x4 s[4];
    f.scores(qf, ks, s);
    const int k0 = blk * kPage + 16 * g;
    if ((blk + 1) * kPage > fewest) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (k0 + 4 * t + e >= seen) s[t][e] = -__builtin_inff();
      // slots past the last token hold anything: 0 * NaN is NaN
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int in = len - (k0 + 4 * e);
        const uint32_t m = in >= 4 ? 0xffffffffu : in <= 0 ? 0u : (1u << (8 * in)) - 1;
#pragma unroll
        for (int dt = 0; dt < F::NDT; ++dt) f.v[dt][e] &= m;
      }
    }
    if (score != nullptr && n < ncol) {
      float* to = score + ((size_t)(blk - blk0) * o.part_cols + n) * kPage + 16 * g;
#pragma unroll
      for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4*>(to + 4 * t) = s[t];
    }
    float mx = s[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[t][e]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    // the maximum moves only when a page exceeds it by 2^8: probabilities stay below
    // that, and the sums are rescaled on those pages alone
    const float mxs = mx * c_log2;
    const bool need = mxs > m_run + 8.f;
    if (__builtin_amdgcn_ballot_w64(need)) {
      const float m_new = need ? mxs : m_run;
      const float a = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      far = __builtin_amdgcn_ballot_w64(far_max(m_run)) != 0;
      l_run *= a;
#pragma unroll
      for (int dt = 0; dt < F::NDT; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) oacc[dt][e] *= a;
    }
    float c_page = c_log2, m_page = m_run;
    if (far) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[t][e] = far_exponent(s[t][e], c_log2, m_run);
      c_page = 1.f;
      m_page = 0.f;
    }
    bf16x8 p[2];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[t][e], c_page, -m_page));
        l_run += x;
        p[t >> 1][4 * (t & 1) + e] = (bf16)x;
      }
#pragma unroll
    for (int dt = 0; dt < F::NDT; ++dt)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        oacc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            codes_to_bf16(f.v[dt][2 * u], f.v[dt][2 * u + 1], vs), p[u], oacc[dt], 0, 0, 0);
  }
  if (first >= 0 && first * kPage < seen) m_run = fmaxf(m_run, kMSeen);
  // the waves' states, merged in wave order
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);
  __syncthreads();  // what was in LDS before has been read
  if (g == 0) lds.mm[wave][n] = m_run, lds.ll[wave][n] = l_run;
  if (n < ncol) {
#pragma unroll
    for (int dt = 0; dt < F::NDT; ++dt)
      *reinterpret_cast<f32x4*>(&lds.oo[wave][n][16 * dt + 4 * g]) = oacc[dt];
  }
  __syncthreads();
  const bool whole = blk0 == 0 && blk1 == np;
  float* pt = o.part + slot * part_floats(o.part_cols, HD);
  for (int i = tid; i < ncol * HD; i += NW * kWave) {
    const int c = i / HD, d = i % HD;
    float m = lds.mm[0][c], l = 0.f, x = 0.f;
#pragma unroll
    for (int v = 1; v < NW; ++v) m = fmaxf(m, lds.mm[v][c]);
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const float a = __builtin_amdgcn_exp2f(lds.mm[v][c] - m);
      l += lds.ll[v][c] * a;
      x += lds.oo[v][c][d] * a;
    }
    if (whole) {
      const float inv = inv_sum(m, l);
      const int row = bt.first_row(b) + c / bt.nq;
      o.out[(((size_t)row * bt.H + h) * bt.nq + c % bt.nq) * HD + d] = (bf16)(x * inv);
      if (d == 0 && o.stat != nullptr)
        put_stat(NoShape{}, bt, b, h, ctx, rows, c, qrow + c, o, m, inv);
    } else {
      pt[i] = x;
      if (d == 0) reinterpret_cast<float2*>(pt + o.part_cols * HD)[c] = float2{m, l};
    }
  }
}

__device__ __forceinline__ long long uniform64(long long x) {
  return (long long)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// The segments of a range of the few-column form: pages blk0 .. blk1-1 (of np) of sequence b,
// group h, numbered from `unit` on; `slot` is where a part goes.
template <bool WIDE>
struct Segment {
  static constexpr int kStart = WIDE ? kStartPages : 0;
  int b, h, rows, ctx, np, blk0, blk1, left;
  long long unit;
  size_t slot;

  // range `r`'s first one, false where it has none; every thread of the workgroup calls it
  __device__ __forceinline__ bool first(const Units<true, WIDE>& w, const Deal& deal, int r) {
    const CacheBatch& bt = w.bt;
    long long total, off;
    locate<kAttThr>(
        bt.B, [&](int i) { return w.group(i) * bt.H; }, deal, r, w.prefix, total, b, off);
    if (b < 0) return false;
    if constexpr (WIDE) {  // (in scalar registers, and all that follows)
      b = __builtin_amdgcn_readfirstlane(b);
      total = uniform64(total);
      off = uniform64(off);
    }
    // (fits: at most 2^37 pages, of tables of 2^31 entries and 64 groups, and kStartPages for each
    // of 65535 sequences' groups, in 512 ranges or more; fewer ranges have at most kFewLeast pages
    // of the tables each, whose groups are no more than the pages)
    const int per = (int)deal.per(total);
    unit = (long long)r * per;
    left = (int)min((long long)per, total - unit);
    rows = w.rows(b), ctx = bt.context(b), np = w.pages(ctx, rows, 0, 0);
    h = (int)(off / (np + kStart)), blk0 = (int)(off % (np + kStart));
    slot = 2 * (size_t)r;
    if constexpr (WIDE) {
      const int start = max(kStart - blk0, 0);
      left -= start;
      blk0 = max(blk0 - kStart, 0);
      if (left <= 0) return false;
    }
    blk1 = min(np, blk0 + left);
    return true;
  }
  // the next group, or the next sequence with rows; false past the range's end
  __device__ __forceinline__ bool next(const Units<true, WIDE>& w) {
    const CacheBatch& bt = w.bt;
    left -= blk1 - blk0;
    unit += blk1 - blk0;
    if (left <= kStart) return false;
    left -= kStart;
    slot |= 1;
    blk0 = 0;
    if (++h == bt.H) {
      h = 0;
      do {
        if (++b >= bt.B) return false;
        rows = w.rows(b);
      } while (rows <= 0);
      ctx = bt.context(b);
      np = w.pages(ctx, rows, 0, 0);
    }
    blk1 = min(np, left);
    return true;
  }
};

template <int HD>
__global__ __launch_bounds__(kAttThr, 2) void cache_attn_few_kernel(
    const bf16* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
    const float* __restrict__ kv_scale, Units<true> w, Deal deal, float c_log2, AttnOut o,
    float* __restrict__ score) {
  __shared__ FewLds<HD> lds;
  Segment<false> g;
  if (!g.first(w, deal, blockIdx.x)) return;
  do {
    few_columns<HD>(q, kc, vc, kv_scale, w.bt, g.b, g.h, g.rows, g.ctx, g.np, g.blk0, g.blk1,
                    c_log2, o, g.slot,
                    score != nullptr ? score + g.unit * o.part_cols * kPage : nullptr, lds);
  } while (g.next(w));
}

// ---- few columns of other shapes -----------------------------------------------------
// The same products, for up to 128 columns (trees of drafts, and any shaped call of so few).
// The four waves are G groups of 16 NC columns by 4 / G pages: groups of a workgroup read the
// same page at about the same time, from L2 but for the first.  The queries are held in LDS, as
// the waves read them; a page's keys give their registers to the next page's as soon as the
// scores are formed, and its values after the second product, so that two waves of a SIMD
// have room for 32 columns each.  (Pages through a ring of LDS-DMA stages, loaded once for the
// four waves of 128 columns: 460 us for four sequences of 131072 tokens, 64 rows of two heads, 8
// groups, and so 380: the waves wait for one another at each page.)  The next segment's page
// numbers are loaded beside this one's pages, and its first page (of more than 16 columns the keys)
// before this one's states are merged.
// number of a page among the kept scores of shaped calls
__device__ __forceinline__ size_t score_page(const CacheBatch& bt, int b, int h, int blk) {
  return ((size_t)b * bt.H + h) * bt.max_blocks + blk;
}

// Where a page lies: sequence, context, new rows, columns and tokens, number; `some`: not every
// column sees it whole (see plain_tokens).
struct PageOf {
  int b, ctx, rows, ncol, len, blk;
  bool some;
};

// The maximum over a column's four lanes, by register swaps: through LDS, as a shuffle goes, its
// latency stands between a page's scores and their exponentials.
__device__ __forceinline__ float column_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// A wave's 16 NC columns: sums, running maxima and sums of probabilities.
template <int NC, int NDT>
struct ShapedState {
  f32x4 oacc[NC][NDT];
  float m_run[NC], l_run[NC];
  bool saw[NC], far[NC];  // any token; (uniform) a column's maximum is far from 0

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) oacc[j][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
      m_run[j] = kMFloor;
      l_run[j] = 0.f;
      saw[j] = far[j] = false;
    }
  }
  // the page's scores s into probabilities p, in bf16 for the product with the values (the matrix
  // instructions' type: half a step is 2^-8 of a probability, and the codes of the values have
  // four bits; the sums are of the unrounded ones, in fp32); columns col0 on; `score`: where
  // column 0's scores are kept, or null
  template <typename S>
  __device__ __forceinline__ void softmax(const S& sh, const CacheBatch& bt, const PageOf& at,
                                          int col0, int lane, const Column* cols, float c_log2,
                                          f32x4 (*s)[4], bf16x8 (*p)[2], float* score) {
    const int n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      __builtin_amdgcn_sched_barrier(0);  // (a tile of columns after another)
      const int c = col0 + 16 * j + opaque_int(n);  // (not held, nor its slope and place)
      uint64_t sees = 0;
      bool masked = false;
      if (at.some) {
        if (c < at.ncol) sees = keys_seen(sh, bt, at.b, c / bt.nq, at.ctx, at.len, at.blk);
        saw[j] |= sees != 0;
        masked = __builtin_amdgcn_ballot_w64(c < at.ncol && ~sees != 0) != 0;
        sees >>= 16 * g;
      } else {
        saw[j] |= c < at.ncol;
      }
      Column col{};
      if constexpr (S::kTransforms) col = cols[c];
      shape_scores<16>(
          sh, bt, at.b, at.ctx, at.rows, col, at.blk * kPage + 16 * g, !at.some, masked, sees,
          [&](int x) { return s[j][x >> 2][x & 3]; },
          [&](int x, float y) { s[j][x >> 2][x & 3] = y; }, [](int x) { return x; });
      if (NC == 1 && score != nullptr && n < at.ncol) {
        float* to = score + n * kPage + 16 * g;
#pragma unroll
        for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4*>(to + 4 * t) = s[j][t];
      }
      float mx = s[j][0][0];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[j][t][e]);
      mx = column_max(mx);
      // (the maximum moves only when a page exceeds it by 2^8, as with causal columns)
      const float mxs = mx * c_log2;
      const bool need = mxs > m_run[j] + 8.f;
      if (__builtin_amdgcn_ballot_w64(need)) {
        const float m_new = need ? mxs : m_run[j];
        const float x = __builtin_amdgcn_exp2f(m_run[j] - m_new);
        m_run[j] = m_new;
        far[j] = __builtin_amdgcn_ballot_w64(far_max(m_run[j])) != 0;
        l_run[j] *= x;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) oacc[j][dt][e] *= x;
      }
      float c_page = c_log2, m_page = m_run[j];
      if (far[j]) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[j][t][e] = far_exponent(s[j][t][e], c_log2, m_run[j]);
        c_page = 1.f;
        m_page = 0.f;
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[j][t][e], c_page, -m_page));
          l_run[j] += x;
          p[j][t >> 1][4 * (t & 1) + e] = (bf16)x;
        }
      // (formed here, so that the next tile has the scores' registers)
      asm volatile("" : "+v"(p[j][0]), "+v"(p[j][1]));
    }
  }
  // the sums over a column's lanes
  __device__ __forceinline__ void finish(int j) {
    if (saw[j]) m_run[j] = fmaxf(m_run[j], kMSeen);
    l_run[j] += __shfl_xor(l_run[j], 16);
    l_run[j] += __shfl_xor(l_run[j], 32);
  }
};

// Slots past the last token hold anything, and 0 * NaN is NaN: their bytes of values of 16
// tokens from key k0 on are cleared.
template <int NDT>
__device__ __forceinline__ void clear_past(u32x4 (&v)[NDT], int k0, int len) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int in = len - (k0 + 4 * e);
    const uint32_t m = in >= 4 ? 0xffffffffu : in <= 0 ? 0u : (1u << (8 * in)) - 1;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) v[dt][e] &= m;
  }
}

// Writes four dims from d on of column c of a segment: the result where it is a whole tile, else
// the part.
template <int HD, typename S>
__device__ __forceinline__ void put_columns(const S& sh, const CacheBatch& bt,
                                            const Segment<true>& a, const AttnOut& o, size_t qrow,
                                            int c, int d, const f32x4& x, float m, float l) {
  if (a.blk0 == 0 && a.blk1 == a.np) {
    const float inv = inv_sum(m, l);
    const int row = c / bt.nq;
    bf16* to = o.out +
               (((size_t)(bt.first_row(a.b) + row) * bt.H + a.h) * bt.nq + c - row * bt.nq) * HD;
    *reinterpret_cast<bf16x4*>(to + d) = bf16x4{(bf16)(x[0] * inv), (bf16)(x[1] * inv),
                                                (bf16)(x[2] * inv), (bf16)(x[3] * inv)};
    if (d == 0 && o.stat != nullptr)
      put_stat(sh, bt, a.b, a.h, a.ctx, a.rows, c, qrow + c, o, m, inv);
  } else {
    float* pt = o.part + a.slot * part_floats(o.part_cols, HD);
    *reinterpret_cast<f32x4*>(pt + (size_t)c * HD + d) = x;
    if (d == 0) reinterpret_cast<float2*>(pt + o.part_cols * HD)[c] = float2{m, l};
  }
}

template <int HD, int NC, int G, bool T>
struct ShapedLds {
  FewLds<HD> few;
  bf16x8 q[G * NC][HD / 32][kWave];
  Column cols[T ? 16 * NC * G : 1];
};

template <int HD, int NC, int G, typename S>
__global__ __launch_bounds__(kAttThr, 2) void cache_attn_shaped_kernel(
    const bf16* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
    const float* __restrict__ kv_scale, Units<true, true> w, Deal deal, float c_log2, S sh,
    AttnOut o, float* __restrict__ score_base) {
  using F = PageFrags<HD>;
  constexpr int NP = kAttWaves / G;  // pages at a time
  __shared__ ShapedLds<HD, NC, G, S::kTransforms> lds;
  const CacheBatch& bt = w.bt;
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), cg = wave % G, pl = wave / G;
  const int n = lane & 15, g = lane >> 4;
  const int col0 = 16 * NC * cg;

  // the numbers of 64 of the wave's pages from its i-th on, one a lane
  auto pages64 = [&](const Segment<true>& a, int i) {
    const int blk = a.blk0 + pl + NP * (i + lane);
    return blk < a.blk1 ? bt.page(a.b, blk) : -1;
  };
  auto count = [&](const Segment<true>& a) { return (a.blk1 - a.blk0 - pl + NP - 1) / NP; };
  int pid;
  F f, next;  // (NC == 1: the page in flight has registers of its own)
  F& to = NC == 1 ? next : f;
  float2 scale;
  auto at = [&](int h, int i) {  // (an absent page loads page 0)
    return (size_t)max(__builtin_amdgcn_readlane(pid, i & 63), 0) * bt.H + h;
  };
  // (the lane's addresses in a page are not held where registers are short)
  auto place = [&]() { return NC == 1 ? lane : opaque_int(lane); };
  auto load_k = [&](int h, int i) {
    scale = *reinterpret_cast<const float2*>(kv_scale + at(h, i) * 2);
    to.load_k(kc + at(h, i) * (kPage * HD), place());
  };
  auto load_v = [&](int h, int i) { to.load_v(vc + at(h, i) * (kPage * HD), place()); };

  Segment<true> a;
  if (!a.first(w, deal, blockIdx.x)) return;
  pid = pages64(a, 0);
  if (count(a) > 0) {
    load_k(a.h, 0);
    if (NC == 1) load_v(a.h, 0);
  }
  while (true) {
    Segment<true> ahead = a;
    const bool another = ahead.next(w);
    const int b = a.b, h = a.h, rows = a.rows, ctx = a.ctx, ncol = rows * bt.nq;
    const size_t qrow = ((size_t)h * bt.N + bt.first_row(b)) * bt.nq;
    int pid_ahead = -1;
    if (another) pid_ahead = pages64(ahead, 0);
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = col0 + 16 * j + n;
      if (pl == 0) {
        if constexpr (S::kTransforms) lds.cols[c] = column_of(sh, bt, b, h, ctx, c, ncol);
        bf16x8 qf[F::NST];
        load_q<HD>(q + qrow * HD, c, ncol, g, qf);
#pragma unroll
        for (int ks = 0; ks < F::NST; ++ks) lds.q[NC * cg + j][ks][lane] = qf[ks];
      }
    }
    const int len = min(ctx + rows, bt.cap());  // tokens the cache holds now
    const int fewest = min(plain_tokens(sh, ctx, 0), bt.cap());
    float* score = NC == 1 && score_base != nullptr
                       ? score_base + score_page(bt, b, h, a.blk0) * o.part_cols * kPage
                       : nullptr;
    ShapedState<NC, F::NDT> st;
    st.clear();
    const int mine = count(a);
    __syncthreads();
    for (int i = 0; i < mine; ++i) {
      const int blk = a.blk0 + pl + NP * i;
      const int page = __builtin_amdgcn_readlane(pid, i & 63);
      const float ks = scale.x, vs = scale.y;
      const bool more = i + 1 < mine;
      if constexpr (NC == 1) {
        f = next;
        if (more) {
          if (((i + 1) & 63) == 0) pid = pages64(a, i + 1);
          load_k(h, i + 1);
          load_v(h, i + 1);
        }
      } else {
        // (here and not behind the last page's product, the same moment, and the next page's keys
        // below even if there is none: in one block and always as many, so that a wait for keys
        // leaves the values on their way and the other way round.  48 trees of 25 rows, hd 96, 100
        // to 4096 tokens: 44 us, and 46 with a wait for both)
        load_v(h, i);
        __builtin_amdgcn_sched_barrier(0);
      }
      f32x4 s[NC][4];
#pragma unroll
      for (int j = 0; j < NC; ++j)
#pragma unroll
        for (int t = 0; t < 4; ++t) s[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int step = 0; step < F::NST; ++step) {
        bf16x8 qf[NC];
#pragma unroll
        for (int j = 0; j < NC; ++j) qf[j] = lds.q[NC * cg + j][step][lane];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const bf16x8 kf = f.key(t, step, ks);
#pragma unroll
          for (int j = 0; j < NC; ++j)
            s[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[j], s[j][t], 0, 0, 0);
        }
      }
      if constexpr (NC > 1) {
        if (more && ((i + 1) & 63) == 0) pid = pages64(a, i + 1);
        load_k(h, i + 1);
      }
      if (page >= 0) {
        const int k0 = blk * kPage + 16 * g;
        const bool some = (blk + 1) * kPage > fewest;
        bf16x8 p[NC][2];
        const PageOf at_page{b, ctx, rows, ncol, len, blk, some};
        st.softmax(sh, bt, at_page, col0, lane, lds.cols, c_log2, s, p,
                   NC == 1 && score != nullptr
                       ? score + (size_t)(blk - a.blk0) * o.part_cols * kPage
                       : nullptr);
        if (some) clear_past(f.v, k0, len);
#pragma unroll
        for (int dt = 0; dt < F::NDT; ++dt)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const bf16x8 vf = codes_to_bf16(f.v[dt][2 * u], f.v[dt][2 * u + 1], vs);
#pragma unroll
            for (int j = 0; j < NC; ++j)
              st.oacc[j][dt] =
                  __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[j][u], st.oacc[j][dt], 0, 0, 0);
          }
      }
    }
    if (another) {
      pid = pid_ahead;
      if (count(ahead) > 0) {
        load_k(ahead.h, 0);
        if (NC == 1) load_v(ahead.h, 0);
      }
    }
    const int me = opaque_int(lane), n1 = me & 15, g1 = me >> 4;  // (not held over the pages)
    const auto put = [&](int c, int d, const f32x4& x, float m, float l) {
      put_columns<HD>(sh, bt, a, o, qrow, c, d, x, m, l);
    };
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      st.finish(j);
      if constexpr (NP == 1) {  // the wave has all of its columns' pages
        const int c = col0 + 16 * j + n1;
        if (c < ncol) {
#pragma unroll
          for (int dt = 0; dt < F::NDT; ++dt)
            put(c, 16 * dt + 4 * g1, st.oacc[j][dt], st.m_run[j], st.l_run[j]);
        }
      } else {
        // the states of the waves of a column group, merged in wave order, 16 columns of each
        // group at a time
        if (16 * j >= ncol) break;  // (uniform)
        __syncthreads();  // what was in LDS before has been read
        if (g1 == 0) lds.few.mm[wave][n1] = st.m_run[j], lds.few.ll[wave][n1] = st.l_run[j];
#pragma unroll
        for (int dt = 0; dt < F::NDT; ++dt)
          *reinterpret_cast<f32x4*>(&lds.few.oo[wave][n1][16 * dt + 4 * g1]) = st.oacc[j][dt];
        __syncthreads();
        for (int i = opaque_int(threadIdx.x); i < G * 16 * (HD / 4); i += kAttThr) {
          const int gr = i / (16 * (HD / 4)), c = i / (HD / 4) % 16, d = i % (HD / 4) * 4;
          const int cc = 16 * (NC * gr + j) + c;
          if (cc >= ncol) break;
          float m = lds.few.mm[gr][c], l = 0.f;
          f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int v = 1; v < NP; ++v) m = fmaxf(m, lds.few.mm[v * G + gr][c]);
#pragma unroll
          for (int v = 0; v < NP; ++v) {
            const float y = __builtin_amdgcn_exp2f(lds.few.mm[v * G + gr][c] - m);
            const f32x4 z = *reinterpret_cast<const f32x4*>(&lds.few.oo[v * G + gr][c][d]);
            l += lds.few.ll[v * G + gr][c] * y;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] += z[e] * y;
          }
          put(cc, d, x, m, l);
        }
      }
    }
    if (!another) return;
    a = ahead;
    if constexpr (NP == 1) __syncthreads();  // the queries have been read
  }
}

// ---- many columns -----------------------------------------------------------------
// Eight waves of 32 columns.  Each page is converted to bf16 once, by all threads, on
// its way into LDS (the loads of the next page are in flight meanwhile):
//   K tile   [64 keys][128 dims], 256-byte rows, 16-byte chunk c in slot c ^ (key & 15);
//   V^T tile [HD dims][64 keys], 128-byte rows, chunk c in slot c ^ swz(dim), the keys
//            of each 16 in the order 0-3, 8-11, 4-7, 12-15.
// Scores come out transposed (v_mfma_f32_32x32x16_bf16, A = K rows, B = Q^T in
// registers): lane l holds 32 scores of column l % 32, at keys 32 t + 8 (v / 4) +
// 4 (l / 32) + v % 4 of tile t; its 8 scores of 16 keys are the B operand of O^T += V^T
// P^T in the order that the V^T tile stores.  A page's P V product runs one iteration
// late, beside the next page's softmax, so K is held for two pages and V^T for three.
template <int HD, typename S>
__global__ __launch_bounds__(kTileThr) __attribute__((amdgpu_waves_per_eu(2, 2))) void
cache_attn_tile_kernel(const bf16* __restrict__ q, const uint8_t* __restrict__ kc,
                       const uint8_t* __restrict__ vc, const float* __restrict__ kv_scale,
                       Units<false, is_shaped<S>> w, Deal deal, float c_log2, S sh, AttnOut o) {
  constexpr bool SHAPED = is_shaped<S>;
  constexpr int KT = kPage * 256;       // K tile bytes
  constexpr int VT = HD * kPage * 2;    // V^T tile bytes
  constexpr int NST = HD / 16;          // score k-steps
  constexpr int NDT = HD / 32;          // output tiles
  constexpr int CPR = HD / 16;          // 16-byte pieces of a key row
  __shared__ __align__(1024) unsigned char smem[2 * KT + 3 * VT];
  __shared__ float2 cols[SHAPED ? kTileCols : 1];  // slope and place of each column
  const CacheBatch& bt = w.bt;
  const int tid = threadIdx.x, lane = lane_id();
  const int wave = SHAPED ? __builtin_amdgcn_readfirstlane(tid >> 6) : tid >> 6;
  const int qi = lane & 31, hl = lane >> 5;
  // neighbouring ranges, which share a sequence's pages, on one XCD (workgroups go
  // round the eight XCDs; the grid is a multiple of 8)
  const int range = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  long long total, off;
  int b;
  locate<kTileThr>(
      bt.B, [&](int i) { return w.group(i) * bt.H; }, deal, range, w.prefix, total, b, off);
  if (b < 0) return;
  const long long per = deal.per(total);
  long long left = min(per, total - range * per);
  int rows = w.rows(b), ctx = bt.context(b), nt = w.tiles(rows), h, t, blk0;
  int least = SHAPED ? w.least(b, ctx, rows) : 0;
  {
    const long long each = w.group(b);
    h = (int)(off / each);
    off -= h * each;
    int lo = 0, hi = nt - 1;  // the tile: largest t with before(t) <= off
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (w.before(ctx, mid, least) <= off) lo = mid;
      else hi = mid - 1;
    }
    t = lo;
    blk0 = (int)(off - w.before(ctx, t, least));
    if constexpr (SHAPED) {  // (in scalar registers)
      b = __builtin_amdgcn_readfirstlane(b);
      h = __builtin_amdgcn_readfirstlane(h);
      t = __builtin_amdgcn_readfirstlane(t);
      blk0 = __builtin_amdgcn_readfirstlane(blk0);
      left = uniform64(left);
    }
  }
  size_t slot = 2 * (size_t)range;

  // staging: thread -> 16 bytes of a key row, and 16 tokens of a value dim
  const bool stages = tid < kPage * CPR;
  int vg;
  uint32_t ks0, ks1, vs0, vs1;
  auto places = [&](int i) {
    const int krow = i / CPR, kch = i % CPR, vd = i % HD;
    vg = i / HD;
    const uint32_t kdst = krow * 256, vdst = vd * (kPage * 2);
    ks0 = kdst + (((2 * kch) ^ (krow & 15)) << 4);
    ks1 = kdst + (((2 * kch + 1) ^ (krow & 15)) << 4);
    const int vsw = (vd & 7) ^ ((vd >> 3) & 1);
    vs0 = vdst + (((2 * vg) ^ vsw) << 4);
    vs1 = vdst + (((2 * vg + 1) ^ vsw) << 4);
  };
  places(tid);
  // (formed again where they are used, if a Shape's values need the registers)
  auto fresh = [&](int x) { return SHAPED ? opaque_int(x) : x; };

  while (true) {
    const int np = w.pages(ctx, rows, t, least);
    const int blk1 = segment_end(np, blk0, left);
    const int row0 = t << w.log2r;
    const int ncol = (min(rows, (t + 1) << w.log2r) - row0) * bt.nq;
    const size_t qrow = ((size_t)h * bt.N + bt.first_row(b) + row0) * bt.nq;
    const int col = wave * 32 + qi;
    bf16x8 qf[NST];
#pragma unroll
    for (int st = 0; st < NST; ++st) {
      qf[st] = bf16x8{};
      if (col < ncol)
        qf[st] = *reinterpret_cast<const bf16x8*>(q + (qrow + col) * HD + st * 16 + fresh(hl) * 8);
    }
    const int len = min(ctx + rows, bt.cap());
    const int seen = col < ncol ? min(ctx + row0 + col / bt.nq + 1, bt.cap()) : 0;
    const int c0 = __builtin_amdgcn_readfirstlane(wave * 32);
    const int fewest =  // tokens that every column of this wave sees (see plain_tokens)
        min(plain_tokens(sh, ctx, row0 + c0 / bt.nq), bt.cap());
    if constexpr (SHAPED) {  // (read back by its own lanes)
      const Column cl = column_of(sh, bt, b, h, ctx, row0 * bt.nq + col, row0 * bt.nq + ncol);
      cols[col] = float2{cl.slope, __int_as_float(cl.place)};
    }
    // pages that a column of this wave sees some of
    int npw = c0 < ncol ? (min(ctx + row0 + min(c0 + 31, ncol - 1) / bt.nq + 1, bt.cap()) +
                           kPage - 1) / kPage : 0;
    if (SHAPED && c0 < ncol) npw = max(npw, least);
    f32x16 oacc[NDT];
#pragma unroll
    for (int i = 0; i < NDT; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) oacc[i][v] = 0.f;
    float m_run = kMFloor, l_run = 0.f, alpha = 1.f;
    bool resc = false;
    bf16x8 pf[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) pf[u] = bf16x8{};

    // page numbers and scales of 64 pages, one a lane
    int pid = -1;
    float2 psc{0.f, 0.f};
    auto pages64 = [&](int base) {
      pid = base + lane < blk1 ? bt.page(b, base + lane) : -1;
      psc = float2{0.f, 0.f};
      if (pid >= 0)
        psc = *reinterpret_cast<const float2*>(kv_scale + ((size_t)pid * bt.H + h) * 2);
    };
    u32x4 kreg, vreg;
    auto fetch = [&](int blk) {  // (pid holds the lanes of blk's 64)
      const int p = __builtin_amdgcn_readlane(pid, (blk - blk0) & 63);
      kreg = vreg = zero_u32x4();
      if (p >= 0 && stages) {
        const size_t at = ((size_t)p * bt.H + h) * (kPage * HD) + fresh(tid) * 16;
        kreg = *reinterpret_cast<const u32x4*>(kc + at);
        vreg = *reinterpret_cast<const u32x4*>(vc + at);
      }
    };
    auto stage = [&](int i, int blk, float ks, float vs) {  // i-th page of the segment
      if constexpr (SHAPED) places(opaque_int(tid));
      if ((blk + 1) * kPage > len) {  // slots past the last token hold anything
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int in = len - (blk * kPage + vg * 16 + 4 * e);
          vreg[e] &= in >= 4 ? 0xffffffffu : in <= 0 ? 0u : (1u << (8 * in)) - 1;
        }
      }
      if (!stages) return;
      unsigned char* kb = smem + (i & 1) * KT;
      unsigned char* vb = smem + 2 * KT + (i % 3) * VT;
      *reinterpret_cast<bf16x8*>(kb + ks0) = codes_to_bf16(kreg[0], kreg[1], ks);
      *reinterpret_cast<bf16x8*>(kb + ks1) = codes_to_bf16(kreg[2], kreg[3], ks);
      *reinterpret_cast<bf16x8*>(vb + vs0) = codes_to_bf16(vreg[0], vreg[2], vs);
      *reinterpret_cast<bf16x8*>(vb + vs1) = codes_to_bf16(vreg[1], vreg[3], vs);
    };
    auto scale_of = [&](float x, int blk) {
      return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), (blk - blk0) & 63));
    };
    auto pv = [&](const unsigned char* vb) {
      const int r0 = fresh(qi);
#pragma unroll
      for (int i = 0; i < NDT; ++i) {
        const int row = i * 32 + r0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const bf16x8 vf = *reinterpret_cast<const bf16x8*>(
              vb + row * 128 + (((u * 2 + hl) ^ ((row & 7) ^ ((row >> 3) & 1))) << 4));
          oacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[u], oacc[i], 0, 0, 0);
        }
      }
    };
    auto rescale = [&]() {
      if (!resc) return;
#pragma unroll
      for (int i = 0; i < NDT; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[i][v] *= alpha;
    };

    const int niter = blk1 - blk0;
    pages64(blk0);
    fetch(blk0);
    __syncthreads();  // the previous tile's last reads are done
    stage(0, blk0, scale_of(psc.x, blk0), scale_of(psc.y, blk0));
    for (int it = 0; it < niter; ++it) {
      const int blk = blk0 + it;
      const bool absent = __builtin_amdgcn_readlane(pid, it & 63) < 0;
      __syncthreads();
      if (it + 1 < niter) {
        if (((it + 1) & 63) == 0) pages64(blk + 1);
        fetch(blk + 1);
      }
      rescale();
      const unsigned char* kb = smem + (it & 1) * KT;
      const unsigned char* vb = smem + 2 * KT + ((it + 2) % 3) * VT;  // the previous page's
      if (blk >= npw || absent) {
        if (it > 0) pv(vb);
        resc = false;
#pragma unroll
        for (int u = 0; u < 4; ++u) pf[u] = bf16x8{};
      } else {
        f32x16 sacc[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[i][v] = 0.f;
        const int r0 = fresh(qi);
#pragma unroll
        for (int st = 0; st < NST; ++st)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = i * 32 + r0;
            const bf16x8 kf = *reinterpret_cast<const bf16x8*>(
                kb + row * 256 + (((st * 2 + hl) ^ (row & 15)) << 4));
            sacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[st], sacc[i], 0, 0, 0);
          }
        const bool some = (blk + 1) * kPage > fewest;
        uint64_t sees = 0;  // (SHAPED, some)
        if constexpr (SHAPED) {
          __builtin_amdgcn_sched_barrier(0);
          if (some && fresh(col) < ncol)
            sees = keys_seen(sh, bt, b, row0 + fresh(col) / bt.nq, ctx, len, blk);
          const int k4 = 4 * fresh(hl);
          const float2 sp = cols[fresh(col)];
          const Column cl{sp.x, __float_as_int(sp.y)};
          shape_scores<32>(
              sh, bt, b, ctx, rows, cl, blk * kPage + k4, !some,
              some && __builtin_amdgcn_ballot_w64(fresh(col) < ncol && ~sees != 0) != 0, sees >> k4,
              [&](int x) { return sacc[x >> 4][x & 15]; },
              [&](int x, float y) { sacc[x >> 4][x & 15] = y; },
              [](int x) { return 32 * (x >> 4) + 8 * ((x & 15) >> 2) + (x & 3); });
          __builtin_amdgcn_sched_barrier(0);
        } else if (some) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const int key = blk * kPage + i * 32 + (v >> 2) * 8 + hl * 4 + (v & 3);
              if (key >= seen) sacc[i][v] = -__builtin_inff();
            }
        }
        float mx = sacc[0][0];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int v = 0; v < 16; ++v) mx = fmaxf(mx, sacc[i][v]);
        {
          const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx),
                                                           __float_as_uint(mx), false, false);
          mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        }
        const float mxs = mx * c_log2;
        const bool need = mxs > m_run + 8.f;
        float m_new = need ? mxs : m_run;
        const float a_new = need ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
        if (SHAPED ? (some ? sees != 0 : col < ncol) : blk * kPage < seen)
          m_new = fmaxf(m_new, kMSeen);
        m_run = m_new;
        float c_page = c_log2;
        if (__builtin_amdgcn_ballot_w64(far_max(m_new))) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) sacc[i][v] = far_exponent(sacc[i][v], c_log2, m_new);
          c_page = 1.f;
          m_new = 0.f;
        }
        if (it > 0) pv(vb);
        float ps = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          bf16x8 p8;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = __builtin_amdgcn_exp2f(
                fmaf(sacc[u >> 1][(u & 1) * 8 + e], c_page, -m_new));
            ps += x;
            p8[e] = (bf16)x;
          }
          pf[u] = p8;
        }
        resc = __builtin_amdgcn_ballot_w64(need) != 0;
        alpha = a_new;
        l_run = l_run * a_new + ps;
      }
      if (it + 1 < niter)
        stage(it + 1, blk + 1, scale_of(psc.x, blk + 1), scale_of(psc.y, blk + 1));
    }
    rescale();
    pv(smem + 2 * KT + ((niter + 2) % 3) * VT);

    float l;
    if constexpr (SHAPED) {  // (the lane's number of the shuffle would be held over the pages)
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run),
                                                       __float_as_uint(l_run), false, false);
      l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    } else {
      l = l_run + __shfl_xor(l_run, 32);
    }
    const bool whole = blk0 == 0 && blk1 == np;
    const int ec = fresh(col), eh = fresh(hl);
    if (ec < ncol) {
      // lane holds dims 32 i + 8 g + 4 hl + [0, 4)
      if (whole) {
        const float inv = inv_sum(m_run, l);
        const int row = bt.first_row(b) + row0 + ec / bt.nq;
        bf16* dst = o.out + (((size_t)row * bt.H + h) * bt.nq + ec % bt.nq) * HD;
#pragma unroll
        for (int i = 0; i < NDT; ++i)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            bf16x4 x;
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] = (bf16)(oacc[i][g * 4 + v] * inv);
            *reinterpret_cast<bf16x4*>(dst + i * 32 + g * 8 + eh * 4) = x;
          }
        if (o.stat != nullptr && eh == 0)
          put_stat(sh, bt, b, h, ctx, rows, row0 * bt.nq + ec, qrow + ec, o, m_run, inv);
      } else {
        float* pt = o.part + slot * part_floats(kTileCols, HD);
#pragma unroll
        for (int i = 0; i < NDT; ++i)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(pt + ((i * 8 + g * 2 + eh) * kTileCols + ec) * 4) =
                f32x4{oacc[i][g * 4], oacc[i][g * 4 + 1], oacc[i][g * 4 + 2], oacc[i][g * 4 + 3]};
        if (eh == 0) reinterpret_cast<float2*>(pt + kTileCols * HD)[ec] = float2{m_run, l};
      }
    }
    left -= niter;
    if (left <= 0) return;
    // the next tile, group, or sequence with rows
    slot |= 1;
    blk0 = 0;
    if (++t == nt) {
      t = 0;
      if (++h == bt.H) {
        h = 0;
        do {
          if (++b >= bt.B) return;
          rows = w.rows(b);
        } while (rows <= 0);
        ctx = bt.context(b);
        nt = w.tiles(rows);
        if constexpr (SHAPED) least = w.least(b, ctx, rows);
      }
    }
  }
}

// ---- joining the parts ---------------------------------------------------------------
// The parts of a tile: ranges r0 .. r1, the first in slot 2 r0 + 1 unless the tile starts
// its range.
struct Parts {
  const float* part;
  int cols, hd, r0, r1;
  bool first_late;
  __device__ __forceinline__ const float* at(int r) const {
    return part + (2 * (size_t)r + (r == r0 && first_late)) * part_floats(cols, hd);
  }
  __device__ __forceinline__ const float2* stats(int r) const {  // (maximum, sum) by column
    return reinterpret_cast<const float2*>(at(r) + (size_t)cols * hd);
  }
};
// units u0 .. of a tile of np pages; false where one range wrote it whole
template <bool FEW, bool WIDE>
__device__ __forceinline__ bool find_parts(const Units<FEW, WIDE>& w, const Deal& deal,
                                           long long u0, int np, Parts& p) {
  const long long per = deal.per(w.prefix[w.bt.B]);
  if constexpr (FEW && WIDE) {  // (a range that starts before the pages has none of a tile's)
    p.r0 = (int)((u0 + kStartPages) / per);
    p.r1 = (int)((u0 + kStartPages + np - 1) / per);
    p.first_late = u0 > p.r0 * per;
  } else {
    p.r0 = (int)(u0 / per);
    p.r1 = (int)((u0 + np - 1) / per);
    p.first_late = u0 % per != 0;
  }
  return p.r0 != p.r1;
}

// Few columns: one workgroup per (group h, column c of sequence b).  8 groups of 32 lanes (a
// lane 4 dims) each sum every eighth part, and are then summed in order.  (A sequence's
// columns one after another in a workgroup: 13.7 us instead of 4.3 for 16 sequences of 1000 to
// 4000 tokens, 4 groups of 8 heads.)
template <int HD, typename S>
__device__ __forceinline__ void join_few(const Units<true, is_shaped<S>>& w, const Deal& deal,
                                         const S& sh,
                                         const AttnOut& o, int h, int b, int c) {
  __shared__ f32x4 osum[8][32];
  const CacheBatch& bt = w.bt;
  const int rows = w.rows(b);
  if (c >= rows * bt.nq) return;
  const int np = w.pages(bt.context(b), rows, 0, 0);
  Parts p{o.part, o.part_cols, HD};
  if (!find_parts(w, deal, w.prefix[b] + w.group(b) * h, np, p)) return;
  const int grp = threadIdx.x >> 5, l5 = threadIdx.x & 31, d = 4 * l5;
  float m = kMFloor, l = 0.f;
  for (int r = p.r0 + l5; r <= p.r1; r += 32) {
    const float2 x = p.stats(r)[c];
    const float mn = fmaxf(m, x.x);
    l = l * __builtin_amdgcn_exp2f(m - mn) + x.y * __builtin_amdgcn_exp2f(x.x - mn);
    m = mn;
  }
#pragma unroll
  for (int i = 1; i < 32; i <<= 1) {
    const float mo = __shfl_xor(m, i), lo = __shfl_xor(l, i), mn = fmaxf(m, mo);
    l = l * __builtin_amdgcn_exp2f(m - mn) + lo * __builtin_amdgcn_exp2f(mo - mn);
    m = mn;
  }
  f32x4 x{0.f, 0.f, 0.f, 0.f};
  if (d < HD) {
#pragma unroll 4
    for (int r = p.r0 + grp; r <= p.r1; r += 8) {
      const float a = __builtin_amdgcn_exp2f(p.stats(r)[c].x - m);
      const f32x4 y = *reinterpret_cast<const f32x4*>(p.at(r) + (size_t)c * HD + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += y[e] * a;
    }
  }
  osum[grp][l5] = x;
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int k = 1; k < 8; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += osum[k][l5][e];
  const float inv = inv_sum(m, l);
  if (d < HD) {
    const int row = bt.first_row(b) + c / bt.nq;
    bf16* dst = o.out + (((size_t)row * bt.H + h) * bt.nq + c % bt.nq) * HD + d;
    *reinterpret_cast<bf16x4*>(dst) = bf16x4{(bf16)(x[0] * inv), (bf16)(x[1] * inv),
                                             (bf16)(x[2] * inv), (bf16)(x[3] * inv)};
  }
  if (o.stat != nullptr && l5 == 0)
    put_stat(sh, bt, b, h, bt.context(b), rows, c,
             ((size_t)h * bt.N + bt.first_row(b)) * bt.nq + c, o, m, inv);
}

// The same for a workgroup's eight columns from c0 on, 32 lanes each, where the sequences have
// many columns and few parts: their sums need no second step, and what finds the parts is shared.
// us for 64 sequences of 32 columns, 2 or 3 parts each, 8 groups: a workgroup a column 39.
template <int HD, typename S>
__device__ __forceinline__ void join_few8(const Units<true, true>& w, const Deal& deal, const S& sh,
                                          const AttnOut& o, int h, int b, int c0) {
  const CacheBatch& bt = w.bt;
  const int rows = w.rows(b), ncol = rows * bt.nq;
  if (c0 >= ncol) return;
  const int np = w.pages(bt.context(b), rows, 0, 0);
  Parts p{o.part, o.part_cols, HD};
  if (!find_parts(w, deal, w.prefix[b] + w.group(b) * h, np, p)) return;
  const int l5 = threadIdx.x & 31, c = c0 + (threadIdx.x >> 5), d = 4 * l5;
  if (c >= ncol) return;
  float m = kMFloor, l = 0.f;
  f32x4 x{0.f, 0.f, 0.f, 0.f};
  constexpr int AT_ONCE = 4;
  for (int r0 = p.r0; r0 <= p.r1; r0 += AT_ONCE) {
    float2 z[AT_ONCE];
    f32x4 y[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      z[i] = float2{kMFloor, 0.f};
      y[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (r0 + i > p.r1) continue;
      z[i] = p.stats(r0 + i)[c];
      if (d < HD) y[i] = *reinterpret_cast<const f32x4*>(p.at(r0 + i) + (size_t)c * HD + d);
    }
    float mn = m;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) mn = fmaxf(mn, z[i].x);
    const float a0 = __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    l *= a0;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= a0;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const float a = __builtin_amdgcn_exp2f(z[i].x - m);
      l += z[i].y * a;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += y[i][e] * a;
    }
  }
  const float inv = inv_sum(m, l);
  if (d < HD) {
    const int row = c / bt.nq;
    bf16* dst =
        o.out + (((size_t)(bt.first_row(b) + row) * bt.H + h) * bt.nq + c - row * bt.nq) * HD + d;
    *reinterpret_cast<bf16x4*>(dst) = bf16x4{(bf16)(x[0] * inv), (bf16)(x[1] * inv),
                                             (bf16)(x[2] * inv), (bf16)(x[3] * inv)};
  }
  if (o.stat != nullptr && l5 == 0)
    put_stat(sh, bt, b, h, bt.context(b), rows, c,
             ((size_t)h * bt.N + bt.first_row(b)) * bt.nq + c, o, m, inv);
}

// Many columns: one workgroup per (32 columns of a tile, group h), 8 threads a column; a
// thread loads its dims of four parts at a time.
constexpr int kJoinCols = 32;

template <int HD, typename S>
__device__ __forceinline__ void join_tile(const Units<false, is_shaped<S>>& w, const Deal& deal,
                                          const S& sh, const AttnOut& o, int h, int x32) {
  constexpr int CB = kTileCols / kJoinCols, NV = HD / 32, AT_ONCE = 4;
  const CacheBatch& bt = w.bt;
  int b, t;
  if (!find_tile<256>(bt.B, x32 / CB, [&](int i) { return w.tiles(w.rows(i)); }, b, t)) return;
  const int c = x32 % CB * kJoinCols + (threadIdx.x & 31), l3 = threadIdx.x >> 5;
  const int rows = w.rows(b), ctx = bt.context(b), row0 = t << w.log2r;
  const int ncol = (min(rows, (t + 1) << w.log2r) - row0) * bt.nq;
  const int least = w.least(b, ctx, rows), np = w.pages(ctx, rows, t, least);
  Parts p{o.part, kTileCols, HD};
  if (!find_parts(w, deal, w.prefix[b] + w.group(b) * h + w.before(ctx, t, least), np, p) ||
      c >= ncol)
    return;
  float m = kMFloor, l = 0.f;
  f32x4 x[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) x[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int r0 = p.r0; r0 <= p.r1; r0 += AT_ONCE) {
    float2 z[AT_ONCE];
    f32x4 y[AT_ONCE][NV];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      z[i] = float2{kMFloor, 0.f};
#pragma unroll
      for (int k = 0; k < NV; ++k) y[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (r0 + i > p.r1) continue;
      z[i] = p.stats(r0 + i)[c];
#pragma unroll
      for (int k = 0; k < NV; ++k)
        y[i][k] = *reinterpret_cast<const f32x4*>(p.at(r0 + i) +
                                                  ((size_t)(l3 + 8 * k) * kTileCols + c) * 4);
    }
    float mn = m;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) mn = fmaxf(mn, z[i].x);
    const float a0 = __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    l *= a0;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[k][e] *= a0;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const float a = __builtin_amdgcn_exp2f(z[i].x - m);
      l += z[i].y * a;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[k][e] += y[i][k][e] * a;
    }
  }
  const float inv = inv_sum(m, l);
  const int row = bt.first_row(b) + row0 + c / bt.nq;
  bf16* dst = o.out + (((size_t)row * bt.H + h) * bt.nq + c % bt.nq) * HD;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    *reinterpret_cast<bf16x4*>(dst + 4 * (l3 + 8 * k)) =
        bf16x4{(bf16)(x[k][0] * inv), (bf16)(x[k][1] * inv), (bf16)(x[k][2] * inv),
               (bf16)(x[k][3] * inv)};
  if (o.stat != nullptr && l3 == 0)
    put_stat(sh, bt, b, h, ctx, rows, row0 * bt.nq + c,
             ((size_t)h * bt.N + bt.first_row(b) + row0) * bt.nq + c, o, m, inv);
}

// What a form's launches share: its units, how they are dealt out, and where it writes.
template <bool FEW, bool WIDE = false>
struct Form {
  Units<FEW, WIDE> w;
  Deal deal;
  AttnOut o;
};

// One launch joins both forms' parts: `many_blocks` by H workgroups those of tiles, the rest
// those of few columns.
template <int HD, typename S>
__global__ __launch_bounds__(256) void cache_join_kernel(Form<true, is_shaped<S>> few,
                                                         Form<false, is_shaped<S>> many, S sh,
                                                         int many_blocks, int few_each) {
  int x = blockIdx.x;
  const int h = blockIdx.y;
  if (x < many_blocks) {
    join_tile<HD>(many.w, many.deal, sh, many.o, h, x);
    return;
  }
  x -= many_blocks;
  if constexpr (is_shaped<S>) {
    if (few_each == 8) {
      const int each = (few.o.part_cols + 7) / 8;
      join_few8<HD>(few.w, few.deal, sh, few.o, h, x / each, x % each * 8);
      return;
    }
  }
  join_few<HD>(few.w, few.deal, sh, few.o, h, x / few.o.part_cols, x % few.o.part_cols);
}

// ---- mass ---------------------------------------------------------------------------
// A token's mass is the sum of its probabilities over the columns, each from its score
// and its column's final maximum and sum, so it follows the joining.  With few columns the
// scores were kept; else they are formed again.

// Few columns: equal ranges of the units again; a wave takes every fourth page, a lane a
// token.
__device__ __forceinline__ void mass_few(const float* __restrict__ score, const Units<true>& w,
                                         const Deal& deal, int range, int part_cols,
                                         float c_log2, const f32x2* __restrict__ stat,
                                         const float* __restrict__ mass_in,
                                         float* __restrict__ mass_out) {
  __shared__ int found;
  const CacheBatch& bt = w.bt;
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  const long long total = w.prefix[bt.B], per = deal.per(total);
  const long long unit = range * per;
  if (unit >= total) return;
  for (int i = threadIdx.x; i < bt.B; i += kAttThr)
    if (w.prefix[i] <= unit && unit < w.prefix[i + 1]) found = i;
  __syncthreads();
  int b = found;
  int left = (int)min(per, total - unit);
  int rows = w.rows(b), ctx = bt.context(b), np = w.pages(ctx, rows, 0, 0);
  const int off = (int)(unit - w.prefix[b]);
  int h = off / np, blk0 = off % np;
  score += unit * part_cols * kPage;
  while (true) {
    const int blk1 = min(np, blk0 + left), ncol = rows * bt.nq;
    float2 z{0.f, 0.f};  // of column `lane`
    if (lane < ncol) {
      const f32x2 y = stat[((size_t)h * bt.N + bt.first_row(b)) * bt.nq + lane];
      z = float2{y[0], y[1]};
    }
    for (int blk = blk0 + wave; blk < blk1; blk += kAttWaves) {
      const int page = bt.page(b, blk), slot = blk * kPage + lane;
      if (page < 0) continue;
      const size_t at = ((size_t)page * bt.H + h) * kPage + lane;
      const float before = slot < ctx ? mass_in[at] : 0.f;
      float y = 0.f;
      const float* s = score + (size_t)(blk - blk0) * part_cols * kPage + lane;
      int last = ctx, head = 0;  // the last token that column c sees
      for (int c = 0; c < ncol; ++c) {
        const float m = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(z.x), c));
        const float inv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(z.y), c));
        // (the sum of a NaN row is NaN: 0 * inv would be NaN for the tokens behind it too)
        const float x = s[c * kPage];
        const float p = __builtin_amdgcn_exp2f(inv < 0.f ? far_exponent(x, c_log2, m)
                                                         : fmaf(x, c_log2, -m)) * fabsf(inv);
        y += slot <= last ? p : 0.f;
        if (++head == bt.nq) head = 0, ++last;
      }
      if (slot < min(ctx + rows, bt.cap())) mass_out[at] = before + y;
    }
    left -= blk1 - blk0;
    score += (size_t)(blk1 - blk0) * part_cols * kPage;
    if (left <= 0) return;
    blk0 = 0;
    if (++h == bt.H) {
      h = 0;
      do {
        if (++b >= bt.B) return;
        rows = w.rows(b);
      } while (rows <= 0);
      ctx = bt.context(b);
      np = w.pages(ctx, rows, 0, 0);
    }
  }
}

// The same for shaped calls, whose scores are -inf for the tokens that a column does not see.
template <typename S>
__device__ __forceinline__ void mass_scores(const float* __restrict__ score_base,
                                            const Units<true, true>& w, const Deal& deal, int range,
                                            int part_cols, float c_log2, const S& sh,
                                            const f32x4* __restrict__ stat,
                                            const float* __restrict__ mass_in,
                                            float* __restrict__ mass_out) {
  const CacheBatch& bt = w.bt;
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  Segment<true> a;
  if (!a.first(w, deal, range)) return;
  do {
    const int ncol = a.rows * bt.nq, len = min(a.ctx + a.rows, bt.cap());
    f32x4 z{0.f, 0.f, 0.f, 0.f};  // of column `lane`
    if (lane < ncol) z = stat[((size_t)a.h * bt.N + bt.first_row(a.b)) * bt.nq + lane];
    for (int blk = a.blk0 + wave; blk < a.blk1; blk += kAttWaves) {
      const int page = bt.page(a.b, blk), slot = blk * kPage + lane;
      if (page < 0) continue;
      const size_t at = ((size_t)page * bt.H + a.h) * kPage + lane;
      const float before = slot < a.ctx ? mass_in[at] : 0.f;
      const float* s = score_base + score_page(bt, a.b, a.h, blk) * part_cols * kPage + lane;
      float y = 0.f;
      for (int c = 0; c < ncol; ++c) {
        const float m = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(z[0]), c));
        const float inv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(z[1]), c));
        const float x = s[c * kPage];
        float p = __builtin_amdgcn_exp2f(inv < 0.f ? far_exponent(x, c_log2, m)
                                                   : fmaf(x, c_log2, -m)) * fabsf(inv);
        // (a NaN row counts for the tokens that it sees alone)
        if (inv != inv && (keys_seen(sh, bt, a.b, c / bt.nq, a.ctx, len, blk) >> lane & 1) == 0)
          p = 0.f;
        y += p;
      }
      if (slot < len) mass_out[at] = before + y;
    }
  } while (a.next(w));
}

// Shaped calls of more than 16 columns, or whose scores take too much room: the scores are
// formed again from the keys alone, a page a wave, as in the attention; the probabilities of a
// lane's 16 keys are summed over its tiles' columns and then over the 16 lanes of a key.
// us for 48 trees of 25 rows (hd 96, 100 to 4096 tokens): 30; as sequences of many columns
// (mass_any) 53.
template <int HD, typename S>
__global__ __launch_bounds__(kAttThr, 2) void cache_mass_shaped_kernel(
    const bf16* __restrict__ q, const uint8_t* __restrict__ kc, const float* __restrict__ kv_scale,
    Units<true, true> w, Deal deal, float c_log2, S sh, const f32x4* __restrict__ stat,
    const float* __restrict__ mass_in, float* __restrict__ mass_out) {
  using F = PageFrags<HD>;
  constexpr int MT = kShapedCols / 16;
  __shared__ bf16x8 qs[MT][F::NST][kWave];
  __shared__ f32x4 zs[MT * 16];
  const CacheBatch& bt = w.bt;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  Segment<true> a;
  if (!a.first(w, deal, blockIdx.x)) return;
  do {
    const int ncol = a.rows * bt.nq, len = min(a.ctx + a.rows, bt.cap());
    const int tiles = (ncol + 15) / 16;
    const size_t qrow = ((size_t)a.h * bt.N + bt.first_row(a.b)) * bt.nq;
    int pid = -1;  // of the wave's next 64 pages, one a lane
    auto pages64 = [&](int blk) {
      const int mine = blk + kAttWaves * lane;
      pid = mine < a.blk1 ? bt.page(a.b, mine) : -1;
    };
    F f;
    float ks = 0.f, before = 0.f;
    auto load = [&](int i) {  // (an absent page loads page 0)
      const size_t pg = (size_t)max(__builtin_amdgcn_readlane(pid, i & 63), 0) * bt.H + a.h;
      ks = kv_scale[pg * 2];
      f.load_k(kc + pg * (kPage * HD), lane);
      before = mass_in[pg * kPage + lane];
    };
    if (a.blk0 + wave < a.blk1) pages64(a.blk0 + wave), load(0);
    __syncthreads();  // the last segment's queries have been read
    for (int j = wave; j < tiles; j += kAttWaves) {
      bf16x8 qf[F::NST];
      load_q<HD>(q + qrow * HD, 16 * j + n, ncol, g, qf);
#pragma unroll
      for (int st = 0; st < F::NST; ++st) qs[j][st][lane] = qf[st];
    }
    for (int c = threadIdx.x; c < tiles * 16; c += kAttThr)
      zs[c] = c < ncol ? stat[qrow + c] : f32x4{0.f, 0.f, 0.f, 0.f};
    const int fewest = min(plain_tokens(sh, a.ctx, 0), bt.cap());
    __syncthreads();
    int i = 0;
    for (int blk = a.blk0 + wave; blk < a.blk1; blk += kAttWaves, ++i) {
      const int page = __builtin_amdgcn_readlane(pid, i & 63);
      const bool some = (blk + 1) * kPage > fewest;
      const float was = before;
      float sum[16];
#pragma unroll
      for (int x = 0; x < 16; ++x) sum[x] = 0.f;
      bf16x8 kf[4][F::NST];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int st = 0; st < F::NST; ++st) kf[t][st] = f.key(t, st, ks);
      if (blk + kAttWaves < a.blk1) {
        if (((i + 1) & 63) == 0) pages64(blk + kAttWaves);
        load(i + 1);
      }
      if (page < 0) continue;
      for (int j = 0; j < tiles; ++j) {
        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < F::NST; ++st) {
          const bf16x8 qf = qs[j][st][lane];
#pragma unroll
          for (int t = 0; t < 4; ++t)
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][st], qf, s[t], 0, 0, 0);
        }
        const f32x4 z = zs[16 * j + n];
        uint64_t sees = 0;
        bool masked = false;
        if (some) {
          if (16 * j + n < ncol)
            sees = keys_seen(sh, bt, a.b, (16 * j + n) / bt.nq, a.ctx, len, blk);
          masked = __builtin_amdgcn_ballot_w64(~sees != 0) != 0;
          sees >>= 16 * g;
        }
        shape_scores<16>(
            sh, bt, a.b, a.ctx, a.rows, Column{z[2], __float_as_int(z[3])}, blk * kPage + 16 * g,
            !some, masked, sees, [&](int x) { return s[x >> 2][x & 3]; },
            [&](int x, float y) { s[x >> 2][x & 3] = y; }, [](int x) { return x; });
        float m = z[0], c_tile = c_log2;
        if (__builtin_amdgcn_ballot_w64(z[1] < 0.f)) {
#pragma unroll
          for (int x = 0; x < 16; ++x) s[x >> 2][x & 3] = far_exponent(s[x >> 2][x & 3], c_log2, m);
          m = 0.f;
          c_tile = 1.f;
        }
        const float inv = fabsf(z[1]);
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[x >> 2][x & 3], c_tile, -m));
          // (a NaN row counts for the tokens that it sees alone)
          sum[x] = fmaf(p, masked && (sees >> x & 1) == 0 ? 0.f : inv, sum[x]);
        }
      }
      // over the 16 lanes of a key: each step halves the keys of a lane, which ends with key n
      auto fold = [&](auto halfv) {
        constexpr int half = decltype(halfv)::value;
        const bool up = (n & half) != 0;
#pragma unroll
        for (int x = 0; x < half; ++x) {
          const float mine = up ? sum[x + half] : sum[x], other = up ? sum[x] : sum[x + half];
          sum[x] = mine + __shfl_xor(other, half);
        }
      };
      fold(std::integral_constant<int, 8>{});
      fold(std::integral_constant<int, 4>{});
      fold(std::integral_constant<int, 2>{});
      fold(std::integral_constant<int, 1>{});
      const int slot = blk * kPage + lane;
      if (slot < len)
        mass_out[((size_t)page * bt.H + a.h) * kPage + lane] = (slot < a.ctx ? was : 0.f) + sum[0];
    }
  } while (a.next(w));
}

// Any columns: a workgroup takes pairs of pages, a wave 32 of their keys, held in
// registers as A operand of v_mfma_f32_32x32x16_bf16.  Tiles of 32 columns go by through a
// ring of four in LDS, filled by LDS-DMA three tiles ahead (256-byte rows, 16-byte chunk
// c in slot c ^ (column & 15); the columns' maxima and sums behind them), since a tile
// takes less time than a load.  Four workgroups fit a CU: many of them do little (a
// decoding sequence's pages) and wait for their first loads.
// us of this kernel for 4096 rows over 4096 tokens, 8 groups of two heads, and for a 512-row
// chunk beside 16 decoding sequences: tiles through registers, one ahead 224 and 46; the
// ring 176 and 40 (two tiles at a time 170, with registers for three workgroups); equal
// ranges of the pairs that exist, so that no launch follows the tables' width, 183 and 25.
constexpr int kMassThr = 256, kMassCols = 32;
constexpr int kMassStages = 4;

template <int HD, typename S>
__device__ __forceinline__ void mass_any(const bf16* __restrict__ q, const uint8_t* __restrict__ kc,
                                         const float* __restrict__ kv_scale,
                                         const Units<false, is_shaped<S>>& w, const Deal& deal,
                                         int range, float c_log2, const S& sh,
                                         const Stat<S>* __restrict__ stat,
                                         const float* __restrict__ mass_in,
                                         float* __restrict__ mass_out) {
  constexpr bool SHAPED = is_shaped<S>;
  constexpr int NST = HD / 16, ST = sizeof(Stat<S>);
  // bytes of a tile, and with its statistics
  constexpr int QT = kMassCols * 256, STAGE = QT + kMassCols * ST;
  constexpr int QI = QT / 1024 / (kMassThr / kWave);     // 1 KB DMA instructions of a wave
  __shared__ __align__(1024) unsigned char smem[kMassStages * STAGE];
  __shared__ float sum[kMassThr / kWave][32];
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int qi = lane & 31, hl = lane >> 5;
  const CacheBatch& bt = w.bt;
  // pairs of a sequence, all groups; numbered by sequence, pair and group
  auto pairs = [&](int i) -> long long {
    const int n = w.rows(i);
    const int len = min(bt.context(i) + n, bt.cap());
    return n > 0 ? (long long)((len + 2 * kPage - 1) / (2 * kPage)) * bt.H : 0;
  };
  long long total, first;
  int b;
  locate<kMassThr>(bt.B, pairs, deal, range, nullptr, total, b, first);
  if (b < 0) return;
  const long long per = deal.per(total);
  // (in scalar registers: the keys and sums fill the others)
  b = __builtin_amdgcn_readfirstlane(b);
  int off = __builtin_amdgcn_readfirstlane((int)first);  // (of 2^17 pairs in 64 groups)
  int left = __builtin_amdgcn_readfirstlane((int)min(per, total - range * per));
  while (true) {
    const int h = off % bt.H, blk0 = off / bt.H * 2;
    const int rows = w.rows(b), ctx = bt.context(b);
    const int len = min(ctx + rows, bt.cap());
    const int key0 = blk0 * kPage + wave * 32;  // the wave's first key
    const int page = bt.page(b, key0 / kPage);
    const bool works = page >= 0 && key0 < len;  // (wave-uniform)
    const size_t pg = (size_t)max(page, 0) * bt.H + h;
    // key qi; in steps st, st + 1 the lane halves hold dims 32 (st / 2) + 16 hl + 8 (st % 2)
    bf16x8 kf[NST];
    {
      const float ks = works ? kv_scale[pg * 2] : 0.f;
      const uint8_t* row = kc + pg * (kPage * HD) + ((wave & 1) * 32 + qi) * HD + 16 * hl;
#pragma unroll
      for (int st = 0; st < NST; st += 2) {
        u32x4 x = zero_u32x4();
        if (works) x = *reinterpret_cast<const u32x4*>(row + 16 * st);
        kf[st] = codes_to_bf16(x[0], x[1], ks);
        kf[st + 1] = codes_to_bf16(x[2], x[3], ks);
      }
    }
    // arrived before the loop, whose loads are counted
#pragma unroll
    for (int st = 0; st < NST; ++st) asm volatile("" ::"v"(kf[st]));
    const int ncol = rows * bt.nq;
    const size_t qrow = ((size_t)h * bt.N + bt.first_row(b)) * bt.nq;
    float acc[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
    // tiles before the first column that sees the pages are left out
    long long c_first = (long long)max(blk0 * kPage - ctx, 0) * bt.nq;
    if constexpr (SHAPED)
      if (blk0 < w.least(b, ctx, rows)) c_first = 0;
    const int t0 = (int)(c_first / kMassCols), t1 = (ncol + kMassCols - 1) / kMassCols;
    // columns past the last read zeros: no query, maximum 0 and 1 / sum 0
    const __amdgpu_buffer_rsrc_t rq = make_rsrc_u(q + qrow * HD, (uint32_t)ncol * (HD * 2));
    const __amdgpu_buffer_rsrc_t rz = make_rsrc_u(stat + qrow, (uint32_t)ncol * (uint32_t)ST);
    rsrc_settle(rq, rz);
    uint32_t qoff[QI];
#pragma unroll
    for (int i = 0; i < QI; ++i) {
      const int c = 4 * (wave * QI + i) + (lane >> 4), ch = (lane & 15) ^ (c & 15);
      qoff[i] = ch < HD / 8 ? (uint32_t)(c * (HD * 2) + ch * 16) : kOob;
    }
    const uint32_t lds = lds_addr(smem);
    auto issue = [&](int t) {
      const uint32_t to = lds + (uint32_t)((t & (kMassStages - 1)) * STAGE);
      const uint32_t step = (uint32_t)t * (kMassCols * HD * 2);
#pragma unroll
      for (int i = 0; i < QI; ++i)
        dma16(rq, qoff[i] + step, to + (uint32_t)wave_u * (QI * 1024), i * 1024);
      // (every wave loads the statistics, so that all count the same)
#pragma unroll
      for (int i = 0; i < ST / 8; ++i)
        dma4(rz, (uint32_t)t * (kMassCols * ST) + i * 256u + lane * 4u, to, QT + i * 256);
    };
    constexpr int OPS = QI + ST / 8;  // DMA instructions of a wave and tile
#pragma unroll
    for (int i = 0; i < kMassStages - 1; ++i)
      if (t0 + i < t1) issue(t0 + i);
    for (int t = t0; t < t1; ++t) {
      // this tile has landed for every wave, and the one before is done with
      if (t + 2 < t1) vm_barrier<2 * OPS>();
      else if (t + 1 < t1) vm_barrier<OPS>();
      else vm_barrier<0>();
      if (t + kMassStages - 1 < t1) issue(t + kMassStages - 1);
      const unsigned char* tile = smem + (t & (kMassStages - 1)) * STAGE;
      if (works) {
        const Stat<S> zs = *reinterpret_cast<const Stat<S>*>(tile + QT + qi * ST);
        float2 z{zs[0], zs[1]};
        const uint32_t qat = (uint32_t)((t & (kMassStages - 1)) * STAGE + qi * 256 +
                                        (((2 * hl) ^ (qi & 15)) << 4));
        // (formed before the products, so that nothing waits for it behind them)
        uint64_t special = __builtin_amdgcn_ballot_w64(!(z.y >= 0.f));
        asm volatile("" : "+s"(special));
        f32x16 x;
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = 0.f;
#pragma unroll
        for (int st = 0; st < NST; ++st) {
          // chunk 4 (st / 2) + 2 hl + st % 2; in bits 4 to 7 of the address, for all stages
          const bf16x8 qf = *reinterpret_cast<const bf16x8*>(
              smem + (qat ^ (uint32_t)((4 * (st / 2) + st % 2) << 4)));
          x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[st], qf, x, 0, 0, 0);
        }
        const int col = t * kMassCols + qi;
        if constexpr (SHAPED) {
          const int i0 = t * kMassCols / bt.nq;
          const bool all = plain_tokens(sh, ctx, i0) >= min(key0 + 32, len + 1);
          uint64_t sees = 0;
          bool masked = false;
          if (!all) {
            if (col < ncol) sees = keys_seen(sh, bt, b, col / bt.nq, ctx, len, key0 / kPage);
            masked = __builtin_amdgcn_ballot_w64(~sees != 0) != 0;
            sees >>= (wave & 1) * 32 + 4 * hl;
          }
          shape_scores<16>(
              sh, bt, b, ctx, rows, Column{zs[2], __float_as_int(zs[3])}, key0 + 4 * hl, all,
              masked, sees, [&](int v) { return x[v]; }, [&](int v, float y) { x[v] = y; },
              [](int v) { return 8 * (v >> 2) + (v & 3); });
        } else if (ctx + t * kMassCols / bt.nq + 1 < min(key0 + 32, len + 1)) {
          // (the tile's first column sees the fewest)
          const int seen = col < ncol ? ctx + col / bt.nq + 1 : 0;
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (key0 + 8 * (v >> 2) + 4 * hl + (v & 3) >= seen) x[v] = -__builtin_inff();
        }
        float c_tile = c_log2;
        if (special) {
          // a NaN row counts, as NaN, for the tokens that it sees alone (0 * NaN is NaN)
          if (z.y != z.y) {
            const int seen = ctx + col / bt.nq + 1;
            uint64_t sees = 0;
            if constexpr (SHAPED)
              sees = keys_seen(sh, bt, b, col / bt.nq, ctx, len, key0 / kPage) >>
                     ((wave & 1) * 32 + 4 * hl);
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (SHAPED ? (sees >> (8 * (v >> 2) + (v & 3)) & 1) != 0
                         : key0 + 8 * (v >> 2) + 4 * hl + (v & 3) < seen)
                acc[v] = z.y;
            z.y = 0.f;
          }
#pragma unroll
          for (int v = 0; v < 16; ++v) x[v] = far_exponent(x[v], c_log2, z.x);
          c_tile = 1.f;
          z = float2{0.f, fabsf(z.y)};
        }
#pragma unroll
        for (int v = 0; v < 16; ++v)
          acc[v] = fmaf(__builtin_amdgcn_exp2f(fmaf(x[v], c_tile, -z.x)), z.y, acc[v]);
      }
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) acc[v] += __shfl_xor(acc[v], o);
      if (qi == 0) sum[wave][8 * (v >> 2) + 4 * hl + (v & 3)] = acc[v];
    }
    __syncthreads();
    const int slot = key0 + lane;
    if (works && lane < 32 && slot < len) {
      const size_t at = pg * kPage + (wave & 1) * 32 + lane;
      mass_out[at] = (slot < ctx ? mass_in[at] : 0.f) + sum[wave][lane];
    }
    if (--left == 0) return;
    __syncthreads();  // the ring and the sums have been read
    if (++off == pairs(b)) {
      off = 0;
      do {
        if (++b >= bt.B) return;
      } while (w.rows(b) <= 0);
    }
  }
}

// One launch for both: `any_ranges` workgroups for the sequences of `any`, the rest for
// those of few columns, from their scores.
template <int HD, typename S>
__global__ __launch_bounds__(kMassThr, S::kTransforms ? 3 : 4) void cache_mass_kernel(
    const bf16* __restrict__ q, const uint8_t* __restrict__ kc, const float* __restrict__ kv_scale,
    Units<false, is_shaped<S>> any, int any_ranges, Form<true, is_shaped<S>> few,
    const float* __restrict__ score, float c_log2, S sh, const Stat<S>* __restrict__ stat,
    const float* __restrict__ mass_in, float* __restrict__ mass_out) {
  static_assert(kMassThr == kAttThr, "one workgroup size");
  const int x = blockIdx.x;
  if (x >= any_ranges) {
    const Deal deal{few.deal.ranges, few.deal.least, 0};
    if constexpr (is_shaped<S>)
      mass_scores(score, few.w, deal, x - any_ranges, few.o.part_cols, c_log2, sh, stat, mass_in,
                  mass_out);
    else
      mass_few(score, few.w, deal, x - any_ranges, few.o.part_cols, c_log2, stat, mass_in,
               mass_out);
    return;
  }
  mass_any<HD>(q, kc, kv_scale, any, Deal{any_ranges, 1, 0}, x, c_log2, sh, stat, mass_in,
               mass_out);
}

// Host side of the two forms: ranges (workgroups) and scratch.
constexpr int kFewLeast = 4;   // pages of a range at least: one for each wave
// With 128 columns every wave takes every page.  us for 64 rows of two heads over 300, 1500 and
// 5000 tokens, 8 groups: 22 22 26, with four 28 24 28.
constexpr int kFullLeast = 2;
constexpr int kManyLeast = 2;
// Pages of the tables from which a shaped call of 65 to 128 columns whose other sequences have few
// takes both forms: in the 128-column one each wave would form 128 columns of every sequence.  us
// for one tree of 64 rows of two heads beside single rows, 8 groups, the 128-column form and both,
// in brackets with the mass: 15 rows over 256 to 2000 tokens (4096 pages) 35 39 (55 52), over 256
// to 8192 (16384) 63 62 (102 81), 63 rows over 256 to 2000 84 61 (133 82), over 256 to 8192 224 150
// (354 202).  Of 32 rows (64 columns, with the 64-column form) 63 rows 144 147, 15 rows 40 59.
constexpr long long kMixedPages = 16384;
constexpr int kJoinParts = 24;  // parts up to which eight columns are joined by a workgroup
// The scores of few columns are kept for the mass where the tables' room for them is up to
// this many bytes of workspace; beyond, they are formed again.  us kept and formed again, 8
// groups of two heads: 16 sequences of 1000 to 4000 tokens 35 53, 64 of 1000 to 8000 155 264,
// one of 100000 68 112.
constexpr size_t kScoreBytes = (size_t)1 << 30;

// One form of a call: what it launches and where its scratch is.
struct FormPlan {
  bool on;
  int lo, hi;                 // columns of its sequences
  int ranges, least, cols, log2r, tiles;
  size_t prefix, part;
};
struct AttnPlan {
  FormPlan few, many;
  int few_cols;  // that the few-column form holds
  bool scores;
  size_t stat, score, total;
};

AttnPlan attn_plan(int H, int B, int N, int nq, int hd, int max_blocks, int max_rows, bool mass,
                   bool shaped) {
  AttnPlan p{};
  const long long most = (long long)max_rows * nq;
  const long long pages = (long long)B * H * max_blocks;
  // Both forms where the sequences beside the longest have few columns on average (us for a
  // 512-row chunk beside 16 decoding sequences, with mass: 85, and 114 in the second form
  // alone); where they are all chunks the first would be a launch for nothing.
  const bool mixed = B > 1 && (long long)(N - max_rows) * nq <= kFewCols * (B - 1LL);
  p.few_cols = kFewCols;
  if (shaped && most <= kShapedCols &&
      !(mixed && most > kShapedCols / 2 && pages >= kMixedPages))
    while (p.few_cols < most) p.few_cols *= 2;
  p.few.on = most <= p.few_cols || mixed;
  p.many.on = most > p.few_cols;
  p.few.hi = p.few_cols;
  p.many.lo = p.few.on ? p.few_cols : 0;
  p.many.hi = INT_MAX;
  auto take = [&](size_t& field, size_t bytes) {
    field = p.total;
    p.total = align_up(p.total + bytes, 256);
  };
  auto scratch = [&](FormPlan& f, size_t part_bytes) {
    take(f.prefix, (size_t)(B + 1) * 8);
    take(f.part, part_bytes);
  };
  auto least_of = [](int few_cols) { return few_cols == kShapedCols ? kFullLeast : kFewLeast; };
  auto ranges_of = [&](int few_cols) {
    return (int)std::min<long long>((few_cols <= 32 ? 4LL : 2LL) * kCus,
                                    (pages + least_of(few_cols) - 1) / least_of(few_cols));
  };
  auto parts_of = [&](int ranges, int cols) {
    return 2 * (size_t)ranges * part_floats(cols, hd) * 4;
  };
  p.few.cols = (int)std::min<long long>(p.few_cols, most);
  p.few.least = least_of(p.few_cols);
  p.few.ranges = ranges_of(p.few_cols);
  p.many.cols = kTileCols;
  p.many.ranges = kCus;
  p.many.least = kManyLeast;
  while ((2 << p.many.log2r) * nq <= kTileCols) ++p.many.log2r;
  // tiles of the batch: at most n / 2^log2r, rounded up, of each sequence
  p.many.tiles = (int)std::min<long long>(N, ((long long)N >> p.many.log2r) + B);
  // Every region has room for any call of no larger sizes, whichever forms and widths that takes,
  // so that a caller's one workspace for its largest batch serves the smaller ones: the parts of
  // each width that so many columns or fewer take, the scores of the first 16 columns.
  size_t few_parts = 0;
  for (int w = kFewCols; w <= (shaped ? kShapedCols : kFewCols); w *= 2)
    if (w == kFewCols || most > w / 2)
      few_parts = std::max(few_parts,
                           parts_of(ranges_of(w), (int)std::min<long long>(w, most)));
  scratch(p.few, few_parts);
  if (most > (shaped ? kShapedCols / 2 : kFewCols))
    scratch(p.many, parts_of(p.many.ranges, p.many.cols));
  if (mass) {
    take(p.stat, (size_t)H * N * nq * (shaped ? sizeof(Stat<Shape<true>>) : sizeof(Stat<NoShape>)));
    const size_t bytes = (size_t)pages * std::min<long long>(kFewCols, most) * kPage * 4;
    p.scores = p.few.on && p.few_cols == kFewCols && bytes <= kScoreBytes;
    take(p.score, std::min(bytes, kScoreBytes));
  }
  return p;
}

template <bool T>
Shape<T> shape_of(const CacheScores& a, int hd) {
  constexpr double kLog2e = 1.4426950408889634;
  Shape<T> sh{};
  sh.a = a;
  sh.scale = (float)(kLog2e / sqrt((double)hd));
  if (a.cap != 0.f) {
    const double k = 1.0 / (a.cap * sqrt((double)hd));
    sh.cap = (float)(a.cap * kLog2e);
    sh.x_of = (float)k;
    // (beyond, the squares and coefficients could leave fp32)
    const bool fits = a.cap >= 0x1p-8f && a.cap <= 0x1p10f;
    sh.bound = fits ? (float)(kTanhBound / k) : -1.f;
    sh.near = fits ? (float)(kTanhNear / k) : -1.f;
    auto factor = [&](double c, int i) {
      return fits ? (float)(a.cap * kLog2e * c * pow(k, 2 * i + 1)) : 0.f;
    };
    for (int i = 0; i < 5; ++i) sh.poly[i] = factor(kTanhPoly[i], i);
    for (int i = 0; i < 3; ++i) sh.low[i] = factor(kTanhLow[i], i);
  }
  return sh;
}
}  // namespace

size_t cache_attention_scratch_bytes(int H, int B, int N, int nq, int hd, int max_blocks,
                                     int max_rows, bool mass, bool shaped) {
  return attn_plan(H, B, N, nq, hd, max_blocks, max_rows, mass, shaped).total;
}

hipError_t launch_cache_attention(const CacheArgs& a, int nq, int N, int max_rows, const void* q,
                                  const int32_t* row_start, const float* mass_in, float* mass_out,
                                  void* out, void* scratch, hipStream_t s,
                                  const CacheScores* scores) {
  const CacheBatch bt{a.H, a.B, N, nq, a.n_pages, a.max_blocks, a.block_table, a.length, row_start};
  const AttnPlan p = attn_plan(a.H, a.B, N, nq, a.hd, a.max_blocks, max_rows, mass_out != nullptr,
                               scores != nullptr);
  unsigned char* base = static_cast<unsigned char*>(scratch);
  const bf16* qb = static_cast<const bf16*>(q);
  void* stat = mass_out != nullptr ? base + p.stat : nullptr;
  float* score = p.scores ? reinterpret_cast<float*>(base + p.score) : nullptr;
  const Reach reach =
      scores != nullptr ? Reach{scores->prefix, scores->tree != nullptr} : Reach{nullptr, false};
  auto form = [&](const FormPlan& f, int round, auto few, auto wide) {
    return Form<decltype(few)::value, decltype(wide)::value>{
        {bt, max_rows, f.log2r, f.lo, f.hi, reach, reinterpret_cast<long long*>(base + f.prefix)},
        {f.ranges, f.least, round},
        {static_cast<bf16*>(out), stat, reinterpret_cast<float*>(base + f.part), f.cols}};
  };
  auto go = [&](auto hdv, auto sh) {
    constexpr int HD = decltype(hdv)::value;
    using S = decltype(sh);
    constexpr std::integral_constant<bool, is_shaped<S>> wide;
    const auto few = form(p.few, std::min(p.few.ranges, 2 * kCus), std::true_type{}, wide);
    const auto many = form(p.many, 0, std::false_type{}, wide);
    float c_log2 = 1.4426950408889634f / sqrtf((float)a.hd);
    if constexpr (is_shaped<S>)
      if (S::kTransforms) c_log2 = 1.f;
    if (p.few.on) {
      if constexpr (is_shaped<S>) {
        ProfileScope ps("cache_attn_shaped", s);
        auto launch = [&](auto kernel) {
          FOE_LAUNCH(kernel, dim3(few.deal.ranges), dim3(kAttThr), 0, s, qb, a.k, a.v, a.kv_scale,
                     few.w, few.deal, c_log2, sh, few.o, score);
        };
        if (p.few_cols == 16) launch(cache_attn_shaped_kernel<HD, 1, 1, S>);
        else if (p.few_cols == 32) launch(cache_attn_shaped_kernel<HD, 2, 1, S>);
        else if (p.few_cols == 64) launch(cache_attn_shaped_kernel<HD, 2, 2, S>);
        else launch(cache_attn_shaped_kernel<HD, 2, 4, S>);
      } else {
        ProfileScope ps("cache_attn_few", s);
        FOE_LAUNCH(cache_attn_few_kernel<HD>, dim3(few.deal.ranges), dim3(kAttThr), 0, s, qb, a.k,
                   a.v, a.kv_scale, few.w, few.deal, c_log2, few.o, score);
      }
    }
    if (p.many.on) {
      ProfileScope ps("cache_attn_tile", s);
      FOE_LAUNCH((cache_attn_tile_kernel<HD, S>), dim3(many.deal.ranges), dim3(kTileThr), 0, s, qb,
                 a.k, a.v, a.kv_scale, many.w, many.deal, c_log2, sh, many.o);
    }
    {
      ProfileScope ps("cache_join", s);
      const int many_blocks = p.many.on ? p.many.tiles * (kTileCols / kJoinCols) : 0;
      // with many parts of a (sequence, group) a column's are shared by a workgroup
      const int few_each = is_shaped<S> && p.few.cols >= 8 &&
                                   few.deal.ranges <= (long long)kJoinParts * a.B * a.H
                               ? 8
                               : 1;
      const int few_blocks = p.few.on ? a.B * ceil_div(few.o.part_cols, few_each) : 0;
      FOE_LAUNCH((cache_join_kernel<HD, S>), dim3(many_blocks + few_blocks, a.H), dim3(256), 0, s,
                 few, many, sh, many_blocks, few_each);
    }
    if constexpr (is_shaped<S>) {
      if (mass_out != nullptr && !p.many.on && score == nullptr) {
        ProfileScope ps("cache_mass", s);
        Deal deal = few.deal;
        deal.round = 0;
        FOE_LAUNCH((cache_mass_shaped_kernel<HD, S>), dim3(deal.ranges), dim3(kAttThr), 0, s, qb,
                   a.k, a.kv_scale, few.w, deal, c_log2, sh, static_cast<const f32x4*>(stat),
                   mass_in, mass_out);
        return;
      }
    }
    if (mass_out != nullptr) {
      ProfileScope ps("cache_mass", s);
      // without scores the sequences of both forms; at most 16 workgroups a CU: four rounds,
      // which evens out what pages near a chunk's end have less to do
      auto any = many.w;
      if (score == nullptr) any.lo = 0;
      const long long pairs = (long long)ceil_div(a.max_blocks, 2) * a.H * a.B;
      const int any_ranges =
          p.many.on || score == nullptr ? (int)std::min(16LL * kCus, pairs) : 0;
      FOE_LAUNCH((cache_mass_kernel<HD, S>),
                 dim3(any_ranges + (score != nullptr ? few.deal.ranges : 0)), dim3(kMassThr), 0, s,
                 qb, a.k, a.kv_scale, any, any_ranges, few, score, c_log2, sh,
                 static_cast<const Stat<S>*>(stat), mass_in, mass_out);
    }
  };
  auto with = [&](auto sh) {
    if (a.hd == 96) go(std::integral_constant<int, 96>{}, sh);
    else go(std::integral_constant<int, 128>{}, sh);
  };
  if (scores == nullptr) with(NoShape{});
  else if (scores->cap != 0.f || scores->slope != nullptr) with(shape_of<true>(*scores, a.hd));
  else with(shape_of<false>(*scores, a.hd));
  return hipGetLastError();
}

}  // namespace foe
