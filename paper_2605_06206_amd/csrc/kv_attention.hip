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

// ---- dealing out the work -------------------------------------------------------

// The units of a batch in a form, numbered by sequence, group, tile and page.  A tile of
// many columns has 2^log2r rows, tile t reaches page ceil((ctx + last row + 1) / 64), and
// the sums over tiles are closed forms (which count pages past the table's end too).
template <bool FEW>
struct Units {
  CacheBatch bt;
  int max_rows;
  int log2r;   // (many)
  int lo, hi;  // columns that a sequence of this form has: lo < columns <= hi
  long long* prefix;  // [B + 1]: units before each sequence, and in all (for the launches after)

  // rows of sequence b in this form
  __device__ __forceinline__ int rows(int b) const {
    const int n = min(bt.rows(b), max_rows);
    return n * bt.nq > lo && n * bt.nq <= hi ? n : 0;
  }
  __device__ __forceinline__ int tiles(int n) const { return (n + (1 << log2r) - 1) >> log2r; }
  // pages of the tiles before tile t (t < tiles)
  __device__ __forceinline__ long long before(int ctx, int t) const {
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
  __device__ __forceinline__ int pages(int ctx, int n, int t) const {
    if (FEW) return min((ctx + n + kPage - 1) / kPage, bt.max_blocks);
    return (ctx + min((t + 1) << log2r, n) + kPage - 1) / kPage;
  }
  // units of one group of sequence b
  __device__ __forceinline__ long long group(int b) const {
    const int n = rows(b);
    if (n <= 0) return 0;
    const int ctx = bt.context(b), t = FEW ? 0 : tiles(n) - 1;
    return (FEW ? 0 : before(ctx, t)) + pages(ctx, n, t);
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
  // scores of the page: s[t][v] = key 16 g + 4 t + v of column n
  __device__ __forceinline__ void scores(const bf16x8* qf, float ks, f32x4* s) const {
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < NST; ++st)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const u32x4 w = k[t][st / 2];
        const bf16x8 a = codes_to_bf16(w[2 * (st % 2)], w[2 * (st % 2) + 1], ks);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[st], s[t], 0, 0, 0);
      }
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
  float2* stat;      // of each column (see column_stat), or null
  float* part;
  int part_cols;
};

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
      if (d == 0 && o.stat != nullptr) o.stat[qrow + c] = column_stat(m, inv);
    } else {
      pt[i] = x;
      if (d == 0) reinterpret_cast<float2*>(pt + o.part_cols * HD)[c] = float2{m, l};
    }
  }
}

template <int HD>
__global__ __launch_bounds__(kAttThr, 2) void cache_attn_few_kernel(
    const bf16* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
    const float* __restrict__ kv_scale, Units<true> w, Deal deal, float c_log2, AttnOut o,
    float* __restrict__ score) {
  __shared__ FewLds<HD> lds;
  const CacheBatch& bt = w.bt;
  long long total, off;
  int b;
  locate<kAttThr>(
      bt.B, [&](int i) { return w.group(i) * bt.H; }, deal, blockIdx.x, w.prefix, total, b, off);
  if (b < 0) return;
  // (at most 2^37 units, of tables of 2^31 entries and 64 groups, in a quarter of them or 1024
  // ranges)
  const int per = (int)deal.per(total);
  long long unit = (long long)blockIdx.x * per;
  int left = (int)min((long long)per, total - unit);
  int rows = w.rows(b), ctx = bt.context(b), np = w.pages(ctx, rows, 0);
  int h = (int)(off / np), blk0 = (int)(off % np);
  size_t slot = 2 * (size_t)blockIdx.x;
  while (true) {
    const int blk1 = min(np, blk0 + left);
    few_columns<HD>(q, kc, vc, kv_scale, bt, b, h, rows, ctx, np, blk0, blk1, c_log2, o, slot,
                    score != nullptr ? score + unit * o.part_cols * kPage : nullptr, lds);
    left -= blk1 - blk0;
    unit += blk1 - blk0;
    if (left <= 0) return;
    // the next group, or the next sequence with rows
    slot |= 1;
    blk0 = 0;
    if (++h == bt.H) {
      h = 0;
      do {
        if (++b >= bt.B) return;
        rows = w.rows(b);
      } while (rows <= 0);
      ctx = bt.context(b);
      np = w.pages(ctx, rows, 0);
    }
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
template <int HD>
__global__ __launch_bounds__(kTileThr) __attribute__((amdgpu_waves_per_eu(2, 2))) void
cache_attn_tile_kernel(const bf16* __restrict__ q, const uint8_t* __restrict__ kc,
                       const uint8_t* __restrict__ vc, const float* __restrict__ kv_scale,
                       Units<false> w, Deal deal, float c_log2, AttnOut o) {
  constexpr int KT = kPage * 256;       // K tile bytes
  constexpr int VT = HD * kPage * 2;    // V^T tile bytes
  constexpr int NST = HD / 16;          // score k-steps
  constexpr int NDT = HD / 32;          // output tiles
  constexpr int CPR = HD / 16;          // 16-byte pieces of a key row
  __shared__ __align__(1024) unsigned char smem[2 * KT + 3 * VT];
  const CacheBatch& bt = w.bt;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
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
  {
    const long long each = w.group(b);
    h = (int)(off / each);
    off -= h * each;
    int lo = 0, hi = nt - 1;  // the tile: largest t with before(t) <= off
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (w.before(ctx, mid) <= off) lo = mid;
      else hi = mid - 1;
    }
    t = lo;
    blk0 = (int)(off - w.before(ctx, t));
  }
  size_t slot = 2 * (size_t)range;

  // staging: thread -> 16 bytes of a key row, and 16 tokens of a value dim
  const bool stages = tid < kPage * CPR;
  const int krow = tid / CPR, kch = tid % CPR, vg = tid / HD, vd = tid % HD;
  const uint32_t kdst = krow * 256, vdst = vd * (kPage * 2);
  const uint32_t ks0 = kdst + (((2 * kch) ^ (krow & 15)) << 4);
  const uint32_t ks1 = kdst + (((2 * kch + 1) ^ (krow & 15)) << 4);
  const int vsw = (vd & 7) ^ ((vd >> 3) & 1);
  const uint32_t vs0 = vdst + (((2 * vg) ^ vsw) << 4), vs1 = vdst + (((2 * vg + 1) ^ vsw) << 4);

  while (true) {
    const int np = w.pages(ctx, rows, t);
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
        qf[st] = *reinterpret_cast<const bf16x8*>(q + (qrow + col) * HD + st * 16 + hl * 8);
    }
    const int len = min(ctx + rows, bt.cap());
    const int seen = col < ncol ? min(ctx + row0 + col / bt.nq + 1, bt.cap()) : 0;
    const int c0 = __builtin_amdgcn_readfirstlane(wave * 32);
    const int fewest = min(ctx + row0 + c0 / bt.nq + 1, bt.cap());
    // pages that a column of this wave sees some of
    const int npw = c0 < ncol ? (min(ctx + row0 + min(c0 + 31, ncol - 1) / bt.nq + 1, bt.cap()) +
                                 kPage - 1) / kPage : 0;
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
        const size_t at = ((size_t)p * bt.H + h) * (kPage * HD) + tid * 16;
        kreg = *reinterpret_cast<const u32x4*>(kc + at);
        vreg = *reinterpret_cast<const u32x4*>(vc + at);
      }
    };
    auto stage = [&](int i, int blk, float ks, float vs) {  // i-th page of the segment
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
#pragma unroll
      for (int i = 0; i < NDT; ++i) {
        const int row = i * 32 + qi;
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
#pragma unroll
        for (int st = 0; st < NST; ++st)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = i * 32 + qi;
            const bf16x8 kf = *reinterpret_cast<const bf16x8*>(
                kb + row * 256 + (((st * 2 + hl) ^ (row & 15)) << 4));
            sacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[st], sacc[i], 0, 0, 0);
          }
        if ((blk + 1) * kPage > fewest) {
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
        if (blk * kPage < seen) m_new = fmaxf(m_new, kMSeen);
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

    const float l = l_run + __shfl_xor(l_run, 32);
    const bool whole = blk0 == 0 && blk1 == np;
    if (col < ncol) {
      // lane holds dims 32 i + 8 g + 4 hl + [0, 4)
      if (whole) {
        const float inv = inv_sum(m_run, l);
        const int row = bt.first_row(b) + row0 + col / bt.nq;
        bf16* dst = o.out + (((size_t)row * bt.H + h) * bt.nq + col % bt.nq) * HD;
#pragma unroll
        for (int i = 0; i < NDT; ++i)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            bf16x4 x;
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] = (bf16)(oacc[i][g * 4 + v] * inv);
            *reinterpret_cast<bf16x4*>(dst + i * 32 + g * 8 + hl * 4) = x;
          }
        if (o.stat != nullptr && hl == 0) o.stat[qrow + col] = column_stat(m_run, inv);
      } else {
        float* pt = o.part + slot * part_floats(kTileCols, HD);
#pragma unroll
        for (int i = 0; i < NDT; ++i)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(pt + ((i * 8 + g * 2 + hl) * kTileCols + col) * 4) =
                f32x4{oacc[i][g * 4], oacc[i][g * 4 + 1], oacc[i][g * 4 + 2], oacc[i][g * 4 + 3]};
        if (hl == 0) reinterpret_cast<float2*>(pt + kTileCols * HD)[col] = float2{m_run, l};
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
// units u0 .. u0 + np - 1 of the tile; false where one range wrote it whole
template <bool FEW>
__device__ __forceinline__ bool find_parts(const Units<FEW>& w, const Deal& deal, long long u0,
                                           int np, Parts& p) {
  const long long per = deal.per(w.prefix[w.bt.B]);
  p.r0 = (int)(u0 / per);
  p.r1 = (int)((u0 + np - 1) / per);
  p.first_late = u0 % per != 0;
  return p.r0 != p.r1;
}

// Few columns: one workgroup per (group h, column c of sequence b).  8 groups of 32 lanes (a
// lane 4 dims) each sum every eighth part, and are then summed in order.  (A sequence's
// columns one after another in a workgroup: 13.7 us instead of 4.3 for 16 sequences of 1000 to
// 4000 tokens, 4 groups of 8 heads.)
template <int HD>
__device__ __forceinline__ void join_few(const Units<true>& w, const Deal& deal,
                                         const AttnOut& o, int h, int b, int c) {
  __shared__ f32x4 osum[8][32];
  const CacheBatch& bt = w.bt;
  const int rows = w.rows(b);
  if (c >= rows * bt.nq) return;
  const int np = w.pages(bt.context(b), rows, 0);
  Parts p{o.part, o.part_cols, HD};
  if (!find_parts(w, deal, w.prefix[b] + (long long)np * h, np, p)) return;
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
    o.stat[((size_t)h * bt.N + bt.first_row(b)) * bt.nq + c] = column_stat(m, inv);
}

// Many columns: one workgroup per (32 columns of a tile, group h), 8 threads a column; a
// thread loads its dims of four parts at a time.
constexpr int kJoinCols = 32;

template <int HD>
__device__ __forceinline__ void join_tile(const Units<false>& w, const Deal& deal,
                                          const AttnOut& o, int h, int x32) {
  constexpr int CB = kTileCols / kJoinCols, NV = HD / 32, AT_ONCE = 4;
  const CacheBatch& bt = w.bt;
  int b, t;
  if (!find_tile<256>(bt.B, x32 / CB, [&](int i) { return w.tiles(w.rows(i)); }, b, t)) return;
  const int c = x32 % CB * kJoinCols + (threadIdx.x & 31), l3 = threadIdx.x >> 5;
  const int rows = w.rows(b), ctx = bt.context(b), row0 = t << w.log2r;
  const int ncol = (min(rows, (t + 1) << w.log2r) - row0) * bt.nq;
  const int np = w.pages(ctx, rows, t);
  Parts p{o.part, kTileCols, HD};
  if (!find_parts(w, deal, w.prefix[b] + w.group(b) * h + w.before(ctx, t), np, p) ||
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
    o.stat[((size_t)h * bt.N + bt.first_row(b) + row0) * bt.nq + c] = column_stat(m, inv);
}

// What a form's launches share: its units, how they are dealt out, and where it writes.
template <bool FEW>
struct Form {
  Units<FEW> w;
  Deal deal;
  AttnOut o;
};

// One launch joins both forms' parts: `many_blocks` by H workgroups those of tiles, the rest
// those of few columns.
template <int HD>
__global__ __launch_bounds__(256) void cache_join_kernel(Form<true> few, Form<false> many,
                                                         int many_blocks) {
  const int x = blockIdx.x, h = blockIdx.y;
  if (x < many_blocks) join_tile<HD>(many.w, many.deal, many.o, h, x);
  else join_few<HD>(few.w, few.deal, few.o, h, (x - many_blocks) / few.o.part_cols,
                    (x - many_blocks) % few.o.part_cols);
}

// ---- mass ---------------------------------------------------------------------------
// A token's mass is the sum of its probabilities over the columns, each from its score
// and its column's final maximum and sum, so it follows the joining.  With few columns the
// scores were kept; else they are formed again.

// Few columns: equal ranges of the units again; a wave takes every fourth page, a lane a
// token.
__device__ __forceinline__ void mass_few(const float* __restrict__ score, const Units<true>& w,
                                         const Deal& deal, int range, int part_cols,
                                         float c_log2, const float2* __restrict__ stat,
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
  int rows = w.rows(b), ctx = bt.context(b), np = w.pages(ctx, rows, 0);
  const int off = (int)(unit - w.prefix[b]);
  int h = off / np, blk0 = off % np;
  score += unit * part_cols * kPage;
  while (true) {
    const int blk1 = min(np, blk0 + left), ncol = rows * bt.nq;
    float2 z{0.f, 0.f};  // of column `lane`
    if (lane < ncol) z = stat[((size_t)h * bt.N + bt.first_row(b)) * bt.nq + lane];
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
      np = w.pages(ctx, rows, 0);
    }
  }
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

template <int HD>
__device__ __forceinline__ void mass_any(const bf16* __restrict__ q, const uint8_t* __restrict__ kc,
                                         const float* __restrict__ kv_scale, const Units<false>& w,
                                         const Deal& deal, int range, float c_log2,
                                         const float2* __restrict__ stat,
                                         const float* __restrict__ mass_in,
                                         float* __restrict__ mass_out) {
  constexpr int NST = HD / 16;
  constexpr int QT = kMassCols * 256, STAGE = QT + 256;  // bytes of a tile, and with its statistics
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
    const long long c_first = (long long)max(blk0 * kPage - ctx, 0) * bt.nq;
    const int t0 = (int)(c_first / kMassCols), t1 = (ncol + kMassCols - 1) / kMassCols;
    // columns past the last read zeros: no query, maximum 0 and 1 / sum 0
    const __amdgpu_buffer_rsrc_t rq = make_rsrc_u(q + qrow * HD, (uint32_t)ncol * (HD * 2));
    const __amdgpu_buffer_rsrc_t rz = make_rsrc_u(stat + qrow, (uint32_t)ncol * 8u);
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
      dma4(rz, (uint32_t)t * (kMassCols * 8) + lane * 4u, to, QT);
    };
    constexpr int OPS = QI + 1;  // DMA instructions of a wave and tile
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
        float2 z = *reinterpret_cast<const float2*>(tile + QT + qi * 8);
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
        // (the tile's first column sees the fewest)
        if (ctx + t * kMassCols / bt.nq + 1 < min(key0 + 32, len + 1)) {
          const int col = t * kMassCols + qi, seen = col < ncol ? ctx + col / bt.nq + 1 : 0;
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (key0 + 8 * (v >> 2) + 4 * hl + (v & 3) >= seen) x[v] = -__builtin_inff();
        }
        float c_tile = c_log2;
        if (special) {
          // a NaN row counts, as NaN, for the tokens that it sees alone (0 * NaN is NaN)
          if (z.y != z.y) {
            const int seen = ctx + (t * kMassCols + qi) / bt.nq + 1;
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (key0 + 8 * (v >> 2) + 4 * hl + (v & 3) < seen) acc[v] = z.y;
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
template <int HD>
__global__ __launch_bounds__(kMassThr, 4) void cache_mass_kernel(
    const bf16* __restrict__ q, const uint8_t* __restrict__ kc, const float* __restrict__ kv_scale,
    Units<false> any, int any_ranges, Form<true> few, const float* __restrict__ score, float c_log2,
    const float2* __restrict__ stat, const float* __restrict__ mass_in,
    float* __restrict__ mass_out) {
  static_assert(kMassThr == kAttThr, "one workgroup size");
  const int x = blockIdx.x;
  if (x >= any_ranges) {
    mass_few(score, few.w, Deal{few.deal.ranges, few.deal.least, 0}, x - any_ranges,
             few.o.part_cols, c_log2, stat, mass_in, mass_out);
    return;
  }
  mass_any<HD>(q, kc, kv_scale, any, Deal{any_ranges, 1, 0}, x, c_log2, stat, mass_in, mass_out);
}

// Host side of the two forms: ranges (workgroups) and scratch.
constexpr int kFewLeast = 4;   // pages of a range at least: one for each wave
constexpr int kManyLeast = 2;
// The scores of few columns are kept for the mass where the tables' room for them is up to
// this many bytes of workspace; beyond, they are formed again.  us kept and formed again, 8
// groups of two heads: 16 sequences of 1000 to 4000 tokens 35 53, 64 of 1000 to 8000 155 264,
// one of 100000 68 112.
constexpr size_t kScoreBytes = (size_t)1 << 30;

// One form of a call: what it launches and where its scratch is.
struct FormPlan {
  bool on;
  int lo, hi;                 // columns of its sequences
  int ranges, cols, log2r, tiles;
  size_t prefix, part;
};
struct AttnPlan {
  FormPlan few, many;
  bool scores;
  size_t stat, score, total;
};

AttnPlan attn_plan(int H, int B, int N, int nq, int hd, int max_blocks, int max_rows, bool mass) {
  AttnPlan p{};
  const long long most = (long long)max_rows * nq;
  // Both forms where the sequences beside the longest have few columns on average (us for a
  // 512-row chunk beside 16 decoding sequences, with mass: 85, and 114 in the second form
  // alone); where they are all chunks the first would be a launch for nothing.
  p.few.on = most <= kFewCols || (B > 1 && (long long)(N - max_rows) * nq <= kFewCols * (B - 1LL));
  p.many.on = most > kFewCols;
  p.few.hi = kFewCols;
  p.many.lo = p.few.on ? kFewCols : 0;
  p.many.hi = INT_MAX;
  auto take = [&](size_t& field, size_t bytes) {
    field = p.total;
    p.total = align_up(p.total + bytes, 256);
  };
  auto scratch = [&](FormPlan& f) {
    if (!f.on) return;
    take(f.prefix, (size_t)(B + 1) * 8);
    take(f.part, 2 * (size_t)f.ranges * part_floats(f.cols, hd) * 4);
  };
  const long long pages = (long long)B * H * max_blocks;
  p.few.cols = (int)std::min<long long>(kFewCols, most);
  p.few.ranges = (int)std::min<long long>(4LL * kCus, (pages + kFewLeast - 1) / kFewLeast);
  p.many.cols = kTileCols;
  p.many.ranges = kCus;
  while ((2 << p.many.log2r) * nq <= kTileCols) ++p.many.log2r;
  // tiles of the batch: at most n / 2^log2r, rounded up, of each sequence
  p.many.tiles = (int)std::min<long long>(N, ((long long)N >> p.many.log2r) + B);
  scratch(p.few);
  scratch(p.many);
  if (mass) {
    take(p.stat, (size_t)H * N * nq * sizeof(float2));
    const size_t bytes = (size_t)pages * p.few.cols * kPage * 4;
    p.scores = p.few.on && bytes <= kScoreBytes;
    if (p.scores) take(p.score, bytes);
  }
  return p;
}
}  // namespace

size_t cache_attention_scratch_bytes(int H, int B, int N, int nq, int hd, int max_blocks,
                                     int max_rows, bool mass) {
  return attn_plan(H, B, N, nq, hd, max_blocks, max_rows, mass).total;
}

hipError_t launch_cache_attention(const CacheArgs& a, int nq, int N, int max_rows, const void* q,
                                  const int32_t* row_start, const float* mass_in, float* mass_out,
                                  void* out, void* scratch, hipStream_t s) {
  const CacheBatch bt{a.H, a.B, N, nq, a.n_pages, a.max_blocks, a.block_table, a.length, row_start};
  const AttnPlan p = attn_plan(a.H, a.B, N, nq, a.hd, a.max_blocks, max_rows, mass_out != nullptr);
  unsigned char* base = static_cast<unsigned char*>(scratch);
  const float c_log2 = 1.4426950408889634f / sqrtf((float)a.hd);
  const bf16* qb = static_cast<const bf16*>(q);
  float2* stat = mass_out != nullptr ? reinterpret_cast<float2*>(base + p.stat) : nullptr;
  float* score = p.scores ? reinterpret_cast<float*>(base + p.score) : nullptr;
  auto form = [&](const FormPlan& f, int least, int round, auto few) {
    return Form<decltype(few)::value>{
        {bt, max_rows, f.log2r, f.lo, f.hi, reinterpret_cast<long long*>(base + f.prefix)},
        {f.ranges, least, round},
        {static_cast<bf16*>(out), stat, reinterpret_cast<float*>(base + f.part), f.cols}};
  };
  const Form<true> few = form(p.few, kFewLeast, std::min(p.few.ranges, 2 * kCus), std::true_type{});
  const Form<false> many = form(p.many, kManyLeast, 0, std::false_type{});
  auto go = [&](auto hdv) {
    constexpr int HD = decltype(hdv)::value;
    if (p.few.on) {
      ProfileScope ps("cache_attn_few", s);
      FOE_LAUNCH(cache_attn_few_kernel<HD>, dim3(few.deal.ranges), dim3(kAttThr), 0, s, qb, a.k,
                 a.v, a.kv_scale, few.w, few.deal, c_log2, few.o, score);
    }
    if (p.many.on) {
      ProfileScope ps("cache_attn_tile", s);
      FOE_LAUNCH(cache_attn_tile_kernel<HD>, dim3(many.deal.ranges), dim3(kTileThr), 0, s, qb, a.k,
                 a.v, a.kv_scale, many.w, many.deal, c_log2, many.o);
    }
    {
      ProfileScope ps("cache_join", s);
      const int many_blocks = p.many.on ? p.many.tiles * (kTileCols / kJoinCols) : 0;
      const int few_blocks = p.few.on ? a.B * few.o.part_cols : 0;
      FOE_LAUNCH(cache_join_kernel<HD>, dim3(many_blocks + few_blocks, a.H), dim3(256), 0, s, few,
                 many, many_blocks);
    }
    if (mass_out != nullptr) {
      ProfileScope ps("cache_mass", s);
      // without scores the sequences of both forms; at most 16 workgroups a CU: four rounds,
      // which evens out what pages near a chunk's end have less to do
      Units<false> any = many.w;
      if (score == nullptr) any.lo = 0;
      const long long pairs = (long long)ceil_div(a.max_blocks, 2) * a.H * a.B;
      const int any_ranges =
          p.many.on || score == nullptr ? (int)std::min(16LL * kCus, pairs) : 0;
      FOE_LAUNCH(cache_mass_kernel<HD>, dim3(any_ranges + (score != nullptr ? few.deal.ranges : 0)),
                 dim3(kMassThr), 0, s, qb, a.k, a.kv_scale, any, any_ranges, few, score, c_log2,
                 stat, mass_in, mass_out);
    }
  };
  if (a.hd == 96) go(std::integral_constant<int, 96>{});
  else go(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace foe
