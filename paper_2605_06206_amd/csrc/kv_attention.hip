// Causal attention over the 8-bit key/value cache, and the attention weight that
// each cached token receives.
//
// A column is one query: row i of a sequence and head j of a group, numbered
// i * nq + j (the heads share the group's keys and values).  Two forms, by the
// sequence's columns:
// - few (at most 16: decode steps): a tile of 16 columns walks the pages with
//   16x16x32 MFMAs fed from registers; reading the pages is all the work;
// - many (chunks): tiles of up to 256 columns share each page through LDS.
// In both, S^T = K Q^T and O^T += V^T P^T with an online softmax in base 2, and the
// work is dealt out alike: the (sequence, group, tile, page) units of the batch,
// numbered in that order, are cut into equal ranges, one for each workgroup of a
// grid that fills the chip, whatever the lengths are.  A workgroup walks the tiles in
// its range; a tile that lies in one range is written at once, the others leave their
// unnormalised parts, which a second launch joins in page order.  (One workgroup per
// tile of 16 columns: 1151 us instead of 200 for four sequences of 131072 tokens, 8 groups.)
#include <algorithm>
#include <type_traits>

#include "kv_cache.hpp"

namespace foe {
namespace {

constexpr int kAttThr = 256;          // few columns: four waves, each taking every fourth page
constexpr int kAttWaves = kAttThr / kWave;
constexpr int kFewCols = 16;
constexpr int kTileThr = 512;         // many columns: eight waves of 32 columns
constexpr int kTileCols = 256;
constexpr int kMaxCus = 256;          // the workspace holds the parts of this many units
constexpr float kMFloor = -1.0e30f;   // the running maximum's start: finite, below any score

// ---- dealing out the work -------------------------------------------------------

// The units of a batch in one of the two forms, numbered by sequence, group, tile
// and page.  A tile of the many form has 2^log2r rows, tile t reaches page
// ceil((ctx + last row + 1) / 64), and the sums over tiles are closed forms.
struct Units {
  CacheBatch bt;
  int max_rows;
  int log2r;  // few: -1
  long long* prefix;  // [B + 1]: units before each sequence, and in all (written for the join)

  __device__ __forceinline__ int rows(int b) const { return min(bt.rows(b), max_rows); }
  // rows of sequence b in this form
  __device__ __forceinline__ int mine(int b) const {
    const int n = rows(b);
    return (n * bt.nq <= kFewCols) == (log2r < 0) ? n : 0;
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
    const int last = log2r < 0 ? n : min((t + 1) << log2r, n);
    return (ctx + last + kPage - 1) / kPage;
  }
  // units of one group of sequence b
  __device__ __forceinline__ long long group(int b) const {
    const int n = mine(b);
    if (n <= 0) return 0;
    const int ctx = bt.context(b), t = log2r < 0 ? 0 : tiles(n) - 1;
    return (log2r < 0 ? 0 : before(ctx, t)) + pages(ctx, n, t);
  }
};

// units of a workgroup's range
__device__ __forceinline__ long long range_units(long long total, int ranges, int least) {
  const long long per = (total + ranges - 1) / ranges;
  return per < least ? least : per;
}

// Total of the units, and the sequence that unit range * per falls in (b, or -1 past the
// end) with its offset there.  Every thread of the workgroup calls it; range 0 writes
// the prefix.
template <int NT>
__device__ __forceinline__ void locate(const Units& w, int ranges, int range, int least,
                                       long long& total, int& b, long long& off) {
  constexpr int NW = NT / kWave;
  __shared__ long long wave_sum[NW];
  __shared__ long long found[2];
  const int B = w.bt.B, lane = lane_id(), wave = threadIdx.x >> 6;
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
  const long long first = (int)threadIdx.x < B ? w.group(threadIdx.x) * w.bt.H : 0;
  long long mine = first;
  for (int i = threadIdx.x + NT; i < B; i += NT) mine += w.group(i) * w.bt.H;
  long long incl = scan(mine, total);
  const long long u0 = range * range_units(total, ranges, least);
  if (threadIdx.x == 0) found[0] = -1;
  if (B > NT && (u0 < total || range == 0)) {  // (uniform) again, a row of threads at a time
    long long run = 0, all;
    for (int base = 0; base < B; base += NT) {
      const int i = base + (int)threadIdx.x;
      const long long c = base == 0 ? first : i < B ? w.group(i) * w.bt.H : 0;
      incl = run + scan(c, all);
      if (u0 >= incl - c && u0 < incl) found[0] = i, found[1] = u0 - (incl - c);
      if (range == 0 && i < B) w.prefix[i] = incl - c;
      run += all;
    }
  } else if (B <= NT) {
    __syncthreads();
    const int i = threadIdx.x;
    if (u0 >= incl - first && u0 < incl) found[0] = i, found[1] = u0 - (incl - first);
    if (range == 0 && i < B) w.prefix[i] = incl - first;
  }
  if (range == 0 && threadIdx.x == 0) w.prefix[B] = total;
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
  u32x4 k[4][(HD + 63) / 64];          // tile t: 16 bytes at 64 h + 16 g (8 at 64 + 8 g for HD = 96)
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

// A part of a tile that several workgroups share: [columns][HD] unnormalised sums,
// then [columns] (maximum, sum).  Workgroup r leaves at most two: of its first tile
// (slot 2 r), and of its last one if another (2 r + 1).
__host__ __device__ inline size_t part_floats(int cols, int hd) { return (size_t)cols * (hd + 2); }

template <int HD>
__global__ __launch_bounds__(kAttThr) void cache_attn_few_kernel(
    const bf16* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
    const float* __restrict__ kv_scale, Units w, int least, int part_cols, float c_log2,
    bf16* __restrict__ out, float2* __restrict__ stat, float* __restrict__ part) {
  using F = PageFrags<HD>;
  __shared__ float mm[kAttWaves][16], ll[kAttWaves][16];
  __shared__ __align__(16) float oo[kAttWaves][HD][16];
  const CacheBatch& bt = w.bt;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const int n = lane & 15, g = lane >> 4;
  long long total, off;
  int b;
  locate<kAttThr>(w, gridDim.x, blockIdx.x, least, total, b, off);
  if (b < 0) return;
  const int per = (int)range_units(total, gridDim.x, least);
  int left = (int)min((long long)per, total - (long long)blockIdx.x * per);
  int rows = w.mine(b), ctx = bt.context(b), np = w.pages(ctx, rows, 0);
  int h = (int)(off / np), blk0 = (int)(off % np);
  bool first_tile = true;
  while (true) {
    const int blk1 = min(np, blk0 + left);
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
    for (int blk = blk0 + wave; blk < blk1; blk += kAttWaves) {
      const int page = bt.page(b, blk);
      if (page < 0) continue;
      const size_t pg = (size_t)page * bt.H + h;
      const float ks = kv_scale[pg * 2], vs = kv_scale[pg * 2 + 1];
      F f;
      f.load_k(kc + pg * (kPage * HD), lane);
      f.load_v(vc + pg * (kPage * HD), lane);
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
        l_run *= a;
#pragma unroll
        for (int dt = 0; dt < F::NDT; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) oacc[dt][e] *= a;
      }
      bf16x8 p[2];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[t][e], c_log2, -m_run));
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
    // the four waves' states, merged in wave order
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
    __syncthreads();  // the previous tile's merge has been read
    if (g == 0) mm[wave][n] = m_run, ll[wave][n] = l_run;
    if (n < ncol) {
#pragma unroll
      for (int dt = 0; dt < F::NDT; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) oo[wave][16 * dt + 4 * g + e][n] = oacc[dt][e];
    }
    __syncthreads();
    const int c = tid >> 4;  // column; its 16 threads take every 16th dim
    if (c < ncol) {
      float m = mm[0][c], l = 0.f, a[kAttWaves];
#pragma unroll
      for (int v = 1; v < kAttWaves; ++v) m = fmaxf(m, mm[v][c]);
#pragma unroll
      for (int v = 0; v < kAttWaves; ++v) {
        a[v] = __builtin_amdgcn_exp2f(mm[v][c] - m);
        l += ll[v][c] * a[v];
      }
      const bool whole = blk0 == 0 && blk1 == np;
      // a column that sees no token gives zeros
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int row = bt.first_row(b) + c / bt.nq;
      bf16* dst = out + (((size_t)row * bt.H + h) * bt.nq + c % bt.nq) * HD;
      float* pt = part + (2 * (size_t)blockIdx.x + (first_tile ? 0 : 1)) * part_floats(part_cols, HD);
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        const int d = i * 16 + (tid & 15);
        float x = 0.f;
#pragma unroll
        for (int v = 0; v < kAttWaves; ++v) x += oo[v][d][c] * a[v];
        if (whole) dst[d] = (bf16)(x * inv);
        else pt[c * HD + d] = x;
      }
      if ((tid & 15) == 0) {
        if (!whole) reinterpret_cast<float2*>(pt + part_cols * HD)[c] = float2{m, l};
        else if (stat != nullptr) stat[qrow + c] = float2{m, inv};
      }
    }
    left -= blk1 - blk0;
    if (left <= 0) return;
    // the next group, or the next sequence with rows of this form
    first_tile = false;
    blk0 = 0;
    if (++h == bt.H) {
      h = 0;
      do {
        if (++b >= bt.B) return;
        rows = w.mine(b);
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
                       const uint8_t* __restrict__ vc, const float* __restrict__ kv_scale, Units w,
                       int least, float c_log2, bf16* __restrict__ out, float2* __restrict__ stat,
                       float* __restrict__ part) {
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
  locate<kTileThr>(w, gridDim.x, range, least, total, b, off);
  if (b < 0) return;
  const int per = (int)range_units(total, gridDim.x, least);
  int left = (int)min((long long)per, total - (long long)range * per);
  int rows = w.mine(b), ctx = bt.context(b), nt = w.tiles(rows), h, t, blk0;
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
  bool first_tile = true;

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
    const int blk1 = min(np, blk0 + left);
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
        const float m_new = need ? mxs : m_run;
        const float a_new = need ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
        if (it > 0) pv(vb);
        float ps = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          bf16x8 p8;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = __builtin_amdgcn_exp2f(
                fmaf(sacc[u >> 1][(u & 1) * 8 + e], c_log2, -m_new));
            ps += x;
            p8[e] = (bf16)x;
          }
          pf[u] = p8;
        }
        resc = __builtin_amdgcn_ballot_w64(need) != 0;
        alpha = a_new;
        m_run = m_new;
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
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int row = bt.first_row(b) + row0 + col / bt.nq;
        bf16* dst = out + (((size_t)row * bt.H + h) * bt.nq + col % bt.nq) * HD;
#pragma unroll
        for (int i = 0; i < NDT; ++i)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            bf16x4 o;
#pragma unroll
            for (int v = 0; v < 4; ++v) o[v] = (bf16)(oacc[i][g * 4 + v] * inv);
            *reinterpret_cast<bf16x4*>(dst + i * 32 + g * 8 + hl * 4) = o;
          }
        if (stat != nullptr && hl == 0) stat[qrow + col] = float2{m_run, inv};
      } else {
        float* pt = part + (2 * (size_t)range + (first_tile ? 0 : 1)) * part_floats(kTileCols, HD);
#pragma unroll
        for (int i = 0; i < NDT; ++i)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(pt + col * HD + i * 32 + g * 8 + hl * 4) =
                f32x4{oacc[i][g * 4], oacc[i][g * 4 + 1], oacc[i][g * 4 + 2], oacc[i][g * 4 + 3]};
        if (hl == 0) reinterpret_cast<float2*>(pt + kTileCols * HD)[col] = float2{m_run, l};
      }
    }
    left -= niter;
    if (left <= 0) return;
    // the next tile, group, or sequence with rows of this form
    first_tile = false;
    blk0 = 0;
    if (++t == nt) {
      t = 0;
      if (++h == bt.H) {
        h = 0;
        do {
          if (++b >= bt.B) return;
          rows = w.mine(b);
        } while (rows <= 0);
        ctx = bt.context(b);
        nt = w.tiles(rows);
      }
    }
  }
}

// ---- joining the parts ---------------------------------------------------------------
// One workgroup per (32 columns of a tile, group, sequence), 8 groups of 32 lanes, a
// lane taking 4 dims: a few columns have their parts dealt to the 8 groups (each sums
// every eighth, then the groups are summed in order), many columns are dealt
// themselves.  A tile that lies in one range has been written already.
template <int HD, bool FEW>
__global__ __launch_bounds__(256) void cache_join_kernel(Units w, int ranges, int least,
                                                         int part_cols, const float* __restrict__ part,
                                                         bf16* __restrict__ out,
                                                         float2* __restrict__ stat) {
  constexpr int TILE = FEW ? 1 : kTileCols / 32;  // workgroups of a tile
  __shared__ f32x4 osum[FEW ? 8 : 1][32];
  const CacheBatch& bt = w.bt;
  const int t = blockIdx.x / TILE, h = blockIdx.y, b = blockIdx.z;
  const int c0 = (blockIdx.x % TILE) * 32;
  const int rows = w.mine(b);
  if (rows <= 0 || (!FEW && t >= w.tiles(rows))) return;
  const int ctx = bt.context(b), row0 = FEW ? 0 : t << w.log2r;
  const int ncol = ((FEW ? rows : min(rows, (t + 1) << w.log2r)) - row0) * bt.nq;
  if (c0 >= ncol) return;
  const long long total = w.prefix[bt.B], per = range_units(total, ranges, least);
  const long long u0 = w.prefix[b] + (w.group(b) * h + (FEW ? 0 : w.before(ctx, t)));
  const int np = w.pages(ctx, rows, t);
  const int r0 = (int)(u0 / per), r1 = (int)((u0 + np - 1) / per);
  if (r0 == r1) return;
  const size_t pf = part_floats(part_cols, HD);
  auto slot = [&](int r) { return part + (2 * (size_t)r + (r == r0 && u0 % per != 0)) * pf; };
  const int grp = threadIdx.x >> 5, l5 = threadIdx.x & 31;
  const int d = 4 * l5;
  auto ml = [&](int r, int c) {
    return reinterpret_cast<const float2*>(slot(r) + (size_t)part_cols * HD)[c];
  };
  for (int c = c0 + (FEW ? 0 : grp); c < min(ncol, c0 + 32); c += FEW ? 1 : 8) {
    float m = kMFloor, l = 0.f;
    for (int r = r0 + l5; r <= r1; r += 32) m = fmaxf(m, ml(r, c).x);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    for (int r = r0 + l5; r <= r1; r += 32) {
      const float2 x = ml(r, c);
      l += x.y * __builtin_amdgcn_exp2f(x.x - m);
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) l += __shfl_xor(l, o);
    f32x4 x{0.f, 0.f, 0.f, 0.f};
    if (d < HD)
      for (int r = r0 + (FEW ? grp : 0); r <= r1; r += FEW ? 8 : 1) {
        const float a = __builtin_amdgcn_exp2f(ml(r, c).x - m);
        const f32x4 y = *reinterpret_cast<const f32x4*>(slot(r) + (size_t)c * HD + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += y[e] * a;
      }
    if constexpr (FEW) {
      __syncthreads();
      osum[grp][l5] = x;
      __syncthreads();
      x = osum[0][l5];
#pragma unroll
      for (int k = 1; k < 8; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += osum[k][l5][e];
      if (grp != 0) continue;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (d < HD) {
      const int row = bt.first_row(b) + row0 + c / bt.nq;
      bf16* dst = out + (((size_t)row * bt.H + h) * bt.nq + c % bt.nq) * HD + d;
      *reinterpret_cast<bf16x4*>(dst) = bf16x4{(bf16)(x[0] * inv), (bf16)(x[1] * inv),
                                               (bf16)(x[2] * inv), (bf16)(x[3] * inv)};
    }
    if (stat != nullptr && l5 == 0)
      stat[((size_t)h * bt.N + bt.first_row(b) + row0) * bt.nq + c] = float2{m, inv};
  }
}

// ---- mass ---------------------------------------------------------------------------
// Mass: one workgroup per (page, group, sequence); the scores again, each
// probability from its column's maximum and sum, summed over the columns.
template <int HD>
__global__ __launch_bounds__(kAttThr) void cache_mass_kernel(
    const bf16* __restrict__ q, const uint8_t* __restrict__ kc, const float* __restrict__ kv_scale,
    CacheBatch bt, int max_rows, float c_log2, const float2* __restrict__ stat,
    const float* __restrict__ mass_in, float* __restrict__ mass_out) {
  using F = PageFrags<HD>;
  __shared__ float sum[kAttWaves][kPage];
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const int blk = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int n = lane & 15, g = lane >> 4;
  const int rows = min(bt.rows(b), max_rows), ctx = bt.context(b);
  const int len = min(ctx + rows, bt.cap());
  if (rows == 0 || blk * kPage >= len) return;
  const int page = bt.page(b, blk);
  if (page < 0) return;
  const size_t pg = (size_t)page * bt.H + h;
  F f;
  f.load_k(kc + pg * (kPage * HD), lane);
  const float ks = kv_scale[pg * 2];
  const int ncol = rows * bt.nq, k0 = blk * kPage + 16 * g;
  const size_t qrow = ((size_t)h * bt.N + bt.first_row(b)) * bt.nq;
  float acc[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  // columns before the first that sees the page are left out
  const int first = max(blk * kPage - ctx, 0) * bt.nq / 16;
  for (int t0 = first + wave; t0 * 16 < ncol; t0 += kAttWaves) {
    const int col = t0 * 16 + n;
    bf16x8 qf[F::NST];
    load_q<HD>(q + qrow * HD, col, ncol, g, qf);
    const float2 z = col < ncol ? stat[qrow + col] : float2{0.f, 0.f};  // maximum, 1 / sum
    const int seen = col < ncol ? min(ctx + col / bt.nq + 1, bt.cap()) : 0;
    f32x4 s[4];
    f.scores(qf, ks, s);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[t][e], c_log2, -z.x)) * z.y;
        acc[4 * t + e] += k0 + 4 * t + e < seen ? x : 0.f;
      }
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) acc[e] += __shfl_xor(acc[e], o);
    if (n == 0) sum[wave][16 * g + e] = acc[e];
  }
  __syncthreads();
  const int slot = blk * kPage + tid;
  if (tid < kPage && slot < len) {
    float x = slot < ctx ? mass_in[pg * kPage + tid] : 0.f;
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < kAttWaves; ++w) y += sum[w][tid];
    mass_out[pg * kPage + tid] = x + y;
  }
}

}  // namespace

namespace {
int device_cus() {
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 8)
    return 256;
  return n / 8 * 8;
}

// Host side of the two forms: ranges (workgroups) and scratch.
struct AttnPlan {
  bool few, many;           // launches
  int few_ranges, many_ranges, few_cols, log2r, max_tiles;
  size_t few_prefix, many_prefix, few_part, many_part, stat, total;
};
constexpr int kFewLeast = 4;   // pages of a range at least: one for each wave
constexpr int kManyLeast = 2;

AttnPlan attn_plan(int H, int B, int N, int nq, int hd, int max_blocks, int max_rows, bool mass,
                   int cus) {
  AttnPlan p{};
  p.many = (long long)max_rows * nq > kFewCols;
  p.few = nq <= kFewCols;
  p.few_cols = std::min(kFewCols, max_rows * nq);
  const long long most = (long long)B * H * max_blocks;  // few units at most
  p.few_ranges = (int)std::min<long long>(4LL * cus, (most + kFewLeast - 1) / kFewLeast);
  p.many_ranges = cus;
  while ((2 << p.log2r) * nq <= kTileCols) ++p.log2r;
  p.max_tiles = ceil_div(max_rows, 1 << p.log2r);
  size_t off = 0;
  auto take = [&](size_t& field, size_t bytes) {
    field = off;
    off = align_up(off + bytes, 256);
  };
  if (p.few) {
    take(p.few_prefix, (size_t)(B + 1) * 8);
    take(p.few_part, 2 * (size_t)p.few_ranges * part_floats(p.few_cols, hd) * 4);
  }
  if (p.many) {
    take(p.many_prefix, (size_t)(B + 1) * 8);
    take(p.many_part, 2 * (size_t)p.many_ranges * part_floats(kTileCols, hd) * 4);
  }
  if (mass) take(p.stat, (size_t)H * N * nq * sizeof(float2));
  p.total = off;
  return p;
}
}  // namespace

size_t cache_attention_scratch_bytes(int H, int B, int N, int nq, int hd, int max_blocks,
                                     int max_rows, bool mass) {
  return attn_plan(H, B, N, nq, hd, max_blocks, max_rows, mass, kMaxCus).total;
}

hipError_t launch_cache_attention(const CacheArgs& a, int nq, int N, int max_rows, const void* q,
                                  const int32_t* row_start, const float* mass_in, float* mass_out,
                                  void* out, void* scratch, hipStream_t s) {
  const CacheBatch bt{a.H, a.B, N, nq, a.n_pages, a.max_blocks, a.block_table, a.length, row_start};
  const AttnPlan p = attn_plan(a.H, a.B, N, nq, a.hd, a.max_blocks, max_rows, mass_out != nullptr,
                               std::min(device_cus(), kMaxCus));
  unsigned char* base = static_cast<unsigned char*>(scratch);
  float2* stat = mass_out != nullptr ? reinterpret_cast<float2*>(base + p.stat) : nullptr;
  const float c_log2 = 1.4426950408889634f / sqrtf((float)a.hd);
  const bf16* qb = static_cast<const bf16*>(q);
  bf16* ob = static_cast<bf16*>(out);
  auto go = [&](auto hdv) {
    constexpr int HD = decltype(hdv)::value;
    if (p.few) {
      const Units w{bt, max_rows, -1, reinterpret_cast<long long*>(base + p.few_prefix)};
      float* part = reinterpret_cast<float*>(base + p.few_part);
      {
        ProfileScope ps("cache_attn_few", s);
        FOE_LAUNCH(cache_attn_few_kernel<HD>, dim3(p.few_ranges), dim3(kAttThr), 0, s, qb, a.k, a.v,
                   a.kv_scale, w, kFewLeast, p.few_cols, c_log2, ob, stat, part);
      }
      ProfileScope ps("cache_join_few", s);
      FOE_LAUNCH((cache_join_kernel<HD, true>), dim3(1, a.H, a.B), dim3(256), 0, s, w, p.few_ranges,
                 kFewLeast, p.few_cols, part, ob, stat);
    }
    if (p.many) {
      const Units w{bt, max_rows, p.log2r, reinterpret_cast<long long*>(base + p.many_prefix)};
      float* part = reinterpret_cast<float*>(base + p.many_part);
      {
        ProfileScope ps("cache_attn_tile", s);
        FOE_LAUNCH(cache_attn_tile_kernel<HD>, dim3(p.many_ranges), dim3(kTileThr), 0, s, qb, a.k,
                   a.v, a.kv_scale, w, kManyLeast, c_log2, ob, stat, part);
      }
      ProfileScope ps("cache_join_tile", s);
      FOE_LAUNCH((cache_join_kernel<HD, false>), dim3(p.max_tiles * (kTileCols / 32), a.H, a.B),
                 dim3(256), 0, s, w, p.many_ranges, kManyLeast, kTileCols, part, ob, stat);
    }
    if (mass_out != nullptr) {
      ProfileScope ps("cache_mass", s);
      FOE_LAUNCH(cache_mass_kernel<HD>, dim3(a.max_blocks, a.H, a.B), dim3(kAttThr), 0, s, qb, a.k,
                 a.kv_scale, bt, max_rows, c_log2, stat, mass_in, mass_out);
    }
  };
  if (a.hd == 96) go(std::integral_constant<int, 96>{});
  else go(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace foe
