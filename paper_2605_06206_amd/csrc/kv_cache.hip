// The 8-bit key/value cache: appending new tokens (rotation and quantisation)
// and evicting the tokens that received the least attention.
#include <algorithm>

#include "kv_cache.hpp"
#include "lds_dma.hpp"

namespace foe {
namespace {

// ---- append -------------------------------------------------------------------
// One workgroup per (touched page, group).  Thread (row, u) holds the key pairs
// 4u .. 4u+3 (dims i and i + HD/2) and the value dims 8u .. 8u+7 of a row, and of the
// rows 16, 32 and 48 further on; all rows' loads of a head are in flight together, the
// next head's behind them.
// (1) Rotary embedding with the angle (p / scale) * theta^(-2i/HD) formed in double and
// reduced modulo 2 pi, for every eighth of the page's positions and for the distances
// 0 .. 7; a position's sine and cosine follow from the two (a quarter of the sines).
// q goes out in bf16, the rotated key is quantised from its fp32 value.  (2) The page's
// scales from the largest new magnitudes and, if the page held tokens, its old scales;
// a scale that grows rescales the page's other codes.  (3) Key rows are stored as they
// are held; values go through LDS into 16-byte pieces of one dim and 16 tokens, the
// tokens around the new ones kept.
// us for 4096 rows of 8 groups, two query heads, hd 128 (59 MB: 11.5): a sine a position
// and a row's heads one after another 22, so 16.
constexpr int kAppThr = 256;

template <int HD>
__global__ __launch_bounds__(kAppThr) void cache_append_kernel(
    const bf16* __restrict__ qkv, bf16* __restrict__ q_out, uint8_t* __restrict__ kc,
    uint8_t* __restrict__ vc, float* __restrict__ kv_scale, CacheBatch bt,
    const int32_t* __restrict__ pos, double log2_theta, double rope_scale) {
  constexpr int NIT = kPage * 16 / kAppThr;  // rows of a thread
  constexpr int VROW = kPage + 4;            // bytes of a value dim's row in LDS
  // (cosine, sine) of pair i at positions first + 8 a (rows 0-7) and b (rows 8-15)
  __shared__ float2 turn[16][HD / 2];
  __shared__ __align__(16) uint8_t vt[HD * VROW];
  __shared__ double inv_freq[HD / 2];
  const int tid = threadIdx.x, h = blockIdx.y;
  // (the first frequency is 1 for an infinite base too, where 0 * log2 is NaN)
  if (tid < HD / 2) inv_freq[tid] = tid == 0 ? 1.0 : exp2(-2.0 * tid / HD * log2_theta);
  int b, local;
  const bool any = find_tile<kAppThr>(
      bt.B, blockIdx.x,
      [&](int i) {
        const int n = bt.rows(i), c = bt.context(i);
        return n > 0 ? (c + n - 1) / kPage - c / kPage + 1 : 0;
      },
      b, local);
  if (!any) return;
  const int c0 = bt.context(b), r0 = bt.first_row(b);
  const int blk = c0 / kPage + local;
  const int lo = max(c0 - blk * kPage, 0), hi = min(c0 + bt.rows(b) - blk * kPage, kPage);
  const int page = bt.page(b, blk);
  const int i0 = blk * kPage + lo - c0;  // the sequence's row at slot lo

  const int u = tid & 15, rr = tid >> 4;
  const bool act = u < HD / 8;
  // row of the thread's it-th slot; rows past the last are loaded as it and not stored
  const int cnt = hi - lo;
  const size_t row0 = (size_t)h * bt.N + r0 + i0;
  auto row_of = [&](int it) { return row0 + min(it * (kAppThr / 16) + rr, cnt - 1); };
  auto has = [&](int it) { return act && it * (kAppThr / 16) + rr < cnt; };
  auto some = [&](int it) { return it * (kAppThr / 16) < cnt; };  // (uniform)
  const int uc = act ? u : 0;
  bf16x8 v[NIT];
  bf16x4 x1[NIT], x2[NIT];
  auto load_head = [&](int j) {
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
      if (!some(it)) continue;
      const bf16* src = qkv + (row_of(it) * (bt.nq + 2) + j) * HD + 4 * uc;
      x1[it] = *reinterpret_cast<const bf16x4*>(src);
      x2[it] = *reinterpret_cast<const bf16x4*>(src + HD / 2);
    }
  };
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    x1[it] = x2[it] = bf16x4{};
    v[it] = bf16x8{};
    if (some(it))
      v[it] = *reinterpret_cast<const bf16x8*>(qkv + (row_of(it) * (bt.nq + 2) + bt.nq + 1) * HD +
                                               8 * uc);
  }
  load_head(0);
  // what the page holds that the new tokens are put beside: its scales, and the value
  // pieces that they share with other tokens
  constexpr int NV = ((kPage / kSub) * HD + kAppThr - 1) / kAppThr;
  float* sp = kv_scale + ((size_t)max(page, 0) * bt.H + h) * 2;
  uint8_t* kp = kc + ((size_t)max(page, 0) * bt.H + h) * (kPage * HD);
  uint8_t* vp = vc + ((size_t)max(page, 0) * bt.H + h) * (kPage * HD);
  const float2 scale_was =
      lo > 0 && page >= 0 ? *reinterpret_cast<const float2*>(sp) : float2{0.f, 0.f};
  auto touched = [&](int t0) { return t0 < hi && t0 + kSub > lo; };
  auto full = [&](int t0) { return t0 >= lo && t0 + kSub <= hi; };
  u32x4 beside[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = k * kAppThr + tid, t0 = i / HD * kSub;
    beside[k] = zero_u32x4();
    if (page >= 0 && t0 < kPage && touched(t0) && !full(t0))
      beside[k] = *reinterpret_cast<const u32x4*>(vp + i * 16);
  }
  {
    const long long first = (pos != nullptr ? pos[b] : c0) + (long long)i0;
    constexpr double kTwoPi = 6.283185307179586476925286766559;
    const int na = (cnt + 7) / 8, nb = min(cnt, 8);
    for (int e = tid; e < (na + nb) * (HD / 2); e += kAppThr) {
      const int k = e / (HD / 2), i = e % (HD / 2);
      double a = (double)(k < na ? first + 8 * k : k - na) / rope_scale * inv_freq[i];
      a -= kTwoPi * floor(a / kTwoPi);
      float2 t;
      sincosf((float)a, &t.y, &t.x);
      turn[k < na ? k : 8 + k - na][i] = t;
    }
  }
  __syncthreads();
  float cs[NIT][4], sn[NIT][4];
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    const int i = min(it * (kAppThr / 16) + rr, cnt - 1);  // position - first
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 a = turn[i >> 3][4 * uc + e], d = turn[8 + (i & 7)][4 * uc + e];
      cs[it][e] = a.x * d.x - a.y * d.y;
      sn[it][e] = a.y * d.x + a.x * d.y;
    }
  }
  auto rotate = [&](int it, float* y) {  // dims 4u .. +3, then HD/2 on
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float a1 = (float)x1[it][e], a2 = (float)x2[it][e];
      y[e] = a1 * cs[it][e] - a2 * sn[it][e];
      y[4 + e] = a2 * cs[it][e] + a1 * sn[it][e];
    }
  };
  for (int j = 0; j < bt.nq; ++j) {
    bf16x8 y8[NIT];
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
      float y[8];
      rotate(it, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) y8[it][e] = (bf16)y[e];
    }
    load_head(j + 1);  // (the key follows the last query)
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
      if (!has(it)) continue;
      bf16* dst = q_out + (row_of(it) * bt.nq + j) * HD + 4 * u;
      *reinterpret_cast<bf16x4*>(dst) = bf16x4{y8[it][0], y8[it][1], y8[it][2], y8[it][3]};
      *reinterpret_cast<bf16x4*>(dst + HD / 2) = bf16x4{y8[it][4], y8[it][5], y8[it][6], y8[it][7]};
    }
  }
  bool bad[NIT];  // a row that no codes hold
  float2 amax{0.f, 0.f};
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    bool too_large = false;  // or NaN
    float2 m{0.f, 0.f};
    float y[8];
    rotate(it, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float k = fabsf(y[e]), w = fabsf((float)v[it][e]);
      too_large |= !(k < kTooLarge) || !(w < kTooLarge);
      m.x = fmaxf(m.x, k);
      m.y = fmaxf(m.y, w);
    }
    // such a row counts for no scale
    const uint64_t any_bad = __builtin_amdgcn_ballot_w64(too_large && has(it));
    bad[it] = ((any_bad >> (lane_id() & 48)) & 0xffffu) != 0;
    if (!bad[it] && has(it)) amax = float2{fmaxf(amax.x, m.x), fmaxf(amax.y, m.y)};
  }
  if (page < 0) return;  // (uniform) nowhere to store
  amax = block_max<kAppThr>(amax);
  // (scale_was is 0 where the page held no token: its other codes are left)
  const float ks = fmaxf(block_scale(amax.x), scale_was.x);
  const float vs = fmaxf(block_scale(amax.y), scale_was.y);
  const float ki = pow2_inv(ks), vi = pow2_inv(vs);
  const float kratio = lo > 0 ? scale_was.x * ki : 1.f, vratio = lo > 0 ? scale_was.y * vi : 1.f;

#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    if (!has(it)) continue;
    const int t = lo + it * (kAppThr / 16) + rr;
    float k[8], w[8];
    rotate(it, k);  // (again: its registers are not held meanwhile)
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = (float)v[it][e] * vi;
    uint32_t c0w = to_codes4(k[0] * ki, k[1] * ki, k[2] * ki, k[3] * ki);
    uint32_t c1w = to_codes4(k[4] * ki, k[5] * ki, k[6] * ki, k[7] * ki);
    uint32_t v0w = to_codes4(w[0], w[1], w[2], w[3]), v1w = to_codes4(w[4], w[5], w[6], w[7]);
    if (bad[it]) c0w = c1w = 0x7f7f7f7fu, v0w = v1w = 0u;
    *reinterpret_cast<uint32_t*>(kp + t * HD + 4 * u) = c0w;
    *reinterpret_cast<uint32_t*>(kp + t * HD + HD / 2 + 4 * u) = c1w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      vt[(8 * u + e) * VROW + t] = (uint8_t)(v0w >> (8 * e));
      vt[(8 * u + 4 + e) * VROW + t] = (uint8_t)(v1w >> (8 * e));
    }
  }
  if (kratio != 1.f)  // the page's other rows, in units of the new scale
    for (int i = tid; i < kPage * (HD / 16); i += kAppThr) {
      if (i >= lo * (HD / 16) && i < hi * (HD / 16)) continue;
      u32x4* w = reinterpret_cast<u32x4*>(kp + i * 16);
      u32x4 x = *w;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = rescale4(x[e], kratio);
      *w = x;
    }
  __syncthreads();
  if (tid == 0) *reinterpret_cast<float2*>(sp) = float2{ks, vs};
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int i = n * kAppThr + tid, d = i % HD, t0 = i / HD * kSub;
    if (t0 >= kPage || (!touched(t0) && vratio == 1.f)) continue;
    u32x4* w = reinterpret_cast<u32x4*>(vp + i * 16);
    u32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x[e] = *reinterpret_cast<const uint32_t*>(vt + d * VROW + t0 + 4 * e);
    if (full(t0)) {
      *w = x;
      continue;
    }
    u32x4 old = touched(t0) ? beside[n] : *w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t fresh = 0;  // bytes of the new tokens
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int t = t0 + 4 * e + k;
        if (t >= lo && t < hi) fresh |= 0xffu << (8 * k);
      }
      const uint32_t o = vratio != 1.f ? rescale4(old[e], vratio) : old[e];
      old[e] = (o & ~fresh) | (x[e] & fresh);
    }
    *w = old;
  }
}

// ---- eviction -------------------------------------------------------------------
// Selection of the keep - recent largest masses among the tokens before the recent
// ones, per (sequence, group).  The masses are mapped to unsigned keys of the same
// order; the smallest kept key is found digit by digit, 11, 11 and 10 bits, counted in
// LDS (the first digit ends inside the significand, so masses of similar size spread
// over counters); the tokens above it, and the first ones equal to it, are listed in
// token order from ballots.  A workgroup holds the keys of 32768 tokens in registers,
// four neighbouring tokens to a register group.  Where the table has room for more, each
// 32768 tokens have a workgroup, their counts are joined between launches, one for each
// digit and one that lists.
// us for two sequences of 131072 tokens, 8 groups: one workgroup a sequence and group
// with 8-bit digits, each pass from memory 398, with these digits 113 (its compute unit's
// vector instructions are the bound), spread 53, of which the last launch 22 as it found all
// three digits again; with the state handed on 45.  24 of at most 16000 tokens: 76, 17.
constexpr int kSelThr = 1024;
constexpr int kSelWaves = kSelThr / kWave;
constexpr int kSelRegs = 8;                          // 4-token pieces of a thread
constexpr int kSelTokens = kSelThr * 4 * kSelRegs;   // tokens of a workgroup
constexpr int kSelBins = 2048;

__device__ __forceinline__ int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ int digit_bits(int pass) { return pass == 2 ? 10 : 11; }

__device__ __forceinline__ uint32_t mass_key(float m) {
  if (m != m) return 0xffffffffu;  // NaN ranks first
  const uint32_t u = m == 0.f ? 0u : __float_as_uint(m);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Keys of tokens base + (j * 1024 + thread) * 4 + e.  Tokens past the old ones, and of
// absent pages, get the lowest key: they come after every other of the same key, and
// fewer than `old` are kept.
__device__ __forceinline__ void load_keys(const float* mass, const CacheBatch& bt, int b, int h,
                                          int old, int base, u32x4* key) {
  int page[kSelRegs];
  f32x4 m[kSelRegs];
#pragma unroll
  for (int j = 0; j < kSelRegs; ++j)  // (a token's page is within the table)
    page[j] = bt.table[(size_t)b * bt.max_blocks +
                       min(base + (j * kSelThr + (int)threadIdx.x) * 4, old - 1) / kPage];
#pragma unroll
  for (int j = 0; j < kSelRegs; ++j) {
    const int t = (base + (j * kSelThr + (int)threadIdx.x) * 4) % kPage;
    const size_t p = page[j] >= 0 && page[j] < bt.n_pages ? page[j] : 0;
    m[j] = *reinterpret_cast<const f32x4*>(mass + (p * bt.H + h) * kPage + t);
  }
#pragma unroll
  for (int j = 0; j < kSelRegs; ++j) {
    const int t = base + (j * kSelThr + (int)threadIdx.x) * 4;
    const bool absent = page[j] < 0 || page[j] >= bt.n_pages;
#pragma unroll
    for (int e = 0; e < 4; ++e) key[j][e] = absent || t + e >= old ? 0u : mass_key(m[j][e]);
  }
}

// Counts the next digit of the keys that have the prefix; np pieces hold tokens.
__device__ __forceinline__ void count_keys(const u32x4* key, int np, int pass, uint32_t prefix,
                                           int* hist) {
  const int shift = digit_shift(pass), bits = digit_bits(pass), lane = lane_id();
  __syncthreads();
  hist[threadIdx.x] = 0;
  hist[threadIdx.x + kSelThr] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSelRegs; ++j) {
    if (j >= np) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t k = key[j][e];
      if (pass > 0 && (k >> (shift + bits)) != (prefix >> (shift + bits))) continue;
      const int d = (k >> shift) & ((1 << bits) - 1);
      // lanes with the first lane's digit count together (equal masses)
      const int d0 = __builtin_amdgcn_readfirstlane(d);
      const uint64_t same = __builtin_amdgcn_ballot_w64(d == d0);
      if (d != d0) atomicAdd(&hist[d], 1);
      else if ((same & (((uint64_t)1 << lane) - 1)) == 0) atomicAdd(&hist[d], __popcll(same));
    }
  }
  __syncthreads();
}

// A thread's digits, two by two from the largest: first_digit and the one below (negative:
// none).
__device__ __forceinline__ int first_digit(int pass) {
  return (1 << digit_bits(pass)) - 1 - 2 * (int)threadIdx.x;
}
// The digit of the want-th largest key, and how many keys have a larger one, from the counts
// of the thread's digits.
__device__ __forceinline__ void find_digit(int pass, int c1, int c2, uint32_t& prefix, int& want) {
  __shared__ int wsum[kSelWaves];
  __shared__ int sh[2];
  const int lane = lane_id(), wave = threadIdx.x >> 6, hi = first_digit(pass);
  int incl = c1 + c2;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int up = __shfl_up(incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == kWave - 1) wsum[wave] = incl;
  __syncthreads();
  for (int w = 0; w < wave; ++w) incl += wsum[w];
  const int above = incl - c1 - c2;
  if (above < want && want <= incl) {
    const bool first = want <= above + c1;
    sh[0] = first ? hi : hi - 1;
    sh[1] = first ? above : above + c1;
  }
  __syncthreads();
  prefix |= (uint32_t)sh[0] << digit_shift(pass);
  want -= sh[1];
}

// Lists the tokens above the prefix and the first `want` equal to it; gt and eq tokens
// came before.
__device__ __forceinline__ void list_keys(const u32x4* key, int np, int base, uint32_t prefix,
                                          int want, int gt, int eq, int32_t* out) {
  constexpr int NC = kSelRegs * kSelWaves;
  __shared__ int2 cnt[NC];  // tokens (above, equal) of a wave's piece, then of those before
  __shared__ int2 half;
  const int lane = lane_id(), wave = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < kSelRegs; ++j) {
    int g = 0, q = 0;
    if (j < np) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g += __popcll(__builtin_amdgcn_ballot_w64(key[j][e] > prefix));
        q += __popcll(__builtin_amdgcn_ballot_w64(key[j][e] == prefix));
      }
    }
    if (lane == 0) cnt[j * kSelWaves + wave] = int2{g, q};
  }
  __syncthreads();
  static_assert(NC == 2 * kWave, "two waves' scan");
  int2 mine{0, 0}, incl{0, 0};
  if (threadIdx.x < NC) {
    mine = incl = cnt[threadIdx.x];
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int ug = __shfl_up(incl.x, o), uq = __shfl_up(incl.y, o);
      if (lane >= o) incl.x += ug, incl.y += uq;
    }
    if (threadIdx.x == kWave - 1) half = incl;
  }
  __syncthreads();
  if (threadIdx.x < NC) {
    if (wave == 1) incl.x += half.x, incl.y += half.y;
    cnt[threadIdx.x] = int2{gt + incl.x - mine.x, eq + incl.y - mine.y};
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSelRegs; ++j) {
    if (j >= np) continue;
    const int2 x = cnt[j * kSelWaves + wave];
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    int pg = x.x, pe = x.y;  // before this lane's first token
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      pg += __popcll(__builtin_amdgcn_ballot_w64(key[j][e] > prefix) & below);
      pe += __popcll(__builtin_amdgcn_ballot_w64(key[j][e] == prefix) & below);
    }
    const int t = base + (j * kSelThr + (int)threadIdx.x) * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool g = key[j][e] > prefix, q = key[j][e] == prefix;
      if (g || (q && pe < want)) out[pg + min(pe, want)] = t + e;
      pg += g;
      pe += q;
    }
  }
}

// pieces that hold tokens of a workgroup's
__device__ __forceinline__ int key_pieces(int old, int base) {
  return min(kSelRegs, (old - base + kSelThr * 4 - 1) / (kSelThr * 4));
}

// The whole of a sequence's old tokens in one workgroup.
__global__ __launch_bounds__(kSelThr) void cache_select_kernel(
    const float* __restrict__ mass, CacheBatch bt, int keep, int recent, int32_t* __restrict__ kept,
    int32_t* __restrict__ new_len) {
  __shared__ int hist[kSelBins];
  const int tid = threadIdx.x, h = blockIdx.x, b = blockIdx.y;
  const int n = bt.context(b);
  int32_t* out = kept + ((size_t)b * bt.H + h) * keep;
  if (h == 0 && tid == 0) new_len[b] = min(n, keep);
  if (n <= keep) {
    for (int j = tid; j < keep; j += kSelThr) out[j] = j < n ? j : -1;
    return;
  }
  const int old = n - recent, need = keep - recent;  // 0 <= need < old
  for (int j = tid; j < recent; j += kSelThr) out[need + j] = old + j;
  if (need == 0) return;
  u32x4 key[kSelRegs];
  load_keys(mass, bt, b, h, old, 0, key);
  const int np = key_pieces(old, 0);
  uint32_t prefix = 0;
  int want = need;  // of the keys with this prefix, the largest `want` are kept
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    count_keys(key, np, pass, prefix, hist);
    const int d = first_digit(pass);
    find_digit(pass, d > 0 ? hist[d] : 0, d > 0 ? hist[d - 1] : 0, prefix, want);
  }
  list_keys(key, np, 0, prefix, want, 0, 0, out);
}

// One workgroup per 32768 tokens: launch `pass` counts that digit into
// counts[pass][b][h][slice], launch 3 lists.  Each launch finds the digit counted before it;
// what the earlier ones are is in state[b][h][slice]: (prefix, want, tokens of the slices
// before that are above the prefix).
template <int PASS>
__global__ __launch_bounds__(kSelThr) void cache_select_slice_kernel(
    const float* __restrict__ mass, CacheBatch bt, int keep, int recent, int* __restrict__ counts,
    int4* __restrict__ state, int32_t* __restrict__ kept, int32_t* __restrict__ new_len) {
  __shared__ int hist[kSelBins];
  __shared__ int before[2];
  const int tid = threadIdx.x, slice = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int n = bt.context(b);
  const int old = n - recent, need = keep - recent, base = slice * kSelTokens;
  int32_t* out = kept + ((size_t)b * bt.H + h) * keep;
  if (PASS == 3) {
    if (h == 0 && slice == 0 && tid == 0) new_len[b] = min(n, keep);
    const int at = slice * kSelThr + tid, step = gridDim.x * kSelThr;
    if (n <= keep) {
      for (int j = at; j < keep; j += step) out[j] = j < n ? j : -1;
    } else {
      for (int j = at; j < recent; j += step) out[need + j] = old + j;
    }
  }
  if (n <= keep || need == 0 || base >= old) return;
  u32x4 key[kSelRegs];
  load_keys(mass, bt, b, h, old, base, key);
  const int np = key_pieces(old, base), slices = (old + kSelTokens - 1) / kSelTokens;
  auto counts_of = [&](int pass) {
    return counts + (((size_t)pass * bt.B + b) * bt.H + h) * gridDim.x * kSelBins;
  };
  state += ((size_t)b * bt.H + h) * gridDim.x + slice;
  uint32_t prefix = 0;
  int want = need, gt = 0, eq = 0;
  if constexpr (PASS > 1) {
    const int4 x = *state;
    prefix = (uint32_t)x.x, want = x.y, gt = x.z;
  }
  if constexpr (PASS > 0) {
    const int d = first_digit(PASS - 1);
    const int* c = counts_of(PASS - 1) + d - 1;
    int2 all{0, 0}, ahead{0, 0};  // digits (d - 1, d), of all slices and of those before
    if (d > 0) {
#pragma unroll 4
      for (int s = 0; s < slices; ++s) {
        const int2 x = *reinterpret_cast<const int2*>(c + (size_t)s * kSelBins);
        all.x += x.x, all.y += x.y;
        if (s < slice) ahead.x += x.x, ahead.y += x.y;
      }
    }
    if (tid == 0) before[0] = before[1] = 0;
    find_digit(PASS - 1, all.y, all.x, prefix, want);
    // tokens of the slices before with a larger digit, and at last with the same
    const int at = (prefix >> digit_shift(PASS - 1)) & ((1 << digit_bits(PASS - 1)) - 1);
    const int larger = (d > at ? ahead.y : 0) + (d - 1 > at ? ahead.x : 0);
    const int same = d == at ? ahead.y : d - 1 == at ? ahead.x : 0;
    if (larger > 0) atomicAdd(&before[0], larger);
    if (PASS == 3 && same > 0) atomicAdd(&before[1], same);
    __syncthreads();
    gt += before[0];
    eq = before[1];
    if (PASS < 3 && tid == 0) *state = int4{(int)prefix, want, gt, 0};
  }
  if constexpr (PASS == 3) {
    list_keys(key, np, base, prefix, want, gt, eq, out);
  } else {
    count_keys(key, np, PASS, prefix, hist);
    int* c = counts_of(PASS) + (size_t)slice * kSelBins;
    for (int d = tid; d < 1 << digit_bits(PASS); d += kSelThr) c[d] = hist[d];
  }
}

// Moving the kept tokens: one workgroup per (page of the result, group, sequence).
// Keys: thread -> 16 bytes of a row.  Values: the 128 threads of group g = 0..3 (a thread
// a dim) gather the 16 tokens 16 g .. +15 of the page; a token is the same for all of
// them, so its address and its byte within 4 bytes are scalars, and a byte permutation puts
// it in its place.  Where the 16 tokens come out of at most four 16-byte pieces of the
// source (tokens kept thickly), a wave loads the pieces into its own LDS and takes the
// bytes from there; else it loads 4 bytes of each token, which touch the same cache lines
// once a token.  A token's place is a chain of loads (its number, its page, the page's
// scales, the codes), hidden by the four workgroups that a CU has room for.
// us for 16 sequences of 16000 tokens, 8 groups, cut to 12000, 8000, 5300, 4000, 2000:
// always 4 bytes 272 176 124 102 64; so 210 144 116 100 65; pieces alone, four at a time,
// 222 148 116 100 67.  For two of 131072 cut to half (the sources' cache lines and the
// results are 640 MB: 125) 147; a load for each byte 249; bytes taken out of pieces in
// registers 193 to 383; a wave for each page's keys and one for its values 401; each
// wave finding its tokens for itself, without barriers, 197.
constexpr int kMoveThr = 512;
constexpr int kMovePieces = 4;  // (32 KB of LDS)

template <int HD>
__global__ __launch_bounds__(kMoveThr, 8) void cache_move_kernel(
    uint8_t* __restrict__ kc, uint8_t* __restrict__ vc, float* __restrict__ kv_scale,
    float* __restrict__ mass, CacheBatch bt, const int32_t* __restrict__ dst_table, int dst_blocks,
    int keep, const int32_t* __restrict__ kept) {
  constexpr int CPR = HD / 16;
  __shared__ __align__(16) uint8_t vstage[kMoveThr / kWave * kMovePieces * 1024];
  __shared__ int sp[kPage], st[kPage];
  __shared__ float2 ss[kPage];
  const int tid = threadIdx.x, blk = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cnt = min(min(bt.context(b), keep) - blk * kPage, kPage);
  if (cnt <= 0) return;
  const int dp = dst_table[(size_t)b * dst_blocks + blk];
  auto lane_f = [&](float x, int i) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i));
  };
  if (tid < kPage) {
    const int t = tid < cnt ? kept[((size_t)b * bt.H + h) * keep + blk * kPage + tid] : -1;
    const int p = t >= 0 ? bt.page(b, t / kPage) : -1;
    sp[tid] = p;
    st[tid] = t >= 0 ? t % kPage : 0;
    ss[tid] = p >= 0 ? *reinterpret_cast<const float2*>(kv_scale + ((size_t)p * bt.H + h) * 2)
                     : float2{0.f, 0.f};
  }
  __syncthreads();
  const int kt = tid / CPR;            // key row
  const int g = tid >> 7, d = tid & 127;
  u32x4 kw = zero_u32x4();
  const bool has_k = kt < cnt && sp[kt] >= 0;
  if (has_k)
    kw = *reinterpret_cast<const u32x4*>(kc + ((size_t)sp[kt] * bt.H + h) * (kPage * HD) +
                                         st[kt] * HD + (tid % CPR) * 16);
  float m = 0.f;
  if (tid < cnt && sp[tid] >= 0) m = mass[((size_t)sp[tid] * bt.H + h) * kPage + st[tid]];
  // values: token 16 g + i in lane i of every wave
  const int my_page = sp[g * kSub + (lane & 15)], my_tok = st[g * kSub + (lane & 15)];
  const float my_scale = ss[g * kSub + (lane & 15)].y;
  // where its 4 bytes are in dim 0, and the permutation that puts its byte at i % 4
  // (an absent token: a zero byte)
  const int at = (lane & 3) * 8;
  const uint32_t my_sel = (0x03020100u & ~(0xffu << at)) |
                          ((my_page < 0 ? 0x0cu : 4u + (my_tok & 3)) << at);
  const uint64_t my_off =
      my_page < 0 ? 0
                  : ((uint64_t)my_page * bt.H + h) * (kPage * HD) +
                        (uint32_t)((my_tok / kSub) * (HD * kSub) + (my_tok % kSub & ~3));
  const uint32_t dim = min(d, HD - 1) * kSub;
  auto place_of = [&](int i) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(my_off >> 32), i) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((uint32_t)my_off, i);
  };
  // tokens whose 16-byte pieces differ from the previous token's
  const uint32_t piece_lo = (uint32_t)my_off & ~15u, piece_hi = (uint32_t)(my_off >> 32);
  // (all lanes take part in the shuffles)
  const uint32_t last_lo = __shfl_up(piece_lo, 1), last_hi = __shfl_up(piece_hi, 1);
  const bool turns = lane == 0 || piece_lo != last_lo || piece_hi != last_hi;
  const uint32_t turn = (uint32_t)__builtin_amdgcn_ballot_w64(turns) & 0xffffu;
  const int my_piece = __popc(turn & ((2u << (lane & 15)) - 1)) - 1;
  const bool staged = __popc(turn) <= kMovePieces;  // (uniform)
  const uint32_t mine = lds_addr(vstage) + wave * (kMovePieces * 1024);
  uint32_t got[kSub / 2];
  if (staged) {
    uint32_t rest = turn;
#pragma unroll
    for (int k = 0; k < kMovePieces; ++k) {
      if (rest == 0) continue;
      const uint64_t off = place_of(__builtin_ctz(rest)) & ~(uint64_t)15;
      rest &= rest - 1;
      const __amdgpu_buffer_rsrc_t piece = make_rsrc_u(vc + off, HD * kSub);
      rsrc_settle(piece);
      dma16(piece, dim, mine, k * 1024);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kSub / 2; ++i)
      got[i] = *reinterpret_cast<const uint32_t*>(vc + place_of(i) + dim);
  }
  float2 amax{0.f, 0.f};  // (a NaN code counts for no scale)
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float x = fmaxf(fabsf(__builtin_amdgcn_cvt_f32_fp8(kw[e], 0)),
                    fabsf(__builtin_amdgcn_cvt_f32_fp8(kw[e], 1)));
    x = fmaxf(x, fmaxf(fabsf(__builtin_amdgcn_cvt_f32_fp8(kw[e], 2)),
                       fabsf(__builtin_amdgcn_cvt_f32_fp8(kw[e], 3))));
    if (has_k) amax.x = fmaxf(amax.x, x * ss[kt].x);
  }
  u32x4 vw = zero_u32x4();
  auto place_byte = [&](int i, uint32_t x) {
    vw[i / 4] = __builtin_amdgcn_perm(x, vw[i / 4], __builtin_amdgcn_readlane(my_sel, i));
  };
  if (staged) {
    vm_wait<0>();
    const uint32_t from = my_piece * 1024 + (my_tok % kSub & ~3);
#pragma unroll
    for (int i = 0; i < kSub; ++i)
      place_byte(i, *reinterpret_cast<const uint32_t*>(
                        vstage + wave * (kMovePieces * 1024) + lane * 16 +
                        __builtin_amdgcn_readlane(from, i)));
  } else {
#pragma unroll
    for (int i = 0; i < kSub / 2; ++i) {
      place_byte(i, got[i]);
      got[i] = *reinterpret_cast<const uint32_t*>(vc + place_of(kSub / 2 + i) + dim);
    }
#pragma unroll
    for (int i = 0; i < kSub / 2; ++i) place_byte(kSub / 2 + i, got[i]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x0 = fabsf(__builtin_amdgcn_cvt_f32_fp8(vw[e], 0)) * lane_f(my_scale, 4 * e);
    const float x1 = fabsf(__builtin_amdgcn_cvt_f32_fp8(vw[e], 1)) * lane_f(my_scale, 4 * e + 1);
    const float x2 = fabsf(__builtin_amdgcn_cvt_f32_fp8(vw[e], 2)) * lane_f(my_scale, 4 * e + 2);
    const float x3 = fabsf(__builtin_amdgcn_cvt_f32_fp8(vw[e], 3)) * lane_f(my_scale, 4 * e + 3);
    amax.y = fmaxf(fmaxf(amax.y, x0), fmaxf(fmaxf(x1, x2), x3));
  }
  amax = block_max<kMoveThr>(amax);
  const float ks = block_scale(amax.x), vs = block_scale(amax.y);
  const float ki = pow2_inv(ks), vi = pow2_inv(vs);
  if (dp >= 0 && dp < bt.n_pages) {
    const size_t dst = (size_t)dp * bt.H + h;
    if (tid == 0) *reinterpret_cast<float2*>(kv_scale + dst * 2) = float2{ks, vs};
    if (tid < cnt) mass[dst * kPage + tid] = m;
    if (kt < cnt) {
      const float r = scale_ratio(ss[kt].x, ki);
      if (r != 1.f) {
#pragma unroll
        for (int e = 0; e < 4; ++e) kw[e] = rescale4(kw[e], r);
      }
      *reinterpret_cast<u32x4*>(kc + dst * (kPage * HD) + tid * 16) = kw;
    }
    if (g * kSub < cnt && d < HD) {
      u32x4* w = reinterpret_cast<u32x4*>(vc + dst * (kPage * HD) + (g * HD + d) * kSub);
      const int left = cnt - g * kSub;  // slots past the kept tokens stay as they were
      const u32x4 was = left < kSub ? *w : zero_u32x4();
      const float r = scale_ratio(my_scale, vi);
      if (__builtin_amdgcn_ballot_w64(r != 1.f)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t x = vw[e];
          vw[e] = to_codes4(__builtin_amdgcn_cvt_f32_fp8(x, 0) * lane_f(r, 4 * e),
                            __builtin_amdgcn_cvt_f32_fp8(x, 1) * lane_f(r, 4 * e + 1),
                            __builtin_amdgcn_cvt_f32_fp8(x, 2) * lane_f(r, 4 * e + 2),
                            __builtin_amdgcn_cvt_f32_fp8(x, 3) * lane_f(r, 4 * e + 3));
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int in = left - 4 * e;
        const uint32_t mk = in >= 4 ? 0xffffffffu : in <= 0 ? 0u : (1u << (8 * in)) - 1;
        vw[e] = (vw[e] & mk) | (was[e] & ~mk);
      }
      *w = vw;
    }
  }
}

}  // namespace

hipError_t launch_cache_append(const CacheArgs& a, int nq, int N, const void* qkv, void* q,
                               const int32_t* row_start, const int32_t* pos, float theta,
                               float scale, hipStream_t s) {
  const CacheBatch bt{a.H, a.B, N, nq, a.n_pages, a.max_blocks, a.block_table, a.length, row_start};
  // pages that n rows touch: at most (n + 62) / 64 + 1, and n
  const long long tiles = std::min<long long>(N, ((long long)N + 62LL * a.B) / kPage + a.B);
  ProfileScope ps("cache_append", s);
  auto go = [&](auto kern) {
    FOE_LAUNCH(kern, dim3((unsigned)tiles, a.H), dim3(kAppThr), 0, s,
               static_cast<const bf16*>(qkv), static_cast<bf16*>(q), a.k, a.v, a.kv_scale, bt, pos,
               log2((double)theta), (double)scale);
  };
  if (a.hd == 96) go(cache_append_kernel<96>);
  else go(cache_append_kernel<128>);
  return hipGetLastError();
}

// the table has room for more tokens than a workgroup holds
static int select_slices(int max_blocks) {
  return ceil_div((long long)max_blocks * kPage, kSelTokens);
}

static size_t select_counts(int H, int B, int slices) {
  return (size_t)3 * B * H * slices * kSelBins;
}

size_t cache_evict_scratch_bytes(int H, int B, int max_blocks) {
  const int slices = select_slices(max_blocks);
  return slices > 1 ? select_counts(H, B, slices) * 4 + (size_t)B * H * slices * sizeof(int4) : 0;
}

hipError_t launch_cache_evict(const CacheArgs& a, float* mass, int keep, int recent,
                              const int32_t* dst_table, int dst_blocks, int32_t* kept,
                              int32_t* new_len, void* scratch, hipStream_t s) {
  const CacheBatch bt{a.H, a.B, 0, 0, a.n_pages, a.max_blocks, a.block_table, a.length, nullptr};
  const int slices = select_slices(a.max_blocks);
  if (slices == 1) {
    ProfileScope ps("cache_select", s);
    FOE_LAUNCH(cache_select_kernel, dim3(a.H, a.B), dim3(kSelThr), 0, s, mass, bt, keep, recent,
               kept, new_len);
  } else {
    int* counts = static_cast<int*>(scratch);
    int4* state = reinterpret_cast<int4*>(counts + select_counts(a.H, a.B, slices));
    auto go = [&](auto kern, const char* name) {
      ProfileScope ps(name, s);
      FOE_LAUNCH(kern, dim3(slices, a.H, a.B), dim3(kSelThr), 0, s, mass, bt, keep, recent,
                 counts, state, kept, new_len);
    };
    go(cache_select_slice_kernel<0>, "cache_select_0");
    go(cache_select_slice_kernel<1>, "cache_select_1");
    go(cache_select_slice_kernel<2>, "cache_select_2");
    go(cache_select_slice_kernel<3>, "cache_select_3");
  }
  {
    ProfileScope ps("cache_move", s);
    const int blocks = std::min(ceil_div(keep, kPage), a.max_blocks);
    auto go = [&](auto kern) {
      FOE_LAUNCH(kern, dim3(blocks, a.H, a.B), dim3(kMoveThr), 0, s, a.k, a.v,
                 a.kv_scale, mass, bt, dst_table, dst_blocks, keep, kept);
    };
    if (a.hd == 96) go(cache_move_kernel<96>);
    else go(cache_move_kernel<128>);
  }
  return hipGetLastError();
}

}  // namespace foe
