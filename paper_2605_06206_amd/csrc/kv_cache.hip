// The 8-bit key/value cache: appending new tokens (rotation and quantisation)
// and evicting the tokens that received the least attention.
#include <algorithm>

#include "kv_cache.hpp"

namespace foe {
namespace {

// ---- append -------------------------------------------------------------------
// One workgroup per (touched page, group).  Thread (row, u) holds the key pairs
// 4u .. 4u+3 (dims i and i + HD/2) and the value dims 8u .. 8u+7 of a row.
// (1) Rotary embedding with the angle (p / scale) * theta^(-2i/HD) formed in
// double and reduced modulo 2 pi, as in the preparation pass of the prompt
// attention; q goes out in bf16, the rotated key is quantised from its fp32
// value.  (2) The page's scales from the largest new magnitudes and, if the
// page held tokens, its old scales; a scale that grows rescales the page's
// other codes.  (3) Key rows are stored as they are held; values go through LDS into
// 16-byte pieces of one dim and 16 tokens, the tokens around the new ones kept.
constexpr int kAppThr = 256;

template <int HD>
__global__ __launch_bounds__(kAppThr) void cache_append_kernel(
    const bf16* __restrict__ qkv, bf16* __restrict__ q_out, uint8_t* __restrict__ kc,
    uint8_t* __restrict__ vc, float* __restrict__ kv_scale, CacheBatch bt,
    const int32_t* __restrict__ pos, double log2_theta, double rope_scale) {
  constexpr int NIT = kPage * 16 / kAppThr;  // rows per thread
  __shared__ double inv_freq[HD / 2];
  __shared__ __align__(16) uint8_t vt[HD * kPage];
  const int tid = threadIdx.x, h = blockIdx.y;
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
  const int c0 = bt.context(b), n = bt.rows(b), r0 = bt.first_row(b);
  const int blk = c0 / kPage + local;
  const int lo = max(c0 - blk * kPage, 0), hi = min(c0 + n - blk * kPage, kPage);
  const int page = bt.page(b, blk);
  const long long p0 = pos != nullptr ? pos[b] : c0;

  const int u = tid & 15;
  const bool act = u < HD / 8;
  float kr[NIT][8], vr[NIT][8];
  bool bad[NIT];
  float2 amax{0.f, 0.f};
  constexpr double kTwoPi = 6.283185307179586476925286766559;
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    const int t = lo + it * (kAppThr / 16) + (tid >> 4);
    bool b_here = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) kr[it][e] = vr[it][e] = 0.f;
    if (act && t < hi) {
      const int i = blk * kPage + t - c0;  // row of the sequence
      float cs[4], sn[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        double a = (double)(p0 + i) / rope_scale * inv_freq[4 * u + e];
        a -= kTwoPi * floor(a / kTwoPi);
        sincosf((float)a, &sn[e], &cs[e]);
      }
      const size_t row = (size_t)h * bt.N + r0 + i;
      const bf16* src = qkv + row * (size_t)(bt.nq + 2) * HD;
      for (int j = 0; j <= bt.nq; ++j) {
        const bf16x4 x1 = *reinterpret_cast<const bf16x4*>(src + (size_t)j * HD + 4 * u);
        const bf16x4 x2 = *reinterpret_cast<const bf16x4*>(src + (size_t)j * HD + HD / 2 + 4 * u);
        float y1[4], y2[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float a1 = (float)x1[e], a2 = (float)x2[e];
          y1[e] = a1 * cs[e] - a2 * sn[e];
          y2[e] = a2 * cs[e] + a1 * sn[e];
        }
        if (j < bt.nq) {
          bf16* dst = q_out + (row * bt.nq + j) * HD + 4 * u;
          *reinterpret_cast<bf16x4*>(dst) =
              bf16x4{(bf16)y1[0], (bf16)y1[1], (bf16)y1[2], (bf16)y1[3]};
          *reinterpret_cast<bf16x4*>(dst + HD / 2) =
              bf16x4{(bf16)y2[0], (bf16)y2[1], (bf16)y2[2], (bf16)y2[3]};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) kr[it][e] = y1[e], kr[it][4 + e] = y2[e];
        }
      }
      const bf16x8 v = *reinterpret_cast<const bf16x8*>(src + (size_t)(bt.nq + 1) * HD + 8 * u);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        vr[it][e] = (float)v[e];
        b_here |= !(fabsf(kr[it][e]) < __builtin_inff()) || !(fabsf(vr[it][e]) < __builtin_inff());
      }
    }
    // a row with a non-finite key or value counts for no scale
    const uint64_t m = __builtin_amdgcn_ballot_w64(b_here);
    bad[it] = ((m >> (lane_id() & 48)) & 0xffffu) != 0;
    if (!bad[it]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        amax.x = fmaxf(amax.x, fabsf(kr[it][e]));
        amax.y = fmaxf(amax.y, fabsf(vr[it][e]));
      }
    }
  }
  if (page < 0) return;  // (uniform) nowhere to store
  amax = block_max<kAppThr>(amax);
  float* sp = kv_scale + ((size_t)page * bt.H + h) * 2;
  float ks = block_scale(amax.x), vs = block_scale(amax.y);
  float kratio = 1.f, vratio = 1.f;
  if (lo > 0) {
    const float ko = sp[0], vo = sp[1];
    ks = fmaxf(ks, ko);
    vs = fmaxf(vs, vo);
    kratio = ko * pow2_inv(ks);
    vratio = vo * pow2_inv(vs);
  }
  const float ki = pow2_inv(ks), vi = pow2_inv(vs);

  uint8_t* kp = kc + ((size_t)page * bt.H + h) * (kPage * HD);
  uint8_t* vp = vc + ((size_t)page * bt.H + h) * (kPage * HD);
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    const int t = lo + it * (kAppThr / 16) + (tid >> 4);
    if (!act || t >= hi) continue;
    const float* k = kr[it];
    const float* v = vr[it];
    uint32_t c0w = to_codes4(k[0] * ki, k[1] * ki, k[2] * ki, k[3] * ki);
    uint32_t c1w = to_codes4(k[4] * ki, k[5] * ki, k[6] * ki, k[7] * ki);
    uint32_t v0w = to_codes4(v[0] * vi, v[1] * vi, v[2] * vi, v[3] * vi);
    uint32_t v1w = to_codes4(v[4] * vi, v[5] * vi, v[6] * vi, v[7] * vi);
    if (bad[it]) c0w = c1w = 0x7f7f7f7fu, v0w = v1w = 0u;
    *reinterpret_cast<uint32_t*>(kp + t * HD + 4 * u) = c0w;
    *reinterpret_cast<uint32_t*>(kp + t * HD + HD / 2 + 4 * u) = c1w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      vt[(8 * u + e) * kPage + t] = (uint8_t)(v0w >> (8 * e));
      vt[(8 * u + 4 + e) * kPage + t] = (uint8_t)(v1w >> (8 * e));
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
  if (tid == 0) sp[0] = ks, sp[1] = vs;
  for (int i = tid; i < (kPage / kSub) * HD; i += kAppThr) {
    const int g = i / HD, d = i % HD;
    const int t0 = g * kSub;
    if ((t0 >= hi || t0 + kSub <= lo) && vratio == 1.f) continue;
    u32x4* w = reinterpret_cast<u32x4*>(vp + i * 16);
    const u32x4 x = *reinterpret_cast<const u32x4*>(vt + d * kPage + t0);
    if (t0 >= lo && t0 + kSub <= hi) {
      *w = x;
      continue;
    }
    u32x4 old = *w;
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
// Selection: one workgroup per (sequence, group).  The keep - recent largest
// masses among the tokens before the recent ones: the masses are mapped to
// unsigned keys of the same order, the smallest kept key is found digit by digit
// (8 bits, counted in LDS), and the tokens above it, and the first ones equal to
// it, are listed in token order by ballots.
constexpr int kSelThr = 1024;

__device__ __forceinline__ uint32_t mass_key(float m) {
  if (m != m) return 0xffffffffu;  // NaN ranks first
  const uint32_t u = m == 0.f ? 0u : __float_as_uint(m);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelThr) void cache_select_kernel(
    const float* __restrict__ mass, CacheBatch bt, int keep, int recent, int32_t* __restrict__ kept,
    int32_t* __restrict__ new_len) {
  __shared__ int hist[256];
  __shared__ int sh[2];
  __shared__ int wgt[kSelThr / kWave], weq[kSelThr / kWave];
  const int tid = threadIdx.x, h = blockIdx.x, b = blockIdx.y;
  const int lane = lane_id(), wave = tid >> 6;
  const int n = bt.context(b);
  int32_t* out = kept + ((size_t)b * bt.H + h) * keep;
  if (h == 0 && tid == 0) new_len[b] = min(n, keep);
  if (n <= keep) {
    for (int j = tid; j < keep; j += kSelThr) out[j] = j < n ? j : -1;
    return;
  }
  const int old = n - recent, need = keep - recent;  // 0 <= need < old
  auto key = [&](int t) {
    const int p = bt.page(b, t / kPage);
    return p < 0 ? 0u : mass_key(mass[((size_t)p * bt.H + h) * kPage + t % kPage]);
  };
  uint32_t prefix = 0;
  int want = need;  // of the keys with this prefix, the largest `want` are kept
  if (need > 0)
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int t = tid; t < old; t += kSelThr) {
        const uint32_t k = key(t);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8)))
          atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int d = 255, above = 0;
        while (d > 0 && above + hist[d] < want) above += hist[d--];
        sh[0] = d;
        sh[1] = above;
      }
      __syncthreads();
      prefix |= (uint32_t)sh[0] << shift;
      want -= sh[1];
      __syncthreads();
    }
  int gt = 0, eq = 0;  // kept above the prefix, and equal to it, so far
  if (need > 0)
    for (int base = 0; base < old; base += kSelThr) {
      const int t = base + tid;
      const uint32_t k = t < old ? key(t) : 0u;
      const bool g = t < old && k > prefix, e = t < old && k == prefix;
      const uint64_t mg = __builtin_amdgcn_ballot_w64(g), me = __builtin_amdgcn_ballot_w64(e);
      if (lane == 0) wgt[wave] = __popcll(mg), weq[wave] = __popcll(me);
      __syncthreads();
      int gb = gt, eb = eq;
      for (int w = 0; w < kSelThr / kWave; ++w) {
        if (w < wave) gb += wgt[w], eb += weq[w];
        gt += wgt[w], eq += weq[w];
      }
      const uint64_t below = ((uint64_t)1 << lane) - 1;
      gb += __popcll(mg & below);
      eb += __popcll(me & below);
      if (g || (e && eb < want)) out[gb + min(eb, want)] = t;
      __syncthreads();
    }
  for (int j = tid; j < recent; j += kSelThr) out[need + j] = old + j;
}

// Moving the kept tokens: one workgroup per (page of the result, group,
// sequence).
constexpr int kMoveThr = 256;

template <int HD>
__global__ __launch_bounds__(kMoveThr) void cache_move_kernel(
    uint8_t* __restrict__ kc, uint8_t* __restrict__ vc, float* __restrict__ kv_scale,
    float* __restrict__ mass, CacheBatch bt, const int32_t* __restrict__ dst_table, int dst_blocks,
    int keep, const int32_t* __restrict__ kept) {
  constexpr int NP = kPage * HD / 16;                       // 16-byte pieces of a page's keys or values
  constexpr int NI = (NP + kMoveThr - 1) / kMoveThr;  // of a thread
  __shared__ int spage[kPage], stok[kPage];
  __shared__ float2 sscale[kPage];
  const int tid = threadIdx.x, blk = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int cnt = min(min(bt.context(b), keep) - blk * kPage, kPage);
  if (cnt <= 0) return;
  const int dp = dst_table[(size_t)b * dst_blocks + blk];
  if (dp < 0 || dp >= bt.n_pages) return;
  const size_t dst = (size_t)dp * bt.H + h;
  if (tid < kPage) {
    int p = -1, t = 0;
    if (tid < cnt) {
      t = kept[((size_t)b * bt.H + h) * keep + blk * kPage + tid];
      p = t >= 0 ? bt.page(b, t / kPage) : -1;
      t %= kPage;
    }
    spage[tid] = p;
    stok[tid] = t;
    float2 s{0.f, 0.f};
    if (p >= 0) {
      const size_t sp = (size_t)p * bt.H + h;
      s = float2{kv_scale[sp * 2], kv_scale[sp * 2 + 1]};
      mass[dst * kPage + tid] = mass[sp * kPage + t];
    } else if (tid < cnt) {
      mass[dst * kPage + tid] = 0.f;
    }
    sscale[tid] = s;
  }
  __syncthreads();
  u32x4 kw[NI], vw[NI];
  float2 amax{0.f, 0.f};
  auto bigger = [](float a, uint32_t w, int i, float s) {
    float x = 0.f;
    switch (i) {
      case 0: x = __builtin_amdgcn_cvt_f32_fp8(w, 0); break;
      case 1: x = __builtin_amdgcn_cvt_f32_fp8(w, 1); break;
      case 2: x = __builtin_amdgcn_cvt_f32_fp8(w, 2); break;
      default: x = __builtin_amdgcn_cvt_f32_fp8(w, 3); break;
    }
    return fmaxf(a, fabsf(x) * s);  // (a NaN code counts for nothing)
  };
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int item = i * kMoveThr + tid, t = item / (HD / 16), c = item % (HD / 16);
    kw[i] = zero_u32x4();
    if (item >= NP) break;
    if (spage[t] >= 0) {
      kw[i] = *reinterpret_cast<const u32x4*>(
          kc + ((size_t)spage[t] * bt.H + h) * (kPage * HD) + stok[t] * HD + c * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) amax.x = bigger(amax.x, kw[i][e], k, sscale[t].x);
    }
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int item = i * kMoveThr + tid, g = item / HD, d = item % HD;
    vw[i] = zero_u32x4();
    if (item >= NP) break;
#pragma unroll
    for (int e = 0; e < kSub; ++e) {
      const int t = g * kSub + e;
      if (spage[t] < 0) continue;
      const uint32_t c = vc[((size_t)spage[t] * bt.H + h) * (kPage * HD) +
                            (stok[t] / kSub) * (HD * kSub) + d * kSub + stok[t] % kSub];
      vw[i][e / 4] |= c << (8 * (e % 4));
      amax.y = bigger(amax.y, c, 0, sscale[t].y);
    }
  }
  amax = block_max<kMoveThr>(amax);
  const float ks = block_scale(amax.x), vs = block_scale(amax.y);
  const float ki = pow2_inv(ks), vi = pow2_inv(vs);
  if (tid == 0) kv_scale[dst * 2] = ks, kv_scale[dst * 2 + 1] = vs;
  uint8_t* kp = kc + dst * (kPage * HD);
  uint8_t* vp = vc + dst * (kPage * HD);
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int item = i * kMoveThr + tid, t = item / (HD / 16);
    if (item >= NP || t >= cnt) continue;
    const float r = sscale[t].x * ki;
#pragma unroll
    for (int e = 0; e < 4; ++e) kw[i][e] = rescale4(kw[i][e], r);
    *reinterpret_cast<u32x4*>(kp + item * 16) = kw[i];
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int item = i * kMoveThr + tid, t0 = item / HD * kSub;
    if (item >= NP || t0 >= cnt) continue;
    u32x4* w = reinterpret_cast<u32x4*>(vp + item * 16);
    const u32x4 was = t0 + kSub > cnt ? *w : zero_u32x4();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = t0 + 4 * e;
      const uint32_t x = vw[i][e];
      uint32_t y = to_codes4(__builtin_amdgcn_cvt_f32_fp8(x, 0) * (sscale[t].y * vi),
                             __builtin_amdgcn_cvt_f32_fp8(x, 1) * (sscale[t + 1].y * vi),
                             __builtin_amdgcn_cvt_f32_fp8(x, 2) * (sscale[t + 2].y * vi),
                             __builtin_amdgcn_cvt_f32_fp8(x, 3) * (sscale[t + 3].y * vi));
      // slots past the kept tokens stay as they were
      const int left = cnt - t;
      const uint32_t m = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1;
      vw[i][e] = (y & m) | (was[e] & ~m);
    }
    *w = vw[i];
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

hipError_t launch_cache_evict(const CacheArgs& a, float* mass, int keep, int recent,
                              const int32_t* dst_table, int dst_blocks, int32_t* kept,
                              int32_t* new_len, hipStream_t s) {
  const CacheBatch bt{a.H, a.B, 0, 0, a.n_pages, a.max_blocks, a.block_table, a.length, nullptr};
  {
    ProfileScope ps("cache_select", s);
    FOE_LAUNCH(cache_select_kernel, dim3(a.H, a.B), dim3(kSelThr), 0, s, mass, bt, keep, recent,
               kept, new_len);
  }
  {
    ProfileScope ps("cache_move", s);
    auto go = [&](auto kern) {
      FOE_LAUNCH(kern, dim3(ceil_div(keep, kPage), a.H, a.B), dim3(kMoveThr), 0, s, a.k, a.v,
                 a.kv_scale, mass, bt, dst_table, dst_blocks, keep, kept);
    };
    if (a.hd == 96) go(cache_move_kernel<96>);
    else go(cache_move_kernel<128>);
  }
  return hipGetLastError();
}

}  // namespace foe
