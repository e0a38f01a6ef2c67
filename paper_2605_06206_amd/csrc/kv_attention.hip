// Causal attention over the 8-bit key/value cache, and the attention weight that
// each cached token receives.
//
// A column is one query: row i of a sequence and head j of a group, numbered
// i * nq + j (the heads share the group's keys and values).  A tile of 16
// columns walks the sequence's pages with v_mfma_f32_16x16x32_bf16:
//   S^T = K Q^T   (A = keys, B = the tile's queries, held in registers)
//   O^T += V^T P^T
// with an online softmax in base 2.  The page layouts feed both products from
// registers, without LDS.  With lane (n, g) = (lane % 16, lane / 16):
// - score tile t (0..3) of a page takes as row r key 16 (r / 4) + 4 t + r % 4, so
//   that a lane ends with the scores of the 16 consecutive keys 16 g .. 16 g + 15 of
//   column n, the four tiles one after another;
// - those are, eight at a time, the B operand of the second product, whose A operand
//   is then 8 consecutive tokens of one dim: the value layout's 16-byte pieces (16
//   tokens of one dim) hold them for both k-steps.
#include <algorithm>
#include <type_traits>

#include "kv_cache.hpp"

namespace foe {
namespace {

constexpr int kAttThr = 256;          // four waves, each taking every fourth page
constexpr int kAttWaves = kAttThr / kWave;
constexpr float kMFloor = -1.0e30f;   // the running maximum's start: finite, below any score

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

// One workgroup per (16 columns of a sequence, group).
template <int HD>
__global__ __launch_bounds__(kAttThr) void cache_attn_kernel(
    const bf16* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
    const float* __restrict__ kv_scale, CacheBatch bt, int max_rows, float c_log2,
    bf16* __restrict__ out, float2* __restrict__ stat) {
  using F = PageFrags<HD>;
  __shared__ float mm[kAttWaves][16], ll[kAttWaves][16];
  __shared__ __align__(16) float oo[kAttWaves][HD][16];
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6, h = blockIdx.y;
  const int n = lane & 15, g = lane >> 4;
  int b, tile;
  if (!find_tile<kAttThr>(
          bt.B, blockIdx.x,
          [&](int i) { return (min(bt.rows(i), max_rows) * bt.nq + 15) / 16; }, b, tile))
    return;
  const int rows = min(bt.rows(b), max_rows), ctx = bt.context(b);
  const int ncol = rows * bt.nq, col = tile * 16 + n;
  const size_t qrow = ((size_t)h * bt.N + bt.first_row(b)) * bt.nq;
  bf16x8 qf[F::NST];
  load_q<HD>(q + qrow * HD, col, ncol, g, qf);
  // tokens that this column, and the tile's last column, see
  const int len = min(ctx + rows, bt.cap());  // tokens the cache holds now
  const int seen = col < ncol ? min(ctx + col / bt.nq + 1, bt.cap()) : 0;
  const int most = min(ctx + min(tile * 16 + 15, ncol - 1) / bt.nq + 1, bt.cap());
  const int least = min(ctx + tile * 16 / bt.nq + 1, bt.cap());
  f32x4 oacc[F::NDT];
#pragma unroll
  for (int dt = 0; dt < F::NDT; ++dt) oacc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kMFloor, l_run = 0.f;
  for (int blk = wave; blk * kPage < most; blk += kAttWaves) {
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
    if ((blk + 1) * kPage > least) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (k0 + 4 * t + e >= seen) s[t][e] = -__builtin_inff();
      // slots past the last token hold anything: 0 * NaN is NaN
      if ((blk + 1) * kPage > len) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int left = len - (k0 + 4 * e);
          const uint32_t m = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
          for (int dt = 0; dt < F::NDT; ++dt) f.v[dt][e] &= m;
        }
      }
    }
    float mx = s[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[t][e]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
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
  if (g == 0) mm[wave][n] = m_run, ll[wave][n] = l_run;
#pragma unroll
  for (int dt = 0; dt < F::NDT; ++dt)
#pragma unroll
    for (int e = 0; e < 4; ++e) oo[wave][16 * dt + 4 * g + e][n] = oacc[dt][e];
  __syncthreads();
  // thread (column, dims): columns 16 threads apart
  const int c = tid >> 4, oc = tile * 16 + c;
  if (oc >= ncol) return;
  float m = mm[0][c], l = 0.f, a[kAttWaves];
#pragma unroll
  for (int w = 1; w < kAttWaves; ++w) m = fmaxf(m, mm[w][c]);
#pragma unroll
  for (int w = 0; w < kAttWaves; ++w) {
    a[w] = __builtin_amdgcn_exp2f(mm[w][c] - m);
    l += ll[w][c] * a[w];
  }
  // a column that sees no token gives zeros
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int row = bt.first_row(b) + oc / bt.nq;
  bf16* dst = out + (((size_t)row * bt.H + h) * bt.nq + oc % bt.nq) * HD;
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) {
    const int d = i * 16 + (tid & 15);
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kAttWaves; ++w) x += oo[w][d][c] * a[w];
    dst[d] = (bf16)(x * inv);
  }
  if (stat != nullptr && (tid & 15) == 0) stat[qrow + oc] = float2{m, inv};
}

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

size_t cache_attention_scratch_bytes(int H, int B, int N, int nq, int hd, int max_blocks,
                                     int max_rows, bool mass) {
  return mass ? align_up((size_t)H * N * nq * sizeof(float2), 256) : 0;
}

hipError_t launch_cache_attention(const CacheArgs& a, int nq, int N, int max_rows, const void* q,
                                  const int32_t* row_start, const float* mass_in, float* mass_out,
                                  void* out, void* scratch, hipStream_t s) {
  const CacheBatch bt{a.H, a.B, N, nq, a.n_pages, a.max_blocks, a.block_table, a.length, row_start};
  float2* stat = mass_out != nullptr ? static_cast<float2*>(scratch) : nullptr;
  const float c_log2 = 1.4426950408889634f / sqrtf((float)a.hd);
  const long long cols = (long long)N * nq;
  const long long tiles = std::min<long long>(cols, (cols + 15LL * a.B) / 16);
  auto go = [&](auto hdv) {
    constexpr int HD = decltype(hdv)::value;
    {
      ProfileScope ps("cache_attn", s);
      FOE_LAUNCH(cache_attn_kernel<HD>, dim3((unsigned)tiles, a.H), dim3(kAttThr), 0, s,
                 static_cast<const bf16*>(q), a.k, a.v, a.kv_scale, bt, max_rows, c_log2,
                 static_cast<bf16*>(out), stat);
    }
    if (mass_out != nullptr) {
      ProfileScope ps("cache_mass", s);
      FOE_LAUNCH(cache_mass_kernel<HD>, dim3(a.max_blocks, a.H, a.B), dim3(kAttThr), 0, s,
                 static_cast<const bf16*>(q), a.k, a.kv_scale, bt, max_rows, c_log2, stat, mass_in,
                 mass_out);
    }
  };
  if (a.hd == 96) go(std::integral_constant<int, 96>{});
  else go(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace foe
