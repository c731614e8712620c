// Attention of new tokens over [bank; paged window cache] on gfx950.
//
// out = softmax(q K^T * scale) V over the tokens that a query sees (dkv_cache.hpp:
// seen_by) and the live slots of its bank.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "dkv_cache_format.hpp"

namespace dkv {
namespace {

// One wave per (token, head): scores of 64 keys at a time, one key per lane, an online
// softmax, then the weighted values with 8 columns per lane.
template <int DT, int FMT, int D>
__global__ __launch_bounds__(64) void k_cache_attn_row(Pages c, Mask mask, BankRows bank, CacheQueries qs) {
  constexpr int CH = D / 8, KG = 64 / CH;
  const unsigned nrow = (unsigned)c.max_new * qs.nh;
  const int s = (int)(blockIdx.x / nrow), row = (int)(blockIdx.x % nrow), i = row / qs.nh, hq = row % qs.nh;
  const NewRows nr = new_rows(c, s);
  if (i >= nr.n) return;
  const int l = threadIdx.x, h = hq / qs.G, b = s * c.H + h;
  const int len = seq_length(c, s);
  const Seen seen = seen_by(mask, len, nr.n, i);
  __shared__ float ql[D];
  __shared__ float pl[64];
  const size_t t = (size_t)nr.first + i;
  for (int j = l; j < D; j += 64) ql[j] = load_elem<DT>(qs.q, t * qs.qt + (size_t)hq * qs.qh + j);
  __syncthreads();
  float mx = -INFINITY, sum = 0.0f, o[8] = {};
  bool any = false;
  auto tile = [&](int n, auto valid, auto load_k, auto load_v) {
    for (int j0 = 0; j0 < n; j0 += 64) {
      const int j = j0 + l;
      const bool ok = j < n && valid(j);
      if (!__any(ok)) continue;
      any = true;
      float sc = -INFINITY;
      if (ok) {
        float dot = 0.0f, x[8];
        for (int ch = 0; ch < CH; ++ch) {
          load_k(j, ch, x);
#pragma unroll
          for (int e = 0; e < 8; ++e) dot = __builtin_fmaf(x[e], ql[8 * ch + e], dot);
        }
        sc = dot * qs.scale_log2;
      }
      float tm = sc;
      for (int w = 32; w; w >>= 1) tm = fmaxf(tm, __shfl_xor(tm, w, 64));
      const float mn = fmaxf(mx, tm), ref = mn == -INFINITY ? 0.0f : mn;
      const float corr = exp2f(mx - ref);
      mx = mn;
      const float p = ok ? exp2f(sc - ref) : 0.0f;
      __syncthreads();
      pl[l] = ok ? p : -1.0f;
      __syncthreads();
      float ps = p;
      for (int w = 32; w; w >>= 1) ps += __shfl_xor(ps, w, 64);
      sum = sum * corr + ps;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] *= corr;
      for (int g = l / CH; g < 64; g += KG) {
        const float pg = pl[g];
        if (pg == -1.0f) continue;
        float x[8];
        load_v(j0 + g, l % CH, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = __builtin_fmaf(pg, x[e], o[e]);
      }
    }
  };
  if (bank.cap > 0) {
    const int m = bound(bank.occupancy[b], 0, bound(bank.budget[b], 0, bank.cap));
    const size_t r0 = (size_t)b * bank.cap;
    tile(m, [](int) { return true; },
         [&](int j, int ch, float *x) { load_f32x8<DT, DKV_CACHE_FULL, D>((const unsigned char *)bank.k, nullptr, r0 + j, ch, x); },
         [&](int j, int ch, float *x) { load_f32x8<DT, DKV_CACHE_FULL, D>((const unsigned char *)bank.v, nullptr, r0 + j, ch, x); });
  }
  tile(seen.hi, [&](int j) { return sees(seen, mask.sink, j) && page_of(c, s, j) >= 0; },
       [&](int j, int ch, float *x) { load_f32x8<DT, FMT, D>(c.k, c.ks, pool_row(c, page_of(c, s, j), h, j), ch, x); },
       [&](int j, int ch, float *x) { load_f32x8<DT, FMT, D>(c.v, c.vs, pool_row(c, page_of(c, s, j), h, j), ch, x); });
  for (int w = CH; w < 64; w <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] += __shfl_xor(o[e], w, 64);
  if (l >= CH) return;
  // nothing seen: zeros; scores of -inf alone: NaN
  const float inv = sum > 0.0f ? 1.0f / sum : (any ? NAN : 0.0f);
  const size_t at = t * qs.ot + (size_t)hq * qs.oh + 8 * l;
  if constexpr (DT == DKV_BF16)
    *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(qs.out) + at) =
        uint4{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv), pack_bf16x2(o[4] * inv, o[5] * inv),
              pack_bf16x2(o[6] * inv, o[7] * inv)};
  else {
    float4 *f = reinterpret_cast<float4 *>(static_cast<float *>(qs.out) + at);
    f[0] = float4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    f[1] = float4{o[4] * inv, o[5] * inv, o[6] * inv, o[7] * inv};
  }
}

template <int DT, int FMT, int D>
hipError_t attn_impl(const Pages &c, const Mask &mask, const BankRows &bank, const CacheQueries &qs, hipStream_t s) {
  const int64_t grid = (int64_t)c.S * c.max_new * qs.nh;
  if (grid == 0) return hipSuccess;
  if (grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  k_cache_attn_row<DT, FMT, D><<<(unsigned)grid, 64, 0, s>>>(c, mask, bank, qs);
  return hipGetLastError();
}

}  // namespace

int cache_attention_splits(const Pages &, int, int, int, const Mask &, const BankRows &, int, size_t *bytes) {
  *bytes = 0;
  return 1;
}

hipError_t launch_cache_attention(const Pages &c, int dtype, int fmt, int d, const Mask &mask, const BankRows &bank,
                                  const CacheQueries &qs, void *, int, hipStream_t s) {
#define DKV_CASE(DT, FMT, D) \
  if (dtype == DT && fmt == FMT && d == D) return attn_impl<DT, FMT, D>(c, mask, bank, qs, s);
  DKV_CASE(DKV_BF16, DKV_CACHE_FULL, 64) DKV_CASE(DKV_BF16, DKV_CACHE_FULL, 128)
  DKV_CASE(DKV_BF16, DKV_CACHE_FP8, 64) DKV_CASE(DKV_BF16, DKV_CACHE_FP8, 128)
  DKV_CASE(DKV_BF16, DKV_CACHE_FP4, 64) DKV_CASE(DKV_BF16, DKV_CACHE_FP4, 128)
  DKV_CASE(DKV_F32, DKV_CACHE_FULL, 64) DKV_CASE(DKV_F32, DKV_CACHE_FULL, 128)
  DKV_CASE(DKV_F32, DKV_CACHE_FP8, 64) DKV_CASE(DKV_F32, DKV_CACHE_FP8, 128)
  DKV_CASE(DKV_F32, DKV_CACHE_FP4, 64) DKV_CASE(DKV_F32, DKV_CACHE_FP4, 128)
#undef DKV_CASE
  return hipErrorInvalidValue;
}

}  // namespace dkv
