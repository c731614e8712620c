// Rows of the paged window cache: written (quantised on the way) and read back.
//
// Both are one pass over the data with 8 elements per thread: 16 bytes of a bf16 row in or out.  A write takes the heads of a
// token one after the other, which lie page_size rows apart in a page: rows of 128 bytes and more go out as whole lines,
// shorter ones (4 bits, 8 bits at d = 64) as 64 or 32 bytes of one, the scales as 2 or 4.  A reading takes the rows of one
// head, which lie together.  The largest magnitude of a group of 32 comes from four neighbouring lanes.  Bound by memory.
// Two sets of buffers in turn, d = 128, 12 heads: 8 x 4,680 tokens into 8 bits 87 us (349 MB, 119 of them written, 4.0 TB/s),
// in bf16 88 us (460 MB, 5.2 TB/s); read back 50 us (7.0 TB/s: the pages come out of caches in part) and 81 us.  30 layers'
// blocks into 4 bits 301 us (1,092 MB, 229 written, 3.6 TB/s), read out of them 250 (863 MB written, 4.4 TB/s; a large copy
// reaches 4.65 on this card).  Two and four rows per thread, with their loads side by side, gained nothing.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "dkv_cache_format.hpp"

namespace dkv {
namespace {

constexpr int kThreads = 256;

// Thread = 8 elements of one row (token, head) of K (z = 0) or V (z = 1).  nb workgroups for each z, and for each sequence
// where the places are by sequences (BY; the choice at run time cost 10.2 -> 11.0 us on a block of 4,680 tokens).
template <int DT, int FMT, int D, bool BY>
__global__ __launch_bounds__(kThreads) void k_cache_write(Pages c, NewKv in, int nb) {
  constexpr int CH = D / 8;
  const int part = (int)(blockIdx.x / (unsigned)nb), z = part & 1;
  const int ch = (int)threadIdx.x % CH;
  const unsigned row = (blockIdx.x % (unsigned)nb) * (kThreads / CH) + threadIdx.x / CH;  // (token, head)
  int i = (int)(row / (unsigned)c.H), s = part >> 1;
  const int h = (int)(row % (unsigned)c.H);
  if constexpr (!BY) {
    if (i >= c.T) return;
    s = seq_of<CH>(c, i);
    if (s < 0) return;
  }
  const NewRows nr = new_rows(c, s);
  if constexpr (!BY) i -= nr.first;
  if (i >= min(nr.n, c.max_new)) return;  // whole groups of four lanes leave together
  const int pos = seq_length(c, s) - nr.n + i;
  if (pos < 0) return;
  // the row is on its way while the page number is
  constexpr int W = DT == DKV_BF16 ? 1 : 2;  // 16-byte words of 8 elements
  const char *src = static_cast<const char *>(z ? in.v : in.k) +
                    ((int64_t)(nr.first + i) * (z ? in.vt : in.kt) + h * (z ? in.vh : in.kh) + 8 * ch) * (2 * W);
  uint4 x[W];
#pragma unroll
  for (int j = 0; j < W; ++j) x[j] = reinterpret_cast<const uint4 *>(src)[j];
  const int p = page_of(c, s, pos);
  if (p < 0) return;
  unsigned char *dst = z ? c.v : c.k;
  const size_t r = pool_row(c, p, h, pos);
  if constexpr (FMT == DKV_CACHE_FULL) {
    uint4 *o = reinterpret_cast<uint4 *>(dst + r * (2 * W * D) + 16 * W * ch);
#pragma unroll
    for (int j = 0; j < W; ++j) o[j] = x[j];
  } else {
    float f[8];
    if constexpr (DT == DKV_BF16) {
      unpack_bf16x8(x[0], f);
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        f[4 * j] = __uint_as_float(x[j].x), f[4 * j + 1] = __uint_as_float(x[j].y);
        f[4 * j + 2] = __uint_as_float(x[j].z), f[4 * j + 3] = __uint_as_float(x[j].w);
      }
    }
    // magnitudes compare as integers, NaN above infinity
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(f[j]) & 0x7fffffffu);
    m = max(m, (uint32_t)__shfl_xor((int)m, 1, 64));
    m = max(m, (uint32_t)__shfl_xor((int)m, 2, 64));
    const int code = scale_code<FMT>(__uint_as_float(m));
    if (code == kScaleNan) {  // a group that reads as NaN stores zeros
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = 0.0f;
    }
    below_infinity<FMT>(f, code);
    const float sc = scale_of(code == kScaleNan ? kScaleBias : code);
    if constexpr (FMT == DKV_CACHE_FP8) *reinterpret_cast<uint2 *>(dst + r * D + 8 * ch) = quantise_fp8(f, sc);
    else *reinterpret_cast<uint32_t *>(dst + r * (D / 2) + 4 * ch) = quantise_fp4(f, sc);
    if ((ch & 3) == 0) (z ? c.vs : c.ks)[r * (D / kGroup) + ch / 4] = (uint8_t)code;
  }
}

// A store past the caches: the rows read back are more than they hold where it matters (30 layers' blocks of 4,680 rows,
// 863 MB out of 4-bit pages: 292 us with ordinary stores, 255 so; rows in bf16 327 and 296).
__device__ __forceinline__ void store_once(void *p, uint4 x) {
  typedef uint32_t word4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(__builtin_bit_cast(word4, x), static_cast<word4 *>(p));
}

// Thread = 8 elements of row i of bank (s, h), K or V.
template <int DT, int FMT, int D>
__global__ __launch_bounds__(kThreads) void k_cache_read(Pages c, const int32_t *__restrict__ first, int n, void *k, void *v,
                                                         int nb) {
  constexpr int CH = D / 8;
  const int bz = (int)(blockIdx.x / (unsigned)nb), z = bz & 1, b = bz >> 1, s = b / c.H, h = b % c.H;
  const int ch = (int)threadIdx.x % CH, i = (int)(blockIdx.x % (unsigned)nb) * (kThreads / CH) + (int)threadIdx.x / CH;
  if (i >= n) return;
  const int64_t pos = (int64_t)(first ? first[s] : 0) + i;
  int p = -1;
  if (pos >= 0 && pos < seq_length(c, s)) p = page_of(c, s, (int)pos);
  const size_t r = p < 0 ? 0 : pool_row(c, p, h, (int)pos);
  const unsigned char *src = z ? c.v : c.k;
  const uint8_t *sc = z ? c.vs : c.ks;
  const size_t o = (((size_t)b * n + i) * CH + ch) * 8;
  if constexpr (DT == DKV_BF16) {
    uint4 x = {0, 0, 0, 0};
    if (p >= 0) x = load_bf16x8<FMT, D>(src, sc, r, ch);
    store_once(static_cast<uint16_t *>(z ? v : k) + o, x);
  } else {
    float x[8] = {};
    if (p >= 0) load_f32x8<DT, FMT, D>(src, sc, r, ch, x);
    float *f = static_cast<float *>(z ? v : k) + o;
    store_once(f, __builtin_bit_cast(uint4, float4{x[0], x[1], x[2], x[3]}));
    store_once(f + 4, __builtin_bit_cast(uint4, float4{x[4], x[5], x[6], x[7]}));
  }
}

// Where the longest sequence is known, its rows are given to every sequence as long as no more than half of them are
// empty: searching for the sequence of a row takes a latency more (16 sequences of 150 to 300 tokens, 12 heads, 8 bits:
// 9.0 us by sequences, 10.5 by packed rows, 28 by sequences with a bound of all the tokens).
template <int DT, int FMT, int D>
hipError_t write_impl(const Pages &c, const NewKv &x, hipStream_t s) {
  constexpr int kRows = kThreads / (D / 8);
  if (c.max_new == 0) return hipSuccess;
  const auto blocks = [&](int tokens) { return ((int64_t)tokens * c.H + kRows - 1) / kRows; };
  const bool by = !c.start || ((int64_t)c.S * c.max_new <= 2 * (int64_t)c.T &&
                               grid_fits(2 * blocks(c.max_new) * c.S, kThreads));  // only starts can be searched
  const int64_t nb = blocks(by ? c.max_new : c.T), grid = 2 * nb * (by ? c.S : 1);
  if (!grid_fits(grid, kThreads)) return hipErrorInvalidConfiguration;
  if (by) k_cache_write<DT, FMT, D, true><<<(unsigned)grid, kThreads, 0, s>>>(c, x, (int)nb);
  else k_cache_write<DT, FMT, D, false><<<(unsigned)grid, kThreads, 0, s>>>(c, x, (int)nb);
  return hipGetLastError();
}
template <int DT, int FMT, int D>
hipError_t read_impl(const Pages &c, const int32_t *first, int n, void *k, void *v, hipStream_t s) {
  constexpr int kRows = kThreads / (D / 8);
  const int64_t nb = ((int64_t)n + kRows - 1) / kRows, grid = nb * c.S * c.H * 2;
  if (grid == 0) return hipSuccess;
  if (!grid_fits(grid, kThreads)) return hipErrorInvalidConfiguration;
  k_cache_read<DT, FMT, D><<<(unsigned)grid, kThreads, 0, s>>>(c, first, n, k, v, (int)nb);
  return hipGetLastError();
}

template <class F>
hipError_t by_format(int dtype, int fmt, int d, F f) {
#define DKV_CASE(DT, FMT, D) \
  if (dtype == DT && fmt == FMT && d == D) return f(std::integral_constant<int, DT>(), std::integral_constant<int, FMT>(), \
                                                    std::integral_constant<int, D>());
  DKV_CASE(DKV_BF16, DKV_CACHE_FULL, 64) DKV_CASE(DKV_BF16, DKV_CACHE_FULL, 128)
  DKV_CASE(DKV_BF16, DKV_CACHE_FP8, 64) DKV_CASE(DKV_BF16, DKV_CACHE_FP8, 128)
  DKV_CASE(DKV_BF16, DKV_CACHE_FP4, 64) DKV_CASE(DKV_BF16, DKV_CACHE_FP4, 128)
  DKV_CASE(DKV_F32, DKV_CACHE_FULL, 64) DKV_CASE(DKV_F32, DKV_CACHE_FULL, 128)
  DKV_CASE(DKV_F32, DKV_CACHE_FP8, 64) DKV_CASE(DKV_F32, DKV_CACHE_FP8, 128)
  DKV_CASE(DKV_F32, DKV_CACHE_FP4, 64) DKV_CASE(DKV_F32, DKV_CACHE_FP4, 128)
#undef DKV_CASE
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_cache_write(const Pages &c, int dtype, int fmt, int d, const NewKv &x, hipStream_t s) {
  return by_format(dtype, fmt, d, [&](auto dt, auto f, auto dd) {
    return write_impl<decltype(dt)::value, decltype(f)::value, decltype(dd)::value>(c, x, s);
  });
}

hipError_t launch_cache_read(const Pages &c, int dtype, int fmt, int d, const int32_t *first, int n, void *k, void *v,
                             hipStream_t s) {
  return by_format(dtype, fmt, d, [&](auto dt, auto f, auto dd) {
    return read_impl<decltype(dt)::value, decltype(f)::value, decltype(dd)::value>(c, first, n, k, v, s);
  });
}

}  // namespace dkv
