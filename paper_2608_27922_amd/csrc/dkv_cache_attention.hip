// Attention of new tokens over [bank; paged window cache] on gfx950.
//
// out = softmax(q K^T * scale) V over the tokens that a query sees (dkv_cache.hpp:
// seen_by) and the live slots of its bank.  The rows of one (sequence, kv head) are
// its (token, query head) pairs, tokens first; a row block of them walks key tiles in
// the order bank, first tokens, window with a streaming softmax in fp32:
//   m' = max(m, max_j s_j),  w_j = exp(s_j - m'),
//   l' = l exp(m - m') + sum_j w_j,  o' = o exp(m - m') + sum_j w_j v_j,  out = o / l.
// Partial results (m, l, o) of disjoint keys join by the same rule, so the keys of a row
// block may lie over waves (k_cache_attn_few, k_cache_attn_f32) and over workgroups (splits,
// k_cache_combine).  Many rows are bound by the matrix cores, a single token's rows by the
// reading of the cache, small calls by the latency of a launch; the figures are at each kernel.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "dkv_cache_format.hpp"

namespace dkv {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kBufferRsrcWord3 = 0x00020000;  // raw buffer, 32-bit data, no swizzle
constexpr float kLazyLimit = 65536.0f;        // weights of a tile's row under the running reference, see exps()
constexpr float kFarScore = 4096.0f;          // references from which the rounding of their product shows, see is_far()

// Partial results of split keys: for each split, and row (place of the token, see Pages) * nh + head, the
// running maximum (bf16: raw scores) and weight sum, and the unnormalised output.
struct Part {
  float *o;    // [nsplit, rows, D]
  float2 *ml;  // [nsplit, rows]; null without splits
};
// Values from the caller's arrays are the same for all lanes, but loaded like any others: this makes them
// known as uniform, and the branches and loops on them scalar.
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Key tiles (KT keys each) of the rows of tokens i0..i1: nb bank tiles, a1 tiles of the
// first tokens, then the window's tiles from b0.  hi, lo: positions that any row sees.
struct Plan {
  int nb, a1, b0, total, hi, lo, m;
};
template <int KT>
__device__ __forceinline__ Plan plan_of(const Mask &mask, const BankRows &bank, int b, int len, int n, int i0, int i1) {
  Plan p;
  p.m = bank.cap > 0 ? bound(bank.occupancy[b], 0, bound(bank.budget[b], 0, bank.cap)) : 0;
  p.hi = seen_by(mask, len, n, i1).hi;
  p.lo = min(seen_by(mask, len, n, i0).lo, p.hi);
  p.nb = (p.m + KT - 1) / KT;
  p.a1 = p.lo > 0 ? (min(mask.sink, p.hi) + KT - 1) / KT : 0;
  p.b0 = max(p.lo / KT, p.a1);
  p.total = p.nb + p.a1 + max(0, (p.hi + KT - 1) / KT - p.b0);
  return p;
}
__device__ __forceinline__ Plan uni(const Plan &p) {
  return Plan{uni(p.nb), uni(p.a1), uni(p.b0), uni(p.total), uni(p.hi), uni(p.lo), uni(p.m)};
}
__device__ __forceinline__ int tile_pos(const Plan &p, int KT, int t) {
  const int u = t - p.nb;
  return KT * (u < p.a1 ? u : u - p.a1 + p.b0);
}

// One piece of a call: row block rb of R rows of (sequence, kv head), key split `split`; place: of the sequence's first
// token among those of all splits.
struct Piece {
  int s, h, rb, split, place;
  NewRows nr;
};
// How the row blocks of all sequences are numbered: `slots` > 0, so many of each sequence (uniform chunks, one row block each
// at most, or where T has many rows of no sequence); kCounted, without gaps, counted by every workgroup from the starts; kSearched, from slot_base on, found by
// a search, with an empty slot for some sequences.  Up to 256 sequences are counted: 16 single tokens of 32 heads without a
// bound take 46 us so and 61 searched (45 with it), 250 chunks of up to 30 tokens 172 and 199 (162); counting costs a wave's
// scan for each 64 of them, so 250 single tokens are 3 us slower than searched, and 2,000, counted in a loop, took 1,138 us
// where they take 439 (410 with the bound).
constexpr int kCounted = 0, kSearched = -1, kCountedSeqs = 256;

// The piece of this workgroup; false where it has none.  The pieces are numbered one sequence after the other (row blocks
// fastest), and each XCD (workgroup L runs on XCD L % 8) takes an equal run of them: row blocks that read the same keys
// share an L2, and no XCD has more work than the others (5 sequences of up to 777 tokens, 16 heads on 4, with the row
// blocks of the longest for each: 107 us, some XCDs have 33 pieces and others 22; 62 without gaps).  Empty slots stand
// together at the end of a sequence's: spread among the pieces they leave the shader engines uneven (64 single tokens, a
// quarter more slots than pieces: 213 in place of 169 us).
// Every wave takes part.
template <int R>
__device__ __forceinline__ bool my_piece(const Pages &c, const CacheQueries &qs, int nsplit, int slots, Piece &w) {
  const int l = threadIdx.x & 63;
  const unsigned per = (unsigned)(c.H * nsplit), L = blockIdx.x, xcd = L % 8;
  auto blocks = [&](int n) { return (min(n, c.max_new) * qs.G + R - 1) / R; };
  // number of this workgroup's piece among N
  auto piece = [&](unsigned N) { return L < N ? xcd * (N / 8) + min(xcd, N % 8) + L / 8 : N; };
  unsigned p;
  int first = 0;  // row blocks before the sequence's
  if (slots == kCounted) {
    constexpr int kLoads = kCountedSeqs / 64;
    NewRows r[kLoads];
    int upto[kLoads], total = 0;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      r[j] = NewRows{0, 0};
      if (64 * j + l < c.S) r[j] = new_rows(c, 64 * j + l);
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      upto[j] = 0;
      if (64 * j >= c.S) continue;
      int n = blocks(r[j].n);
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(n, o, 64);
        if (l >= o) n += y;
      }
      upto[j] = total + n;
      total = __builtin_amdgcn_readlane(upto[j], 63);
    }
    p = piece((unsigned)total * per);
    if (p >= (unsigned)total * per) return false;
    const int u = (int)(p / per);
    w.s = -1;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const uint64_t later = __ballot(upto[j] > u);
      if (w.s < 0 && later != 0) {
        const int i = __ffsll((unsigned long long)later) - 1;
        w.s = 64 * j + i;
        w.nr = NewRows{__builtin_amdgcn_readlane(r[j].first, i), __builtin_amdgcn_readlane(r[j].n, i)};
        first = __builtin_amdgcn_readlane(upto[j], i) - blocks(w.nr.n);
      }
    }
    if (w.s < 0) return false;  // starts that do not ascend, whose sum overflows
  } else {
    p = piece(gridDim.x);
    if (slots != kSearched) {
      w.s = (int)(p / ((unsigned)slots * per));
      first = w.s * slots;
    } else {
      const int u = (int)(p / per);
      w.s = uni(last_at_most<64>(c.S, [&](int lo, int step, int hi) {
        const int at = lo + l * step;
        return 63 - __clzll((long long)__ballot(at < hi && slot_base(c, qs.G, R, at) <= u));
      }));
      if (w.s < 0) return false;
      first = uni(slot_base(c, qs.G, R, w.s));
    }
    const NewRows r = new_rows(c, w.s);
    w.nr = NewRows{uni(r.first), uni(r.n)};
  }
  const unsigned cnt = (unsigned)blocks(w.nr.n), at = p - (unsigned)first * per;
  if (at >= cnt * per) return false;
  const int hs = (int)(at / cnt);
  w.rb = (int)(cnt - 1 - at % cnt);  // later row blocks see more under a causal mask: first
  w.h = hs / nsplit;
  w.split = hs % nsplit;
  w.place = w.split * (int)places(c) + (c.by_seq ? w.s * c.max_new : w.nr.first);
  return true;
}

// The host sizes the splits by the largest sequence; of them a row block takes as many as
// are full with LEAST tiles each (one at least), in equal runs of whole rounds of ROUND tiles (one
// for each wave that has tiles of its own).
template <int LEAST>
__device__ __forceinline__ int splits_used(int total, int nsplit) {
  return max(1, min(nsplit, (total + LEAST - 1) / LEAST));
}
template <int ROUND>
__device__ __forceinline__ void split_range(int total, int used, int split, int &t0, int &t1) {
  const int per = ((total + used - 1) / used + ROUND - 1) / ROUND * ROUND;
  t0 = min(total, split * per);
  t1 = min(total, t0 + per);
}

// s_waitcnt immediate: at most n vector-memory operations and no LDS operation outstanding.
constexpr int waitcnt_vm_lgkm0(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4); }
__device__ __forceinline__ void stage_barrier() { asm volatile("s_barrier" ::: "memory"); }

// Page numbers of 64 consecutive columns of a sequence's table in a register of a wave (one
// per lane), and of the 64 after them on their way to LDS: values in flight in a register
// would make the compiler wait for all loads wherever the register is moved.
struct PageWindow {
  const int32_t *row;
  int *next;      // 64 entries, of this wave
  int cols, P, base, cur;
  int tiles;      // since the numbers were loaded, the present one included
  uint64_t gone;  // bit i: column base + i is absent
  __device__ __forceinline__ int clamped(int c0) const {  // columns past the table repeat its last one: never asked for
    return min(c0 + (int)(threadIdx.x & 63), cols - 1);
  }
  __device__ __forceinline__ void init(const Pages &c, int s, int *lds) {
    row = c.table + (size_t)s * c.cols;
    cols = c.cols;
    P = c.P;
    next = lds;
    base = -256;
    cur = 0;
    tiles = 0;
    gone = 0;
  }
  // Columns col .. col + 7 may be asked for after seek(col) (those of a tile; col a multiple of their number); one call for
  // each tile, followed by its loads, two of them at least.  After eight tiles at least 16 loads are younger than that of
  // `next`: all but the 16 youngest being done, it is there, and the tiles on their way are not waited for.  Earlier (the
  // window may begin soon behind the first tokens) the numbers are loaded again.
  __device__ __forceinline__ void seek(int col) {
    ++tiles;
    if (col >= base && col < base + 64) return;
    if (col >= base + 64 && col < base + 128 && tiles > 8) {
      __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(16));
      asm volatile("" ::: "memory");
      cur = ((const __attribute__((address_space(3))) int *)next)[threadIdx.x & 63];
      base += 64;
      __builtin_amdgcn_s_waitcnt(0xc07f);
    } else {
      base = col;
      cur = row[clamped(base)];
      __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
    }
    tiles = 1;
    asm volatile("" ::: "memory");
    gone = __ballot((unsigned)cur >= (unsigned)P);  // the numbers come from the caller's array and are bounded here
    if ((unsigned)cur >= (unsigned)P) cur = 0;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)row, (short)0, 4 * cols, kBufferRsrcWord3);
    const int off = 4 * clamped(base + 64);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)next, 4, off, 0, 0, 0);
  }
  // Page of a column (any page if it is absent), and the absent ones of n columns, bit 0 the first.
  __device__ __forceinline__ int page(int col) const { return __builtin_amdgcn_readlane(cur, col - base); }
  __device__ __forceinline__ uint32_t absent(int col, int n) const { return (uint32_t)(gone >> (col - base)) & ((1u << n) - 1u); }
};

// Byte offset in the pool of position pos of a head in a page: pages are less than 2^31 bytes (checked by the
// caller), so only the page number takes a 64-bit product.
struct PoolAt {
  uint32_t page_bytes, head_bytes, mask;
  int row;
  __device__ __forceinline__ PoolAt(const Pages &c, int h, int row_bytes)
      : page_bytes((uint32_t)(c.H << c.lps) * row_bytes), head_bytes((uint32_t)(h << c.lps) * row_bytes),
        mask((1u << c.lps) - 1), row(row_bytes) {}
  __device__ __forceinline__ size_t at(int page, int pos) const {
    return (uint64_t)(uint32_t)page * page_bytes + (head_bytes + ((uint32_t)pos & mask) * row);
  }
};

// Physical 16-byte chunk of logical chunk c of row r (K: conflict-free 16-byte reads of
// one chunk across 16 rows; V: conflict-free transposed 8-byte reads of 4 chunks across 4
// rows, or of 2 chunks across 8 rows).
template <int D>
__device__ __forceinline__ int k_swz(int r, int c) { return c ^ (r % (D / 8)); }
template <int D>
__device__ __forceinline__ int v_swz(int r, int c) {
  return c ^ (D == 128 ? 4 * (r % 4) : 4 * ((r >> 1) % 2)) ^ (2 * ((r >> 2) % 2));
}

// Direct-to-LDS loads of 8 rows (2 D bytes each, `valid` of them, the others as zeros)
// of K and V into rows r0 .. r0 + 7 of a tile.  Lane i of a 1 KB load fetches the
// logical chunk that belongs at 16 i.
template <int D>
struct Rows8 {
  static constexpr int kLoads = 16 * D / 1024;  // per tensor
  int rsub, pc, v[kLoads];                      // row and physical chunk of this lane in a load; V's byte offsets
};
template <int D>
__device__ __forceinline__ Rows8<D> rows8_offsets() {
  constexpr int CH = D / 8, RPL = 64 / CH;
  const int l = threadIdx.x & 63;
  Rows8<D> o;
  o.rsub = l / CH;
  o.pc = l % CH;
#pragma unroll
  for (int q = 0; q < Rows8<D>::kLoads; ++q) {
    const int r = q * RPL + o.rsub;
    o.v[q] = r * (2 * D) + 16 * v_swz<D>(r, o.pc);
  }
  return o;
}
// K's swizzle depends on the row modulo D / 8, V's modulo 8.
template <int D>
__device__ __forceinline__ void rows8_issue(int rsub, int pc, const int *voff, const unsigned char *kp,
                                            const unsigned char *vp, int valid, int r0, char *kt, char *vt) {
  constexpr int RPL = 512 / D;
  // uniform: the clamp to 0..8 would otherwise leave it in a vector register, and each load in a loop over its values
  const int extent = __builtin_amdgcn_readfirstlane(valid) * (2 * D);
  const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void *)kp, (short)0, extent, kBufferRsrcWord3);
  const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void *)vp, (short)0, extent, kBufferRsrcWord3);
#pragma unroll
  for (int q = 0; q < Rows8<D>::kLoads; ++q) {
    const int r = q * RPL + rsub, koff = r * (2 * D) + 16 * k_swz<D>(r0 + r, pc);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void *)(kt + r0 * (2 * D) + q * 1024), 16, koff, 0, 0, 0);
  }
#pragma unroll
  for (int q = 0; q < Rows8<D>::kLoads; ++q)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void *)(vt + r0 * (2 * D) + q * 1024), 16, voff[q], 0, 0, 0);
}

// A quarter of a quantised row on its way from memory to an LDS tile through registers: of
// each run of four pieces of a row a lane takes its own, so that four lanes read 64 bytes
// in a row.  The loads are buffer loads whose extent ends after the valid rows (the others
// are zeros): without branches the compiler can count the loads in flight.
template <int FMT, int D>
struct Quarter {
  static constexpr int kRow = FMT == DKV_CACHE_FP8 ? D : D / 2;                // bytes of a row
  static constexpr int kPiece = kRow == 32 ? 8 : 16;                           // bytes
  static constexpr int kElems = FMT == DKV_CACHE_FP8 ? kPiece : 2 * kPiece;    // elements of a piece
  static constexpr int kPieces = kRow / (4 * kPiece);
  u32x4 x[kPieces];
  uint32_t codes;  // of the whole row
  // base, scale: the first of the group's rows; r, part: this lane's row and piece
  __device__ __forceinline__ void load(const unsigned char *base, const uint8_t *scale, int valid, int r, int part) {
    const int n = __builtin_amdgcn_readfirstlane(valid);
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void *)base, (short)0, n * kRow, kBufferRsrcWord3);
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc((void *)scale, (short)0, n * (D / kGroup), kBufferRsrcWord3);
    const int at = r * kRow + part * kPiece, sat = r * (D / kGroup);
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
      if constexpr (kPiece == 16) {
        x[e] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, at + 64 * e, 0, 0));
      } else {
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rx, at + 32 * e, 0, 0));
        x[e] = u32x4{y[0], y[1], 0, 0};
      }
    }
    if constexpr (D == 128) codes = __builtin_amdgcn_raw_buffer_load_b32(rs, sat, 0, 0);
    else codes = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, sat, 0, 0);
  }
  template <bool V>
  __device__ __forceinline__ void store(char *tile, int r, int part) const {
    asm volatile("" : "+v"(r), "+v"(part));  // addresses computed here, not kept in registers over the loop
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
      const int first = (4 * e + part) * kElems;
      const int code = (int)(codes >> (8 * (first / kGroup))) & 255;
#pragma unroll
      for (int j = 0; j < kElems / 8; ++j) {
        uint4 y;
        if constexpr (FMT == DKV_CACHE_FP8) y = bf16_of_fp8(uint2{x[e][2 * j], x[e][2 * j + 1]}, code);
        else y = bf16_of_fp4(x[e][j], code);
        const int ch = first / 8 + j;
        *reinterpret_cast<uint4 *>(tile + r * (2 * D) + 16 * (V ? v_swz<D>(r, ch) : k_swz<D>(r, ch))) = y;
      }
    }
  }
};

// Whether this lane or the row's other lane says so (every lane takes part in the exchange).
__device__ __forceinline__ bool either_half(bool x) {
  const int y = __shfl_xor((int)x, 32, 64);
  return x | (y != 0);
}

// Weight sum of a row: NaN-marked (-1) where its keys' scores were all -inf.
__device__ __forceinline__ float row_sum(float mx, float l, bool keys) {
  return keys && mx == -INFINITY && l == 0.0f ? -1.0f : l;
}
__device__ __forceinline__ float inv_sum(float l) { return l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : NAN); }

// What one wave (32 rows, row n = lane % 32, half h = lane / 32) keeps while it walks keys.
template <int D>
struct Rows {
  f32x16 o[D / 32];  // O^T: register i of tile t is element 32 t + 8 (i / 4) + 4 h + i % 4
  float mrun, off, lrun;  // reference, its offset in the weights' exponents (see is_far), sum of weights
  bool any;               // this lane saw a key of its row
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int t = 0; t < D / 32; ++t) o[t] = f32x16{};
    mrun = -INFINITY, off = NAN, lrun = 0.0f, any = false;
  }
  // (maximum, sum) of the row, and the outputs: put(chunk of 4 elements, values)
  __device__ __forceinline__ float2 stats() const {
    return float2{mrun, row_sum(mrun, lrun + __shfl_xor(lrun, 32, 64), either_half(any))};
  }
  template <class F>
  __device__ __forceinline__ void outputs(F put) const {
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g) put(8 * t + 2 * g + h, float4{o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]});
  }
};

// 1 for +inf, 128 for -inf, 16384 for NaN, 0 for finite values, as bf16: sums of 64 of them
// are exact in fp32.
__device__ __forceinline__ uint32_t kind_of(uint32_t half) {
  const uint32_t a = half & 0x7fffu;
  return a < 0x7f80u ? 0u : (a > 0x7f80u ? 0x4680u : ((half & 0x8000u) ? 0x4300u : 0x3f80u));
}
__device__ __forceinline__ float value_of_kinds(float c) {
  if (c == 0.0f) return 0.0f;
  const bool nan = c >= 16384.0f;
  const int r = (int)c & 16383;
  const bool neg = r >= 128, pos = (r & 127) != 0;
  return nan || (pos && neg) ? NAN : (neg ? -INFINITY : INFINITY);
}

// S^T = K Q^T for NSUB x 32 keys of an LDS tile.
template <int D, int NSUB>
__device__ __forceinline__ void scores(const char *kt, const bf16x8 *qf, f32x16 *sc) {
  const int l = threadIdx.x & 63, h = l >> 5, n = l & 31;
#pragma unroll
  for (int sub = 0; sub < NSUB; ++sub) {
    const int key = 32 * sub + n;
    bf16x8 a[D / 16];
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
      a[kk] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(kt + key * (2 * D) + 16 * k_swz<D>(key, 2 * kk + h)));
    f32x16 acc = {};
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[kk], qf[kk], acc, 0, 0, 0);
    sc[sub] = acc;
  }
  // LDS fragment reads run 6 MFMAs ahead of their use
  constexpr int N = NSUB * D / 16, A = N < 6 ? N : 6;
  __builtin_amdgcn_sched_group_barrier(0x100, A, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (i + A < N) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
}

// A operand of 16 keys (K step kst of sub-tile sub) of V^T, columns 32 t2 ..: the transposing
// LDS reads give lane groups of 16 their 4 x 16 blocks; the key order inside the step is
// that of the weights' registers.
template <int D>
__device__ __forceinline__ u32x4 v_operand(const char *vt, int sub, int kst, int t2) {
  const int l = threadIdx.x & 63, gq = l >> 4, cq = l & 15;
  const int ka = 32 * sub + 16 * kst + 4 * (gq >> 1) + (cq >> 2), kb = ka + 8;
  const int dvb = 8 * t2 + 4 * (gq & 1) + (cq & 3);
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_i16x4 *)(vt + ka * (2 * D) + 16 * v_swz<D>(ka, dvb >> 1) + 8 * (dvb & 1)));
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_i16x4 *)(vt + kb * (2 * D) + 16 * v_swz<D>(kb, dvb >> 1) + 8 * (dvb & 1)));
  const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
  return u32x4{a[0], a[1], b[0], b[1]};
}

// The exponents (x - ref) c of the weights are taken as fma(x, c, off), off = -(ref c): the rounding of ref c is one factor
// for all weights of a row under this reference, 2^-13 at most while |ref c| is below 2^12.  From there on (softmax
// scales of hundreds, or as large queries) it grows to all that a float holds, so that weights vanish or overflow: such a
// row keeps off as NaN, which sends it through the path of raised references in every tile, where it takes the
// difference first.  Rows without a reference yet (-inf) go there too.
__device__ __forceinline__ bool is_far(float off) { return !(fabsf(off) < kFarScore); }

// Softmax update of one tile of one wave from its scores (masked ones are -inf); pb: the
// weights in bf16, pairs of registers.  The reference maximum is raised only when a lane's
// sum of weights exceeds 2^16 (or is not finite): weights and sums stay far from overflow,
// and the final division removes the common factor.
template <int D, int NSUB>
__device__ __forceinline__ void softmax_update(Rows<D> &r, f32x16 *sc, uint32_t (*pb)[8], float c) {
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
  float psum = 0.0f;
  auto exps = [&](float off) __attribute__((always_inline)) {
    psum = 0.0f;
#pragma unroll
    for (int sub = 0; sub < NSUB; ++sub) {
      float ps = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[sub][i], c, off));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[sub][i + 1], c, off));
        pb[sub][i >> 1] = pack_bf16x2(p0, p1);
        // row sum of the bf16 weights that are multiplied into O: their rounding (2^-8) enters
        // numerator and denominator alike.  It is a choice for speed: weights in two parts (two_parts) double
        // the product with V and cost 432 -> 622 us on the large block, 214 -> 279 on the 8-bit one, and with 32 rows a
        // wave 232 -> 275 (64 sequences x 64 rows a head, 8 bits), for an error of 1.7 in place of 2.4e-3 (2-norm, of
        // which the rounding of the outputs to bf16 is 1.66)
        ps = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pb[sub][i >> 1]), ones, ps, false);
      }
      psum += ps;
    }
  };
  exps(r.off);
  const bool over = !(psum <= kLazyLimit);
  if (__builtin_expect(__any(over), 0)) {
    // only the rows concerned, so that a row's result does not depend on the rows beside it
    const bool raise = either_half(over);
    float tmax = sc[0][0];
#pragma unroll
    for (int sub = 0; sub < NSUB; ++sub)
#pragma unroll
      for (int i = 0; i < 16; ++i) tmax = fmaxf(tmax, sc[sub][i]);
    tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
    const float mnew = raise ? fmaxf(r.mrun, tmax) : r.mrun;
    const float mref = mnew == -INFINITY ? 0.0f : mnew;  // scores of -inf alone: weights 0, not inf - inf
    const float corr = raise ? __builtin_amdgcn_exp2f((r.mrun - mref) * c) : 1.0f;
    r.mrun = mnew;
    r.lrun *= corr;
#pragma unroll
    for (int t2 = 0; t2 < D / 32; ++t2)
#pragma unroll
      for (int i = 0; i < 16; ++i) r.o[t2][i] *= corr;
    const float noff = -mref * c;
    const bool far = is_far(noff);
    r.off = far || mnew == -INFINITY ? NAN : noff;
    if (__any(far)) {
#pragma unroll
      for (int sub = 0; sub < NSUB; ++sub)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[sub][i] = far ? sc[sub][i] - mref : sc[sub][i];
    }
    exps(far ? 0.0f : noff);
  }
  r.lrun += psum;
}

// O^T += V^T P^T.
template <int D, int NSUB>
__device__ __forceinline__ void product(Rows<D> &r, const uint32_t (*pb)[8], const char *vt) {
#pragma unroll
  for (int sub = 0; sub < NSUB; ++sub) {
#pragma unroll
    for (int kst = 0; kst < 2; ++kst) {
      const u32x4 bp = {pb[sub][4 * kst], pb[sub][4 * kst + 1], pb[sub][4 * kst + 2], pb[sub][4 * kst + 3]};
#pragma unroll
      for (int t2 = 0; t2 < D / 32; ++t2)
        r.o[t2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v_operand<D>(vt, sub, kst, t2)),
                                                          __builtin_bit_cast(bf16x8, bp), r.o[t2], 0, 0, 0);
    }
  }
  // the two transposed reads of an MFMA run 4 MFMAs ahead of it
  constexpr int N = 2 * NSUB * D / 32, A = N < 4 ? N : 4;
  __builtin_amdgcn_sched_group_barrier(0x100, 2 * A, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (i + A < N) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
  }
}

// Whether a tile of BYTES in LDS holds a NaN or an infinity (bf16; asked by whole waves).
template <int BYTES>
__device__ __forceinline__ bool has_nonfinite(const char *vt) {
  const int l = threadIdx.x & 63;
  uint32_t bad = 0;
#pragma unroll 4
  for (int j = 0; j < BYTES / 1024; ++j) {
    const u32x4 x = *reinterpret_cast<const u32x4 *>(vt + j * 1024 + 16 * l);
#pragma unroll
    for (int e = 0; e < 4; ++e)  // an exponent of all ones plus one carries into its half's sign bit
      bad |= ((x[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  }
  return __any(bad != 0);
}
// Such values become zeros, by NT threads.
template <int BYTES, int NT>
__device__ __forceinline__ void zero_nonfinite(char *vt) {
  for (int j = threadIdx.x % NT; j < BYTES / 16; j += NT) {
    u32x4 x = *reinterpret_cast<const u32x4 *>(vt + 16 * j);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u;
      if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu;
    }
    *reinterpret_cast<u32x4 *>(vt + 16 * j) = x;
  }
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
}

// In a tile that some rows see in part, a NaN or an infinity of V would reach the others
// through 0 x inf.  Such values are added to the rows that see them (vis: as from
// visible_bits), as sums of the kinds that a row sees, and become zeros in
// the tile.  NT threads share the tile (all of them call this), one wave or a workgroup.
template <int D, int NSUB, int NT>
__device__ __forceinline__ void purge(Rows<D> &r, char *vt, const uint32_t *vis, bool work) {
  constexpr int kBytes = NSUB * 32 * 2 * D;
  if (!has_nonfinite<kBytes>(vt)) return;
  if (work) {
#pragma unroll 1
    for (int e = 0; e < (D / 32) * ((NSUB + 1) / 2); ++e) {  // column tile, 64 keys
      const int t2 = e % (D / 32), st0 = 4 * (e / (D / 32));
      f32x16 kinds = {};
#pragma unroll 1
      for (int st = st0; st < st0 + (NSUB < 2 ? 2 : 4); ++st) {
        u32x4 a = v_operand<D>(vt, st >> 1, st & 1, t2), bv;
        uint32_t w = vis[0];
#pragma unroll
        for (int u = 1; u < NSUB; ++u)
          if (st >> 1 == u) w = vis[u];
        w >>= 16 * (st & 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a[e] = kind_of(a[e] & 0xffffu) | (kind_of(a[e] >> 16) << 16);
          const int k = 8 * (e >> 1) + 2 * (e & 1);  // registers 2 e and 2 e + 1 of the step
          bv[e] = ((w >> k) & 1 ? 0x3f80u : 0u) | ((w >> (k + 1)) & 1 ? 0x3f800000u : 0u);
        }
        kinds = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, bv), kinds,
                                                        0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = value_of_kinds(kinds[i]);
#pragma unroll
        for (int u = 0; u < D / 32; ++u)
          if (u == t2) r.o[u][i] += x;
      }
    }
  }
  if constexpr (NT > 64) {
    __builtin_amdgcn_s_waitcnt(0xc07f);
    stage_barrier();  // every wave has read the tile
  }
  zero_nonfinite<kBytes, NT>(vt);
  if constexpr (NT > 64) stage_barrier();
}

// Which of the wave's rows see which keys of a tile.
struct WaveMask {
  Seen first, last, row;  // of the wave's first and last row, and of this lane's
  int sink;
  __device__ __forceinline__ bool none(int pos, int KT) const {
    return pos >= last.hi || (pos + KT <= first.lo && pos >= sink);
  }
  __device__ __forceinline__ bool all(int pos, int KT) const {
    return pos + KT <= first.hi && (pos >= last.lo || pos + KT <= sink);
  }
};

// Bits below x of 32.
__device__ __forceinline__ uint32_t bits_below(int x) { return x <= 0 ? 0u : (x >= 32 ? ~0u : (1u << x) - 1u); }

// Which of the 32 keys at pos this lane's row sees, bit k for key k + 4 g (so that the bits of
// the lane's score registers are in the same places for every lane group g).  They are keys
// first .. first + 31 of a tile of which absent (PageWindow) says the pages that are not there.
__device__ __forceinline__ uint32_t visible_bits(const WaveMask &w, int pos, int first, uint32_t absent, int lps, int g) {
  const uint32_t there = ((absent >> (first >> lps)) & 1 ? 0u : 0xffffu) | ((absent >> ((first + 16) >> lps)) & 1 ? 0u : 0xffff0000u);
  const uint32_t m = bits_below(w.row.hi - pos) & (~bits_below(w.row.lo - pos) | bits_below(w.sink - pos)) & there;
  return m >> (4 * g);
}
template <int NSUB>
__device__ __forceinline__ bool mask_cache(f32x16 *sc, const uint32_t *vis) {
  uint32_t some = 0;
#pragma unroll
  for (int sub = 0; sub < NSUB; ++sub) {
    some |= vis[sub];
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!(vis[sub] & (1u << (8 * (i >> 2) + (i & 3))))) sc[sub][i] = -INFINITY;
  }
  return (some & 0x0f0f0f0fu) != 0;
}
template <int NSUB>
__device__ __forceinline__ void mask_bank(f32x16 *sc, int nvalid) {
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int sub = 0; sub < NSUB; ++sub)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (32 * sub + 8 * (i >> 2) + 4 * h + (i & 3) >= nvalid) sc[sub][i] = -INFINITY;
}

// Row r (token, head of the group) of a row block -> its packed row and query head.
struct RowAt {
  size_t t;
  int i, hq;
};
__device__ __forceinline__ RowAt row_at(const NewRows &nr, const CacheQueries &qs, int h, int r) {
  const int i = (int)((unsigned)r / (unsigned)qs.G);
  return RowAt{(size_t)(nr.first + i), i, h * qs.G + (r - i * qs.G)};
}

template <int D>
__device__ __forceinline__ void load_q(bf16x8 *qf, const CacheQueries &qs, const RowAt &a, bool ok) {
  const int h = (threadIdx.x & 63) >> 5;
  const uint16_t *q = static_cast<const uint16_t *>(qs.q) + a.t * qs.qt + (size_t)a.hq * qs.qh;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    u32x4 x = {0, 0, 0, 0};
    if (ok) x = *reinterpret_cast<const u32x4 *>(q + 16 * kk + 8 * h);
    qf[kk] = __builtin_bit_cast(bf16x8, x);
  }
}

// ---------------------------------------------------------------------------
// Many rows (bf16): a workgroup of 8 waves owns 256 rows, 32 per wave, and walks tiles of
// 64 keys (d = 64: 128) that its waves load together.  256 rows read a tile once for 8 waves, so the L2 sees
// an eighth of what the matrix cores take from LDS; 32 rows a wave are what fits 256 registers
// (128 columns: 64 of outputs, 32 each of scores and queries, 16 of weights), two waves a SIMD;
// 128 keys fit them at d = 64 and halve the barriers and the softmax's fixed part (12 heads x 4,680
// tokens over 15,600 keys: 324 -> 287 us, with 8-bit pages 342 -> 312).
// Measured: bf16, 12 heads x 4,680 tokens over 15,600 keys, d = 128, 228 workgroups: 435 to 470 us on different cards, 960
// to 1,030 TFLOP/s (a large library product: 1,175; the matrix pipe is busy 47% of the cycles of the 228 CUs,
// the rest is a tile's softmax and its barrier: both waves of a SIMD come to them together).  8-bit pages, 12 x 1,560 over
// 9,360 bank and 9,360 cache keys: 213 to 222 us with the joining of three splits, 810 to 840 TFLOP/s: the conversion of a tile
// runs between two matrix blocks of the same wave, and two tiles ahead do not fit the registers.  d = 64 has
// half the matrix work for the same softmax: 8-bit pages, 5 ragged chunks of 478 to 777 tokens that see
// 2,000 tokens each, 63 us, 393 TFLOP/s (13 us before the first product, 200 workgroups of 18 tiles).
// No vector register is spilled but one in the path of raised references; 25 to 63 scalar ones are, into lanes of vector
// registers (kernel arguments, the plan of the tiles and buffer descriptors that stay live over the loops).
// Four waves a SIMD at d = 64 (128 registers) would spill 50 to 90 of them.
// ---------------------------------------------------------------------------
constexpr int kWWaves = 8, kWRows = 32 * kWWaves;
constexpr int wide_keys(int D) { return D == 64 ? 128 : 64; }   // per tile
constexpr int wide_least(int D) { return 256 / wide_keys(D); }  // tiles of a split

template <int FMT, int D>
__global__ __launch_bounds__(64 * kWWaves, 1) void k_cache_attn_wide(Pages c, Mask mask, BankRows bank, CacheQueries qs,
                                                                    int nsplit, int slots, Part part) {
  constexpr int KT = wide_keys(D), NSUB = KT / 32, TB = KT * 2 * D;
  constexpr bool FULL = FMT == DKV_CACHE_FULL;
  Piece w;
  if (!my_piece<kWRows>(c, qs, nsplit, slots, w)) return;
  const int s = w.s, h = w.h, b = s * c.H + h, split = w.split;
  const NewRows nr = w.nr;
  const int nrows = min(nr.n, c.max_new) * qs.G, r0 = w.rb * kWRows;
  const int len = uni(seq_length(c, s));
  const int r1 = min(r0 + kWRows, nrows) - 1;
  const Plan pl = uni(plan_of<KT>(mask, bank, b, len, nr.n, r0 / qs.G, r1 / qs.G));
  const int used = splits_used<wide_least(D)>(pl.total, nsplit);
  if (split >= used) return;
  int tb, nt;
  split_range<1>(pl.total, used, split, tb, nt);
  tb = uni(tb), nt = uni(nt);

  __shared__ __attribute__((aligned(1024))) char k0[TB], k1[TB], k2[TB];
  __shared__ __attribute__((aligned(1024))) char v0[TB], v1[TB], v2[TB];
  __shared__ __attribute__((aligned(256))) int pages_lds[64 * kWWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, lh = l >> 5, n = l & 31;
  const int w0 = r0 + 32 * wave;
  const bool work = w0 < nrows;  // a wave past the last row only loads
  const int r = min(w0 + n, nrows - 1);
  const RowAt at = row_at(nr, qs, h, r);
  const bool rv = w0 + n < nrows;
  bf16x8 qf[D / 16];
  load_q<D>(qf, qs, at, rv);
  // here, so that no use of a query inside the loops waits for the tiles on their way
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
  Rows<D> rows;
  rows.init();
  WaveMask wm;
  wm.sink = mask.sink;
  wm.row = seen_by(mask, len, nr.n, at.i);
  wm.first = seen_by(mask, len, nr.n, min(w0, nrows - 1) / qs.G);
  wm.last = seen_by(mask, len, nr.n, min(w0 + 31, nrows - 1) / qs.G);
  PageWindow pw;   // of the tile being loaded
  pw.init(c, s, pages_lds + 64 * wave);

  const unsigned char *bk = static_cast<const unsigned char *>(bank.k) + (size_t)b * bank.cap * (2 * D);
  const unsigned char *bv = static_cast<const unsigned char *>(bank.v) + (size_t)b * bank.cap * (2 * D);

  const int kcols = max(1, KT >> c.lps);  // pages that a tile lies in
  const Seen bfirst = seen_by(mask, len, nr.n, r0 / qs.G), blast = seen_by(mask, len, nr.n, r1 / qs.G);
  auto compute = [&](bool isbank, int t, const char *kt, char *vt, uint32_t absent) __attribute__((always_inline)) {
    const int pos = tile_pos(pl, KT, t);
    const bool act = work && (isbank || !wm.none(pos, KT));
    // whether every row of the workgroup sees all of the tile: the same for all its waves
    const bool whole = isbank || (absent == 0 && pos + KT <= bfirst.hi && (pos >= blast.lo || pos + KT <= mask.sink));
    uint32_t pb[NSUB][8];
    uint32_t vis[NSUB] = {};
    if (act) {
      f32x16 sc[NSUB];
      scores<D, NSUB>(kt, qf, sc);
      if (isbank) {
        const int nv = pl.m - t * KT;
        if (nv < KT) mask_bank<NSUB>(sc, nv);
        rows.any = true;
      } else if (whole) {
        rows.any = true;
      } else {
#pragma unroll
        for (int u = 0; u < NSUB; ++u) vis[u] = visible_bits(wm, pos + 32 * u, 32 * u, absent, c.lps, lh);
        rows.any |= mask_cache<NSUB>(sc, vis);
      }
      softmax_update<D, NSUB>(rows, sc, pb, qs.scale_log2);
    }
    if (!whole) purge<D, NSUB, 64 * kWWaves>(rows, vt, vis, act);
    if (act) product<D, NSUB>(rows, pb, vt);
  };

  // Tiles [t0, t1) of rows held in bf16 go global -> LDS without registers, three stages: two
  // tiles in flight while one is used.  A wave loads KT / 8 (8 or 16) rows of each tile, which lie in one page.
  const Rows8<D> ld = rows8_offsets<D>();
  const PoolAt pool(c, h, FULL ? 2 * D : Quarter<FULL ? DKV_CACHE_FP8 : FMT, D>::kRow);
  auto run_direct = [&](int t0, int t1) __attribute__((always_inline)) {
    constexpr int kOwn = KT / kWWaves;
    uint32_t pr[3] = {0, 0, 0};
    // Every call has the same number of loads (behind the last tile they read nothing and leave
    // zeros), so that the waits can count them.
    auto issue = [&](int t, char *kd, char *vd) __attribute__((always_inline)) -> uint32_t {
      const unsigned char *kp = bk, *vp = bv;
      int valid = 0;
      uint32_t absent = 0;
      if (t < t1) {
        if (!FULL || t < pl.nb) {
          const int r = t * KT + kOwn * wave;
          kp = bk + (size_t)r * (2 * D), vp = bv + (size_t)r * (2 * D);
          valid = bound(pl.m - r, 0, kOwn);
        } else {
          const int pos = tile_pos(pl, KT, t), p = pos + kOwn * wave;
          pw.seek(pos >> c.lps);
          valid = kOwn;
          if (pw.gone != 0 || pos < pl.lo || pos + KT > pl.hi) {
            absent = pw.absent(pos >> c.lps, kcols);
            valid = !pw.absent(p >> c.lps, 1) && (p + kOwn > pl.lo || p < mask.sink) ? bound(pl.hi - p, 0, kOwn) : 0;
          }
          const size_t off = pool.at(pw.page(p >> c.lps), p);
          kp = c.k + off, vp = c.v + off;
        }
      }
#pragma unroll
      for (int g = 0; g < kOwn / 8; ++g)
        rows8_issue<D>(ld.rsub, ld.pc, ld.v, kp + g * (16 * D), vp + g * (16 * D), bound(valid - 8 * g, 0, 8),
                       kOwn * wave + 8 * g, kd, vd);
      return absent;
    };
    constexpr int kTileLoads = kOwn / 8 * 2 * Rows8<D>::kLoads;
    auto step = [&](int t, const char *kt, char *vt, uint32_t absent, char *kn, char *vn) __attribute__((always_inline)) {
      __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(kTileLoads));  // the next tile may still be on its way
      stage_barrier();
      const uint32_t nx = issue(t + 2, kn, vn);
      if (t < t1) compute(!FULL || t < pl.nb, t, kt, vt, absent);
      return nx;
    };
    pr[0] = issue(t0, k0, v0);
    pr[1] = issue(t0 + 1, k1, v1);
    // whole rounds of the stages, so that the loads in flight are the same wherever a round begins
    for (int t = t0; t < t1; t += 3) {
      pr[2] = step(t, k0, v0, pr[0], k2, v2);
      pr[0] = step(t + 1, k1, v1, pr[1], k0, v0);
      pr[1] = step(t + 2, k2, v2, pr[2], k1, v1);
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));  // nothing is on its way to the stages
  };
  if constexpr (FULL) {
    run_direct(tb, nt);
  } else {
    const int t0 = max(tb, min(nt, pl.nb));
    if (tb < t0) {
      run_direct(tb, t0);
      stage_barrier();
    }
    // Quantised rows come through registers, a tile ahead (a second one does not fit beside the scores), and
    // are stored as bf16: waves 0-3 a quarter row of K per lane and 16 rows, waves 4-7 of V; 16 rows lie in one page.
    // Of the two waves of a SIMD one converts before its matrix work and one after it.
    constexpr int kQ = KT / 64;
    const bool isv = wave >= 4;
    const int row16 = 16 * kQ * (wave & 3), lr = row16 + (l >> 2), qpart = l & 3;
    Quarter<FMT, D> x[kQ];
    uint32_t ahead = 0;  // absent pages of the tile in registers
    auto fetch = [&](int t) __attribute__((always_inline)) {
      size_t row[kQ] = {};
      int valid[kQ] = {};
      ahead = 0;
      if (t < nt) {
        const int pos = tile_pos(pl, KT, t), p16 = pos + row16;
        pw.seek(pos >> c.lps);
#pragma unroll
        for (int g = 0; g < kQ; ++g) valid[g] = 16;
        if (pw.gone != 0 || pos < pl.lo || pos + KT > pl.hi) {
          ahead = pw.absent(pos >> c.lps, kcols);
#pragma unroll
          for (int g = 0; g < kQ; ++g) {
            const int p = p16 + 16 * g;
            valid[g] = !pw.absent(p >> c.lps, 1) && (p + 16 > pl.lo || p < mask.sink) ? bound(pl.hi - p, 0, 16) : 0;
          }
        }
#pragma unroll
        for (int g = 0; g < kQ; ++g) row[g] = pool.at(pw.page((p16 + 16 * g) >> c.lps), p16 + 16 * g);
      }
#pragma unroll
      for (int g = 0; g < kQ; ++g)
        x[g].load((isv ? c.v : c.k) + row[g], (isv ? c.vs : c.ks) + row[g] / (Quarter<FMT, D>::kRow / (D / kGroup)), valid[g],
                  l >> 2, qpart);
    };
    auto store = [&](auto V, char *tile) __attribute__((always_inline)) {
#pragma unroll
      for (int g = 0; g < kQ; ++g) x[g].template store<decltype(V)::value>(tile, lr + 16 * g, qpart);
    };
    uint32_t absent = 0;
    auto step = [&](int t, const char *kt, char *vt, char *kn, char *vn) __attribute__((always_inline)) {
      const uint32_t now = absent, next = ahead;
      if (!isv) store(std::false_type(), kn);
      asm volatile("" ::: "memory");
      if (!isv) fetch(t + 2);
      if (t < nt) compute(false, t, kt, vt, now);
      if (isv) store(std::true_type(), vn);
      asm volatile("" ::: "memory");
      if (isv) fetch(t + 2);
      asm volatile("" ::: "memory");
      absent = next;
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave's stores have landed
      stage_barrier();
    };
    if (t0 < nt) {
      fetch(t0);
      asm volatile("" ::: "memory");
      if (isv) store(std::true_type(), v0);
      else store(std::false_type(), k0);
      absent = ahead;
      asm volatile("" ::: "memory");
      fetch(t0 + 1);
      __builtin_amdgcn_s_waitcnt(0xc07f);
      stage_barrier();
    }
    for (int t = t0; t < nt; t += 2) {
      step(t, k0, v0, k1, v1);
      step(t + 1, k1, v1, k0, v0);
    }
  }
  if (!work) return;
  const float2 ml = rows.stats();
  if (!rv) return;
  if (part.ml) {
    const size_t row = (size_t)(w.place + at.i) * qs.nh + at.hq;
    if (lh == 0) part.ml[row] = ml;
    rows.outputs([&](int chunk, float4 x) { *reinterpret_cast<float4 *>(part.o + row * D + 4 * chunk) = x; });
    return;
  }
  const float inv = inv_sum(ml.y);
  uint16_t *out = static_cast<uint16_t *>(qs.out) + at.t * qs.ot + (size_t)at.hq * qs.oh;
  rows.outputs([&](int chunk, float4 x) {
    *reinterpret_cast<u32x2 *>(out + 4 * chunk) = u32x2{pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv)};
  });
}

// ---------------------------------------------------------------------------
// Few rows (bf16), 16 per wave: the same steps on v_mfma_f32_16x16x32_bf16 over tiles of 32
// keys.  Lane (g, n) = (l / 16, l % 16) holds row n; register i of score tile st is key
// 16 st + 4 g + i, register i of output tile t is element 16 t + 4 g + i.  Half the registers
// and matrix cycles of a 32-row tile, so that a CU holds enough waves to keep its loads coming.
// ---------------------------------------------------------------------------
typedef float f32x4 __attribute__((ext_vector_type(4)));

// A pair of weights as two bf16 numbers each, their leading bits and the rest: 15 bits that the product with V keeps.  The
// rest of a weight that is not zero is not zero either, so that its product with an infinity is that infinity.  With 16
// rows a wave the matrix pipe has the time (error 2.4 -> 1.7e-3 as at softmax_update; single tokens of 64 sequences over
// 8 bits 166 -> 168 us, over 4 bits 116 -> 122, over bf16 289 -> 290; at d = 64, where the vector work bounds quantised
// pages, 4 bits 73 -> 80 and 20 sequences of 8 bits 57 -> 61).
__device__ __forceinline__ void two_parts(float p0, float p1, uint32_t &lead, uint32_t &rest) {
  const uint32_t a = __float_as_uint(p0), b = __float_as_uint(p1);
  lead = __builtin_amdgcn_perm(b, a, 0x07060302u);
  const float r0 = fmaxf(p0 - __uint_as_float(a & 0xffff0000u), fminf(p0, 0x1p-126f));
  const float r1 = fmaxf(p1 - __uint_as_float(b & 0xffff0000u), fminf(p1, 0x1p-126f));
  rest = pack_bf16x2(r0, r1);
}

template <int D>
struct Wave16 {
  static constexpr int R = 16;
  bf16x8 qf[D / 32];
  f32x4 o[D / 16];
  float mrun, off, lrun;
  bool any;
  __device__ __forceinline__ void init(const uint16_t *q, bool ok) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
      u32x4 x = {0, 0, 0, 0};
      if (ok) x = *reinterpret_cast<const u32x4 *>(q + 32 * kk + 8 * g);
      qf[kk] = __builtin_bit_cast(bf16x8, x);
    }
#pragma unroll
    for (int t = 0; t < D / 16; ++t) o[t] = f32x4{};
    mrun = -INFINITY, off = NAN, lrun = 0.0f, any = false;
  }
  static __device__ __forceinline__ u32x4 v_op(const char *vt, int t) {
    const int l = threadIdx.x & 63, g = l >> 4, cq = l & 15;
    const int ka = 4 * g + (cq >> 2), kb = ka + 16, dvb = 4 * t + (cq & 3);
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_i16x4 *)(vt + ka * (2 * D) + 16 * v_swz<D>(ka, dvb >> 1) + 8 * (dvb & 1)));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_i16x4 *)(vt + kb * (2 * D) + 16 * v_swz<D>(kb, dvb >> 1) + 8 * (dvb & 1)));
    const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
    return u32x4{a[0], a[1], b[0], b[1]};
  }
  // One tile: nvalid keys (bank tiles), or the keys of vis where not `whole`.
  __device__ __forceinline__ void step(const char *kt, char *vt, float c, int nvalid, bool whole, uint32_t vis) {
    const int l = threadIdx.x & 63, g = l >> 4, n = l & 15;
    f32x4 sc[2];
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      const int key = 16 * st + n;
      f32x4 acc = {};
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(kt + key * (2 * D) + 16 * k_swz<D>(key, 4 * kk + g))),
            qf[kk], acc, 0, 0, 0);
      sc[st] = acc;
    }
    if (!whole) {
      bool some = false;
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (vis & (1u << (16 * st + i))) some = true;
          else sc[st][i] = -INFINITY;
        }
      any |= some;
    } else {
      any = true;
      if (nvalid < 32) {
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * st + 4 * g + i >= nvalid) sc[st][i] = -INFINITY;
      }
    }
    uint32_t pb[4], pl[4];
    float psum = 0.0f;
    auto exps = [&](float ref, float off) __attribute__((always_inline)) {
      psum = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e >> 1][2 * (e & 1)] - ref, c, off));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e >> 1][2 * (e & 1) + 1] - ref, c, off));
        two_parts(p0, p1, pb[e], pl[e]);
        psum += p0 + p1;
      }
    };
    exps(0.0f, off);
    const bool over = !(psum <= kLazyLimit);
    if (__any(over)) {  // as softmax_update
      int raise = over;
      raise |= __shfl_xor(raise, 16, 64);
      raise |= __shfl_xor(raise, 32, 64);
      float tmax = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                         fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 16, 64));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
      const float mnew = raise ? fmaxf(mrun, tmax) : mrun;
      const float mref = mnew == -INFINITY ? 0.0f : mnew;
      const float corr = raise ? __builtin_amdgcn_exp2f((mrun - mref) * c) : 1.0f;
      mrun = mnew;
      lrun *= corr;
#pragma unroll
      for (int t = 0; t < D / 16; ++t) o[t] *= corr;
      const float noff = -mref * c;
      const bool far = is_far(noff);
      off = far || mnew == -INFINITY ? NAN : noff;
      exps(far ? mref : 0.0f, far ? 0.0f : noff);
    }
    lrun += psum;
    if (!whole) purge(vt, vis);
    const u32x4 bp = {pb[0], pb[1], pb[2], pb[3]}, bl = {pl[0], pl[1], pl[2], pl[3]};
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      const bf16x8 a = __builtin_bit_cast(bf16x8, v_op(vt, t));
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, bp), o[t], 0, 0, 0);
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, bl), o[t], 0, 0, 0);
    }
  }
  // As the function of that name for 32 rows.
  __device__ __forceinline__ void purge(char *vt, uint32_t vis) {
    if (!has_nonfinite<64 * D>(vt)) return;
    u32x4 bv;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = 16 * (e >> 1) + 2 * (e & 1);
      bv[e] = ((vis >> k) & 1 ? 0x3f80u : 0u) | ((vis >> (k + 1)) & 1 ? 0x3f800000u : 0u);
    }
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      u32x4 a = v_op(vt, t);
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = kind_of(a[e] & 0xffffu) | (kind_of(a[e] >> 16) << 16);
      f32x4 kinds = {};
      kinds = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, bv), kinds, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[t][i] += value_of_kinds(kinds[i]);
    }
    zero_nonfinite<64 * D, 64>(vt);
  }
  // (maximum, sum) of the row, and the outputs as float4 chunks: put(chunk of 4 elements, values)
  __device__ __forceinline__ float2 stats() const {
    int a = any;
    a |= __shfl_xor(a, 16, 64);
    a |= __shfl_xor(a, 32, 64);
    float l = lrun + __shfl_xor(lrun, 16, 64);
    l += __shfl_xor(l, 32, 64);
    return float2{mrun, row_sum(mrun, l, a != 0)};
  }
  template <class F>
  __device__ __forceinline__ void outputs(F put) const {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) put(4 * t + g, float4{o[t][0], o[t][1], o[t][2], o[t][3]});
  }
};

// 32 rows per wave, tiles of 32 keys.
template <int D>
struct Wave32 {
  static constexpr int R = 32;
  bf16x8 qf[D / 16];
  Rows<D> r;
  __device__ __forceinline__ void init(const uint16_t *q, bool ok) {
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      u32x4 x = {0, 0, 0, 0};
      if (ok) x = *reinterpret_cast<const u32x4 *>(q + 16 * kk + 8 * h);
      qf[kk] = __builtin_bit_cast(bf16x8, x);
    }
    r.init();
  }
  __device__ __forceinline__ void step(const char *kt, char *vt, float c, int nvalid, bool whole, uint32_t vis) {
    f32x16 sc[1];
    uint32_t pb[1][8];
    scores<D, 1>(kt, qf, sc);
    if (whole) {
      r.any = true;
      if (nvalid < 32) mask_bank<1>(sc, nvalid);
    } else {
      r.any |= mask_cache<1>(sc, &vis);
    }
    softmax_update<D, 1>(r, sc, pb, c);
    if (!whole) purge<D, 1, 64>(r, vt, &vis, true);
    product<D, 1>(r, pb, vt);
  }
  __device__ __forceinline__ float2 stats() const { return r.stats(); }
  template <class F>
  __device__ __forceinline__ void outputs(F put) const { r.outputs(put); }
};

// ---------------------------------------------------------------------------
// Few rows, and fp32: a workgroup of 4 waves owns up to 32 rows; each wave walks tiles of 32 keys
// of its own (every fourth), and the four results are joined at the end.  No wave waits for another
// before that, so the loads of all are in flight the whole time.  Measured: 64 sequences x 32 heads
// on 8 over 4,096 to 8,192 tokens of 8 bits: 168 us, 4.9 TB/s of cache (826 MB; a large read reaches 6.0, a copy
// 4.65), of 4 bits 123 us (426 MB: the conversion and the softmax); with a bank of 4,680 in bf16 beside 8 bits 376 us,
// 5.5 TB/s; 2 x 32 heads on 8 over 131,071 tokens in bf16, 16 splits: 180 us, 5.5 TB/s; one token of 12
// heads over 1,028 tokens of 4 bits: 13 us, of which two launches are 8.
// ---------------------------------------------------------------------------
constexpr int kFWaves = 4, kFK = 32, kFLeast = 4;

// What a workgroup of 4 waves knows about its row block of R rows and its run of key tiles.
template <int R>
struct Block {
  int s, h, b, place, len, here, r0, tb, nt;
  NewRows nr;
  Plan pl;
  // False where it has nothing to do.
  __device__ __forceinline__ bool init(const Pages &c, const Mask &mask, const BankRows &bank, const CacheQueries &qs,
                                       int nsplit, int slots) {
    Piece w;
    if (!my_piece<R>(c, qs, nsplit, slots, w)) return false;
    s = w.s, h = w.h, place = w.place, nr = w.nr;
    b = s * c.H + h;
    r0 = w.rb * R;
    here = min(R, min(nr.n, c.max_new) * qs.G - r0);
    len = uni(seq_length(c, s));
    pl = uni(plan_of<kFK>(mask, bank, b, len, nr.n, r0 / qs.G, (r0 + here - 1) / qs.G));
    const int used = splits_used<kFLeast>(pl.total, nsplit);
    if (w.split >= used) return false;
    split_range<kFWaves>(pl.total, used, w.split, tb, nt);
    tb = uni(tb), nt = uni(nt);
    return true;
  }
  __device__ __forceinline__ WaveMask wave_mask(const Mask &mask, const CacheQueries &qs, int i) const {
    return WaveMask{seen_by(mask, len, nr.n, r0 / qs.G), seen_by(mask, len, nr.n, (r0 + here - 1) / qs.G),
                    seen_by(mask, len, nr.n, i), mask.sink};
  }
};

// The four waves' results (in LDS, 16 rows of D floats a wave in lo, 16 more in hi; 16-byte chunk j of row r at
// j ^ (r % 8); wml: maxima and sums) joined under their common maximum, and written out, or as partial results of a
// split call.  unit: the factor of the maxima's unit to log2.
template <int DT, int D, int R>
__device__ __forceinline__ void join_waves(const char *lo, const char *hi, const float2 (*wml)[R], const Block<R> &k, const Pages &c,
                                           const CacheQueries &qs, const Part &part, float unit) {
  for (int e = threadIdx.x; e < k.here * (D / 4); e += 64 * kFWaves) {
    const int rr = e / (D / 4), j = 4 * (e % (D / 4));
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kFWaves; ++w) M = fmaxf(M, wml[w][rr].x);
    float lt = 0.0f, a[4] = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kFWaves; ++w) {
      const float2 ml = wml[w][rr];
      const float f = ml.x == M ? 1.0f : __builtin_amdgcn_exp2f((ml.x - M) * unit);
      const float4 x = *reinterpret_cast<const float4 *>((rr < 16 ? lo : hi) + 4 * ((16 * w + rr % 16) * D + (j ^ (4 * (rr % 8)))));
      lt = __builtin_fmaf(ml.y, f, lt);
      a[0] = __builtin_fmaf(x.x, f, a[0]);
      a[1] = __builtin_fmaf(x.y, f, a[1]);
      a[2] = __builtin_fmaf(x.z, f, a[2]);
      a[3] = __builtin_fmaf(x.w, f, a[3]);
    }
    const RowAt ra = row_at(k.nr, qs, k.h, k.r0 + rr);
    if (part.ml) {
      const size_t row = (size_t)(k.place + ra.i) * qs.nh + ra.hq;
      if (j == 0) part.ml[row] = float2{M, lt};
      *reinterpret_cast<float4 *>(part.o + row * D + j) = float4{a[0], a[1], a[2], a[3]};
      continue;
    }
    const float inv = inv_sum(lt);
    const size_t o = ra.t * qs.ot + (size_t)ra.hq * qs.oh + j;
    if constexpr (DT == DKV_BF16)
      *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(qs.out) + o) =
          u32x2{pack_bf16x2(a[0] * inv, a[1] * inv), pack_bf16x2(a[2] * inv, a[3] * inv)};
    else
      *reinterpret_cast<float4 *>(static_cast<float *>(qs.out) + o) = float4{a[0] * inv, a[1] * inv, a[2] * inv, a[3] * inv};
  }
}

// R rows per workgroup: 16 or 32.
template <int FMT, int D, int R>
__global__ __launch_bounds__(64 * kFWaves, FMT == DKV_CACHE_FULL && D == 128 ? 1 : 2) void k_cache_attn_few(
    Pages c, Mask mask, BankRows bank, CacheQueries qs, int nsplit, int slots, Part part) {
  constexpr bool FULL = FMT == DKV_CACHE_FULL;
  constexpr int TB = kFK * 2 * D;  // one tile of K or V
  // Stages of a K and a V tile per wave; the first holds the waves' results at the end.  Arrays of their own, so
  // that reads of one are known not to wait for loads into another.
  __shared__ __attribute__((aligned(1024))) char k0[kFWaves * TB], v0[kFWaves * TB];
  __shared__ __attribute__((aligned(1024))) char k1[FULL ? kFWaves * TB : 16], v1[FULL ? kFWaves * TB : 16];
  __shared__ float2 wml[kFWaves][R];
  __shared__ __attribute__((aligned(256))) int pages_lds[64 * kFWaves];
  Block<R> k;
  if (!k.init(c, mask, bank, qs, nsplit, slots)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, n = l % R;
  const RowAt at = row_at(k.nr, qs, k.h, k.r0 + min(n, k.here - 1));
  const WaveMask wm = k.wave_mask(mask, qs, at.i);
  PageWindow pw;
  pw.init(c, k.s, pages_lds + 64 * wave);
  const unsigned char *bk = static_cast<const unsigned char *>(bank.k) + (size_t)k.b * bank.cap * (2 * D);
  const unsigned char *bv = static_cast<const unsigned char *>(bank.v) + (size_t)k.b * bank.cap * (2 * D);
  char *ka = k0 + wave * TB, *va = v0 + wave * TB, *kb = k1 + (FULL ? wave * TB : 0), *vb = v1 + (FULL ? wave * TB : 0);
  std::conditional_t<R == 16, Wave16<D>, Wave32<D>> w;
  w.init(static_cast<const uint16_t *>(qs.q) + at.t * qs.qt + (size_t)at.hq * qs.qh, n < k.here);
  // here, so that no use of a query inside the loops waits for the tiles on their way
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
  auto compute = [&](bool isbank, int t, const char *kt, char *vt, uint32_t absent) __attribute__((always_inline)) {
    const int pos = tile_pos(k.pl, kFK, t);
    const bool whole = isbank || (absent == 0 && wm.all(pos, kFK));
    w.step(kt, vt, qs.scale_log2, isbank ? k.pl.m - t * kFK : kFK, whole, whole ? 0 : visible_bits(wm, pos, 0, absent, c.lps, l / R));
  };
  const int kcols = max(1, kFK >> c.lps);  // pages that a tile lies in
  const Rows8<D> ld = rows8_offsets<D>();
  const PoolAt pool(c, k.h, FULL ? 2 * D : Quarter<FULL ? DKV_CACHE_FP8 : FMT, D>::kRow);
  // Loads of tile t, always the same number: behind the last tile they read nothing.
  auto issue = [&](int t, char *kd, char *vd) __attribute__((always_inline)) -> uint32_t {
    uint32_t absent = 0;
    const bool isbank = !FULL || t < k.pl.nb, in = t < k.nt;
    const int pos = tile_pos(k.pl, kFK, t);
    bool edge = false;
    if (in && !isbank) {
      pw.seek(pos >> c.lps);
      edge = pw.gone != 0 || pos < k.pl.lo || pos + kFK > k.pl.hi;
      if (edge) absent = pw.absent(pos >> c.lps, kcols);
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const unsigned char *kp = bk, *vp = bv;
      int valid = 0;
      if (in) {
        if (isbank) {
          const int r8 = t * kFK + 8 * g;
          kp = bk + (size_t)r8 * (2 * D), vp = bv + (size_t)r8 * (2 * D);
          valid = bound(k.pl.m - r8, 0, 8);
        } else {
          const int p8 = pos + 8 * g;
          valid = 8;
          if (edge) valid = !pw.absent(p8 >> c.lps, 1) && (p8 + 8 > k.pl.lo || p8 < mask.sink) ? bound(k.pl.hi - p8, 0, 8) : 0;
          const size_t off = pool.at(pw.page(p8 >> c.lps), p8);
          kp = c.k + off, vp = c.v + off;
        }
      }
      rows8_issue<D>(ld.rsub, ld.pc, ld.v, kp, vp, valid, 8 * g, kd, vd);
    }
    return absent;
  };
  if constexpr (FULL) {
    // two stages: a tile in flight while the other is used
    constexpr int kTileLoads = 4 * 2 * Rows8<D>::kLoads;
    auto step = [&](int t, const char *kt, char *vt, uint32_t absent, char *kn, char *vn) __attribute__((always_inline)) {
      const uint32_t nx = issue(t + kFWaves, kn, vn);
      __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(kTileLoads));  // the next tile may still be on its way
      asm volatile("" ::: "memory");
      if (t < k.nt) compute(t < k.pl.nb, t, kt, vt, absent);
      __builtin_amdgcn_s_waitcnt(0xc07f);  // its reads are done before the stage is loaded again
      asm volatile("" ::: "memory");
      return nx;
    };
    uint32_t p0 = issue(k.tb + wave, ka, va), p1 = 0;
    for (int t = k.tb + wave; t < k.nt; t += 2 * kFWaves) {  // whole rounds of the stages, as in the other kernel
      p1 = step(t, ka, va, p0, kb, vb);
      p0 = step(t + kFWaves, kb, vb, p1, ka, va);
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));  // nothing is on its way to the stages
    asm volatile("" ::: "memory");
  } else {
    // bank tiles one at a time: the other waves of the CU cover their latency
    int t = k.tb + wave;
    for (; t < min(k.nt, k.pl.nb); t += kFWaves) {
      issue(t, ka, va);
      __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
      asm volatile("" ::: "memory");
      compute(true, t, ka, va, 0);
      __builtin_amdgcn_s_waitcnt(0xc07f);
      asm volatile("" ::: "memory");
    }
    // quantised rows through registers, two tiles ahead (one where two do not fit the registers); a
    // lane: two quarter rows of K and two of V, in rows l / 4 and 16 + l / 4
    constexpr int kAhead = R == 16 || D == 64 ? 2 : 1;
    struct {
      Quarter<FMT, D> k[2], v[2];
      uint32_t absent;
    } f[kAhead];
    const int part4 = l & 3, lr = l >> 2;
    auto fetch = [&](auto &y, int t) __attribute__((always_inline)) {
      size_t row[2] = {0, 0};
      int valid[2] = {0, 0};
      y.absent = 0;
      if (t < k.nt) {
        const int pos = tile_pos(k.pl, kFK, t);
        pw.seek(pos >> c.lps);
        valid[0] = valid[1] = 16;
        if (pw.gone != 0 || pos < k.pl.lo || pos + kFK > k.pl.hi) {
          y.absent = pw.absent(pos >> c.lps, kcols);
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const int p = pos + 16 * g;
            valid[g] = !pw.absent(p >> c.lps, 1) && (p + 16 > k.pl.lo || p < mask.sink) ? bound(k.pl.hi - p, 0, 16) : 0;
          }
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) row[g] = pool.at(pw.page((pos + 16 * g) >> c.lps), pos + 16 * g);
      }
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const size_t srow = row[g] / (Quarter<FMT, D>::kRow / (D / kGroup));  // scales: one byte per group
        y.k[g].load(c.k + row[g], c.ks + srow, valid[g], lr, part4);
        y.v[g].load(c.v + row[g], c.vs + srow, valid[g], lr, part4);
      }
    };
    auto step = [&](auto &y, int t) __attribute__((always_inline)) {
      // the reads of the tile before are done: a wave's LDS operations run in order
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        y.k[g].template store<false>(ka, 16 * g + lr, part4);
        y.v[g].template store<true>(va, 16 * g + lr, part4);
      }
      const uint32_t absent = y.absent;
      asm volatile("" ::: "memory");
      fetch(y, t + kAhead * kFWaves);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
      if (t < k.nt) compute(false, t, ka, va, absent);
      __builtin_amdgcn_wave_barrier();
    };
    fetch(f[0], t);
    asm volatile("" ::: "memory");  // the loads in this order, which the waits count on
    if constexpr (kAhead > 1) fetch(f[kAhead - 1], t + kFWaves);
    asm volatile("" ::: "memory");
    for (; t < k.nt; t += kAhead * kFWaves) {
      step(f[0], t);
      if constexpr (kAhead > 1) step(f[kAhead - 1], t + kFWaves);
    }
  }

  if (n < k.here) {
    float *mo = reinterpret_cast<float *>(n < 16 ? ka : va) + (n % 16) * D;  // in the stages that only this wave uses
    const float2 ml = w.stats();
    if (l < R) wml[wave][n] = ml;
    w.outputs([&](int chunk, float4 x) { *reinterpret_cast<float4 *>(mo + 4 * (chunk ^ (n % 8))) = x; });
  }
  __syncthreads();
  join_waves<DKV_BF16, D, R>(k0, v0, wml, k, c, qs, part, qs.scale_log2);
}

// ---------------------------------------------------------------------------
// fp32: 32 rows per workgroup, the keys over its four waves, scores and products on
// v_mfma_f32_32x32x2_f32 (all of it in fp32; one wave a SIMD, so its loads, matrix work and softmax partly add up).  d = 128:
// 2,000 causal tokens of 12 heads over 4,000: 527 us, 70 TFLOP/s (a large product: 153).  Single tokens of 64 sequences, 32
// heads on 8, over 1,500 to 3,000 tokens: 299 us, 4.1 TB/s (a reading: 204); over 8 bits 292 and over 4 bits 287 us, where
// a reading of the pages takes 53 and 27: 4 rows are padded to 32 in the products, and the values are read from LDS two bytes
// at a time.  Lane (h, n) holds row n; K step 16 kk + j takes the dims 16 kk + j
// (h = 0) and 16 kk + 8 + j of both operands.  Rows of fp32 go to LDS (keys, a tile ahead) or
// to registers (values, asked for before the scores); quantised rows are exact in bf16 and go
// through LDS so.
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ int kf_swz(int r, int c) { return c ^ (r % 16); }  // 16-byte chunks of a row of 4 D bytes

// 8 rows of fp32 keys into rows r0 .. of a tile, `valid` of them, the others as zeros.
template <int D>
__device__ __forceinline__ void rows8_issue_f32(const unsigned char *kp, int valid, int r0, char *kt) {
  constexpr int CH = D / 4, RPL = 64 / CH, kLoads = 8 / RPL;
  const int l = threadIdx.x & 63, extent = uni(valid) * (4 * D);
  const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void *)kp, (short)0, extent, kBufferRsrcWord3);
#pragma unroll
  for (int q = 0; q < kLoads; ++q) {
    const int r = q * RPL + l / CH, off = r * (4 * D) + 16 * kf_swz<D>(r0 + r, l % CH);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void *)(kt + r0 * (4 * D) + q * 1024), 16, off, 0, 0, 0);
  }
}

template <int FMT, int D>
__global__ __launch_bounds__(64 * kFWaves, 1) void k_cache_attn_f32(Pages c, Mask mask, BankRows bank, CacheQueries qs,
                                                                   int nsplit, int slots, Part part) {
  constexpr bool FULL = FMT == DKV_CACHE_FULL;
  constexpr int TB = kFK * 4 * D;  // a tile of fp32 keys; a K and a V tile of bf16
  __shared__ __attribute__((aligned(1024))) char k0[kFWaves * TB], k1[FULL ? kFWaves * TB : 16];
  __shared__ float2 wml[kFWaves][32];
  __shared__ __attribute__((aligned(256))) int pages_lds[64 * kFWaves];
  Block<32> k;
  if (!k.init(c, mask, bank, qs, nsplit, slots)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, lh = l >> 5, n = l & 31;
  const RowAt at = row_at(k.nr, qs, k.h, k.r0 + min(n, k.here - 1));
  const WaveMask wm = k.wave_mask(mask, qs, at.i);
  PageWindow pw;
  pw.init(c, k.s, pages_lds + 64 * wave);
  Rows<D> rows;
  rows.init();
  const unsigned char *bk = static_cast<const unsigned char *>(bank.k) + (size_t)k.b * bank.cap * (4 * D);
  const unsigned char *bv = static_cast<const unsigned char *>(bank.v) + (size_t)k.b * bank.cap * (4 * D);
  char *ka = k0 + wave * TB, *kb = k1 + (FULL ? wave * TB : 0);
  float qf[D / 16][8];
  {
    const float *q = static_cast<const float *>(qs.q) + at.t * qs.qt + (size_t)at.hq * qs.qh;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float4 x = *reinterpret_cast<const float4 *>(q + 16 * kk + 8 * lh + 4 * j);
        qf[kk][4 * j] = x.x, qf[kk][4 * j + 1] = x.y, qf[kk][4 * j + 2] = x.z, qf[kk][4 * j + 3] = x.w;
      }
  }
  const int kcols = max(1, kFK >> c.lps);
  const PoolAt pool(c, k.h, FULL ? 4 * D : Quarter<FULL ? DKV_CACHE_FP8 : FMT, D>::kRow);

  // The 8-row groups of a tile of fp32 rows: where they are and how many rows of each may be read (none behind the
  // last tile).
  struct Groups {
    const unsigned char *kp[4], *vp[4];
    int valid[4];
    uint32_t absent;
  };
  auto groups_of = [&](int t) __attribute__((always_inline)) {
    Groups g;
    g.absent = 0;
    const bool isbank = !FULL || t < k.pl.nb, in = t < k.nt;
    const int pos = tile_pos(k.pl, kFK, t);
    bool edge = false;
    if (in && !isbank) {
      pw.seek(pos >> c.lps);
      edge = pw.gone != 0 || pos < k.pl.lo || pos + kFK > k.pl.hi;
      if (edge) g.absent = pw.absent(pos >> c.lps, kcols);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      size_t off = 0;
      g.valid[j] = 0;
      if (in && isbank) {
        const int r8 = t * kFK + 8 * j;
        off = (size_t)r8 * (4 * D);
        g.valid[j] = uni(bound(k.pl.m - r8, 0, 8));
      } else if (in) {
        const int p8 = pos + 8 * j;
        g.valid[j] = 8;
        if (edge)
          g.valid[j] = uni(!pw.absent(p8 >> c.lps, 1) && (p8 + 8 > k.pl.lo || p8 < mask.sink) ? bound(k.pl.hi - p8, 0, 8) : 0);
        off = pool.at(pw.page(p8 >> c.lps), p8);
      }
      g.kp[j] = (isbank ? bk : c.k) + off;
      g.vp[j] = (isbank ? bv : c.v) + off;
    }
    return g;
  };
  auto issue_keys = [&](const Groups &g, char *kt) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) rows8_issue_f32<D>(g.kp[j], g.valid[j], 8 * j, kt);
  };
  // Value register i of column tile t2: key 8 (i / 4) + 4 h + i % 4, element 32 t2 + n.
  auto load_values = [&](const Groups &g, float (*vx)[16]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const __amdgpu_buffer_rsrc_t rv =
          __builtin_amdgcn_make_buffer_rsrc((void *)g.vp[j], (short)0, g.valid[j] * (4 * D), kBufferRsrcWord3);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t2 = 0; t2 < D / 32; ++t2)
          vx[t2][4 * j + e] = __uint_as_float(
              __builtin_amdgcn_raw_buffer_load_b32(rv, (4 * lh + e) * (4 * D) + 4 * n + 128 * t2, 0, 0));
    }
  };
  auto scores_f32 = [&](const char *kt) __attribute__((always_inline)) {
    f32x16 sc = {};
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float4 x = *reinterpret_cast<const float4 *>(kt + n * (4 * D) + 16 * kf_swz<D>(n, 4 * kk + 2 * lh + j));
        sc = __builtin_amdgcn_mfma_f32_32x32x2f32(x.x, qf[kk][4 * j], sc, 0, 0, 0);
        sc = __builtin_amdgcn_mfma_f32_32x32x2f32(x.y, qf[kk][4 * j + 1], sc, 0, 0, 0);
        sc = __builtin_amdgcn_mfma_f32_32x32x2f32(x.z, qf[kk][4 * j + 2], sc, 0, 0, 0);
        sc = __builtin_amdgcn_mfma_f32_32x32x2f32(x.w, qf[kk][4 * j + 3], sc, 0, 0, 0);
      }
    return sc;
  };
  // Softmax update and products of a tile; not `whole`: only the keys of vis.
  auto finish = [&](f32x16 sc, float (*vx)[16], int nvalid, bool whole, uint32_t vis) __attribute__((always_inline)) {
    if (whole) {
      rows.any = true;
      vis = ~0u;
    } else {
      rows.any |= (vis & 0x0f0f0f0fu) != 0;
    }
    float tmax = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = 8 * (i >> 2) + (i & 3);
      sc[i] = ((vis >> key) & 1) && key + 4 * lh < nvalid ? sc[i] * qs.scale_log2 : -INFINITY;
      tmax = fmaxf(tmax, sc[i]);
    }
    tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
    const float mnew = fmaxf(rows.mrun, tmax);
    const float mref = mnew == -INFINITY ? 0.0f : mnew;  // scores of -inf alone: weights 0, not inf - inf
    const float corr = exp2f(rows.mrun - mref);
    rows.mrun = mnew;
    float w[16], ps = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      w[i] = exp2f(sc[i] - mref);
      ps += w[i];
    }
    rows.lrun = __builtin_fmaf(rows.lrun, corr, ps);
#pragma unroll
    for (int t2 = 0; t2 < D / 32; ++t2) rows.o[t2] *= corr;
    if (!whole) {
#pragma unroll
      for (int t2 = 0; t2 < D / 32; ++t2) {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) bad |= (__float_as_uint(vx[t2][i]) & 0x7f800000u) == 0x7f800000u;
        if (__any(bad)) {  // not finite: out of the product, and added to the rows that see it (see purge)
          f32x16 kinds = {};
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t u = __float_as_uint(vx[t2][i]);
            const uint32_t m = u & 0x7fffffffu;
            const float kind = m < 0x7f800000u ? 0.0f : (m > 0x7f800000u ? 16384.0f : (u >> 31 ? 128.0f : 1.0f));
            kinds = __builtin_amdgcn_mfma_f32_32x32x2f32(kind, (vis >> (8 * (i >> 2) + (i & 3))) & 1 ? 1.0f : 0.0f, kinds, 0, 0, 0);
            if (kind != 0.0f) vx[t2][i] = 0.0f;
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) rows.o[t2][i] += value_of_kinds(kinds[i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int t2 = 0; t2 < D / 32; ++t2)
        rows.o[t2] = __builtin_amdgcn_mfma_f32_32x32x2f32(vx[t2][i], w[i], rows.o[t2], 0, 0, 0);
  };
  auto visible = [&](int t, uint32_t absent, bool &whole) __attribute__((always_inline)) {
    const int pos = tile_pos(k.pl, kFK, t);
    whole = absent == 0 && wm.all(pos, kFK);
    return whole ? 0u : visible_bits(wm, pos, 0, absent, c.lps, lh);
  };

  if constexpr (FULL) {
    // keys two stages: a tile in flight while the other is used
    constexpr int kLoads = D / 8, kYounger = 16 * (D / 32) + kLoads;  // a tile's key loads; and its values before the next keys
    Groups g = groups_of(k.tb + wave);
    issue_keys(g, ka);
    auto step = [&](int t, const char *kt, char *kn) __attribute__((always_inline)) {
      float vx[D / 32][16];
      load_values(g, vx);
      asm volatile("" ::: "memory");
      const uint32_t absent = g.absent;
      g = groups_of(t + kFWaves);
      issue_keys(g, kn);
      __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(kYounger < 63 ? kYounger : 63));  // this tile's keys are there
      asm volatile("" ::: "memory");
      if (t < k.nt) {
        const bool isbank = t < k.pl.nb;
        bool whole = true;
        uint32_t vis = 0;
        if (!isbank) vis = visible(t, absent, whole);
        finish(scores_f32(kt), vx, isbank ? k.pl.m - t * kFK : kFK, whole, vis);
      }
      __builtin_amdgcn_s_waitcnt(0xc07f);  // its reads are done before the stage is loaded again
      asm volatile("" ::: "memory");
    };
    for (int t = k.tb + wave; t < k.nt; t += 2 * kFWaves) {
      step(t, ka, kb);
      step(t + kFWaves, kb, ka);
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));  // nothing is on its way to the stages
  } else {
    int t = k.tb + wave;
    for (; t < min(k.nt, k.pl.nb); t += kFWaves) {
      const Groups g = groups_of(t);
      float vx[D / 32][16];
      issue_keys(g, ka);
      load_values(g, vx);
      __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
      asm volatile("" ::: "memory");
      finish(scores_f32(ka), vx, k.pl.m - t * kFK, true, 0);
      __builtin_amdgcn_s_waitcnt(0xc07f);
      asm volatile("" ::: "memory");
    }
    // quantised rows as in the bf16 kernel, one tile ahead; the tile is read as floats
    char *va = ka + TB / 2;
    Quarter<FMT, D> xk[2], xv[2];
    const int part4 = l & 3, lr = l >> 2;
    uint32_t ahead = 0;
    auto fetch = [&](int t2) __attribute__((always_inline)) {
      const int pos = tile_pos(k.pl, kFK, t2);
      const bool in = t2 < k.nt;
      bool edge = false;
      ahead = 0;
      if (in) {
        pw.seek(pos >> c.lps);
        edge = pw.gone != 0 || pos < k.pl.lo || pos + kFK > k.pl.hi;
        if (edge) ahead = pw.absent(pos >> c.lps, kcols);
      }
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        size_t row = 0;
        int valid = 0;
        if (in) {
          const int p16 = pos + 16 * g;
          valid = 16;
          if (edge)
            valid = !pw.absent(p16 >> c.lps, 1) && (p16 + 16 > k.pl.lo || p16 < mask.sink) ? bound(k.pl.hi - p16, 0, 16) : 0;
          row = pool.at(pw.page(p16 >> c.lps), p16);
        }
        const size_t srow = row / (Quarter<FMT, D>::kRow / (D / kGroup));
        xk[g].load(c.k + row, c.ks + srow, valid, lr, part4);
        xv[g].load(c.v + row, c.vs + srow, valid, lr, part4);
      }
    };
    fetch(t);
    for (; t < k.nt; t += kFWaves) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        xk[g].template store<false>(ka, 16 * g + lr, part4);
        xv[g].template store<true>(va, 16 * g + lr, part4);
      }
      const uint32_t absent = ahead;
      asm volatile("" ::: "memory");
      fetch(t + kFWaves);
      asm volatile("" ::: "memory");
      f32x16 sc = {};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        float x[8];
        unpack_bf16x8(*reinterpret_cast<const uint4 *>(ka + n * (2 * D) + 16 * k_swz<D>(n, 2 * kk + lh)), x);
#pragma unroll
        for (int j = 0; j < 8; ++j) sc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], qf[kk][j], sc, 0, 0, 0);
      }
      float vx[D / 32][16];
#pragma unroll
      for (int t2 = 0; t2 < D / 32; ++t2)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = 8 * (i >> 2) + 4 * lh + (i & 3), col = 32 * t2 + n;
          vx[t2][i] = __uint_as_float(
              (uint32_t)*reinterpret_cast<const uint16_t *>(va + key * (2 * D) + 16 * v_swz<D>(key, col >> 3) + 2 * (col & 7)) << 16);
        }
      bool whole;
      const uint32_t vis = visible(t, absent, whole);
      finish(sc, vx, kFK, whole, vis);
      asm volatile("" ::: "memory");
    }
  }

  __syncthreads();  // the results go where other waves had their tiles
  char *lo = k0, *hi = k0 + kFWaves * 64 * D;
  if (n < k.here) {
    float *mo = reinterpret_cast<float *>(n < 16 ? lo : hi) + (16 * wave + n % 16) * D;
    const float2 ml = rows.stats();
    if (lh == 0) wml[wave][n] = ml;
    rows.outputs([&](int chunk, float4 x) { *reinterpret_cast<float4 *>(mo + 4 * (chunk ^ (n % 8))) = x; });
  }
  __syncthreads();
  join_waves<DKV_F32, D, 32>(lo, hi, wml, k, c, qs, part, 1.0f);  // maxima in log2 units
}

constexpr int kMaxSplit = 64;  // a lane of a wave for each

// Rows of a split attention: the partial outputs under their common maximum, divided by the common sum.  Bound by the
// launch (4-5 us) up to some megabytes of partial results, then by reading them (18,720 rows x 3 splits x 128 columns,
// 29 MB: 9.5 us, 3 TB/s).  D / 4 lanes per row and split; SG splits of a row at a time, joined in LDS, their maxima all
// read at once (one after the other, 64 of them, cost 8 us).  RB rows per row block, KT keys per tile of the kernel that
// wrote them.
template <int DT, int D, int RB, int KT, int LEAST, int SG>
__global__ __launch_bounds__(256) void k_cache_combine(Pages c, Mask mask, BankRows bank, CacheQueries qs, int nsplit,
                                                       Part part) {
  constexpr int LR = D / 4, NR = 256 / LR / SG;  // rows per workgroup
  const size_t nrow = (size_t)places(c) * qs.nh;
  const int lane = threadIdx.x % LR, sub = (threadIdx.x / LR) % SG, rr = threadIdx.x / LR / SG, j = 4 * lane;
  const size_t row = (size_t)blockIdx.x * NR + rr;
  bool live = row < nrow;  // nrow < 2^31
  int s = 0, i = 0, hq = 0, used = 0;
  NewRows nr{0, 0};
  if (live) {
    const unsigned place = (unsigned)row / (unsigned)qs.nh;
    hq = (int)((unsigned)row % (unsigned)qs.nh);
    if (c.by_seq) {
      s = (int)(place / (unsigned)c.max_new), i = (int)(place % (unsigned)c.max_new);
    } else {
      s = seq_of<LR>(c, (int)place), i = (int)place;
    }
    live = s >= 0;
    if (live) {
      nr = new_rows(c, s);
      if (!c.by_seq) i -= nr.first;
    }
    const int n = min(nr.n, c.max_new), h = hq / qs.G;
    live = live && i < n;
    if (live) {
      const int r0 = (i * qs.G + hq - h * qs.G) / RB * RB, r1 = min(r0 + RB, n * qs.G) - 1;
      const Plan pl = plan_of<KT>(mask, bank, s * c.H + h, seq_length(c, s), nr.n, r0 / qs.G, r1 / qs.G);
      used = splits_used<LEAST>(pl.total, nsplit);
    }
  }
  const float unit = DT == DKV_BF16 ? qs.scale_log2 : 1.0f;  // the bf16 maxima are raw scores
  float l = 0.0f, a[4] = {0, 0, 0, 0};
  auto weight = [&](float mx, float M) { return mx == M ? 1.0f : __builtin_amdgcn_exp2f((mx - M) * unit); };
  auto add = [&](int k, float w) {
    const float4 x = *reinterpret_cast<const float4 *>(part.o + (k * nrow + row) * D + j);
    a[0] = __builtin_fmaf(x.x, w, a[0]);
    a[1] = __builtin_fmaf(x.y, w, a[1]);
    a[2] = __builtin_fmaf(x.z, w, a[2]);
    a[3] = __builtin_fmaf(x.w, w, a[3]);
  };
  if constexpr (SG > 1) {  // one row: lane k of every wave takes the maximum and sum of split k, in one latency
    static_assert(NR == 1 && kMaxSplit <= 64, "");
    const int kk = threadIdx.x & 63;
    float2 ml{-INFINITY, 0.0f};
    if (kk < used) ml = part.ml[kk * nrow + row];
    float M = ml.x;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
    const float w = kk < used ? weight(ml.x, M) : 0.0f;
    l = kk < used ? ml.y * w : 0.0f;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
    for (int k0 = 0; k0 < used; k0 += SG) {
      const float wk = __shfl(w, min(k0 + sub, 63), 64);
      if (k0 + sub < used) add(k0 + sub, wk);
    }
    __shared__ float4 la[256];
    la[threadIdx.x] = float4{a[0], a[1], a[2], a[3]};
    __syncthreads();
    if (sub != 0) return;
#pragma unroll
    for (int k = 1; k < SG; ++k) {
      const float4 x = la[threadIdx.x + k * LR];
      a[0] += x.x, a[1] += x.y, a[2] += x.z, a[3] += x.w;
    }
  } else {
    float M = -INFINITY;
    for (int k = 0; k < used; ++k) M = fmaxf(M, part.ml[k * nrow + row].x);
#pragma unroll 4
    for (int k = 0; k < used; ++k) {
      const float2 ml = part.ml[k * nrow + row];
      const float w = weight(ml.x, M);
      l = __builtin_fmaf(ml.y, w, l);
      add(k, w);
    }
  }
  if (!live) return;
  const float inv = inv_sum(l);
  const size_t o = (size_t)(nr.first + i) * qs.ot + (size_t)hq * qs.oh + j;
  if constexpr (DT == DKV_BF16)
    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(qs.out) + o) =
        u32x2{pack_bf16x2(a[0] * inv, a[1] * inv), pack_bf16x2(a[2] * inv, a[3] * inv)};
  else
    *reinterpret_cast<float4 *>(static_cast<float *>(qs.out) + o) = float4{a[0] * inv, a[1] * inv, a[2] * inv, a[3] * inv};
}

constexpr int kCUs = 256;
constexpr int kManySplits = 5;  // splits from which a row's partial results are read 8 (d = 64: 16) at a time

// Rows of a (sequence, kv head) up to which blocks of 16 or 32 rows are taken: 64, or 32 where the two stages of bf16
// rows leave a CU one workgroup (us of 32-row and 256-row blocks, 8 kv heads, up to 8,192 tokens).  8-bit pages, d = 128,
// 32 sequences: 32 rows 93 and 169, 64 rows 125 and 171, 128 rows 214 and 174; 4 sequences: 28 and 35, 33 and 37, 45 and
// 44; d = 64, 32 sequences: 64 rows 81 and 110, 128 rows 141 and 112.  bf16 pages, d = 128, 32 sequences: 32 rows 159 and
// 171, 64 rows 228 and 170.
int few_rows(int fmt, int d) { return fmt == DKV_CACHE_FULL && d == 128 ? 32 : 64; }

// New tokens that a call's sequences have: the bound of the longest where the caller knows one, else their mean.
int new_tokens(const Pages &c) { return c.max_new < c.T ? c.max_new : (int)(((int64_t)c.T + c.S - 1) / c.S); }

// Rows per row block of a call: 16 or 32 with the keys over the waves, or 256.
int block_rows(const Pages &c, int dtype, int fmt, int d, int G) {
  const int64_t rows = (int64_t)new_tokens(c) * G;
  if (dtype != DKV_BF16) return 32;
  return rows <= 16 ? 16 : (rows <= few_rows(fmt, d) ? 32 : kWRows);
}

template <int DT, int D, int RB, int KT, int LEAST>
void combine(const Pages &c, const Mask &mask, const BankRows &bank, const CacheQueries &qs, int nsplit, const Part &part,
             hipStream_t s) {
  constexpr int kGroups = 256 / (D / 4);
  const int64_t nrow = places(c) * qs.nh;  // < 2^31 (checked by the caller)
  if (nsplit >= kManySplits)
    k_cache_combine<DT, D, RB, KT, LEAST, kGroups><<<(unsigned)nrow, 256, 0, s>>>(c, mask, bank, qs, nsplit, part);
  else
    k_cache_combine<DT, D, RB, KT, LEAST, 1><<<(unsigned)((nrow + kGroups - 1) / kGroups), 256, 0, s>>>(c, mask, bank, qs,
                                                                                                       nsplit, part);
}

template <int DT, int FMT, int D>
hipError_t attn_impl(const Pages &c, const Mask &mask, const BankRows &bank, const CacheQueries &qs, void *ws, int nsplit,
                     hipStream_t s) {
  const int64_t nrow = places(c) * qs.nh;
  if (c.T == 0 || c.max_new == 0) return hipSuccess;
  Part part{nullptr, nullptr};
  if (nsplit > 1) {  // the outputs first, then the maxima and sums
    part.o = static_cast<float *>(ws);
    part.ml = reinterpret_cast<float2 *>(part.o + nrow * nsplit * D);
  }
  const int R = block_rows(c, DT, FMT, D, qs.G);
  const int64_t nrb = ((int64_t)c.max_new * qs.G + R - 1) / R;
  const int64_t even = nrb * c.S, packed = packed_slots(c, qs.G, R);  // slots if all are the longest, or of T rows
  const bool counted = c.start && c.S > 1 && c.S <= kCountedSeqs && nrb > 1;
  const int slots = counted ? kCounted : (!c.start || even <= packed ? (int)nrb : kSearched);
  const int64_t grid = (slots == kSearched || (counted && packed < even) ? packed : even) * c.H * nsplit;
  if (!grid_fits(grid, 64 * kWWaves) || (nsplit > 1 && !grid_fits(nrow, 256))) return hipErrorInvalidConfiguration;
  const unsigned g = (unsigned)grid;
  if constexpr (DT == DKV_BF16) {
    if (R == kWRows) {
      k_cache_attn_wide<FMT, D><<<g, 64 * kWWaves, 0, s>>>(c, mask, bank, qs, nsplit, slots, part);
      if (nsplit > 1) combine<DT, D, kWRows, wide_keys(D), wide_least(D)>(c, mask, bank, qs, nsplit, part, s);
    } else if (R == 32) {
      k_cache_attn_few<FMT, D, 32><<<g, 64 * kFWaves, 0, s>>>(c, mask, bank, qs, nsplit, slots, part);
      if (nsplit > 1) combine<DT, D, 32, kFK, kFLeast>(c, mask, bank, qs, nsplit, part, s);
    } else {
      k_cache_attn_few<FMT, D, 16><<<g, 64 * kFWaves, 0, s>>>(c, mask, bank, qs, nsplit, slots, part);
      if (nsplit > 1) combine<DT, D, 16, kFK, kFLeast>(c, mask, bank, qs, nsplit, part, s);
    }
  } else {
    k_cache_attn_f32<FMT, D><<<g, 64 * kFWaves, 0, s>>>(c, mask, bank, qs, nsplit, slots, part);
    if (nsplit > 1) combine<DT, D, 32, kFK, kFLeast>(c, mask, bank, qs, nsplit, part, s);
  }
  return hipGetLastError();
}

}  // namespace

// Splits: the time is about rounds of workgroups over the chip times (tiles per split and
// some tiles' worth of prologue), plus the joining kernel.  Waves with tiles of their own work in
// rounds of four: one token of 12 heads over 8,001 tokens of 4 bits 22 -> 14 us, in fp32 2 x 64 rows over 400 keys
// 17 -> 15 us, against runs that end within a round and a joining that reads the maxima in turn.
int cache_attention_splits(const Pages &c, int dtype, int fmt, int d, const Mask &mask, const BankRows &bank, int nh,
                           size_t *bytes) {
  *bytes = 0;
  const int G = nh / c.H;
  const int64_t nrow = places(c) * nh;
  if (c.T == 0 || c.max_new == 0) return 1;
  const int news = new_tokens(c);
  const int RB = block_rows(c, dtype, fmt, d, G);
  const bool few = RB != kWRows;
  const int KT = few ? kFK : wide_keys(d), least = few ? kFLeast : wide_least(d);
  const int step = few ? kFWaves : 1;
  int64_t keys = (int64_t)c.cols << c.lps;
  if (mask.window > 0) {
    const int64_t seen = (int64_t)mask.window + (mask.causal ? news : 0) + mask.sink + KT;
    if (seen < keys) keys = seen;
  }
  const int64_t tiles = (keys + KT - 1) / KT + (bank.cap + KT - 1) / KT;
  const int64_t nwg = min(((int64_t)news * G + RB - 1) / RB * c.S, packed_slots(c, G, RB)) * c.H;
  const int64_t slots = few && (d == 64 || fmt != DKV_CACHE_FULL) && dtype == DKV_BF16 ? 2 * kCUs : kCUs;
  // us per tile of a workgroup, and per workgroup
  const double tile_us = dtype != DKV_BF16 ? (d == 64 ? 0.8 : 1.3) : (few ? (d == 64 ? 0.4 : 0.7) : (d == 64 ? 2.0 : 1.9));
  const double start_us = few ? 5.0 : 8.0;
  int best = 1;
  double best_cost = 0.0;
  for (int S = 1; S <= kMaxSplit && (S == 1 || S <= (tiles + least - 1) / least); ++S) {
    const double rounds = (double)((nwg * S + slots - 1) / slots);
    const int64_t per = ((tiles + S - 1) / S + step - 1) / step * step;  // tiles of a workgroup
    double cost = rounds * ((double)per * tile_us + start_us);
    if (S > 1) cost += 5.0 + (double)nrow * S * (8.0 * d + 16.0) / 4e6;
    if (S == 1 || cost < 0.95 * best_cost) best = S, best_cost = cost;
  }
  if (best > 1) *bytes = (size_t)nrow * best * (d * 4 + 8);
  return best;
}

hipError_t launch_cache_attention(const Pages &c, int dtype, int fmt, int d, const Mask &mask, const BankRows &bank,
                                  const CacheQueries &qs, void *ws, int nsplit, hipStream_t s) {
#define DKV_CASE(DT, FMT, D) \
  if (dtype == DT && fmt == FMT && d == D) return attn_impl<DT, FMT, D>(c, mask, bank, qs, ws, nsplit, s);
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
