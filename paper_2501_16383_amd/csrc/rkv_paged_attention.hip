// Attention of packed rows over the cache in pages.
//
// Per query head h of KV head g = h / rep: out = sum_t w_t v_t, w = softmax(scale q.k_t).  The rows of a sequence that
// read one KV head - its new tokens times the rep query heads - are the columns of two matrix products,
//   S^T[token][column] = K . Q^T          O^T[channel][column] = V^T . P^T,
// so that a lane of the result owns one column: the running maximum and sum of its softmax are plain registers, and
// the weights a lane gets from the first product are, in their order, an operand of the second.
// (Which token is which index of the sum is free as long as both operands agree.)  Weights are powers of two of
// scores in fp32; the sum of weights is taken in fp32 from unrounded weights.  For the second product weights are rounded to
// the cache's type, which is what a product on the matrix units at the rate of 16 bits costs: against the definition in 64 bits outputs are off by
// up to 0.0022 (bf16) or 0.00026 (fp16) in k_paged_chunk, where the rounding of the output alone makes 0.0017 and 0.00021; few rows: 5 % more than it.
#include <type_traits>

#include "rkv_mfma_ops.h"
#include "rkv_paged.h"

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));

template <int DT> __device__ __forceinline__ f4 paged_mfma16(u32x4 a, u32x4 b, f4 c) {
  if constexpr (DT) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

typedef float f16v __attribute__((ext_vector_type(16)));
template <int DT> __device__ __forceinline__ f16v paged_mfma32(u32x4 a, u32x4 b, f16v c) {
  if constexpr (DT) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

#define LDS_AS __attribute__((address_space(3)))
#define PAGED_INLINE __attribute__((always_inline))
#define PAGED_CONST __attribute__((address_space(4)))      // not written while a kernel runs: scalar loads
// Four rows of sixteen 16-bit elements, transposed: lane i of a row of 16 gives the address of row i >> 2, elements
// 4 (i & 3) .., and gets element i of the four rows.
__device__ __forceinline__ u32x2 paged_transposed(const unsigned short* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s4*)p));
}

// 16 bytes for each lane from base + offset straight to LDS, lane after lane from `to` on (base and `to` are the wave's).  Not the
// builtin: after that one the compiler has every read of LDS wait for the copy, also those of other buffers.  It does
// not know of this one: whoever reads waits for vmcnt(0) first (paged_copies_done) and meets the other waves at a barrier.
__device__ __forceinline__ void paged_copy(const void* base, uint32_t offset, unsigned short* to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               : : "{m0}"((uint32_t)(uintptr_t)(LDS_AS unsigned short*)to), "v"(offset), "s"(base) : "memory");   // (m0: written by the compiler, which knows of it)
}
__device__ __forceinline__ void paged_copies_done() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }

// Is the element in the low half an infinity or NaN?
template <int DT> __device__ __forceinline__ bool paged_odd(uint32_t x) {
  constexpr uint32_t ex = DT ? 0x7f80 : 0x7c00;
  return (x & ex) == ex;
}

// Queries for a scale of zero: what is not finite as NaN, everything else as 0 - a score that is a number then is 0, also where the
// unscaled one would pass fp32
template <int DT> __device__ __forceinline__ uint32_t paged_times_zero(uint32_t x) {
  constexpr uint32_t nan = DT ? 0x7fc0 : 0x7e00;
  return (paged_odd<DT>(x) ? nan : 0) | (paged_odd<DT>(x >> 16) ? nan << 16 : 0);
}

__device__ __forceinline__ float paged_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Weights are held times a power of two that the division by their sum takes out again: in fp16 the largest is
// 2^14 or a little more, so that one of 2^-28 of it still is a normal number (as a subnormal of 2^-25 it would be off by up to its own size).
template <int DT> __device__ constexpr float paged_bias() { return DT ? 0.f : 14.f; }

// The exponent that weights are taken against where the largest score's is `top`.  From 2^24 on fp32's numbers lie 2 and more
// apart: where the difference comes out as 16, 2^16 would be no fp16 number, and the largest weight is 1.
template <int DT> __device__ __forceinline__ float paged_ref(float top) {
  const float r = top - paged_bias<DT>();
  return top - r > 15.f ? top : r;
}

// ... and how far the largest may pass that before it is taken anew.  The difference is exact where it matters; half a power more than
// the bias, because top - 14 is rounded and would look passed again and again.
template <int DT> __device__ constexpr float paged_slack() { return DT ? 0.f : 14.5f; }

// The exponent of the same power in k_paged_chunk, where weights may pass the largest by 2^8
template <int DT> __device__ constexpr float paged_chunk_bias() { return DT ? 0.f : 6.f; }

// score times scale, rounded, less `ref`: not one operation, which would leave the product's rounding in the difference
__device__ __forceinline__ float paged_less(float score, float scale, float ref) {
#pragma clang fp contract(off)
  const float x = score * scale;
  return x - ref;
}

// the value of the lane 32 further
__device__ __forceinline__ float paged_other(float x, float& mine) {
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  mine = __uint_as_float(r[0]);
  return __uint_as_float(r[1]);
}

// maximum / sum over the four rows of 16 lanes
__device__ __forceinline__ float paged_max4(float x) {
  u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float paged_sum4(float x) {
  u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Splits of the sequences' tokens: partial results of a work unit (a sequence's columns or a tile of them, and a KV
// head), as acc [unit][column][split][D] and then (exponent that weights are taken against, their sum) [unit][column][split]
struct PagedSplit {
  int chunk, splits;                  // tokens of a split, most splits of a sequence
  float* acc;
  float2* ml;
};

// What a call asks for beside the batch
struct PagedAsk {
  const unsigned short* q;
  int64_t qs;
  unsigned short* out;
  float* lse;
  float scale2;                       // scale * log2(e)
  int causal, window;
  int few;                            // rows times rep up to which a sequence goes to k_paged_few
  int mixed;                          // sequences with more go to k_paged_chunk (else there are none but bad ones)
  PagedSplit sp;
};

// Log-sum-exp of a sum of weights against 2^ref, times 2^bias
__device__ __forceinline__ float paged_lse(float ref, float sum, float bias) {
  return sum == 0 ? -INFINITY : (ref + (__log2f(sum) - bias)) * 0.69314718055994531f;
}

// Tokens that the row at position p sees: lo .. hi - 1 (none in front of the first token)
__device__ __forceinline__ int paged_hi_of(const PagedAsk& a, const PagedSeq& s, int p) { return p < 0 ? 0 : a.causal ? min(p + 1, s.len) : s.len; }
__device__ __forceinline__ int paged_lo_of(const PagedAsk& a, int p) { return a.window ? max(0, p - a.window + 1) : 0; }

// NaN for every row of a bad sequence that reads this KV head
template <int D, int DT> __device__ __forceinline__ void paged_bad_rows(const PagedView& v, const PagedAsk& a, int first, int last, int kvh) {
  const int n = (last - first) * v.rep;
  for (int64_t i = threadIdx.x; i < (int64_t)n * D; i += blockDim.x) {
    const int c = (int)(i / D);
    a.out[((int64_t)(first + c / v.rep) * v.Hq + kvh * v.rep + c % v.rep) * D + i % D] = DT ? 0x7fc0 : 0x7e00;
  }
  if (a.lse)
    for (int c = threadIdx.x; c < n; c += blockDim.x) a.lse[(int64_t)(first + c / v.rep) * v.Hq + kvh * v.rep + c % v.rep] = __uint_as_float(0x7fc00000);
}

// ---- few rows: single tokens, drafted tokens -----------------------------------------------------
//
// A workgroup takes up to 16 NB columns of one (sequence, KV head) over one split of its tokens, each wave every
// fourth tile of 32.  Keys go from memory into the registers of the lanes that feed them to the matrix unit
// (lane l: token l % 16, a quarter of its channels); values, whose operand runs along the tokens, pass through
// the wave's own LDS as 16-bit rows and come back transposed.  The next tile's values are asked for as soon as
// these are in LDS, its keys as soon as these are multiplied.
//
// What bounds it: the stream of the cache.  32 sequences of 8192 tokens, 8 KV heads of 128, 8 bits: 96 us = 5.8 TB/s, and 94
// with the arithmetic left out; more bytes in flight (three or four workgroups a compute unit) change nothing.  With two blocks of
// columns the registers are not enough: up to 34 scalar ones and, with 16 bits of bf16 and heads of 128, six vector ones are spilled.
template <int D, int BITS, int DT, int NB>
__global__ __launch_bounds__(256, NB == 1 ? 3 : 2) void k_paged_few(PagedView v, PagedAsk a) {
  constexpr int KL = D * BITS / 8 / 4 / 16;                 // 16-byte loads of a quarter row of keys (0: one of 8 bytes)
  constexpr int VP = D * BITS / 8 / 16, VL = 32 * VP / 64;  // 16-byte parts of a row of values; loads of a lane for 32 tokens
  constexpr int rb = paged_row<D, BITS>(), sb = paged_srow<D, BITS>();
  constexpr int PITCH = D + 16;                             // 16-bit elements between two tokens' values in LDS
  constexpr int CB = D / 16, NK = D / 32;
  constexpr int OP = D + 4;                                 // floats between two columns when waves meet
  __shared__ __align__(16) unsigned short lds[4 * 32 * PITCH];
  __shared__ float meet[2][4][16];
  static_assert(4 * 16 * OP * 4 <= 4 * 32 * PITCH * 2, "the waves' results fit the values' rows");

  const int kvh = blockIdx.x, split = blockIdx.y, b = blockIdx.z;   // (the heads of a page at the same time)
  const PagedSeq s = paged_seq(v, b);
  const int rows = s.last - s.first, cols = rows * v.rep;
  if (rows == 0) return;
  if (cols > a.few && a.mixed) return;                      // the other kernel's
  if (s.bad) {
    if (split == 0) paged_bad_rows<D, DT>(v, a, s.first, s.last, kvh);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;

  // tokens that some row sees, and this split's share
  const int all_lo = paged_lo_of(a, s.base), all_hi = paged_hi_of(a, s, s.base + rows - 1);
  const int from = (all_lo & ~31) + split * a.sp.chunk, to = min(all_hi, from + a.sp.chunk);
  if (split && from >= all_hi) return;
  // ... that all rows see
  const int full_lo = paged_lo_of(a, s.base + rows - 1), full_hi = paged_hi_of(a, s, s.base);

  u32x4 q[NB][NK];
  int hi[NB], lo[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int c = 16 * i + n, row = c / v.rep;
    const bool on = c < cols;
    const int p = s.base + row;
    hi[i] = on ? paged_hi_of(a, s, p) : 0;
    lo[i] = on ? paged_lo_of(a, p) : 0;
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      const int ch = BITS == 16 ? 32 * j + 8 * g : g * (D / 4) + 8 * j;
      const u32x4 z = {0, 0, 0, 0};
      q[i][j] = on ? *(const u32x4*)(a.q + (s.first + row) * a.qs + (kvh * v.rep + c % v.rep) * D + ch) : z;
    }
  }

  f4 o[NB][CB];
  float m[NB], l[NB];                                       // what weights are taken against (paged_ref), their sum
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    m[i] = -INFINITY;
    l[i] = 0;
#pragma unroll
    for (int c = 0; c < CB; ++c) o[i][c] = f4{0, 0, 0, 0};
  }
  unsigned short* vl = lds + wave * 32 * PITCH;
  const int mask = (1 << v.page_shift) - 1;
  const int64_t page_bytes = paged_block<D, BITS>(v.page_shift) * v.Hkv;
  const unsigned char* pool = v.pool + paged_block<D, BITS>(v.page_shift) * kvh;
  const int last_page = (s.len - 1) >> v.page_shift;        // (len > 0 where there is a tile at all)
  const PAGED_CONST int* table = (const PAGED_CONST int*)(v.table + (int64_t)b * v.max_pages);
  u32x4 kx[2][KL ? KL : 1], vx[VL];                         // bytes of the tile to come
  uint32_t ks[2], vs[VL];
  int page[2];                                              // of its two sixteens of tokens

  auto pages = [&](int t) PAGED_INLINE {
#pragma unroll
    for (int i = 0; i < 2; ++i) page[i] = table[min((t + 16 * i) >> v.page_shift, last_page)];
  };
  auto block = [&](int i, bool& ok) PAGED_INLINE {
    ok = (unsigned)page[i] < (unsigned)v.n_pages;
    return pool + (ok ? page[i] : 0) * page_bytes;
  };
  auto load_keys = [&](int t) PAGED_INLINE {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      bool ok;
      const unsigned char* blk = block(i, ok);
      const int slot = (t + 16 * i) & mask;
      const unsigned char* kp = blk + slot * rb + (n * rb + (BITS == 16 ? 16 * g : g * (rb / 4)));
      if constexpr (KL == 0) {
        const u32x2 w = *(const u32x2*)kp;
        kx[i][0] = u32x4{w[0], w[1], 0, 0};
      } else {
#pragma unroll
        for (int j = 0; j < KL; ++j) kx[i][j] = *(const u32x4*)(kp + (BITS == 16 ? 64 : 16) * j);
      }
      if constexpr (BITS < 16) {
        ks[i] = (blk + ((2 * rb) << v.page_shift) + slot * sb)[n * sb + (D == 128 ? g : g >> 1)];
        if (!ok) ks[i] = 255;                               // keys of no page: NaN
      } else if (!ok) {
#pragma unroll
        for (int j = 0; j < KL; ++j) kx[i][j] = u32x4{~0u, ~0u, ~0u, ~0u};
      }
    }
  };
  auto load_values = [&](int t) PAGED_INLINE {
    constexpr int TL = 64 / VP;                             // tokens of a wave's load: of one sixteen, or (D = 64, 4 bits) of both
    bool ok[2];
    const unsigned char *at[2], *sat[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned char* blk = block(i, ok[i]);
      const int slot = (t + 16 * i) & mask;
      at[i] = blk + (rb << v.page_shift) + slot * rb;
      sat[i] = blk + ((2 * rb + sb) << v.page_shift) + slot * sb;
    }
    const bool inside = t >= all_lo && t + 32 <= all_hi && ok[0] && ok[1];
#pragma unroll
    for (int r = 0; r < VL; ++r) {
      const int tok = r * TL + lane / VP, part = lane % VP; // token in the tile
      const int i = r * TL / 16;
      const unsigned char* c = TL <= 16 ? at[i] : lane < 32 ? at[0] : at[1];
      const unsigned char* e = TL <= 16 ? sat[i] : lane < 32 ? sat[0] : sat[1];
      vx[r] = *(const u32x4*)(c + ((tok & 15) * rb + part * 16));
      if constexpr (BITS < 16) vs[r] = e[(tok & 15) * sb + part * (128 / BITS) / 32];
      if (!inside) {
        // a value row that no row sees, or of no page, counts as zeros: weight 0 times whatever lies there must be 0
        const bool seen = (TL <= 16 ? ok[i] : lane < 32 ? ok[0] : ok[1]) && t + tok < all_hi && t + tok >= all_lo;
        if (!seen) vx[r] = u32x4{0, 0, 0, 0};
        if (BITS < 16 && !seen) vs[r] = 127;
      }
    }
  };
  auto compute = [&](int t, bool more) PAGED_INLINE {         // tile t; more: tile t + 128 is this wave's next
    const bool whole = t >= full_lo && t + 32 <= full_hi;   // every row sees every token
    const bool mixed_rows = !whole && rows > 1;             // ... or some do
    // values to LDS as 16-bit rows
    bool odd = false;                                       // holds infinities or NaN
#pragma unroll
    for (int r = 0; r < VL; ++r) {
      const int ci = r * 64 + lane, tok = ci / VP, part = ci % VP;
      u32x4* d = (u32x4*)(vl + tok * PITCH + part * (128 / BITS));
      if constexpr (BITS == 16) {
        d[0] = vx[r];
      } else {
        const float sc = paged_scale(vs[r]);
        odd |= vs[r] == 255;
#pragma unroll
        for (int e = 0; e < 16 / BITS; ++e) {
          const u32x2 w = {vx[r][BITS == 8 ? 2 * e : e], BITS == 8 ? vx[r][2 * e + 1] : 0};
          d[e] = paged_decode8<DT, BITS>(w, sc);
        }
      }
    }
    if (BITS == 16 && mixed_rows) {
#pragma unroll
      for (int r = 0; r < VL; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= paged_odd<DT>(vx[r][e]) || paged_odd<DT>(vx[r][e] >> 16);
    }
    if (more) {
      pages(t + 128);
      load_values(t + 128);
    }
    // scores
    f4 sc[NB][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u32x4 kk[NK];
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        if constexpr (BITS == 16) kk[j] = kx[i][j];
        else {
          const int w = j * (BITS / 4);                     // dword of the lane's codes
          const u32x2 c = {kx[i][w / 4][w % 4], BITS == 8 ? kx[i][w / 4][(w % 4) + 1 & 3] : 0};
          kk[j] = paged_decode8<DT, BITS>(c, paged_scale(ks[i]));
        }
      }
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        sc[c][i] = f4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < NK; ++j) sc[c][i] = paged_mfma16<DT>(kk[j], q[c][j], sc[c][i]);
      }
    }
    if (more) load_keys(t + 128);
    u32x4 p[NB];
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = sc[c][e >> 2][e & 3] * a.scale2;
      if (!whole) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int tok = t + 16 * (e >> 2) + 4 * g + (e & 3);
          w[e] = tok >= lo[c] && tok < hi[c] ? w[e] : -INFINITY;
        }
      }
      float top = fmaxf(fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3])), fmaxf(fmaxf(w[4], w[5]), fmaxf(w[6], w[7])));
      top = paged_max4(top);
      const bool up = top - m[c] > paged_slack<DT>();
      if (__any(up)) {
        const float m2 = up ? paged_ref<DT>(top) : m[c], f = up ? paged_exp2(m[c] - m2) : 1.f;   // (of other columns nothing changes)
        m[c] = m2;
        l[c] *= f;
#pragma unroll
        for (int k = 0; k < CB; ++k) o[c][k] *= f;
      }
      const float ref = m[c] == -INFINITY ? 0.f : m[c];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = paged_exp2(w[e] - ref);
        l[c] += w[e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) p[c][e] = paged_pair<DT>(w[2 * e], w[2 * e + 1]);
    }
    wave_lds_fence();
    if (mixed_rows && __any(odd)) {
      // A value that is not finite, and rows that do not see it: 0 times it is not 0.  Rows that see it take it here; the
      // products below find a zero in its place, and give the other rows the bits that they always have.
#pragma unroll 1
      for (int tok = 0; tok < 32; ++tok) {
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          // the weight of token tok is element tok % 4 (+ 4 from token 16 on) of the lanes' row (tok % 16) / 4
          uint32_t pw = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) pw = (tok >> 4) * 2 + ((tok & 3) >> 1) == e ? p[c][e] : pw;
          pw = __shfl(pw, n + 16 * ((tok >> 2) & 3));
          const float pf = tok & 1 ? paged_hi<DT>(pw) : paged_lo<DT>(pw);
          const bool sees = t + tok >= lo[c] && t + tok < hi[c];
#pragma unroll
          for (int k = 0; k < CB; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t bits = vl[tok * PITCH + 16 * k + 4 * g + e];
              if (sees && paged_odd<DT>(bits)) o[c][k][e] += pf * paged_lo<DT>(bits);
            }
        }
      }
      wave_lds_fence();
      for (int i = lane; i < 32 * D; i += 64) {
        unsigned short* e = vl + i / D * PITCH + i % D;
        if (paged_odd<DT>(*e)) *e = 0;
      }
      wave_lds_fence();
    }
    const unsigned short* at = vl + (4 * g + (n >> 2)) * PITCH + 4 * (n & 3);
#pragma unroll
    for (int k = 0; k < CB; ++k) {
      const u32x2 a0 = paged_transposed(at + 16 * k), a1 = paged_transposed(at + 16 * PITCH + 16 * k);
      const u32x4 vv = {a0[0], a0[1], a1[0], a1[1]};
#pragma unroll
      for (int c = 0; c < NB; ++c) o[c][k] = paged_mfma16<DT>(vv, p[c], o[c][k]);
    }
    wave_lds_fence();
  };

  const int first = from + 32 * wave;
  if (first < to) {
    pages(first);
    load_values(first);
    load_keys(first);
  }
  if (a.scale2 == 0)
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < NK; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) q[i][j][e] = paged_times_zero<DT>(q[i][j][e]);
  for (int t = first; t < to; t += 128) compute(t, t + 128 < to);

  // the four waves meet
  float* os = (float*)lds;
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    __syncthreads();                                        // (the waves' values are read, the round before is done)
    const float lt = paged_sum4(l[c]);
    if (g == 0) {
      meet[0][wave][n] = m[c];
      meet[1][wave][n] = lt;
    }
#pragma unroll
    for (int k = 0; k < CB; ++k) *(f4*)(os + (wave * 16 + n) * OP + 16 * k + 4 * g) = o[c][k];
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < 16 * D; i += 256) {
      const int col = i / D, ch = i % D, cc = 16 * c + col;
      if (cc >= cols) break;
      const float m0 = meet[0][0][col], m1 = meet[0][1][col], m2 = meet[0][2][col], m3 = meet[0][3][col];
      const float mm = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)), ref = mm == -INFINITY ? 0.f : mm;
      float sum = 0, acc = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = paged_exp2(meet[0][w][col] - ref);
        sum += f * meet[1][w][col];
        acc += f * os[(w * 16 + col) * OP + ch];
      }
      const int64_t at = (int64_t)(s.first + cc / v.rep) * v.Hq + kvh * v.rep + cc % v.rep;
      if (a.sp.splits == 1) {
        a.out[at * D + ch] = (unsigned short)paged_pair<DT>(sum == 0 ? 0.f : acc / sum, 0.f);
        if (a.lse && ch == 0) a.lse[at] = paged_lse(mm, sum, 0);
      } else {
        const int64_t u = (((int64_t)b * v.Hkv + kvh) * (16 * NB) + cc) * a.sp.splits + split;
        a.sp.acc[u * D + ch] = acc;
        if (ch == 0) a.sp.ml[u] = make_float2(mm, sum);
      }
    }
  }
}

// One column's splits together, by a wave: u0 is the first one's index, `at` the column's place in the output.  Eight at a time are
// asked for together, maxima and all, so that a chain of latencies is what it takes: 4 us for the largest batches.
template <int D, int DT> __device__ __forceinline__ void paged_join(const PagedAsk& a, int64_t u0, int n, int64_t at) {
  constexpr int W = 8, C = D / 64;                          // splits at a time; channels of a lane
  const int lane = threadIdx.x & 63;
  float m = -INFINITY, sum = 0, acc[C] = {};
  for (int i0 = 0; i0 < n; i0 += W) {
    float2 ml[W];
    float x[W][C];
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const int64_t u = u0 + min(i0 + i, n - 1);
      ml[i] = a.sp.ml[u];
#pragma unroll
      for (int j = 0; j < C; ++j) x[i][j] = a.sp.acc[u * D + lane + 64 * j];
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < W; ++i) top = fmaxf(top, ml[i].x);
    const float ref = top == -INFINITY ? 0.f : top, f0 = paged_exp2(m - ref);
    sum *= f0;
#pragma unroll
    for (int j = 0; j < C; ++j) acc[j] *= f0;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float f = i0 + i < n ? paged_exp2(ml[i].x - ref) : 0.f;
      sum += f * (i0 + i < n ? ml[i].y : 0.f);              // (not 0 times a NaN)
#pragma unroll
      for (int j = 0; j < C; ++j) acc[j] += f * (i0 + i < n ? x[i][j] : 0.f);
    }
    m = top;
  }
#pragma unroll
  for (int j = 0; j < C; ++j) a.out[at * D + lane + 64 * j] = (unsigned short)paged_pair<DT>(sum == 0 ? 0.f : acc[j] / sum, 0.f);
  if (a.lse && lane == 0) a.lse[at] = paged_lse(m, sum, 0);
}

template <int D, int DT, int NB>
__global__ __launch_bounds__(256) void k_paged_merge(PagedView v, PagedAsk a) {
  const int c = blockIdx.x * 4 + (threadIdx.x >> 6), kvh = blockIdx.y, b = blockIdx.z;
  const PagedSeq s = paged_seq(v, b);
  const int rows = s.last - s.first, cols = rows * v.rep;
  if (s.bad || cols > a.few || c >= cols) return;
  const int lo = paged_lo_of(a, s.base) & ~31, hi = paged_hi_of(a, s, s.base + rows - 1);
  const int n = max(1, (hi - lo + a.sp.chunk - 1) / a.sp.chunk);
  paged_join<D, DT>(a, (((int64_t)b * v.Hkv + kvh) * (16 * NB) + c) * a.sp.splits, n,
                    (int64_t)(s.first + c / v.rep) * v.Hq + kvh * v.rep + c % v.rep);
}

// ---- many rows: chunks, prompts ----------------------------------------------------------------
//
// A workgroup takes 32 WAVES columns of one (sequence, KV head), 32 a wave, and walks the tokens that they see in
// tiles of 64, which it stages in LDS as 16-bit rows: tile i + 2 comes from memory while tile i is computed, with one
// barrier a tile.  A wave works in half tiles: the softmax of one stands beside the scores of the next and the values of the one
// before, so that matrix and vector unit have work that does not wait for the other.
//
// What bounds it: no unit by itself, but that softmax and staging do not wholly hide behind the products.  8192 tokens, 32 query heads
// on 8 KV heads of 128, 16 bits: 540-570 us (0.96-1.0 PFLOP/s).  The products with their reads of LDS (1 KiB for every 32 x 32 x 16) alone take
// 390 us, the softmax alone 250, staging adds 80; the matrix units are busy in 51 % of the cycles, LDS in 26 %, and 3 % of the waves' cycles
// are spent waiting for it.  64 columns a wave would halve the reads, but their 512 registers leave one wave a SIMD, which took twice as long.
#define PAGED_TILE 64

// The tile of columns that a workgroup takes: sequence and first column, or b = n_seqs.  Sequences of more than `few`
// columns have ceil(columns / COLS) tiles each, numbered through; the last columns, which see most, come first.
__device__ __forceinline__ int paged_find_tile(const PagedView& v, int few, int per, int tile, int& c0) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 0; b0 < v.n_seqs; b0 += 64) {
    int t = 0;
    if (b0 + lane < v.n_seqs) {
      const int f = min(max(v.row_start[b0 + lane], 0), v.n_rows), l = min(max(v.row_start[b0 + lane + 1], f), v.n_rows);
      const int cols = (l - f) * v.rep;
      t = cols > few ? (cols + per - 1) / per : 0;
    }
    int upto = t;                                           // sum over the lanes up to this one
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    const uint64_t m = __ballot(before + upto > tile);
    if (m) {
      const int i = __builtin_ctzll(m);
      const int n = __shfl(t, i), first = before + __shfl(upto, i) - n;
      c0 = (n - 1 - (tile - first)) * per;
      return b0 + i;
    }
    before += __shfl(upto, 63);
  }
  c0 = 0;
  return v.n_seqs;
}

// 0 in the place of infinities and NaN
template <int DT> __device__ __forceinline__ uint32_t paged_finite(uint32_t x) {
  return (paged_odd<DT>(x) ? 0 : x & 0xffffu) | (paged_odd<DT>(x >> 16) ? 0 : x & 0xffff0000u);
}

template <int D, int BITS, int DT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_paged_chunk(PagedView v, PagedAsk a) {
  constexpr int rb = paged_row<D, BITS>(), sb = paged_srow<D, BITS>(), COLS = 32 * WAVES, T = PAGED_TILE, N = WAVES * 64;
  // 16-bit elements between two tokens in LDS.  Codes are converted on their way and written with a pitch that spreads reads of
  // 32 keys' / of 4 values' parts over the banks; 16 bits go there directly, 64 lanes' parts one after the other, so that
  // the parts of a row change places instead (key_part, value_part).
  constexpr bool DIRECT = BITS == 16;
  constexpr int PK = DIRECT ? D : D + 8, PV = DIRECT ? D : D + 32;
  constexpr int VP = rb / 16;                               // 16-byte parts of a row
  constexpr int NS = D / 16, CB = D / 32;
  constexpr float SLACK = 8.f;                              // a maximum may be exceeded by 2^8 before everything is scaled anew
  __shared__ __align__(16) unsigned short lk[3][T * PK], lv[4][T * PV];
  __shared__ int odd_tile[4];                               // the last tile in the buffer that held a value which is not finite
  const int kvh = blockIdx.x % v.Hkv, unit = blockIdx.x / v.Hkv, split = blockIdx.y;
  int c0;
  const int b = __builtin_amdgcn_readfirstlane(paged_find_tile(v, a.few, COLS, unit, c0));
  if (b >= v.n_seqs) return;
  c0 = __builtin_amdgcn_readfirstlane(c0);
  const PagedSeq s = paged_seq(v, b);
  const int rows = s.last - s.first, cols = rows * v.rep;
  const int r0 = c0 / v.rep, r1 = min(c0 + COLS, cols) - 1;   // first row; last column
  if (s.bad) {
    // (rows of this tile's columns; a row whose columns two tiles share is written by both)
    if (split == 0) paged_bad_rows<D, DT>(v, a, s.first + r0, s.first + r1 / v.rep + 1, kvh);
    return;
  }
  const int all_lo = paged_lo_of(a, s.base + r0), all_hi = paged_hi_of(a, s, s.base + r1 / v.rep);
  const int from = (all_lo & ~(T - 1)) + split * a.sp.chunk, to = min(all_hi, from + a.sp.chunk);
  if (split && from >= all_hi) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;

  // this lane's column, and the tokens it sees
  const int cc = c0 + wave * 32 + n, pos = s.base + cc / v.rep;
  const bool mine = cc < cols;
  const int hi = mine ? paged_hi_of(a, s, pos) : 0, lo = mine ? paged_lo_of(a, pos) : 0;
  const int64_t at = (int64_t)(s.first + cc / v.rep) * v.Hq + kvh * v.rep + cc % v.rep;
  u32x4 q[NS];
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const u32x4 z = {0, 0, 0, 0};
    q[j] = mine ? *(const u32x4*)(a.q + (s.first + cc / v.rep) * a.qs + (kvh * v.rep + cc % v.rep) * D + 16 * j + 8 * h) : z;
  }
  const float scale2 = a.scale2 == 0 ? 1.f : fabsf(a.scale2);
  f16v o[CB];
  float m = -INFINITY, l = 0, worst = 0;                    // worst: largest magnitude that m had
#pragma unroll
  for (int k = 0; k < CB; ++k) o[k] = f16v{};

  // Staging: the lanes of a wave take 64 neighbouring parts, which lie in one page (in the pages of two sixteens of tokens
  // where a row is but two parts) and one after the other in memory: a scalar address, and 16 bytes a lane.  A wave
  // takes G such groups of keys and the same of values, or, where a tile's keys are fewer parts than threads, one of either.
  constexpr bool BOTH = T * VP >= N;
  constexpr int G = BOTH ? T * VP / N : 1, R = BOTH ? 2 * G : 1, TL = 64 / VP, NP = TL > 16 ? 2 : 1;   // loads; tokens of one; their pages
  static_assert(!BOTH || T * VP % N == 0, "groups of keys and values fall together");
  const int mask = (1 << v.page_shift) - 1;
  const int64_t page_bytes = paged_block<D, BITS>(v.page_shift) * v.Hkv;
  const unsigned char* pool = v.pool + paged_block<D, BITS>(v.page_shift) * kvh;
  const int last_page = (s.len - 1) >> v.page_shift;
  const PAGED_CONST int* table = (const PAGED_CONST int*)(v.table + (int64_t)b * v.max_pages);
  const bool has = BOTH || wave < 2 * T * VP / 64, val0 = !BOTH && wave >= T * VP / 64;   // (else: this wave's load is of values)
  const int ltok = lane / VP, lpart = lane % VP;
  const int tok0 = (wave * 64 / VP) % T;                    // first token of this wave's first group
  // where part c of token t's keys / values lies in its row (and which part lies in place c)
  auto key_part = [&](int t, int c) PAGED_INLINE { return DIRECT ? c ^ (t & (VP - 1)) : c; };
  auto value_part = [&](int t, int c) PAGED_INLINE { return DIRECT ? c ^ ((D == 128 ? t & 3 : t >> 1 & 1) << 2) : c; };
  // (direct: the part that belongs where this lane's bytes go; its row is lane / VP more than a multiple of 64 / VP)
  const uint32_t lkey = DIRECT ? ltok * rb + key_part(tok0 + ltok, lpart) * 16 : 0, lvalue = DIRECT ? ltok * rb + value_part(tok0 + ltok, lpart) * 16 : 0;
  const uint32_t lcode = lane * 16 % (16 * rb), lscale = (ltok & 15) * sb + lpart * (128 / BITS) / 32;   // (of a sixteen of tokens)
  u32x4 x[R];
  uint32_t xs[R];
  int page[G][NP], was[G][NP];                              // of the tile to load, and of the one in x
  bool gone = false;                                        // a page of it is none of the pool's
  auto pages = [&](int t) PAGED_INLINE {
#pragma unroll
    for (int r = 0; r < G; ++r)
#pragma unroll
      for (int i = 0; i < NP; ++i) page[r][i] = table[min((t + tok0 + r * (N / VP) + 16 * i) >> v.page_shift, last_page)];
  };
  auto load = [&](int t, int kb, int vb) PAGED_INLINE {     // (direct: into these buffers)
    gone = false;
    if (!has) return;
#pragma unroll
    for (int r = 0; r < G; ++r) {
      const unsigned char *at[NP], *sat[NP];                // first key code, first key scale
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        was[r][i] = page[r][i];
        const bool ok = (unsigned)page[r][i] < (unsigned)v.n_pages;
        gone |= !ok;
        const unsigned char* blk = pool + (ok ? page[r][i] : 0) * page_bytes;
        const int slot = (t + tok0 + r * (N / VP) + 16 * i) & mask;
        at[i] = blk + slot * rb + ((val0 ? rb : 0) << v.page_shift);
        sat[i] = blk + ((2 * rb + (val0 ? sb : 0)) << v.page_shift) + slot * sb;
      }
#pragma unroll
      for (int w = 0; w < (BOTH ? 2 : 1); ++w) {            // keys, values
        const unsigned char* c = at[0];
        const unsigned char* e = sat[0];
        if constexpr (NP > 1) {
          c = lane < 32 ? c : at[1];
          e = lane < 32 ? e : sat[1];
        }
        if constexpr (DIRECT) {
          paged_copy(c + ((w * rb) << v.page_shift), w ? lvalue : lkey, (w ? lv[vb] : lk[kb]) + (tok0 + r * (N / VP)) * D);
        } else x[r + w * G] = *(const u32x4*)(c + ((w * rb) << v.page_shift) + lcode);
        if constexpr (BITS < 16) xs[r + w * G] = e[((w * sb) << v.page_shift) + lscale];
      }
    }
  };
  // rows that all columns of the workgroup see whole
  const int wg_lo = paged_lo_of(a, s.base + r1 / v.rep), wg_hi = paged_hi_of(a, s, s.base + r0);
  auto stage = [&](int t, int kb, int vb) PAGED_INLINE {
    if (!has) return;
    const bool plain = t >= wg_lo && t + T <= wg_hi && !gone;
    if constexpr (DIRECT) paged_copies_done();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool val = BOTH ? r >= G : val0;
      const int tok = tok0 + (r % G) * (N / VP) + ltok;
      u32x4* d = (u32x4*)((val ? lv[vb] + tok * PV : lk[kb] + tok * PK) + lpart * (128 / BITS));
      if (__builtin_expect(!plain, 0)) {
        // values that no row of the tile sees, or of no page, count as zeros; keys of no page as NaN
        const int pg = NP > 1 && lane >= 32 ? was[r % G][NP - 1] : was[r % G][0];
        const bool ok = (unsigned)pg < (unsigned)v.n_pages, seen = ok && t + tok < all_hi && t + tok >= all_lo;
        const u32x4 z = {0, 0, 0, 0}, none = {~0u, ~0u, ~0u, ~0u};
        if constexpr (DIRECT) x[r] = *d;
        if (val) x[r] = seen ? x[r] : z;
        else if (BITS == 16) x[r] = ok ? x[r] : none;
        bool odd = false;
        if constexpr (BITS < 16) {
          xs[r] = val ? (seen ? xs[r] : 127) : ok ? xs[r] : 255;
          odd = xs[r] == 255;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) odd |= paged_odd<DT>(x[r][e]) || paged_odd<DT>(x[r][e] >> 16);
        }
        if (val && odd) odd_tile[vb] = t;
        if constexpr (DIRECT) *d = x[r];
      }
      if constexpr (!DIRECT) {
#pragma unroll
        for (int e = 0; e < 16 / BITS; ++e) {
          const u32x2 w = {x[r][BITS == 8 ? 2 * e : e], BITS == 8 ? x[r][2 * e + 1] : 0};
          d[e] = paged_decode8<DT, BITS>(w, paged_scale(xs[r]));
        }
      }
    }
  };

  // scores of 32 tokens: S^T = K Q^T
  auto scores = [&](const unsigned short* kb, f16v& sc) PAGED_INLINE {
    sc = f16v{};
#pragma unroll
    for (int j = 0; j < NS; ++j) sc = paged_mfma32<DT>(*(const u32x4*)(kb + n * PK + key_part(n, 2 * j + h) * 8), q[j], sc);
  };
  // O^T += V^T P^T over 32 tokens from t on.  Lane 16 (2 h + i) + j gives the address of token 4 h + j / 4 (and 8 more), channels
  // 16 i + 4 (j % 4) ..
  auto values = [&](auto fix, const unsigned short* vb, const u32x4* p, int t) PAGED_INLINE {
    if constexpr (decltype(fix)::value) {
      // Values that are not finite, and rows that do not see them: 0 times those is not 0.  Rows that see one take it here; the
      // products below find a zero in its place.
#pragma unroll 1
      for (int tok = 0; tok < 32; ++tok) {
        uint32_t pw = 0;
        const int want = (tok >> 3) * 2 + ((tok & 3) >> 1);
#pragma unroll
        for (int e = 0; e < 8; ++e) pw = want == e ? p[e >> 2][e & 3] : pw;
        pw = __shfl(pw, n + 32 * ((tok >> 2) & 1));
        const float pf = tok & 1 ? paged_hi<DT>(pw) : paged_lo<DT>(pw);
        const bool sees = t + tok >= lo && t + tok < hi;
#pragma unroll
        for (int k = 0; k < CB; ++k)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t bits = vb[tok * PV + value_part(tok, 4 * k + (e >> 2)) * 8 + 4 * h + (e & 3)];
            if (sees && paged_odd<DT>(bits)) o[k][e] += pf * paged_lo<DT>(bits);
          }
      }
    }
    const int row = 4 * h + ((lane & 15) >> 2);
    const unsigned short* from = vb + row * PV + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int k = 0; k < CB; ++k) {
        const unsigned short* at = from + 16 * j * PV + (DIRECT ? value_part(row, 4 * k) * 8 : 32 * k);
        const u32x2 a0 = paged_transposed(at), a1 = paged_transposed(at + 8 * PV);
        u32x4 vv = {a0[0], a0[1], a1[0], a1[1]};
        if constexpr (decltype(fix)::value) {
#pragma unroll
          for (int e = 0; e < 4; ++e) vv[e] = paged_finite<DT>(vv[e]);
        }
        o[k] = paged_mfma32<DT>(vv, p[j], o[k]);
      }
  };
  // Half a tile's step: the softmax of 32 tokens (from t on) beside two products that do not depend on it, the next 32 tokens'
  // scores and the 32 values before.  Those belong to the maximum before this step: O is scaled anew at its end.
  auto step = [&](auto masked, f16v& sc, f16v& next, const unsigned short* kb, u32x4* p, const u32x4* before, const unsigned short* vb,
                  int t, int tb, bool odd) PAGED_INLINE {
    if constexpr (decltype(masked)::value) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int tok = t + 8 * (e >> 2) + 4 * h + (e & 3);
        sc[e] = tok >= lo && tok < hi ? sc[e] : -INFINITY;
      }
    }
    float top = sc[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, sc[e]);
    float own;
    const float other = paged_other(top, own);
    top = fmaxf(own, other) * scale2;
    const bool up = top - m > SLACK;                        // (after none, any score is a new maximum)
    const float m2 = up ? top : m, f = up ? paged_exp2(m - m2) : 1.f;
    const float ref = paged_chunk_bias<DT>() - (m2 == -INFINITY ? 0.f : m2);
    m = m2;
    worst = fmaxf(worst, fabsf(ref));
    __builtin_amdgcn_s_setprio(1);                          // (the other wave of the SIMD has its arithmetic meanwhile)
    scores(kb, next);
    float sum = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      sc[e] = paged_exp2(__builtin_fmaf(sc[e], scale2, ref));
      sum += sc[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e >> 2][e & 3] = paged_pair<DT>(sc[2 * e], sc[2 * e + 1]);
    if constexpr (decltype(masked)::value) {
      if (vb) {
        if (odd) values(std::true_type{}, vb, before, tb);
        else values(std::false_type{}, vb, before, tb);
      }
    } else values(std::false_type{}, vb, before, tb);
    __builtin_amdgcn_s_setprio(0);
    asm volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(sum));   // (before the branch, beside the products, not where they are needed)
    if (__any(up)) {
      l *= f;
#pragma unroll
      for (int k = 0; k < CB; ++k) o[k] *= f;
    }
    l += sum;
  };

  // The tiles' order: those that not all columns see whole first (in front of a window's end, then the last tokens'), in a loop
  // of their own, so that the loop over the others holds nothing else.
  const int whole_from = max(from, (wg_lo + T - 1) & ~(T - 1)), whole_to = min(to, wg_hi & ~(T - 1));
  const int tiles = from < to ? (to - from + T - 1) / T : 0, whole = max(0, (whole_to - whole_from) / T), partial = tiles - whole;
  const int front = whole ? (whole_from - from) / T : tiles;
  auto tile_at = [&](int i) PAGED_INLINE { return i < front ? from + i * T : i < partial ? whole_to + (i - front) * T : whole_from + (i - partial) * T; };
  if (tid < 4) odd_tile[tid] = -1;
  __syncthreads();
  u32x4 p0[2] = {}, p1[2] = {};
  f16v s0, s1;
  if (tiles > 0) {
    int t0 = tile_at(0), t1 = tile_at(1), t2 = tile_at(2), before = 0;   // tiles i, i + 1, i + 2 (where there are such), i - 1
    pages(t0);
    load(t0, 0, 0);
    pages(t1);
    stage(t0, 0, 0);
    if (tiles > 1) {
      load(t1, 1, 1);
      pages(t2);
      stage(t1, 1, 1);
    }
    __syncthreads();
    int i = 0, k0 = 0, k1 = 1, k2 = 2;                      // buffers of keys of tiles i, i + 1, i + 2
    // a wave of no columns only stages
    if (c0 + wave * 32 >= cols) {
      for (; i < tiles; ++i) {
        if (i + 2 < tiles) {
          load(t2, k2, (i + 2) & 3);
          pages(tile_at(i + 3));
          stage(t2, k2, (i + 2) & 3);
        }
        __syncthreads();
        t2 = tile_at(i + 3);
        k2 = k2 == 2 ? 0 : k2 + 1;                          // (the buffer of tile i + 3 is tile i's)
      }
      return;
    }
    if (a.scale2 <= 0) {                                    // (scale2 is its magnitude, or 1)
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) q[j][e] = a.scale2 < 0 ? q[j][e] ^ 0x80008000u : paged_times_zero<DT>(q[j][e]);
    }
    scores(lk[0], s0);
    auto walk = [&](auto masked, int end) PAGED_INLINE {
      constexpr bool M = decltype(masked)::value;
      for (; i < end; ++i) {
        const int t3 = M ? tile_at(i + 3) : t2 + T;         // (M: the next may be elsewhere)
        const bool more = i + 2 < tiles;
        if (more) {
          load(t2, k2, (i + 2) & 3);
          pages(t3);
        }
        // (the keys of a tile that is not there give scores that nothing looks at)
        const bool ob = M && odd_tile[(i - 1) & 3] == before, oc = M && odd_tile[i & 3] == t0;
        step(masked, s0, s1, lk[k0] + 32 * PK, p0, p1, M && !i ? nullptr : lv[(i - 1) & 3] + 32 * PV, t0, before + 32, ob);
        if (more) stage(t2, k2, (i + 2) & 3);               // (nobody reads those buffers)
        step(masked, s1, s0, lk[k1], p1, p0, lv[i & 3], t0 + 32, t0, oc);
        __syncthreads();
        const int k = k0;
        k0 = k1;
        k1 = k2;
        k2 = k;
        before = t0;
        t0 = t1;
        t1 = t2;
        t2 = t3;
      }
    };
    // (the first tile, and the one after a partial one, may have values of a partial tile, or none, before them)
    walk(std::true_type{}, min(partial + 1, tiles));
    walk(std::false_type{}, tiles);
    const int t = tile_at(tiles - 1), vb = (tiles - 1) & 3;
    if (odd_tile[vb] == t) values(std::true_type{}, lv[vb] + 32 * PV, p1, t + 32);
    else values(std::false_type{}, lv[vb] + 32 * PV, p1, t + 32);
  }

  // A weight above is the power of one multiplication and addition, whose error against the rounded maximum grows with the maximum: from
  // 2^25 on fp16 weights would pass their type.  Columns that were beyond 2^20, which are rare, are taken anew: token after token from memory,
  // differences of scores that are rounded alike, weights in fp32.  (Asking for such a maximum in the loop takes
  // 1.5-2.4 % of every call; this way a prompt of 8192 tokens takes 24 ms if all its rows are such.)
  const bool far = worst > 0x1p20f && m != INFINITY;
  if (m == INFINITY) l = NAN;                               // (a score of infinity: infinity less infinity)
  if (__builtin_expect(__any(far), 0)) {
    if (far) {
      m = -INFINITY;
      l = 0;
#pragma unroll
      for (int k = 0; k < CB; ++k) o[k] = f16v{};
    }
#pragma unroll 1
    for (int t = from; t < to; ++t) {
      const int pg = table[t >> v.page_shift], slot = t & mask;
      const bool ok = (unsigned)pg < (unsigned)v.n_pages;
      const unsigned char* blk = pool + (ok ? pg : 0) * page_bytes;
      const unsigned char *kd = blk + slot * rb, *sd = blk + ((2 * rb) << v.page_shift) + slot * sb;
      const unsigned char *vd = kd + (rb << v.page_shift), *vsd = sd + (sb << v.page_shift);
      float x = 0;
#pragma unroll
      for (int j = 0; j < NS; ++j) {                        // this lane's half of the channels
        const unsigned char* at = kd + (16 * j + 8 * h) * BITS / 8;
        u32x4 kk;
        if constexpr (BITS == 16) kk = *(const u32x4*)at;
        else {
          u32x2 c = {0, 0};
          if constexpr (BITS == 8) c = *(const u32x2*)at;
          else c[0] = *(const uint32_t*)at;
          kk = paged_decode8<DT, BITS>(c, paged_scale(sd[j >> 1]));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x = __builtin_fmaf(paged_lo<DT>(kk[e]), paged_lo<DT>(q[j][e]), x);
          x = __builtin_fmaf(paged_hi<DT>(kk[e]), paged_hi<DT>(q[j][e]), x);
        }
      }
      float half;
      const float rest = paged_other(x, half);
      x = ok ? (half + rest) * scale2 : NAN;
      if (far && t >= lo && t < hi) {
        const float m2 = fmaxf(m, x), base = m2 == -INFINITY ? 0.f : m2, f = m2 == m ? 1.f : paged_exp2(m - m2);
        const float w = paged_exp2(paged_less(x, 1.f, base));
        m = m2;
        l = l * f + w;
#pragma unroll
        for (int k = 0; k < CB; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const unsigned char* at = vd + (32 * k + 8 * i + 4 * h) * BITS / 8;
            u32x2 vv;
            if constexpr (BITS == 16) vv = *(const u32x2*)at;
            else {
              const uint32_t c = BITS == 8 ? *(const uint32_t*)at : *(const unsigned short*)at;
              const float sc = paged_scale(vsd[k]);
              vv = u32x2{paged_decode2<DT, BITS, 0>(c, sc), paged_decode2<DT, BITS, 1>(c, sc)};
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              o[k][4 * i + 2 * e] = __builtin_fmaf(w, paged_lo<DT>(vv[e]), o[k][4 * i + 2 * e] * f);
              o[k][4 * i + 2 * e + 1] = __builtin_fmaf(w, paged_hi<DT>(vv[e]), o[k][4 * i + 2 * e + 1] * f);
            }
          }
      }
    }
    if (far) {
      constexpr float unit = DT ? 1.f : 64.f;               // 2^bias, as the other columns
      l = h == 0 ? l * unit : 0.f;                          // (the two lanes of a column are added below)
#pragma unroll
      for (int k = 0; k < CB; ++k) o[k] *= unit;
    }
  }
  float own;
  const float other = paged_other(l, own), sum = own + other;
  if (!mine) return;
  if (a.sp.splits == 1) {
    const float inv = sum == 0 ? 0.f : 1.f / sum;
#pragma unroll
    for (int k = 0; k < CB; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const u32x2 w = {paged_pair<DT>(o[k][4 * e] * inv, o[k][4 * e + 1] * inv), paged_pair<DT>(o[k][4 * e + 2] * inv, o[k][4 * e + 3] * inv)};
        *(u32x2*)(a.out + at * D + 32 * k + 8 * e + 4 * h) = w;
      }
    if (a.lse && h == 0) a.lse[at] = paged_lse(m, sum, paged_chunk_bias<DT>());
  } else {
    const int64_t u = (((int64_t)unit * v.Hkv + kvh) * COLS + (cc - c0)) * a.sp.splits + split;
#pragma unroll
    for (int k = 0; k < CB; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *(f4*)(a.sp.acc + u * D + 32 * k + 8 * e + 4 * h) = f4{o[k][4 * e], o[k][4 * e + 1], o[k][4 * e + 2], o[k][4 * e + 3]};
    if (h == 0) a.sp.ml[u] = make_float2(m, sum);
  }
}

// The splits of k_paged_chunk together.  A lane takes four channels of a column.
template <int D, int DT, int COLS>
__global__ __launch_bounds__(256) void k_paged_chunk_merge(PagedView v, PagedAsk a) {
  const int kvh = blockIdx.x % v.Hkv, unit = blockIdx.x / v.Hkv;
  int c0;
  const int b = paged_find_tile(v, a.few, COLS, unit, c0);
  if (b >= v.n_seqs) return;
  const PagedSeq s = paged_seq(v, b);
  const int cols = (s.last - s.first) * v.rep;
  if (s.bad) return;
  const int lo = paged_lo_of(a, s.base + c0 / v.rep) & ~(PAGED_TILE - 1);
  const int hi = paged_hi_of(a, s, s.base + (min(c0 + COLS, cols) - 1) / v.rep);
  const int n = max(1, (hi - lo + a.sp.chunk - 1) / a.sp.chunk);
  constexpr int LANES = D / 4, STEP = 256 / LANES;          // of a column; columns at a time
  const int ch = threadIdx.x % LANES * 4;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int c = (blockIdx.y * 2 + r) * STEP + threadIdx.x / LANES;
    if (c0 + c >= cols) return;
    const int64_t u0 = (((int64_t)unit * v.Hkv + kvh) * COLS + c) * a.sp.splits;
    constexpr int W = 8;                                    // splits asked for together
    float mm = -INFINITY, sum = 0;
    f4 acc = {0, 0, 0, 0};
    for (int i0 = 0; i0 < n; i0 += W) {
      float2 ml[W];
      f4 x[W];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const int64_t u = u0 + min(i0 + i, n - 1);
        ml[i] = a.sp.ml[u];
        x[i] = *(const f4*)(a.sp.acc + u * D + ch);
      }
      float top = mm;
#pragma unroll
      for (int i = 0; i < W; ++i) top = fmaxf(top, ml[i].x);
      const float ref = top == -INFINITY ? 0.f : top, f0 = paged_exp2(mm - ref);
      sum *= f0;
      acc *= f0;
#pragma unroll
      for (int i = 0; i < W; ++i)
        if (i0 + i < n) {
          const float f = paged_exp2(ml[i].x - ref);
          sum += f * ml[i].y;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] += f * x[i][e];
        }
      mm = top;
    }
    const int64_t at = (int64_t)(s.first + (c0 + c) / v.rep) * v.Hq + kvh * v.rep + (c0 + c) % v.rep;
    const float inv = sum == 0 ? 0.f : 1.f / sum;
    *(u32x2*)(a.out + at * D + ch) = u32x2{paged_pair<DT>(acc[0] * inv, acc[1] * inv), paged_pair<DT>(acc[2] * inv, acc[3] * inv)};
    if (a.lse && ch == 0) a.lse[at] = paged_lse(mm, sum, paged_chunk_bias<DT>());
  }
}

// ---- host side ---------------------------------------------------------------------------------

#define RKV_PAGED_CUS 256             // compute units that a launch should fill
// (8 sequences of 4096 tokens, 8 KV heads of 128, 8 bits: 20 columns 23.7 us in k_paged_few and 34.4 in k_paged_chunk, 32 columns 25.6 and 35.0;
// more than two blocks of columns do not fit k_paged_few's registers: 36 columns take 36.0)
#define RKV_PAGED_FEW 32              // columns (rows times rep) of a sequence that k_paged_few takes ...
#define RKV_PAGED_FEW_MIXED 16        // ... where others go to k_paged_chunk: single tokens, half the registers
#define RKV_PAGED_SPLITS 256          // most splits of a sequence
#define RKV_PAGED_COLS 256            // columns of a workgroup of k_paged_chunk

// Splits of sequences of max_len tokens whose work units (`units` of them) should become `want`: a multiple of `step` tokens each.
// One span of up to `whole` tokens is not cut: the launch that joins splits takes longer than what they save.
static void paged_cut(const PagedView& v, int window, int tile, int64_t units, int64_t want, int step, int whole, int rows, PagedSplit* sp) {
  int64_t span = v.max_len;
  if (window && span > (int64_t)window + rows + tile - 1) span = (int64_t)window + rows + tile - 1;
  int64_t n = span <= whole ? 1 : (want + units - 1) / units;
  if (n > RKV_PAGED_SPLITS) n = RKV_PAGED_SPLITS;
  const int64_t c = ((span + n - 1) / n + step - 1) / step * step;
  sp->chunk = (int)c;
  sp->splits = (int)((span + c - 1) / c);
}
// Bytes of partial results, for any window (a shorter span may be cut into more splits than a longer one, but never into
// more than are wanted)
static size_t paged_cut_bytes(const PagedView& v, int64_t units, int64_t want, int step, int whole, int cols, int D) {
  if (v.max_len <= whole) return 0;
  int64_t n = (want + units - 1) / units, cut = ((int64_t)v.max_len + step - 1) / step;
  if (n > RKV_PAGED_SPLITS) n = RKV_PAGED_SPLITS;
  if (n > cut) n = cut;
  return n > 1 ? (size_t)units * cols * n * (D + 2) * 4 : 0;
}

static bool has_chunk(const PagedView& v) { return (int64_t)v.max_new * v.rep > RKV_PAGED_FEW; }
static bool has_few(const PagedView& v) { return v.n_seqs > 1 || !has_chunk(v); }

// k_paged_few: a unit is a (sequence, KV head); splits of at least 128 tokens (32 for each wave).  Two workgroups for each
// compute unit have enough bytes in flight, and four where a row is 64 bytes or less and the spans are long (32768 tokens, 32 heads of 128,
// 4 bits: 30.4 us with four, 35.6 with two; 8 x 4096 tokens, 8 heads, 8 bits: 19.8 with two, 24.2 with four).  Where the whole batch is short two are
// better with narrow rows as well (2 x 16384 tokens, 8 heads: 16.9 against 18.8 with 4 bits, 13.7 against 15.8 with heads of 64), which the rule does not know.
// One span is not cut up to 512 tokens (one token, 32 heads of 128 in 16 bits: 8.4 us whole, 12.6 cut; at 513-640 tokens 9.8 and 12.5, at 768 11.0
// and 12.6, at 1024 13.8 and 12.6: the crossing is near 900 for this shape).  What a window leaves is counted for RKV_PAGED_FEW rows, also where there is one.
// The number of splits follows the number of sequences and the longest of them, as the host knows no other lengths: one sequence of 32768 tokens among
// seven of 512 takes 58 us, among 63 of them 402, because nothing is cut there.
static int64_t few_units(const PagedView& v) { return (int64_t)v.n_seqs * v.Hkv; }
static int few_cols(const PagedView& v) { return (int64_t)v.max_new * v.rep <= 16 || has_chunk(v) ? 16 : 32; }
static int64_t few_want(int D, int bits) { return (D * bits <= 512 ? 4 : 2) * RKV_PAGED_CUS; }
#define FEW_STEP 128
#define FEW_WHOLE 512
// k_paged_chunk: a unit is a tile of columns and a KV head; a workgroup for each compute unit, splits of at least 512 tokens
static int64_t chunk_units(const PagedView& v) {
  // Every sequence of more than RKV_PAGED_FEW_MIXED columns, and one alone, may have a tile that is not full.  The host cannot tell those from
  // single tokens, so that a chunk beside many of them is cut less than it could be: 1021 rows over 4090 tokens, 32 heads on 8, beside 14 single tokens
  // 113 us in two splits, beside 15 in one 145.  (Over 1100 tokens one split is the better: 57 against 68.)
  const int64_t cols = (int64_t)v.n_rows * v.rep, most = cols / RKV_PAGED_FEW_MIXED, seqs = v.n_seqs < most ? v.n_seqs : most;
  return (cols / RKV_PAGED_COLS + seqs) * v.Hkv;
}
bool rkv_paged_attention_fits(const PagedView& v) { return !has_chunk(v) || chunk_units(v) * 512 < RKV_PAGED_THREADS; }   // (k_paged_few's is Hkv x 256 x n_seqs)
#define CHUNK_WANT RKV_PAGED_CUS
#define CHUNK_STEP 512
// work space: k_paged_few's partial results, then k_paged_chunk's
static size_t few_bytes(const PagedView& v, int D, int bits) {
  const size_t n = has_few(v) ? paged_cut_bytes(v, few_units(v), few_want(D, bits), FEW_STEP, FEW_WHOLE, few_cols(v), D) : 0;
  return (n + 255) & ~(size_t)255;
}
size_t rkv_paged_attention_scratch(const PagedView& v, int D, int bits) {
  return few_bytes(v, D, bits) + (has_chunk(v) ? paged_cut_bytes(v, chunk_units(v), CHUNK_WANT, CHUNK_STEP, CHUNK_STEP, RKV_PAGED_COLS, D) : 0);
}

template <int D, int BITS, int DT, int NB>
static void launch_few(const PagedView& v, PagedAsk a, void* scratch, hipStream_t s) {
  paged_cut(v, a.window, 32, few_units(v), few_want(D, BITS), FEW_STEP, FEW_WHOLE, RKV_PAGED_FEW, &a.sp);
  a.sp.acc = (float*)scratch;
  a.sp.ml = (float2*)(a.sp.acc + few_units(v) * (16 * NB) * a.sp.splits * D);
  k_paged_few<D, BITS, DT, NB><<<dim3(v.Hkv, a.sp.splits, v.n_seqs), 256, 0, s>>>(v, a);
  if (a.sp.splits > 1) k_paged_merge<D, DT, NB><<<dim3(4 * NB, v.Hkv, v.n_seqs), 256, 0, s>>>(v, a);
}

template <int D, int BITS, int DT>
static void launch(const PagedView& v, PagedAsk a, void* scratch, hipStream_t s) {
  a.mixed = has_chunk(v);
  a.few = a.mixed ? RKV_PAGED_FEW_MIXED : RKV_PAGED_FEW;
  if (has_few(v)) {
    if (few_cols(v) == 16) launch_few<D, BITS, DT, 1>(v, a, scratch, s);
    else launch_few<D, BITS, DT, 2>(v, a, scratch, s);
  }
  if (a.mixed) {
    if (!has_few(v)) a.few = 0;
    const int64_t units = chunk_units(v);
    // (rows of a unit; without `causal` its first row sees all behind it)
    const int rows = a.causal && v.max_new > RKV_PAGED_COLS ? RKV_PAGED_COLS : v.max_new;
    paged_cut(v, a.window, PAGED_TILE, units, CHUNK_WANT, CHUNK_STEP, CHUNK_STEP, rows, &a.sp);
    a.sp.acc = (float*)((char*)scratch + few_bytes(v, D, BITS));
    a.sp.ml = (float2*)(a.sp.acc + units * RKV_PAGED_COLS * a.sp.splits * D);
    k_paged_chunk<D, BITS, DT, 8><<<dim3((unsigned)units, a.sp.splits), 512, 0, s>>>(v, a);
    if (a.sp.splits > 1) k_paged_chunk_merge<D, DT, RKV_PAGED_COLS><<<dim3((unsigned)units, RKV_PAGED_COLS * D / 2048), 256, 0, s>>>(v, a);
  }
}

int rkv_launch_paged_attention(const PagedView& v, int D, int bits, int dtype, const void* q, int64_t qs, int causal, int window, float scale,
                               void* out, float* lse, void* scratch, hipStream_t s) {
  PagedAsk a{};
  a.q = (const unsigned short*)q;
  a.qs = qs;
  a.out = (unsigned short*)out;
  a.lse = lse;
  a.scale2 = (float)((double)scale * 1.4426950408889634);
  a.causal = causal;
  a.window = window < 1 << 30 ? window : 1 << 30;            // (no sequence is longer)
#define GO(D_, B_) (dtype ? launch<D_, B_, 1>(v, a, scratch, s) : launch<D_, B_, 0>(v, a, scratch, s))
  if (D == 64) { if (bits == 16) GO(64, 16); else if (bits == 8) GO(64, 8); else GO(64, 4); }
  else { if (bits == 16) GO(128, 16); else if (bits == 8) GO(128, 8); else GO(128, 4); }
#undef GO
  RKV_HIP_CHECK(hipGetLastError());
  return RKV_OK;
}
