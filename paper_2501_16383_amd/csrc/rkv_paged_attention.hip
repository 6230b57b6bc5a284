// Attention of packed rows over the cache in pages.
//
// Per query head h of KV head g = h / rep: out = sum_t w_t v_t, w = softmax(scale q.k_t).  The rows of a sequence that
// read one KV head - its new tokens times the rep query heads - are the columns of two matrix products,
//   S^T[token][column] = K . Q^T          O^T[channel][column] = V^T . P^T,
// so that a lane of the result owns one column: the running maximum and sum of its softmax are plain registers, and
// the four (eight) weights a lane gets from the first product are, in their order, an operand of the second.
// (Which token is which index of the sum is free as long as both operands agree.)  Weights are powers of two of
// scores in fp32; the sum of weights is taken in fp32 from unrounded weights.
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

#define LDS_AS __attribute__((address_space(3)))
// Four rows of sixteen 16-bit elements, transposed: lane i of a row of 16 gives the address of row i >> 2, elements
// 4 (i & 3) .., and gets element i of the four rows.
__device__ __forceinline__ u32x2 paged_transposed(const unsigned short* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s4*)p));
}

// Is the element in the low half an infinity or NaN?
template <int DT> __device__ __forceinline__ bool paged_odd(uint32_t x) {
  constexpr uint32_t ex = DT ? 0x7f80 : 0x7c00;
  return (x & ex) == ex;
}

__device__ __forceinline__ float paged_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Weights are held times a power of two that the division by their sum takes out again: in fp16 the largest is
// 2^14, so that one of 2^-28 of it still is a normal number (as a subnormal of 2^-25 it would be off by up to its own size).
template <int DT> __device__ constexpr float paged_bias() { return DT ? 0.f : 14.f; }

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

// What a call asks for beside the batch
struct PagedAsk {
  const unsigned short* q;
  int64_t qs;
  unsigned short* out;
  float* lse;
  float* part;                        // partial results of splits: [row][head][split][D + 2]
  float scale2;                       // scale * log2(e)
  int causal, window;
  int few;                            // rows times rep up to which a sequence goes to k_paged_few (0: no sequence does)
  int chunk, splits;                  // of k_paged_few: tokens of a split, most splits of a sequence
};

// Tokens that the row at position p sees: lo .. hi - 1
__device__ __forceinline__ int paged_hi_of(const PagedAsk& a, const PagedSeq& s, int p) { return a.causal ? min(max(p + 1, 0), s.len) : s.len; }
__device__ __forceinline__ int paged_lo_of(const PagedAsk& a, int p) { return a.window ? max(0, p - a.window + 1) : 0; }

// NaN for every row of a bad sequence that reads this KV head
template <int D, int DT> __device__ __forceinline__ void paged_bad_rows(const PagedView& v, const PagedAsk& a, int first, int last, int kvh) {
  const int n = (last - first) * v.rep;
  for (int i = threadIdx.x; i < n * D; i += blockDim.x) {
    const int c = i / D;
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
// the wave's own LDS as 16-bit rows and come back transposed.  The next tile's bytes are in flight while
// one is computed.
template <int D, int BITS> struct FewTile {
  static constexpr int KL = D * BITS / 8 / 4 / 16;          // 16-byte loads of a quarter row of keys (0: one of 8 bytes)
  static constexpr int VP = D * BITS / 8 / 16;              // 16-byte parts of a row of values
  static constexpr int VL = 32 * VP / 64;                   // loads of a lane for 32 tokens
  u32x4 k[2][KL ? KL : 1], v[VL];
  uint32_t ks[2], vs[VL];
};

template <int D, int BITS, int DT, int NB>
__global__ __launch_bounds__(256) void k_paged_few(PagedView v, PagedAsk a) {
  using Tile = FewTile<D, BITS>;
  constexpr int rb = paged_row<D, BITS>(), sb = paged_srow<D, BITS>();
  constexpr int PITCH = D + 16;                             // 16-bit elements between two tokens' values in LDS
  constexpr int CB = D / 16, NK = D / 32;
  constexpr int OP = D + 4;                                 // floats between two columns when waves meet
  __shared__ __align__(16) unsigned short lds[4 * 32 * PITCH];
  __shared__ float meet[2][4][16];
  static_assert(4 * 16 * OP * 4 <= 4 * 32 * PITCH * 2, "the waves' results fit the values' rows");

  const int split = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
  const PagedSeq s = paged_seq(v, b);
  const int rows = s.last - s.first, cols = rows * v.rep;
  if (rows == 0) return;
  if (cols > a.few && v.max_new * v.rep > a.few) return;    // the other kernel's
  if (s.bad) {
    if (split == 0) paged_bad_rows<D, DT>(v, a, s.first, s.last, kvh);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;

  // tokens that some row sees, and this split's share
  const int all_lo = paged_lo_of(a, s.base), all_hi = paged_hi_of(a, s, s.base + rows - 1);
  const int from = (all_lo & ~31) + split * a.chunk, to = min(all_hi, from + a.chunk);
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
  float m[NB], l[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    m[i] = -INFINITY;
    l[i] = 0;
#pragma unroll
    for (int c = 0; c < CB; ++c) o[i][c] = f4{0, 0, 0, 0};
  }
  unsigned short* vl = lds + wave * 32 * PITCH;
  const int mask = (1 << v.page_shift) - 1;
  const int64_t bb = paged_block<D, BITS>(v.page_shift);
  const int last_page = (s.len - 1) >> v.page_shift;        // (len > 0 where there is a tile at all)

  auto pages = [&](int t, int* p) {
#pragma unroll
    for (int i = 0; i < 2; ++i) p[i] = v.table[(int64_t)b * v.max_pages + min((t + 16 * i) >> v.page_shift, last_page)];
  };
  auto load = [&](int t, const int* p, Tile& x) {
    const unsigned char* blk[2];
    bool ok[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ok[i] = (unsigned)p[i] < (unsigned)v.n_pages;
      blk[i] = v.pool + ((int64_t)(ok[i] ? p[i] : 0) * v.Hkv + kvh) * bb;
      const int slot = (t + 16 * i) & mask;
      const unsigned char* kp = blk[i] + (slot + n) * rb + (BITS == 16 ? 16 * g : g * (rb / 4));
      if constexpr (Tile::KL == 0) {
        const u32x2 w = *(const u32x2*)kp;
        x.k[i][0] = u32x4{w[0], w[1], 0, 0};
      } else {
#pragma unroll
        for (int j = 0; j < Tile::KL; ++j) x.k[i][j] = *(const u32x4*)(kp + (BITS == 16 ? 64 : 16) * j);
      }
      if constexpr (BITS < 16) {
        x.ks[i] = blk[i][((2 * rb) << v.page_shift) + (slot + n) * sb + (D == 128 ? g : g >> 1)];
        if (!ok[i]) x.ks[i] = 255;
      } else if (!ok[i]) {
#pragma unroll
        for (int j = 0; j < Tile::KL; ++j) x.k[i][j] = u32x4{~0u, ~0u, ~0u, ~0u};
      }
    }
#pragma unroll
    for (int r = 0; r < Tile::VL; ++r) {
      const int ci = r * 64 + lane, tok = ci / Tile::VP, part = ci % Tile::VP;
      const int gi = 64 / Tile::VP <= 16 ? (r * 64 / Tile::VP) / 16 : tok >> 4;   // which sixteen tokens
      const unsigned char* base = 64 / Tile::VP <= 16 ? blk[gi] : gi ? blk[1] : blk[0];
      const bool fine = 64 / Tile::VP <= 16 ? ok[gi] : gi ? ok[1] : ok[0];
      const int slot = ((t + 16 * gi) & mask) + (tok & 15);
      const u32x4 z = {0, 0, 0, 0};
      // a value row that no row sees, or of no page, counts as zeros: weight 0 times whatever lies there must be 0
      const bool seen = fine && t + tok < all_hi && t + tok >= all_lo;
      x.v[r] = seen ? *(const u32x4*)(base + ((int64_t)rb << v.page_shift) + slot * rb + part * 16) : z;
      if constexpr (BITS < 16) x.vs[r] = seen ? base[((2 * rb + sb) << v.page_shift) + slot * sb + part * (128 / BITS) / 32] : 127;
    }
  };
  auto compute = [&](int t, const Tile& x) {
    // values to LDS as 16-bit rows
    bool odd = false;                                       // holds infinities or NaN
#pragma unroll
    for (int r = 0; r < Tile::VL; ++r) {
      const int ci = r * 64 + lane, tok = ci / Tile::VP, part = ci % Tile::VP;
      u32x4* d = (u32x4*)(vl + tok * PITCH + part * (128 / BITS));
      if constexpr (BITS == 16) {
        d[0] = x.v[r];
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= paged_odd<DT>(x.v[r][e]) || paged_odd<DT>(x.v[r][e] >> 16);
      } else {
        const float sc = paged_scale(x.vs[r]);
        odd |= x.vs[r] == 255;
#pragma unroll
        for (int e = 0; e < 16 / BITS; ++e) {
          const u32x2 w = {x.v[r][BITS == 8 ? 2 * e : e], BITS == 8 ? x.v[r][2 * e + 1] : 0};
          d[e] = paged_decode8<DT, BITS>(w, sc);
        }
      }
    }
    // scores
    f4 sc[NB][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u32x4 kk[NK];
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        if constexpr (BITS == 16) kk[j] = x.k[i][j];
        else {
          const int w = j * (BITS / 4);                     // dword of the lane's codes
          const u32x2 c = {x.k[i][w / 4][w % 4], BITS == 8 ? x.k[i][w / 4][(w % 4) + 1 & 3] : 0};
          kk[j] = paged_decode8<DT, BITS>(c, paged_scale(x.ks[i]));
        }
      }
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        sc[c][i] = f4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < NK; ++j) sc[c][i] = paged_mfma16<DT>(kk[j], q[c][j], sc[c][i]);
      }
    }
    const bool whole = t >= full_lo && t + 32 <= full_hi;   // every row sees every token
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
      if (__any(top > m[c])) {
        const float m2 = fmaxf(m[c], top), f = m2 == m[c] ? 1.f : paged_exp2(m[c] - m2);
        m[c] = m2;
        l[c] *= f;
#pragma unroll
        for (int k = 0; k < CB; ++k) o[c][k] *= f;
      }
      const float ref = (m[c] == -INFINITY ? 0.f : m[c]) - paged_bias<DT>();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = paged_exp2(w[e] - ref);
        l[c] += w[e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) p[c][e] = paged_pair<DT>(w[2 * e], w[2 * e + 1]);
    }
    wave_lds_fence();
    if (!whole && rows > 1 && __any(odd)) {
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
#pragma unroll
          for (int k = 0; k < CB; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t bits = vl[tok * PITCH + 16 * k + 4 * g + e];
              if (paged_odd<DT>(bits) && pf != 0) o[c][k][e] += pf * paged_lo<DT>(bits);
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

  {
    const int first = from + 32 * wave;
    int pg[2], pn[2];
    Tile x, y;
    if (first < to) {
      pages(first, pg);
      load(first, pg, x);
      if (first + 128 < to) pages(first + 128, pn);
    }
    for (int t = first; t < to; t += 256) {
      if (t + 128 < to) {
        load(t + 128, pn, y);
        if (t + 256 < to) pages(t + 256, pg);
      }
      compute(t, x);
      if (t + 128 >= to) break;
      if (t + 256 < to) {
        load(t + 256, pg, x);
        if (t + 384 < to) pages(t + 384, pn);
      }
      compute(t + 128, y);
    }
  }

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
      if (a.splits == 1) {
        a.out[at * D + ch] = (unsigned short)paged_pair<DT>(sum == 0 ? 0.f : acc / sum, 0.f);
        if (a.lse && ch == 0) a.lse[at] = sum == 0 ? -INFINITY : (mm + __log2f(sum) - paged_bias<DT>()) * 0.69314718055994531f;
      } else {
        float* part = a.part + (at * a.splits + split) * (D + 2);
        part[ch] = acc;
        if (ch == 0) {
          part[D] = mm;
          part[D + 1] = sum;
        }
      }
    }
  }
}

// The splits of a row and head together: a wave each.
template <int D, int DT>
__global__ __launch_bounds__(256) void k_paged_merge(PagedView v, PagedAsk a) {
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= (int64_t)v.n_rows * v.Hq) return;
  const int row = __builtin_amdgcn_readfirstlane((int)(at / v.Hq));
  const int b = paged_owner(v, row);
  if (b >= v.n_seqs) return;
  const PagedSeq s = paged_seq(v, b);
  const int rows = s.last - s.first;
  if (row < s.first || row >= s.last || s.bad || rows * v.rep > a.few) return;
  const int all_lo = paged_lo_of(a, s.base), all_hi = paged_hi_of(a, s, s.base + rows - 1);
  const int n = max(1, (all_hi - (all_lo & ~31) + a.chunk - 1) / a.chunk);
  const float* part = a.part + at * a.splits * (D + 2);
  float mm = -INFINITY;
  for (int i = lane; i < n; i += 64) mm = fmaxf(mm, part[(int64_t)i * (D + 2) + D]);
  for (int o = 32; o; o >>= 1) mm = fmaxf(mm, __shfl_xor(mm, o));
  const float ref = mm == -INFINITY ? 0.f : mm;
  float sum = 0, acc[D / 64] = {};
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const float* p = part + (int64_t)i * (D + 2);
    const float f = paged_exp2(p[D] - ref);
    sum += f * p[D + 1];
#pragma unroll
    for (int j = 0; j < D / 64; ++j) acc[j] += f * p[lane + 64 * j];
  }
#pragma unroll
  for (int j = 0; j < D / 64; ++j) a.out[at * D + lane + 64 * j] = (unsigned short)paged_pair<DT>(sum == 0 ? 0.f : acc[j] / sum, 0.f);
  if (a.lse && lane == 0) a.lse[at] = sum == 0 ? -INFINITY : (mm + __log2f(sum) - paged_bias<DT>()) * 0.69314718055994531f;
}

// One wave per (row, query head): lanes hold channels, tokens one after the other with the running maximum and
// sum of the softmax.
template <int D, int BITS, int DT>
__global__ __launch_bounds__(64) void k_paged_plain(PagedView v, const unsigned short* __restrict__ q, int64_t qs, int causal, int window,
                                                    float scale, unsigned short* __restrict__ out, float* __restrict__ lse, int few) {
  constexpr int N = D / 64;                                      // channels of a lane
  const int lane = threadIdx.x, row = blockIdx.x / v.Hq, h = blockIdx.x % v.Hq;
  const int b = paged_owner(v, row);
  if (b >= v.n_seqs) return;
  const PagedSeq s = paged_seq(v, b);
  if (row < s.first || row >= s.last || (s.last - s.first) * v.rep <= few) return;
  const int pos = s.base + (row - s.first);
  const int hi = causal ? min(pos + 1, s.len) : s.len;
  const int lo = window ? max(0, pos - window + 1) : 0;
  constexpr int rb = paged_row<D, BITS>(), sb = paged_srow<D, BITS>();
  auto element = [&](const unsigned char* codes, const unsigned char* scales, int c) {
    if constexpr (BITS == 16) return paged_lo<DT>(((const unsigned short*)codes)[c]);
    else {
      const uint32_t byte = scales[c / 32];
      if (byte == 255) return __uint_as_float(0x7fc00000);
      if constexpr (BITS == 8) return paged_lo<DT>(paged_decode2<DT, 8, 0>(codes[c], paged_scale(byte)));
      else return paged_lo<DT>(paged_decode2<DT, 4, 0>(codes[c / 2] >> (4 * (c & 1)), paged_scale(byte)));
    }
  };
  float x[N], acc[N], m = -INFINITY, l = 0;
  for (int j = 0; j < N; ++j) {
    x[j] = paged_lo<DT>(q[row * qs + h * D + lane + 64 * j]);
    acc[j] = 0;
  }
  for (int t = lo; t < hi; ++t) {
    const int page = paged_page(v, b, t);
    const unsigned char* blk = v.pool + ((int64_t)max(page, 0) * v.Hkv + h / v.rep) * paged_block<D, BITS>(v.page_shift);
    const int slot = t & ((1 << v.page_shift) - 1);
    const unsigned char* sc = blk + ((2 * rb) << v.page_shift) + slot * sb;
    float d = 0;
    for (int j = 0; j < N; ++j) d += x[j] * element(blk + slot * rb, sc, lane + 64 * j);
    for (int o = 32; o; o >>= 1) d += __shfl_xor(d, o);
    d = page < 0 ? __uint_as_float(0x7fc00000) : d * scale;
    const float m2 = fmaxf(m, d), ref = m2 == -INFINITY ? 0 : m2;
    const float a = expf(m - ref), p = expf(d - ref);
    l = l * a + p;
    for (int j = 0; j < N; ++j) acc[j] = acc[j] * a + (p > 0 || p != p ? p * element(blk + (rb << v.page_shift) + slot * rb, sc + (sb << v.page_shift), lane + 64 * j) : 0);
    m = m2;
  }
  const float nan = __uint_as_float(0x7fc00000);
  for (int j = 0; j < N; ++j) {
    const float o = s.bad ? nan : l == 0 ? 0 : acc[j] / l;
    out[((int64_t)row * v.Hq + h) * D + lane + 64 * j] = (unsigned short)paged_pair<DT>(o, 0);
  }
  if (lse && lane == 0) lse[(int64_t)row * v.Hq + h] = s.bad ? nan : l == 0 ? -INFINITY : m + logf(l);
}

// ---- host side ---------------------------------------------------------------------------------

#define RKV_PAGED_CUS 256             // compute units that a launch should fill
#define RKV_PAGED_FEW 32              // columns (rows times rep) of a sequence that k_paged_few takes
#define RKV_PAGED_SPLITS 256          // most splits of a sequence

// Splits of k_paged_few: as many tokens each (a multiple of 128: 32 for each wave) as let the workgroups of sequences
// of max_len tokens fill the device twice.
static void few_splits(const PagedView& v, int window, int* chunk, int* splits) {
  int64_t span = v.max_len;                                 // (the rows are a sequence's last tokens, with or without `causal`)
  if (window && span > (int64_t)window + v.max_new + 31) span = (int64_t)window + v.max_new + 31;
  const int64_t pairs = (int64_t)v.n_seqs * v.Hkv, want = (2 * RKV_PAGED_CUS + pairs - 1) / pairs;
  int64_t c = ((span + want - 1) / want + 127) / 128 * 128;
  const int64_t least = ((span + RKV_PAGED_SPLITS - 1) / RKV_PAGED_SPLITS + 127) / 128 * 128;
  if (c < least) c = least;
  *chunk = (int)c;
  *splits = (int)((span + c - 1) / c);
}

// (for any window: a shorter span may be cut into more splits, but not into more than are wanted)
size_t rkv_paged_attention_scratch(const PagedView& v, int D) {
  const int64_t pairs = (int64_t)v.n_seqs * v.Hkv, want = (2 * RKV_PAGED_CUS + pairs - 1) / pairs, cut = ((int64_t)v.max_len + 127) / 128;
  int64_t splits = want < cut ? want : cut;
  if (splits > RKV_PAGED_SPLITS) splits = RKV_PAGED_SPLITS;
  return splits > 1 ? (size_t)v.n_rows * v.Hq * splits * (D + 2) * 4 : 0;
}

template <int D, int BITS, int DT>
static void launch(const PagedView& v, PagedAsk a, hipStream_t s) {
  few_splits(v, a.window, &a.chunk, &a.splits);
  a.few = RKV_PAGED_FEW;
  const dim3 grid(a.splits, v.Hkv, v.n_seqs);
  if (v.max_new * v.rep <= 16) k_paged_few<D, BITS, DT, 1><<<grid, 256, 0, s>>>(v, a);
  else k_paged_few<D, BITS, DT, 2><<<grid, 256, 0, s>>>(v, a);
  if (v.max_new * v.rep > RKV_PAGED_FEW)
    k_paged_plain<D, BITS, DT><<<dim3(v.n_rows * v.Hq), 64, 0, s>>>(v, a.q, a.qs, a.causal, a.window, a.scale2 / 1.4426950408889634f, a.out, a.lse, a.few);
  if (a.splits > 1) k_paged_merge<D, DT><<<dim3((unsigned)(((int64_t)v.n_rows * v.Hq + 3) / 4)), 256, 0, s>>>(v, a);
}

int rkv_launch_paged_attention(const PagedView& v, int D, int bits, int dtype, const void* q, int64_t qs, int causal, int window, float scale,
                               void* out, float* lse, void* scratch, hipStream_t s) {
  PagedAsk a{};
  a.q = (const unsigned short*)q;
  a.qs = qs;
  a.out = (unsigned short*)out;
  a.lse = lse;
  a.part = (float*)scratch;
  a.scale2 = (float)((double)scale * 1.4426950408889634);
  a.causal = causal;
  a.window = window < 1 << 30 ? window : 1 << 30;            // (no sequence is longer)
#define GO(D_, B_) (dtype ? launch<D_, B_, 1>(v, a, s) : launch<D_, B_, 0>(v, a, s))
  if (D == 64) { if (bits == 16) GO(64, 16); else if (bits == 8) GO(64, 8); else GO(64, 4); }
  else { if (bits == 16) GO(128, 16); else if (bits == 8) GO(128, 8); else GO(128, 4); }
#undef GO
  RKV_HIP_CHECK(hipGetLastError());
  return RKV_OK;
}
