// What the kernels of the paged cache share: the batch's description as they see it, the pool's layout, and
// the conversion of stored codes.
#pragma once
#include "rkv_internal.h"

#define RKV_PAGED_BLOCK 32            // channels that share a scale
#define RKV_PAGED_THREADS (1ll << 32)  // threads that a launch has not, in each direction of its grid

struct PagedView {
  unsigned char* pool;
  const int* table;                   // [n_seqs][max_pages]
  const int* row_start;               // [n_seqs + 1]
  const int* lengths;                 // [n_seqs]
  int n_seqs, max_pages, n_rows, max_new, max_len;
  int Hq, Hkv, rep;
  int page_shift, n_pages;            // a page holds 1 << page_shift tokens
};

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// DT: 0 fp16, 1 bf16.  Pairs of elements travel as one dword.
template <int DT> __device__ __forceinline__ float paged_lo(uint32_t x) {
  return DT ? __uint_as_float(x << 16) : (float)__builtin_bit_cast(h2, x)[0];
}
template <int DT> __device__ __forceinline__ float paged_hi(uint32_t x) {
  return DT ? __uint_as_float(x & 0xffff0000u) : (float)__builtin_bit_cast(h2, x)[1];
}
template <int DT> __device__ __forceinline__ uint32_t paged_pair(float a, float b) {   // to nearest, ties to even
  if constexpr (DT) {
    const b2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
  } else {
    const h2 r = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, r);
  }
}

// Bytes of one token's codes / scales, and of the block that a page keeps for a KV head
template <int D, int BITS> __host__ __device__ constexpr int paged_row() { return D * BITS / 8; }
template <int D, int BITS> __host__ __device__ constexpr int paged_srow() { return BITS < 16 ? D / RKV_PAGED_BLOCK : 0; }
template <int D, int BITS> __host__ __device__ inline int64_t paged_block(int page_shift) {
  return (int64_t)(2 * (paged_row<D, BITS>() + paged_srow<D, BITS>())) << page_shift;
}

// Two stored codes (the low 16 bits of w with 8 bits, byte SEL with 4) to a pair of the cache's type, times
// the block's scale: exact, by the choice of the scales.  A scale of infinity (byte 255) gives NaN.
template <int DT, int BITS, int SEL> __device__ __forceinline__ uint32_t paged_decode2(uint32_t w, float scale) {
  if constexpr (BITS == 8 && DT) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, SEL));
  else if constexpr (BITS == 8) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, SEL));
  else if constexpr (DT) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, SEL));
}

__device__ __forceinline__ float paged_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight consecutive codes (two dwords of 8 bits, one of 4) to four pairs
template <int DT, int BITS> __device__ __forceinline__ u32x4 paged_decode8(u32x2 w, float scale) {
  u32x4 r;
  if constexpr (BITS == 8) {
    r[0] = paged_decode2<DT, 8, 0>(w[0], scale);
    r[1] = paged_decode2<DT, 8, 1>(w[0], scale);
    r[2] = paged_decode2<DT, 8, 0>(w[1], scale);
    r[3] = paged_decode2<DT, 8, 1>(w[1], scale);
  } else {
    r[0] = paged_decode2<DT, 4, 0>(w[0], scale);
    r[1] = paged_decode2<DT, 4, 1>(w[0], scale);
    r[2] = paged_decode2<DT, 4, 2>(w[0], scale);
    r[3] = paged_decode2<DT, 4, 3>(w[0], scale);
  }
  return r;
}

// A sequence's rows and tokens, made safe: whatever the arrays hold, first .. last are rows of the tensors
// and 0 <= len <= max_len.
struct PagedSeq {
  int first, last;                    // its rows are first .. last - 1
  int len;                            // its tokens (0 if bad)
  int base;                           // position of row `first`
  bool bad;                           // more rows than max_new, or a length outside 0 .. max_len
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedView& v, int b) {
  PagedSeq s;
  const int f = v.row_start[b], l = v.row_start[b + 1], n = v.lengths[b];
  s.first = min(max(f, 0), v.n_rows);
  s.last = min(max(l, s.first), v.n_rows);
  s.bad = n < 0 || n > v.max_len || s.last - s.first > v.max_new;
  s.len = s.bad ? 0 : n;
  s.base = s.len - (s.last - s.first);
  return s;
}

// The sequence that owns a row: the first whose rows end behind it (n_seqs if none does).  The whole wave
// asks for the same row; 64 ends are compared at a time.
__device__ __forceinline__ int paged_owner(const PagedView& v, int row) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < v.n_seqs; b0 += 64) {
    const bool behind = b0 + lane < v.n_seqs && v.row_start[b0 + lane + 1] > row;
    const uint64_t m = __ballot(behind);
    if (m) return b0 + __builtin_ctzll(m);
  }
  return v.n_seqs;
}

// The page of token t of sequence b, or -1 if there is none in the pool (t < max_len <= the table's tokens)
__device__ __forceinline__ int paged_page(const PagedView& v, int b, int t) {
  const int p = v.table[(int64_t)b * v.max_pages + (t >> v.page_shift)];
  return (unsigned)p < (unsigned)v.n_pages ? p : -1;
}

bool rkv_paged_attention_fits(const PagedView& v);       // do its launches stay under RKV_PAGED_THREADS?
size_t rkv_paged_attention_scratch(const PagedView& v, int D, int bits);
int rkv_launch_paged_attention(const PagedView& v, int D, int bits, int dtype, const void* q, int64_t qs, int causal, int window, float scale,
                               void* out, float* lse, void* scratch, hipStream_t s);
