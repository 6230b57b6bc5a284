// The cache in pages: host side of its calls, and the kernels that write tokens into it and read them back.
#include "rkv_paged.h"

#define RKV_EXPORT extern "C" __attribute__((visibility("default")))

// ---- writing and reading -----------------------------------------------------------------------
//
// Both move every byte once: a thread takes eight channels (16 bytes) of a token's key head and of its value
// head, so that a wave reads and writes 1 KiB runs of the dense rows; four neighbouring lanes are a block of
// 32 channels.  Bound by memory - prompts of 8430 tokens in all, 40 heads of 128, 4 bits: 62 us to write (5.0 TB/s of rows and
// codes), 43 to read back -, and for a few tokens by the chain row -> sequence -> page -> slot, whose loads go out
// beside those of the rows (one token: 2.5 us).

// Where a thread works: row, sequence and slot
struct PagedSlot {
  int row, c;                          // row of the tensors, channel group (of eight) in it
  bool mine;                           // the row belongs to a sequence
  bool bad;                            // its sequence is bad
  int pos;                             // position in the sequence, < 0 in front of its first token
  int64_t at;                          // page * Hkv + head of the slot's block, or -1
  int slot;                            // token in the page
};

template <int D> __device__ __forceinline__ PagedSlot paged_slot(const PagedView& v) {
  PagedSlot p;
  const int G = v.Hkv * (D / 8);
  const int64_t start = (int64_t)blockIdx.x * 256;
  const int row0 = (int)(start / G);
  const int r = (int)(start - (int64_t)row0 * G) + threadIdx.x;
  p.row = row0 + r / G;
  p.c = r % G;
  p.mine = p.bad = false;
  p.pos = -1;
  p.at = -1;
  p.slot = 0;
  int b = paged_owner(v, __builtin_amdgcn_readfirstlane(p.row));
  if (p.row >= v.n_rows || b >= v.n_seqs) return p;
  while (b < v.n_seqs && v.row_start[b + 1] <= p.row) ++b;   // (rows of narrow heads: several in a wave)
  if (b >= v.n_seqs) return p;
  const PagedSeq s = paged_seq(v, b);
  p.mine = p.row >= s.first && p.row < s.last;
  p.bad = s.bad;
  if (!p.mine || s.bad) return p;
  p.pos = s.base + (p.row - s.first);
  if (p.pos < 0) return p;
  const int page = paged_page(v, b, p.pos);
  p.slot = p.pos & ((1 << v.page_shift) - 1);
  if (page >= 0) p.at = (int64_t)page * v.Hkv + p.c / (D / 8);
  return p;
}

// larger of the four lanes of a block's
__device__ __forceinline__ uint32_t paged_quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true));   // quad_perm [1,0,3,2]
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true));   // quad_perm [2,3,0,1]
}

// (a bit cast of a vector's element would take the vector's first)
__device__ __forceinline__ b2 as_b2(uint32_t x) { return __builtin_bit_cast(b2, x); }
__device__ __forceinline__ h2 as_h2(uint32_t x) { return __builtin_bit_cast(h2, x); }

typedef unsigned short us2 __attribute__((ext_vector_type(2)));

// Eight elements of a block that this lane and its three neighbours hold: codes, and the block's scale byte.
// Magnitudes compare as integers, and scaling by a power of two is exact: the only rounding is the
// conversion's own, to nearest with ties to even.
template <int DT, int BITS> __device__ __forceinline__ u32x2 paged_encode8(u32x4 x, uint32_t& byte) {
  constexpr uint32_t top = DT ? (BITS == 8 ? 0x7f70 : 0x7f40) : (BITS == 8 ? 0x7b80 : 0x7a00);   // largest number of both types
  constexpr uint32_t inf = DT ? 0x7f80 : 0x7c00;
  constexpr int e_min = DT ? (BITS == 8 ? -118 : -126) : (BITS == 8 ? -15 : -23);
  us2 m = {0, 0};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t a = x[j] & 0x7fff7fffu;
    m = __builtin_elementwise_max(m, __builtin_bit_cast(us2, a));
    const us2 cap = {(unsigned short)top, (unsigned short)top};
    x[j] = (x[j] & 0x80008000u) | __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(us2, a), cap));
  }
  const uint32_t big = paged_quad_max(max((uint32_t)m[0], (uint32_t)m[1]));
  const uint32_t a = __float_as_uint(paged_lo<DT>(big));
  // A = 1.f 2^k: the exponent that puts it at or under 448 = 1.75 2^8 or 6 = 1.5 2^2
  const int k = (int)(a >> 23) - 127;
  int e = BITS == 8 ? k - 8 + ((a & 0x7fffff) > 0x600000) : k - 2 + ((a & 0x7fffff) > 0x400000);
  e = max(e, e_min);
  const bool bad = big >= inf;
  byte = bad ? 255 : e + 127;
  const float scale = paged_scale(e + 127);
  u32x2 r = {0, 0};
  if (bad) return r;
  typedef short s2 __attribute__((ext_vector_type(2)));
  if constexpr (BITS == 8) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      s2 w = {0, 0};
      if constexpr (DT) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, as_b2(x[2 * j]), scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, as_b2(x[2 * j + 1]), scale, true);
      } else {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, as_h2(x[2 * j]), scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, as_h2(x[2 * j + 1]), scale, true);
      }
      r[j] = __builtin_bit_cast(uint32_t, w);
    }
  } else {
    uint32_t w = 0;
    if constexpr (DT) {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_b2(x[0]), scale, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_b2(x[1]), scale, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_b2(x[2]), scale, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_b2(x[3]), scale, 3);
    } else {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, as_h2(x[0]), scale, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, as_h2(x[1]), scale, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, as_h2(x[2]), scale, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, as_h2(x[3]), scale, 3);
    }
    r[0] = w;
  }
  return r;
}

template <int D, int BITS, int DT>
__global__ __launch_bounds__(256) void k_paged_append(PagedView v, const unsigned short* __restrict__ k, int64_t ks,
                                                      const unsigned short* __restrict__ val, int64_t vs) {
  const PagedSlot p = paged_slot<D>(v);
  const bool in = p.row < v.n_rows;
  const u32x4 z = {0, 0, 0, 0};
  const u32x4 kx = in ? *(const u32x4*)(k + p.row * ks + p.c * 8) : z;
  const u32x4 vx = in ? *(const u32x4*)(val + p.row * vs + p.c * 8) : z;
  constexpr int rb = paged_row<D, BITS>(), sb = paged_srow<D, BITS>();
  const int cc = p.c % (D / 8);                                  // channel group in the head
  unsigned char* blk = v.pool + p.at * paged_block<D, BITS>(v.page_shift);
  unsigned char* kd = blk + p.slot * rb + cc * BITS;             // (eight codes: BITS bytes)
  unsigned char* vd = kd + (rb << v.page_shift);
  if constexpr (BITS == 16) {
    if (p.at < 0) return;
    *(u32x4*)kd = kx;
    *(u32x4*)vd = vx;
  } else {
    uint32_t kbyte, vbyte;                                       // (every lane of a block takes part)
    const u32x2 kc = paged_encode8<DT, BITS>(kx, kbyte), vc = paged_encode8<DT, BITS>(vx, vbyte);
    if (p.at < 0) return;
    if constexpr (BITS == 8) {
      *(u32x2*)kd = kc;
      *(u32x2*)vd = vc;
    } else {
      *(uint32_t*)kd = kc[0];
      *(uint32_t*)vd = vc[0];
    }
    if ((cc & 3) == 0) {
      unsigned char* sd = blk + ((2 * rb) << v.page_shift) + p.slot * sb + (cc >> 2);
      sd[0] = (unsigned char)kbyte;
      sd[sb << v.page_shift] = (unsigned char)vbyte;
    }
  }
}

template <int D, int BITS, int DT>
__global__ __launch_bounds__(256) void k_paged_read(PagedView v, unsigned short* __restrict__ k, int64_t ks, unsigned short* __restrict__ val,
                                                    int64_t vs) {
  const PagedSlot p = paged_slot<D>(v);
  if (!p.mine) return;
  constexpr int rb = paged_row<D, BITS>(), sb = paged_srow<D, BITS>();
  constexpr uint32_t nan2 = DT ? 0x7fc07fc0u : 0x7e007e00u;
  const int cc = p.c % (D / 8);
  const uint32_t none = p.bad || p.pos >= 0 ? nan2 : 0;          // a bad sequence or page, else a row in front of the first token
  u32x4 kx = {none, none, none, none}, vx = kx;
  if (p.at >= 0) {
    const unsigned char* blk = v.pool + p.at * paged_block<D, BITS>(v.page_shift);
    const unsigned char* kd = blk + p.slot * rb + cc * BITS;
    const unsigned char* vd = kd + (rb << v.page_shift);
    if constexpr (BITS == 16) {
      kx = *(const u32x4*)kd;
      vx = *(const u32x4*)vd;
    } else {
      const unsigned char* sd = blk + ((2 * rb) << v.page_shift) + p.slot * sb + (cc >> 2);
      u32x2 kc = {0, 0}, vc = {0, 0};
      if constexpr (BITS == 8) {
        kc = *(const u32x2*)kd;
        vc = *(const u32x2*)vd;
      } else {
        kc[0] = *(const uint32_t*)kd;
        vc[0] = *(const uint32_t*)vd;
      }
      const uint32_t kbyte = sd[0], vbyte = sd[sb << v.page_shift];
      kx = paged_decode8<DT, BITS>(kc, paged_scale(kbyte));
      vx = paged_decode8<DT, BITS>(vc, paged_scale(vbyte));
    }
  }
  *(u32x4*)(k + p.row * ks + p.c * 8) = kx;
  *(u32x4*)(val + p.row * vs + p.c * 8) = vx;
}

static int64_t move_blocks(const PagedView& v, int D) { return ((int64_t)v.n_rows * v.Hkv * (D / 8) + 255) / 256; }

template <int D, int BITS>
static void launch_append(const PagedView& v, int dtype, const void* k, int64_t ks, const void* val, int64_t vs, hipStream_t s) {
  const dim3 grid((unsigned)move_blocks(v, D));
  if (dtype) k_paged_append<D, BITS, 1><<<grid, 256, 0, s>>>(v, (const unsigned short*)k, ks, (const unsigned short*)val, vs);
  else k_paged_append<D, BITS, 0><<<grid, 256, 0, s>>>(v, (const unsigned short*)k, ks, (const unsigned short*)val, vs);
}
template <int D, int BITS>
static void launch_read(const PagedView& v, int dtype, void* k, int64_t ks, void* val, int64_t vs, hipStream_t s) {
  const dim3 grid((unsigned)move_blocks(v, D));
  if (dtype) k_paged_read<D, BITS, 1><<<grid, 256, 0, s>>>(v, (unsigned short*)k, ks, (unsigned short*)val, vs);
  else k_paged_read<D, BITS, 0><<<grid, 256, 0, s>>>(v, (unsigned short*)k, ks, (unsigned short*)val, vs);
}

#define PAGED_DISPATCH(CALL)                                                                          \
  do {                                                                                                \
    if (cfg->head_dim == 64) {                                                                        \
      if (cfg->bits == 16) CALL<64, 16>(ARGS); else if (cfg->bits == 8) CALL<64, 8>(ARGS); else CALL<64, 4>(ARGS);      \
    } else {                                                                                          \
      if (cfg->bits == 16) CALL<128, 16>(ARGS); else if (cfg->bits == 8) CALL<128, 8>(ARGS); else CALL<128, 4>(ARGS);   \
    }                                                                                                 \
  } while (0)

// ---- host side ---------------------------------------------------------------------------------

static int check_paged(const rkv_paged_config* c) {
  if (!c) return RKV_EINVAL;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 256 || c->n_q_heads < c->n_kv_heads || c->n_q_heads % c->n_kv_heads != 0) return RKV_EINVAL;
  if (c->n_q_heads / c->n_kv_heads > 256) return RKV_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return RKV_EINVAL;
  if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return RKV_EINVAL;
  if (c->n_pages < 1) return RKV_EINVAL;
  if (c->bits != 16 && c->bits != 8 && c->bits != 4) return RKV_EINVAL;
  if (c->dtype != 0 && c->dtype != 1) return RKV_EINVAL;
  return RKV_OK;
}

static int check_batch(const rkv_paged_config* c, const rkv_paged_batch* b, void* pool, PagedView* v) {
  const int rc = check_paged(c);
  if (rc != RKV_OK) return rc;
  if (!b || b->n_rows < 0) return RKV_EINVAL;
  if (b->n_rows == 0) return RKV_OK;
  if (!b->dev_page_table || !b->dev_row_start || !b->dev_lengths) return RKV_EINVAL;
  if (((uintptr_t)b->dev_page_table | (uintptr_t)b->dev_row_start | (uintptr_t)b->dev_lengths) & 3) return RKV_EINVAL;
  if (b->n_seqs < 1 || b->n_seqs > 65535 || b->max_pages < 1) return RKV_EINVAL;
  if (b->max_new < 1 || b->max_new > b->n_rows) return RKV_EINVAL;
  if (b->max_len < 1 || b->max_len > 1 << 30 || b->max_len > (int64_t)b->max_pages * c->page_tokens) return RKV_EINVAL;
  if ((int64_t)b->n_rows * c->n_q_heads > (int64_t)1 << 30) return RKV_EINVAL;   // (rows and columns are counted in 32 bits)
  if ((uintptr_t)pool & 15) return RKV_EINVAL;
  v->pool = (unsigned char*)pool;
  v->table = b->dev_page_table;
  v->row_start = b->dev_row_start;
  v->lengths = b->dev_lengths;
  v->n_seqs = b->n_seqs;
  v->max_pages = b->max_pages;
  v->n_rows = b->n_rows;
  v->max_new = b->max_new;
  v->max_len = b->max_len;
  v->Hq = c->n_q_heads;
  v->Hkv = c->n_kv_heads;
  v->rep = c->n_q_heads / c->n_kv_heads;
  v->page_shift = __builtin_ctz(c->page_tokens);
  v->n_pages = c->n_pages;
  return RKV_OK;
}

// rows of `heads` heads, `stride` elements apart, from `p` on
static bool rows_ok(const rkv_paged_config* c, const void* p, int64_t stride, int heads) {
  return p && !((uintptr_t)p & 15) && stride >= (int64_t)heads * c->head_dim && !(stride & 7) && stride < ((int64_t)1 << 31);
}

RKV_EXPORT int rkv_paged_sizes(const rkv_paged_config* cfg, size_t* pool_bytes) {
  const int rc = check_paged(cfg);
  if (rc != RKV_OK) return rc;
  const size_t row = 2 * ((size_t)cfg->head_dim * cfg->bits / 8 + (cfg->bits < 16 ? cfg->head_dim / RKV_PAGED_BLOCK : 0));
  if (pool_bytes) *pool_bytes = row * cfg->page_tokens * cfg->n_kv_heads * (size_t)cfg->n_pages;
  return RKV_OK;
}

RKV_EXPORT int rkv_paged_append(const rkv_paged_config* cfg, void* dev_pool, const rkv_paged_batch* batch, const void* dev_k, int64_t k_stride,
                                const void* dev_v, int64_t v_stride, void* stream) {
  PagedView v{};
  const int rc = check_batch(cfg, batch, dev_pool, &v);
  if (rc != RKV_OK || v.n_rows == 0) return rc;
  if (!dev_pool || !rows_ok(cfg, dev_k, k_stride, cfg->n_kv_heads) || !rows_ok(cfg, dev_v, v_stride, cfg->n_kv_heads)) return RKV_EINVAL;
  if (move_blocks(v, cfg->head_dim) * 256 >= RKV_PAGED_THREADS) return RKV_EINVAL;
#define ARGS v, cfg->dtype, dev_k, k_stride, dev_v, v_stride, (hipStream_t)stream
  PAGED_DISPATCH(launch_append);
#undef ARGS
  RKV_HIP_CHECK(hipGetLastError());
  return RKV_OK;
}

RKV_EXPORT int rkv_paged_read(const rkv_paged_config* cfg, const void* dev_pool, const rkv_paged_batch* batch, void* dev_k, int64_t k_stride,
                              void* dev_v, int64_t v_stride, void* stream) {
  PagedView v{};
  const int rc = check_batch(cfg, batch, (void*)dev_pool, &v);
  if (rc != RKV_OK || v.n_rows == 0) return rc;
  if (!dev_pool || !rows_ok(cfg, dev_k, k_stride, cfg->n_kv_heads) || !rows_ok(cfg, dev_v, v_stride, cfg->n_kv_heads)) return RKV_EINVAL;
  if (move_blocks(v, cfg->head_dim) * 256 >= RKV_PAGED_THREADS) return RKV_EINVAL;
#define ARGS v, cfg->dtype, dev_k, k_stride, dev_v, v_stride, (hipStream_t)stream
  PAGED_DISPATCH(launch_read);
#undef ARGS
  RKV_HIP_CHECK(hipGetLastError());
  return RKV_OK;
}

RKV_EXPORT int rkv_paged_scratch(const rkv_paged_config* cfg, const rkv_paged_batch* batch, size_t* scratch_bytes) {
  PagedView v{};
  const int rc = check_batch(cfg, batch, nullptr, &v);
  if (rc != RKV_OK) return rc;
  if (v.n_rows && !rkv_paged_attention_fits(v)) return RKV_EINVAL;
  if (scratch_bytes) *scratch_bytes = v.n_rows ? rkv_paged_attention_scratch(v, cfg->head_dim, cfg->bits) : 0;
  return RKV_OK;
}

RKV_EXPORT int rkv_paged_attention(const rkv_paged_config* cfg, const void* dev_pool, const rkv_paged_batch* batch, const void* dev_q,
                                   int64_t q_stride, int32_t causal, int32_t window, float scale, void* dev_out, float* dev_lse,
                                   void* dev_scratch, size_t scratch_bytes, void* stream) {
  PagedView v{};
  const int rc = check_batch(cfg, batch, (void*)dev_pool, &v);
  if (rc != RKV_OK) return rc;
  if ((causal != 0 && causal != 1) || window < 0 || !__builtin_isfinite(scale * 1.4426950408889634f)) return RKV_EINVAL;
  if (v.n_rows == 0) return RKV_OK;
  if (!dev_pool || !rows_ok(cfg, dev_q, q_stride, cfg->n_q_heads) || !dev_out || ((uintptr_t)dev_out & 15) || ((uintptr_t)dev_lse & 3)) return RKV_EINVAL;
  if (!rkv_paged_attention_fits(v)) return RKV_EINVAL;
  const size_t need = rkv_paged_attention_scratch(v, cfg->head_dim, cfg->bits);
  if (need && (!dev_scratch || ((uintptr_t)dev_scratch & 255) || scratch_bytes < need)) return RKV_EINVAL;
  return rkv_launch_paged_attention(v, cfg->head_dim, cfg->bits, cfg->dtype, dev_q, q_stride, causal, window, scale, dev_out, dev_lse,
                                    dev_scratch, (hipStream_t)stream);
}
