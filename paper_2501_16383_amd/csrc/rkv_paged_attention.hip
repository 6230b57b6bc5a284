// Attention of packed rows over the cache in pages.
#include "rkv_paged.h"

// One wave per (row, query head): lanes hold channels, tokens one after the other with the running maximum and
// sum of the softmax.
template <int D, int BITS, int DT>
__global__ __launch_bounds__(64) void k_paged_plain(PagedView v, const unsigned short* __restrict__ q, int64_t qs, int causal, int window,
                                                    float scale, unsigned short* __restrict__ out, float* __restrict__ lse) {
  constexpr int N = D / 64;                                      // channels of a lane
  const int lane = threadIdx.x, row = blockIdx.x / v.Hq, h = blockIdx.x % v.Hq;
  const int b = paged_owner(v, row);
  if (b >= v.n_seqs) return;
  const PagedSeq s = paged_seq(v, b);
  if (row < s.first || row >= s.last) return;
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

size_t rkv_paged_attention_scratch(const PagedView&, int) { return 0; }

template <int D, int BITS, int DT>
static void launch(const PagedView& v, const void* q, int64_t qs, int causal, int window, float scale, void* out, float* lse, hipStream_t s) {
  k_paged_plain<D, BITS, DT><<<dim3(v.n_rows * v.Hq), 64, 0, s>>>(v, (const unsigned short*)q, qs, causal, window, scale, (unsigned short*)out, lse);
}

int rkv_launch_paged_attention(const PagedView& v, int D, int bits, int dtype, const void* q, int64_t qs, int causal, int window, float scale,
                               void* out, float* lse, void*, hipStream_t s) {
#define GO(D_, B_) (dtype ? launch<D_, B_, 1>(v, q, qs, causal, window, scale, out, lse, s) : launch<D_, B_, 0>(v, q, qs, causal, window, scale, out, lse, s))
  if (D == 64) { if (bits == 16) GO(64, 16); else if (bits == 8) GO(64, 8); else GO(64, 4); }
  else { if (bits == 16) GO(128, 16); else if (bits == 8) GO(128, 8); else GO(128, 4); }
#undef GO
  RKV_HIP_CHECK(hipGetLastError());
  return RKV_OK;
}
