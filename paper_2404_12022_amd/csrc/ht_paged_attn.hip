// Attention of the rows of a batch over its pages.
//
//   out[r][h] = softmax_{j seen by r}( scale q[r][h] . K[j] ) V[j]
//   seen by r = the cached slots 0 .. n-1 of its sequence  U  { n + u : bit u of r's ancestor mask }   (u <= r without masks)
//
// Slots whose page is none of the pool's are seen by nobody; a row that sees nothing is 0.
#include "ht_common.h"

namespace ht {

// Any head width, either type: a wavefront per (row, query head), a lane per key for the scores and per output element for the
// values.  Keys and values that a row does not see are read but never used: what they hold does not matter.
template <typename T>
__global__ __launch_bounds__(64) void paged_attn_simple_kernel(PagedRows b, AttnRows a) {
  __shared__ float qs[256];
  const int seq = blockIdx.z, i = blockIdx.y, h = blockIdx.x, lane = threadIdx.x;
  const SeqSpan sp = seq_span(b, seq);
  if (i >= sp.count) return;
  const int row = sp.row0 + i, hk = h / (a.Hq / b.Hkv), hd = b.hd, in_page = (1 << b.page_shift) - 1;
  const T* q = (const T*)a.q + row * a.q_stride + (size_t)h * hd;
  for (int e = lane; e < hd; e += 64) qs[e] = Conv<T>::load(q + e) * a.scale_log2;
  uint64_t mask[kMaskWords];
#pragma unroll
  for (int w = 0; w < kMaskWords; ++w) {
    const int past = i + 1 - 64 * w;                       // the chain: rows 0 .. i
    mask[w] = a.anc ? a.anc[(size_t)row * kMaskWords + w] : past >= 64 ? ~0ull : past > 0 ? (1ull << past) - 1 : 0ull;
  }
  __syncthreads();
  constexpr int EL = 4;
  float acc[EL] = {}, top = -INFINITY, sum = 0.f;
  const int S = sp.n + sp.count;
  for (int j0 = 0; j0 < S; j0 += 64) {
    const int j = j0 + lane;
    const int page = j < S ? page_of(b, seq, j) : -1;
    const size_t at = ((((size_t)(page < 0 ? 0 : page) * b.Hkv + hk) << b.page_shift) + (j & in_page)) * hd;
    bool seen = page >= 0;
    if (seen && j >= sp.n) {
      const int u = j - sp.n;
      uint64_t word = 0;
#pragma unroll
      for (int w = 0; w < kMaskWords; ++w) word = u >> 6 == w ? mask[w] : word;
      seen = word >> (u & 63) & 1;
    }
    float z = -INFINITY;
    if (seen) {
      const T* k = (const T*)a.k_pages + at;
      z = 0.f;
      for (int e = 0; e < hd; ++e) z = fmaf(qs[e], Conv<T>::load(k + e), z);
    }
    float best = z;
    for (int o = 32; o; o >>= 1) best = fmaxf(best, __shfl_xor(best, o, 64));
    const float now = fmaxf(top, best), safe = now == -INFINITY ? 0.f : now;
    const float p = seen ? exp2f(z - safe) : 0.f, keep = exp2f(top - safe);
    top = now;
    sum = sum * keep + p;
#pragma unroll
    for (int t = 0; t < EL; ++t) acc[t] *= keep;
    const unsigned long long any = __ballot(seen);
    for (int l = 0; l < 64; ++l) {
      if (!(any >> l & 1)) continue;
      const float w = __shfl(p, l, 64);
      const T* v = (const T*)a.v_pages + __shfl((long long)at, l, 64);
#pragma unroll
      for (int t = 0; t < EL; ++t)
        if (lane + 64 * t < hd) acc[t] = fmaf(w, Conv<T>::load(v + lane + 64 * t), acc[t]);
    }
  }
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o, 64);
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  T* out = (T*)a.out + row * a.out_stride + (size_t)h * hd;
#pragma unroll
  for (int t = 0; t < EL; ++t)
    if (lane + 64 * t < hd) Conv<T>::store(out + lane + 64 * t, sum == 0.f ? 0.f : acc[t] * inv);
}

size_t paged_attn_scratch_bytes(int, const PagedRows&, int) { return 0; }

hipError_t launch_paged_attn(int dtype, const PagedRows& b, const AttnRows& a, void*, hipStream_t s) {
  const dim3 grid(a.Hq, b.max_rows, b.seqs);
  if (dtype == 0) hipLaunchKernelGGL(paged_attn_simple_kernel<float>, grid, dim3(64), 0, s, b, a);
  else hipLaunchKernelGGL(paged_attn_simple_kernel<bf16_t>, grid, dim3(64), 0, s, b, a);
  return hipGetLastError();
}

}  // namespace ht
