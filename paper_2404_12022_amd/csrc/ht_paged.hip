// A batch of sequences whose keys and values lie in pages: tables of the trees, append (norm of the heads, rotary, keys and
// values into their pages) and acceptance with compaction.  The attention over the pages is in ht_paged_attn.hip.
//
// Everything that changes from step to step (row starts, lengths, page table, trees) is read on the device, so a captured pass
// can be replayed with new contents.  What the host checked by its bounds (rows, max_rows, max_len, n_pages) the kernels hold
// the device's values to: no value of a table leads outside a buffer.
#include "ht_common.h"

namespace ht {

// ------------------------------------------------------------------------------------------------ trees
// depth[r] and ancestor bits of row r from the parents of its sequence's rows, a workgroup per sequence: every thread walks up
// from its own row through the parents in LDS.  A parent outside 0 .. v-1 ends the walk, so it takes at most v steps.  A chain of LDS reads as long as
// the tree is deep: 4 us for 8 trees of 64 rows and for 256.
__global__ __launch_bounds__(256) void tree_tables_kernel(PagedRows b, const int32_t* __restrict__ parent, int32_t* __restrict__ depth,
                                                          uint64_t* __restrict__ anc) {
  __shared__ int32_t up[kMaxRows];
  const SeqSpan sp = seq_span(b, blockIdx.x);
  const int v = threadIdx.x;
  if (v < sp.count) up[v] = parent[sp.row0 + v];
  __syncthreads();
  if (v >= sp.count) return;
  uint64_t bits[kMaskWords] = {};
  int d = 0, at = v;
  for (;;) {
#pragma unroll
    for (int w = 0; w < kMaskWords; ++w) bits[w] |= at >> 6 == w ? 1ull << (at & 63) : 0ull;
    const int p = up[at];
    if (p < 0 || p >= at) break;
    at = p;
    ++d;
  }
  depth[sp.row0 + v] = d;
#pragma unroll
  for (int w = 0; w < kMaskWords; ++w) anc[(size_t)(sp.row0 + v) * kMaskWords + w] = bits[w];
}
hipError_t launch_tree_tables(const PagedRows& b, const int32_t* parent, int32_t* depth, uint64_t* anc, hipStream_t s) {
  hipLaunchKernelGGL(tree_tables_kernel, dim3(b.seqs), dim3(256), 0, s, b, parent, depth, anc);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------ append
// Any head width (16 trees of 64, 32 heads of 80: 24 us; the kernel below takes 12 for 1.6 times the bytes): a wavefront per head of a row, lane l holds the pairs l, l + 64 of the rotated part and what it passes through.
template <typename T>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedRows b, AppendRows a) {
  const SeqSpan sp = seq_span(b, blockIdx.z);
  const int i = blockIdx.y;
  if (i >= sp.count) return;
  __shared__ float2 factors[128];
  const int row = sp.row0 + i, half = a.rot / 2, slot = sp.n + i;
  const int pos = sp.n + (a.depth ? a.depth[row] : i);
  if ((int)threadIdx.x < half) {
    const int j = threadIdx.x;
    const float2 f = rope_factor(pos, a.inv_freq ? freq_turns(a.inv_freq[j]) : rope_turns(j, a.step));
    factors[j] = make_float2(f.x * a.amplitude, f.y * a.amplitude);
  }
  __syncthreads();
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int h = blockIdx.x * 4 + wave, heads = a.Hq + 2 * b.Hkv;
  if (h >= heads) return;
  const int kind = h < a.Hq ? 0 : h < a.Hq + b.Hkv ? 1 : 2, hk = h - a.Hq - (kind == 2 ? b.Hkv : 0);
  const T* src = kind == 0 ? (const T*)a.q : kind == 1 ? (const T*)a.k : (const T*)a.v;
  if (!src) return;
  T* dst;
  if (kind == 0) {
    src += row * a.q_stride + (size_t)h * b.hd;
    dst = (T*)a.q_out + row * a.q_out_stride + (size_t)h * b.hd;
  } else {
    src += row * (kind == 1 ? a.k_stride : a.v_stride) + (size_t)hk * b.hd;
    const int page = page_of(b, blockIdx.z, slot);
    if (page < 0) return;
    dst = (T*)(kind == 1 ? a.k_pages : a.v_pages) + ((((size_t)page * b.Hkv + hk) << b.page_shift) + (slot & ((1 << b.page_shift) - 1))) * b.hd;
  }
  constexpr int PAIRS = 2;                                   // heads of up to 256
  float x[PAIRS], y[PAIRS];
  int lo[PAIRS], hi[PAIRS];
  const int pairs = b.hd / 2;
  float ss = 0.f;
#pragma unroll
  for (int t = 0; t < PAIRS; ++t) {
    const int j = lane + 64 * t;
    // pair j: of the rotated part, or two neighbours behind it
    lo[t] = j < half ? (a.interleaved ? 2 * j : j) : 2 * j;
    hi[t] = j < half && !a.interleaved ? j + half : lo[t] + 1;
    x[t] = y[t] = 0.f;
    if (j < pairs) {
      x[t] = Conv<T>::load(src + lo[t]);
      y[t] = Conv<T>::load(src + hi[t]);
    }
    ss = fmaf(x[t], x[t], fmaf(y[t], y[t], ss));
  }
  const T* gain = kind == 0 ? (const T*)a.q_gain : kind == 1 ? (const T*)a.k_gain : nullptr;
  if (gain) {
    for (int o = 32; o; o >>= 1) ss += __shfl_xor(ss, o, 64);
    const float r = 1.0f / sqrtf(ss / (float)b.hd + a.eps);
#pragma unroll
    for (int t = 0; t < PAIRS; ++t)
      if (lane + 64 * t < pairs) {
        x[t] = x[t] * r * Conv<T>::load(gain + lo[t]);
        y[t] = y[t] * r * Conv<T>::load(gain + hi[t]);
      }
  }
#pragma unroll
  for (int t = 0; t < PAIRS; ++t) {
    const int j = lane + 64 * t;
    if (j >= pairs) continue;
    float u = x[t], w = y[t];
    if (kind < 2 && j < half) {
      const float2 f = factors[j];
      u = rope_low(x[t], y[t], f);
      w = rope_high(x[t], y[t], f);
    }
    Conv<T>::store(dst + lo[t], u);
    Conv<T>::store(dst + hi[t], w);
  }
}
// Heads of whole 16-byte pieces whose number is a power of two: a row's heads P at a time for every hd / VEC threads, all of them
// requested before the factors are worked out (by as many threads as there are pairs, once for all heads of the workgroup).  Partners of a
// pair lie in one thread, or rot / 2 entries, whole pieces, apart in the same wavefront.  Bound by what the rows stream at once there are
// many (64 x 64 rows of 96 heads of 128, 168 MB: 33 us, 5.1 TB/s; 16 x 64: 12 us, 3.4); for few by the chain row start, length, depth,
// factors (4.7 us).
template <typename T, int P>
__global__ __launch_bounds__(256) void paged_append_vec_kernel(PagedRows b, AppendRows a) {
  constexpr int VEC = 16 / sizeof(T);
  struct __attribute__((packed, aligned(sizeof(T)))) Piece {
    T v[VEC];
  };
  const SeqSpan sp = seq_span(b, blockIdx.z);
  const int i = blockIdx.y;
  if (i >= sp.count) return;
  __shared__ __attribute__((aligned(16))) float2 factors[128];
  const int tid = threadIdx.x, row = sp.row0 + i, half = a.rot / 2, slot = sp.n + i;
  const int per_head = b.hd / VEC, at_once = 256 / per_head, p = tid % per_head, heads = a.Hq + 2 * b.Hkv;
  const int h0 = blockIdx.x * P * at_once + tid / per_head;
  // kind 0: query, 1: key, 2: value, 3: none
  auto kind_of = [&](int h) { return h >= heads ? 3 : h < a.Hq ? (a.q ? 0 : 3) : !a.k ? 3 : h < a.Hq + b.Hkv ? 1 : 2; };
  auto head_of = [&](int h, int kind) { return kind == 0 ? h : h - a.Hq - (kind == 2 ? b.Hkv : 0); };
  Piece x[P];
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int h = h0 + k * at_once, kind = kind_of(h);
    if (kind == 3) continue;
    const T* src = kind == 0 ? (const T*)a.q + row * a.q_stride : kind == 1 ? (const T*)a.k + row * a.k_stride : (const T*)a.v + row * a.v_stride;
    x[k] = *(const Piece*)(src + (size_t)head_of(h, kind) * b.hd + p * VEC);
  }
  const int page = a.k ? page_of(b, blockIdx.z, slot) : -1;
  const int pos = sp.n + (a.depth ? a.depth[row] : i);
  if (tid < half) {
    const float2 f = rope_factor(pos, a.inv_freq ? freq_turns(a.inv_freq[tid]) : rope_turns(tid, a.step));
    factors[tid] = make_float2(f.x * a.amplitude, f.y * a.amplitude);
  }
  __syncthreads();
  const int half_pieces = half / VEC;                      // pairs apart: pieces between partners
  const bool turns = a.interleaved ? p * VEC < a.rot : p < 2 * half_pieces, upper = p >= half_pieces;
  const int partner = (tid & 63) + (!turns || a.interleaved ? 0 : upper ? -half_pieces : half_pieces);
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int h = h0 + k * at_once, kind = kind_of(h);
    float y[VEC];
#pragma unroll
    for (int c = 0; c < VEC; ++c) y[c] = kind == 3 ? 0.f : Conv<T>::load(&x[k].v[c]);
    const T* gain = kind == 0 ? (const T*)a.q_gain : kind == 1 ? (const T*)a.k_gain : nullptr;
    if (a.q_gain || a.k_gain) {                            // (the same for the wavefront: the exchange needs all of it)
      float ss = 0.f;
#pragma unroll
      for (int c = 0; c < VEC; ++c) ss = fmaf(y[c], y[c], ss);
      for (int o = per_head / 2; o; o >>= 1) ss += __shfl_xor(ss, o, 64);
      if (gain) {
        const float r = 1.0f / sqrtf(ss / (float)b.hd + a.eps);
        const Piece g = *(const Piece*)(gain + p * VEC);
#pragma unroll
        for (int c = 0; c < VEC; ++c) y[c] = y[c] * r * Conv<T>::load(&g.v[c]);
      }
    }
    if (a.rot && !a.interleaved) {
      float z[VEC];
#pragma unroll
      for (int c = 0; c < VEC; ++c) z[c] = __shfl(y[c], partner, 64);
      if (kind < 2 && turns) {
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
          const float2 f = factors[(upper ? p - half_pieces : p) * VEC + c];
          y[c] = upper ? rope_high(z[c], y[c], f) : rope_low(y[c], z[c], f);
        }
      }
    } else if (kind < 2 && turns) {
#pragma unroll
      for (int c = 0; c < VEC; c += 2) {
        if (p * VEC + c >= a.rot) break;
        const float2 f = factors[(p * VEC + c) / 2];
        const float lo = rope_low(y[c], y[c + 1], f);
        y[c + 1] = rope_high(y[c], y[c + 1], f);
        y[c] = lo;
      }
    }
    if (kind == 3 || (kind && page < 0)) continue;
    Piece out;
    if (kind == 2) out = x[k];
    else
#pragma unroll
      for (int c = 0; c < VEC; ++c) Conv<T>::store(&out.v[c], y[c]);
    T* dst;
    if (kind == 0) dst = (T*)a.q_out + row * a.q_out_stride + (size_t)h * b.hd;
    else
      dst = (T*)(kind == 1 ? a.k_pages : a.v_pages) +
            ((((size_t)page * b.Hkv + head_of(h, kind)) << b.page_shift) + (slot & ((1 << b.page_shift) - 1))) * b.hd;
    *(Piece*)(dst + p * VEC) = out;
  }
}
template <typename T> void launch_append_of(const PagedRows& b, const AppendRows& a, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  const int heads = a.Hq + 2 * b.Hkv, pieces = b.hd / VEC;
  // pieces of a head: whole, a power of two, within a wavefront; partners whole pieces apart
  if (b.hd % VEC || pieces > 64 || (pieces & (pieces - 1)) || (!a.interleaved && (a.rot / 2) % VEC)) {
    hipLaunchKernelGGL(paged_append_kernel<T>, dim3((heads + 3) / 4, b.max_rows, b.seqs), dim3(256), 0, s, b, a);
    return;
  }
  // two heads to a thread once the rows are many (64 sequences of 64 rows, 32 heads of 128: 33 us, with one 37, with four 40), one
  // before (16 of 64: 12.3 us, with two 12.7, four 15.7; one row: 3.9, 4.7, 6.3)
  const int at_once = 256 / pieces;
  const int64_t rows = (int64_t)b.max_rows * b.seqs;
  const int P = rows >= 2048 ? 2 : 1;
  auto f = P == 2 ? paged_append_vec_kernel<T, 2> : paged_append_vec_kernel<T, 1>;
  hipLaunchKernelGGL(f, dim3((heads + P * at_once - 1) / (P * at_once), b.max_rows, b.seqs), dim3(256), 0, s, b, a);
}
hipError_t launch_paged_append(int dtype, const PagedRows& b, const AppendRows& a, hipStream_t s) {
  if (dtype == 0) launch_append_of<float>(b, a, s);
  else launch_append_of<bf16_t>(b, a, s);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------ acceptance
// From the root of a sequence's tree on, the lowest child that carries the token answered after the node so far is accepted;
// path[j] >= j rises, so row path[j] may move to slot n + j, j ascending, in place: no source is overwritten before it is read.
// blockIdx.x: pieces of a cache row (keys, then values), blockIdx.y: layer, blockIdx.z: sequence.  U: the unit that moves.  Every workgroup walks
// its sequence's tree for itself, a ballot a level: a chain of some 3 us, next to which the few rows that move are nothing (8 trees of
// 64 in 80 layers 4.8 us, 64 trees 19).
template <typename U>
__global__ __launch_bounds__(256) void paged_accept_kernel(PagedRows b, AcceptRows a, int unit_elems, int units) {
  __shared__ int32_t up[kMaxRows], own[kMaxRows], next[kMaxRows], path[kMaxRows];
  __shared__ int32_t found;
  const int seq = blockIdx.z, tid = threadIdx.x;
  const SeqSpan sp = seq_span(b, seq);
  if (tid < sp.count) {
    up[tid] = a.parent[sp.row0 + tid];
    own[tid] = a.tokens[sp.row0 + tid];
    next[tid] = a.answers[sp.row0 + tid];
  }
  __syncthreads();
  if (tid < 64) {
    int cur = 0, m = sp.count > 0;
    if (tid == 0) path[0] = 0;
    while (m && m < a.max_path) {
      int child = -1;
      for (int c0 = (cur + 1) & ~63; c0 < sp.count && child < 0; c0 += 64) {
        const int c = c0 + tid;
        const uint64_t match = __ballot(c > cur && c < sp.count && up[c] == cur && own[c] == next[cur]);
        if (match) child = c0 + __builtin_ctzll(match);
      }
      if (child < 0) break;
      if (tid == 0) path[m] = child;
      cur = child;
      ++m;
    }
    if (tid == 0) found = m;
  }
  __syncthreads();
  const int m = found;
  const int at = blockIdx.x * 256 + tid;
  if (at < 2 * units) {
    const int c = at < units ? at : at - units, per_head = b.hd / unit_elems;
    const int hk = c / per_head, e = c % per_head;
    U* pool = (U*)(at < units ? a.k_pages : a.v_pages) + (size_t)blockIdx.y * a.layer_elems / unit_elems;
    auto place = [&](int slot) -> U* {
      const int page = page_of(b, seq, slot);
      return page < 0 ? nullptr : pool + ((((size_t)page * b.Hkv + hk) << b.page_shift) + (slot & ((1 << b.page_shift) - 1))) * per_head + e;
    };
    for (int j = 1; j < m; ++j) {
      if (path[j] == j) continue;
      const U* from = place(sp.n + path[j]);
      U* to = place(sp.n + j);
      if (from && to) *to = *from;
    }
  }
  if (blockIdx.x || blockIdx.y) return;
  for (int j = tid; j < a.max_path; j += 256) {
    a.path[(size_t)seq * a.max_path + j] = j < m ? path[j] : -1;
    a.emitted[(size_t)seq * a.max_path + j] = j < m ? own[path[j]] : -1;
  }
  if (tid == 0) {
    a.accepted[seq] = m;
    a.next_root[seq] = m ? next[path[m - 1]] : -1;
    a.new_len[seq] = sp.n + m;
  }
}
hipError_t launch_paged_accept(int dtype, const PagedRows& b, const AcceptRows& a, int layers, hipStream_t s) {
  const int elem = dtype == 0 ? 4 : 2;
  const bool wide = b.hd * elem % 16 == 0 && !(((uintptr_t)a.k_pages | (uintptr_t)a.v_pages | a.layer_elems * elem) & 15);
  const int unit = wide ? 16 / elem : 1, units = b.Hkv * b.hd / unit;
  const dim3 grid((2 * units + 255) / 256, layers, b.seqs);
  if (wide) hipLaunchKernelGGL(paged_accept_kernel<uint4>, grid, dim3(256), 0, s, b, a, unit, units);
  else if (dtype == 0) hipLaunchKernelGGL(paged_accept_kernel<float>, grid, dim3(256), 0, s, b, a, unit, units);
  else hipLaunchKernelGGL(paged_accept_kernel<bf16_t>, grid, dim3(256), 0, s, b, a, unit, units);
  return hipGetLastError();
}

}  // namespace ht
