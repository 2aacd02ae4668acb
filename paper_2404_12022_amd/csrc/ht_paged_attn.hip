// Attention of the rows of a batch over its pages.
//
//   out[r][h] = softmax_{j seen by r}( scale q[r][h] . K[j] ) V[j]
//   seen by r = the cached slots 0 .. n-1 of its sequence  U  { n + u : bit u of r's ancestor mask }   (u <= r without masks)
//
// Slots whose page is none of the pool's are seen by nobody; a row that sees nothing is 0.
#include "ht_common.h"
#include <type_traits>

namespace ht {

// Any head width, either type: a workgroup per (row, query head), whose wavefronts take blocks of 64 keys in turn, a lane per key for the
// scores and per output element for the values.  Keys and values that a row does not see are read but never used: what they hold
// does not matter.  Every row reads its sequence's cache for itself and multiplies on the vector units, so this is for
// heads that the matrix kernels below do not take (8 sequences of 1000, 8 heads of 80: 29 us for a row each, 310 us for 64).
template <typename T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void paged_attn_simple_kernel(PagedRows b, AttnRows a) {
  __shared__ float qs[256], lds_o[WAVES][256], lds_m[WAVES], lds_l[WAVES];
  struct Pair {
    T v[2];
  };
  const int seq = blockIdx.z, i = blockIdx.y, h = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const SeqSpan sp = seq_span(b, seq);
  if (i >= sp.count) return;
  const int row = sp.row0 + i, hk = h / (a.Hq / b.Hkv), hd = b.hd, in_page = (1 << b.page_shift) - 1;
  const T* q = (const T*)a.q + row * a.q_stride + (size_t)h * hd;
  for (int e = threadIdx.x; e < hd; e += 64 * WAVES) qs[e] = Conv<T>::load(q + e) * a.scale_log2;
  uint64_t mask[kMaskWords];
#pragma unroll
  for (int w = 0; w < kMaskWords; ++w) {
    const int past = i + 1 - 64 * w;                       // the chain: rows 0 .. i
    mask[w] = a.anc ? a.anc[(size_t)row * kMaskWords + w] : past >= 64 ? ~0ull : past > 0 ? (1ull << past) - 1 : 0ull;
  }
  __syncthreads();
  constexpr int EL = 4, AT_ONCE = 8;                       // keys whose values are requested together
  float acc[EL] = {}, top = -INFINITY, sum = 0.f;
  const int S = sp.n + sp.count;
  for (int j0 = wave * 64; j0 < S; j0 += 64 * WAVES) {
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
      const Pair* k = (const Pair*)((const T*)a.k_pages + at);         // (heads are even, pages on 16 bytes)
      z = 0.f;
#pragma unroll 8
      for (int e = 0; e < hd / 2; ++e) {
        const Pair x = k[e];
        z = fmaf(qs[2 * e], Conv<T>::load(&x.v[0]), fmaf(qs[2 * e + 1], Conv<T>::load(&x.v[1]), z));
      }
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
    for (int l0 = 0; l0 < 64; l0 += AT_ONCE) {
      if (!(any >> l0 & ((1ull << AT_ONCE) - 1))) continue;
      float v[AT_ONCE][EL];
#pragma unroll
      for (int l = 0; l < AT_ONCE; ++l) {
        const T* from = (const T*)a.v_pages + __shfl((long long)at, l0 + l, 64);
#pragma unroll
        for (int t = 0; t < EL; ++t) v[l][t] = lane + 64 * t < hd ? Conv<T>::load(from + lane + 64 * t) : 0.f;
      }
#pragma unroll
      for (int l = 0; l < AT_ONCE; ++l) {
        const float w = __shfl(p, l0 + l, 64);
        const bool in = any >> (l0 + l) & 1;
#pragma unroll
        for (int t = 0; t < EL; ++t) acc[t] = in ? fmaf(w, v[l][t], acc[t]) : acc[t];
      }
    }
  }
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o, 64);
  // ---- join the wavefronts
#pragma unroll
  for (int t = 0; t < EL; ++t) lds_o[wave][lane + 64 * t] = acc[t];
  if (lane == 0) lds_m[wave] = top, lds_l[wave] = sum;
  __syncthreads();
  const int e = threadIdx.x;
  if (e >= hd) return;
  float all = -INFINITY, total = 0.f, out = 0.f;
  for (int w = 0; w < WAVES; ++w) all = fmaxf(all, lds_m[w]);
  const float ref = all == -INFINITY ? 0.f : all;
  for (int w = 0; w < WAVES; ++w) {
    const float f = exp2f(lds_m[w] - ref);
    total = fmaf(f, lds_l[w], total);
    out = fmaf(f, lds_o[w][e], out);
  }
  Conv<T>::store((T*)a.out + row * a.out_stride + (size_t)h * hd + e, total == 0.f ? 0.f : out / total);
}

// ------------------------------------------------------------------------------------------------ bf16, heads of 64 and 128
// The matrix-core kernels work transposed, a column being a (row, query head of the group) pair of one sequence and key/value head:
//   S^T[key][col] = K[key][:] . Q[col][:]      O^T[e][col] += V^T[e][key] P[key][col]
// The 32 keys of a block are assigned to the two 16-row score products in the order key = 8 (r / 4) + 4 b + r % 4, so the eight scores
// a lane holds are the eight consecutive keys that its P operand of the second product wants.  V lies in its pages as rows of a
// key (one row is stored and moved as one piece); its way through LDS ends in transposing reads, four keys of one column e at a time.
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float floatx4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

union Frag {
  u32x4_t nat;
  bf16x8_t v;
  uint2 half[2];
  uint32_t u[4];
};
// 16 and 8 bytes at any address (a caller's rows need not lie on 16)
struct __attribute__((packed, aligned(2))) Loose16 {
  u32x4_t v;
};
struct __attribute__((packed, aligned(2))) Loose8 {
  uint2 v;
};

// Four outputs, over their sum (0 over an empty one)
__device__ __forceinline__ void store_four(bf16_t* out, const floatx4_t& acc, float sum) {
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  ((Loose8*)out)->v = sum == 0.f ? make_uint2(0, 0) : pack4_bf16(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
}
__device__ __forceinline__ void store_four(float* out, const floatx4_t& acc, float sum) {
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = sum == 0.f ? 0.f : acc[i] / sum;
}

constexpr float kRescaleStep = 8.0f;         // log2 units the reference point may lag behind the maximum: probabilities stay below 2^8

__device__ __forceinline__ float max_over_groups(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  auto r2 = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r2[0]), __uint_as_float(r2[1]));
}
__device__ __forceinline__ float sum_over_groups(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  auto r2 = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r2[0]) + __uint_as_float(r2[1]);
}

// Where the 16-byte piece of a key's row lies in LDS, in bytes from the row's start.  K is read 16 rows of one piece at a time (a
// quarter of a wavefront; rows 8 apart and 0 .. 3), V 16 rows of one 32-byte unit: both are spread over the 256 bytes of all banks.
template <int HD> __device__ __forceinline__ int k_place(int row, int piece) {
  const int h = HD == 128 ? (row & 3) | ((row >> 3) & 3) << 2 : ((row >> 1) & 1) | ((row >> 3) & 3) << 1;
  return (piece ^ h) << 4;
}
template <int HD> __device__ __forceinline__ int v_place(int row, int unit) {
  const int f = HD == 128 ? (row & 3) | ((row >> 3) & 1) << 2 : ((row >> 1) & 1) | ((row >> 3) & 1) << 1;
  return (unit ^ f) << 5;
}
// V^T operand of 32 keys: rows e = eb * 16 + r16, keys 8 g .. 8 g + 7
template <int HD> __device__ __forceinline__ Frag v_operand(const unsigned char* rows, int eb, int r16, int g) {
  Frag f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = 8 * g + 4 * h + (r16 >> 2);
    const unsigned char* at = rows + row * (HD * 2) + v_place<HD>(row, eb) + (r16 & 3) * 8;
    const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)at);
    f.half[h] = *(const uint2*)&x;
  }
  return f;
}

// Keys j0 .. j0 + 63 that row `row` of the sequence sees, as bits; w: its mask (NULL: a chain), `there`: the keys that are
__device__ __forceinline__ uint64_t seen_bits(const uint64_t* w, const SeqSpan& sp, int row, int j0, uint64_t there) {
  const int first = j0 - sp.n;                             // the row of the pass that key j0 is
  if (first <= -64 || row >= sp.count) return there;
  uint64_t bits;
  if (!w) {
    const int upto = row - first;                          // rows 0 .. row
    bits = upto < 0 ? 0ull : upto >= 63 ? ~0ull : (2ull << upto) - 1;
  } else {
    if (first < 0) {
      bits = w[0] << -first | ((1ull << -first) - 1);
    } else {
      const int i = first >> 6, s = first & 63;
      bits = i < kMaskWords ? w[i] >> s : 0ull;
      if (s && i + 1 < kMaskWords) bits |= w[i + 1] << (64 - s);
    }
  }
  return bits & there;
}
__device__ __forceinline__ const uint64_t* mask_of(const AttnRows& a, const SeqSpan& sp, int row) {
  return a.anc ? a.anc + (size_t)(sp.row0 + (row < sp.count ? row : 0)) * kMaskWords : nullptr;
}
// Values that are no numbers become 0 (they would reach columns that do not see them); whether there were any
__device__ __forceinline__ bool tidy(u32x4_t& x) {
  bool odd = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const bool lo = (x[w] & 0x7f80u) == 0x7f80u, hi = (x[w] & 0x7f800000u) == 0x7f800000u;
    odd |= lo | hi;
    x[w] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
  }
  return odd;
}
// Four values of a key that one or more columns see, of which those that are no numbers have been left out: added (a share of one is itself)
template <typename F> __device__ __forceinline__ void add_odd(const char* at, F&& add) {
  const uint2 four = ((const Loose8*)at)->v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t v = (i < 2 ? four.x : four.y) >> (i & 1) * 16 & 0xffffu;
    if ((v & 0x7f80u) == 0x7f80u) add(i, __uint_as_float(v << 16));
  }
}
// The pages of a sequence, seen from one key/value head
struct PageView {
  const char *kp, *vp;
  const int32_t* table;
  size_t page_bytes;
  int S, shift, n_pages;
  __device__ __forceinline__ PageView(const PagedRows& b, const AttnRows& a, const SeqSpan& sp, int seq, int hk)
      : table(b.table + (size_t)seq * b.table_width), S(sp.n + sp.count), shift(b.page_shift), n_pages(b.n_pages) {
    page_bytes = (size_t)b.Hkv * b.hd * 2 << shift;
    const size_t head = (size_t)hk * b.hd * 2 << shift;
    kp = (const char*)a.k_pages + head;
    vp = (const char*)a.v_pages + head;
  }
  // of a slot that is the same for the whole wavefront, through scalar registers
  __device__ __forceinline__ int page_at(int slot) const {
    const auto* in = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)table;
    return in[(slot < S ? slot : S - 1) >> shift];
  }
  // the keys j0 .. j0 + 63 that are there (j0 < S), as bits
  __device__ __forceinline__ uint64_t up_to_end(int j0) const { return j0 + 64 > S ? (1ull << (S - j0)) - 1 : ~0ull; }
  __device__ __forceinline__ uint64_t there_at(int j0) const {
    uint64_t t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) t |= (unsigned)page_at(j0 + 8 * i) < (unsigned)n_pages ? 0xffull << 8 * i : 0ull;
    return t & up_to_end(j0);
  }
  __device__ __forceinline__ const char* value_row(int slot, int hd) const {
    return vp + page_at(slot) * page_bytes + (size_t)(slot & ((1 << shift) - 1)) * (hd * 2);
  }
};

// The K place of the kernel with 32 columns to a wavefront, which reads 16 consecutive keys of one piece at a time
template <int HD> __device__ __forceinline__ int wide_k_place(int row, int piece) {
  return (piece ^ (HD == 128 ? row & 15 : (row >> 1) & 7)) << 4;
}

// What a workgroup's four wavefronts bring of a sequence's pages: tiles of 64 keys of K and V, through registers to LDS
template <int HD> struct TileLoader : PageView {
  static constexpr int PIECES = HD / 8, ROWS = 64 / PIECES, PASS = 4 * ROWS, LOADS = 64 / PASS, TILE = 64 * HD * 2;
  static_assert(64 % PASS == 0, "whole passes");
  typedef u32x4_t Part[LOADS];                              // a wavefront's part of a tile
  int wave, lane;

  __device__ __forceinline__ TileLoader(const PagedRows& b, const AttnRows& a, const SeqSpan& sp, int seq, int hk, int wave, int lane)
      : PageView(b, a, sp, seq, hk), wave(wave), lane(lane) {}
  __device__ __forceinline__ int pages(int j0) const {      // of key j0 + lane
    const int slot = j0 + lane;
    return table[(slot < S ? slot : S - 1) >> shift];
  }
  __device__ __forceinline__ uint64_t there_of(int j0, int id) const { return __ballot((unsigned)id < (unsigned)n_pages && j0 + lane < S); }
  __device__ __forceinline__ void load(Part& x, const char* pool, int j0, int id) const {
    const int held = (unsigned)id < (unsigned)n_pages ? id : 0;
#pragma unroll
    for (int p = 0; p < LOADS; ++p) {                       // a load's rows lie in one page: pages hold whole eights
      const int row0 = p * PASS + wave * ROWS;
      const size_t at = __builtin_amdgcn_readlane(held, row0) * page_bytes + (size_t)((j0 + row0) & ((1 << shift) - 1)) * (HD * 2);
      x[p] = ((const Loose16*)(pool + at + (uint32_t)lane * 16u))->v;
    }
  }
  __device__ __forceinline__ void store_k(const Part& x, unsigned char* base) const {
#pragma unroll
    for (int p = 0; p < LOADS; ++p) {
      const int row = p * PASS + wave * ROWS + lane / PIECES, piece = lane % PIECES;
      *(u32x4_t*)(base + row * (HD * 2) + k_place<HD>(row, piece)) = x[p];
    }
  }
  __device__ __forceinline__ void store_v(const Part& x, unsigned char* base) const {
#pragma unroll
    for (int p = 0; p < LOADS; ++p) {
      const int row = p * PASS + wave * ROWS + lane / PIECES, piece = lane % PIECES;
      *(u32x4_t*)(base + row * (HD * 2) + v_place<HD>(row, piece >> 1) + (piece & 1) * 16) = x[p];
    }
  }
  // Values for a tile that not every column sees whole: those of keys that are not there become 0 (0 times what lies there is no 0),
  // and those that are no numbers, for add_odd; whether there were such
  __device__ __forceinline__ bool clear(Part& x, uint64_t there, int lane) const {
    bool odd = false;
#pragma unroll
    for (int p = 0; p < LOADS; ++p) {
      if (!(there >> (p * PASS + wave * ROWS + lane / PIECES) & 1)) x[p] = u32x4_t{0, 0, 0, 0};
      odd |= tidy(x[p]);
    }
    return odd;
  }
  // Tile after tile, the next on its way while one is multiplied, two stages of (K, V), a barrier per tile; a loop for the tiles that
  // every column sees whole, and one for those behind (they hold rows of the pass; or a page is missing):
  // f(masked, first key, keys that are there, tile).  *odd is set where values were left out; returns the first key of the second loop
  template <typename F> __device__ __forceinline__ int run(unsigned char* lds, int* odd, int key0, int key1, int n, F&& f) const {
    Part k, v;
    auto store = [&](unsigned char* base, int j0, uint64_t there) __attribute__((always_inline)) {
      if (there != ~0ull || j0 + 64 > n)
        if (clear(v, there, lane)) *odd = 1;
      store_k(k, base);
      store_v(v, base + TILE);
    };
    int id = pages(key0), j0 = key0, stage = 0;
    uint64_t there = there_of(key0, id);
    load(k, kp, key0, id);
    load(v, vp, key0, id);
    id = pages(key0 + 64);
    if (wave == 0 && lane == 0) *odd = 0;
    __syncthreads();
    store(lds, key0, there);
    __syncthreads();
    auto tiles = [&](auto masked) __attribute__((always_inline)) {
      for (; j0 < key1; j0 += 64, stage ^= 2 * TILE) {
        if (!decltype(masked)::value && (there != ~0ull || j0 + 64 > n)) break;
        const bool more = j0 + 64 < key1;
        const uint64_t there_next = there_of(j0 + 64, id);
        if (more) {
          load(k, kp, j0 + 64, id);
          load(v, vp, j0 + 64, id);
          id = pages(j0 + 128);
        }
        f(masked, j0, there, (const unsigned char*)lds + stage);
        there = there_next;
        if (more) store(lds + (stage ^ 2 * TILE), j0 + 64, there);
        __syncthreads();
      }
    };
    tiles(std::false_type{});
    const int rest = j0;
    tiles(std::true_type{});
    return rest;
  }
};

// The 16 columns of a wavefront
template <int HD> struct Columns {
  static constexpr int ES = HD / 32, EB = HD / 16;
  Frag q[ES];
  floatx4_t o[EB];
  float m, l;                                // reference point (log2 units, scaled) and this lane's part of the sum
  int row, head;                             // row of the sequence (count or more: none) and query head

  __device__ __forceinline__ void start(const AttnRows& a, const SeqSpan& sp, int hk, int group, int col, int g) {
    row = col / group;
    head = hk * group + col % group;
    const int r = row < sp.count ? row : sp.count - 1;
    const bf16_t* src = (const bf16_t*)a.q + (int64_t)(sp.row0 + r) * a.q_stride + (int64_t)head * HD + g * 8;
#pragma unroll
    for (int es = 0; es < ES; ++es) q[es].nat = ((const Loose16*)(src + es * 32))->v;
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int eb = 0; eb < EB; ++eb) o[eb] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  }

  // SUB blocks of 32 keys: k(sub, block, piece) their K operands, V rows in LDS, and with MASKED what the column sees of them
  template <int SUB, bool MASKED, typename K>
  __device__ __forceinline__ void multiply(K&& k, const unsigned char* v_rows, uint64_t vis, float scale, int r16, int g) {
    float p[8 * SUB];
#pragma unroll
    for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        Frag kf[ES];
#pragma unroll
        for (int es = 0; es < ES; ++es) kf[es] = k(sub, b, es);
        floatx4_t s = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int es = 0; es < ES; ++es) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[es].v, q[es].v, s, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[sub * 8 + b * 4 + i] = s[i];
      }
    if (MASKED) {
#pragma unroll
      for (int x = 0; x < 8 * SUB; ++x) {
        const uint32_t word = (uint32_t)(vis >> (x >> 3) * 32) >> g * 8;
        p[x] = word >> (x & 7) & 1 ? p[x] : -INFINITY;
      }
    }
    float top = p[0];
#pragma unroll
    for (int x = 1; x < 8 * SUB; ++x) top = fmaxf(top, p[x]);
    top = max_over_groups(top) * scale;
    const bool grow = top > m + kRescaleStep;              // m = -inf: any number
    if (__any(grow)) {
      const float keep = grow ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
      l *= keep;
#pragma unroll
      for (int eb = 0; eb < EB; ++eb) o[eb] *= keep;
      m = grow ? top : m;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int x = 0; x < 8 * SUB; ++x) {
      p[x] = __builtin_amdgcn_exp2f(fmaf(p[x], scale, -ref));
      sum += p[x];
    }
    l += sum;
#pragma unroll
    for (int sub = 0; sub < SUB; ++sub) {
      Frag pf;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        pf.half[h] = pack4_bf16(p[sub * 8 + 4 * h], p[sub * 8 + 4 * h + 1], p[sub * 8 + 4 * h + 2], p[sub * 8 + 4 * h + 3]);
      const unsigned char* rows = v_rows + sub * 32 * HD * 2;
#pragma unroll
      for (int eb = 0; eb < EB; ++eb) {
        const Frag vf = v_operand<HD>(rows, eb, r16, g);
        o[eb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.v, pf.v, o[eb], 0, 0, 0);
      }
    }
  }
  // The values of keys j0 .. j1 - 1 that are no numbers, to the columns that see them: rare, key by key
  __device__ __forceinline__ void add_odd_values(const AttnRows& a, const SeqSpan& sp, const PageView& in, int j0, int j1, int g) {
    for (; j0 < j1; j0 += 64) {
      const uint64_t there = in.there_at(j0), vis = seen_bits(mask_of(a, sp, row), sp, row, j0, there);
#pragma unroll 1
      for (int k = 0; k < 64 && j0 + k < j1; ++k) {
        if (!(there >> k & 1)) continue;
        const char* values = in.value_row(j0 + k, HD) + g * 8;
#pragma unroll
        for (int eb = 0; eb < EB; ++eb)
          add_odd(values + eb * 32, [&](int i, float v) __attribute__((always_inline)) {
            if (vis >> k & 1) o[eb][i] += v;
          });
      }
    }
  }
  // o over its sum
  __device__ __forceinline__ void finish(const AttnRows& a, const SeqSpan& sp, const floatx4_t& acc, int eb, float sum, int g) const {
    if (row < sp.count)
      store_four((bf16_t*)a.out + (int64_t)(sp.row0 + row) * a.out_stride + (int64_t)head * HD + eb * 16 + g * 4, acc, sum);
  }
};

// A sequence's share of a split launch: keys key0 .. key1 - 1
struct Slice {
  int key0, key1, count;
};
__device__ __forceinline__ Slice slice_of(const SeqSpan& sp, int split, int split_len) {
  const int S = sp.n + sp.count;
  const int count = (S + split_len - 1) / split_len, k0 = split * split_len;
  return Slice{k0, k0 + split_len < S ? k0 + split_len : S, count};
}

// Shared-out work of the bf16 kernels.  An item is a (head, sequence, column tile); a long one is cut into parts, a workgroup each, none
// of more than T tiles of 64 keys with kItemTiles for what starting and ending costs, T the smallest with which all parts fit the
// grid: lengths may be as ragged as they like.  The parts of an item leave partial results, which a second kernel joins.  Every
// wavefront works this out for itself.
constexpr int kShareSeqs = 256;              // sequences that a wavefront can add up
constexpr int kItemTiles = 3;                // tiles that starting and ending a part costs (5 to 6 us; a tile 1.9); 2 or 5: the same within 3%
struct Part {
  int seq, hk, col_tile, key0, key1;
  int parts, part, place;                    // of the item: how many, which, and where in the row of parts this one stands
  SeqSpan sp;
};
// What a workgroup leaves for the join; parts 0: nothing, 1: a whole item
struct PartNote {
  int32_t row0, count, hk, col_tile, part, parts, pad[2];
};
// Running sums over a wavefront, by moves that need no LDS; lane 63 has them all
__device__ __forceinline__ int wave_sums(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);        // from the lanes 1, 2, 4, 8 before in the row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);        // from the last lane of the row before
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);        // from lane 31
  return v;
}
__device__ __forceinline__ int wave_total(int v) { return __builtin_amdgcn_readlane(wave_sums(v), 63); }
__device__ __forceinline__ int wave_largest(int v) {                      // of numbers >= 0
  auto step = [&](int other) { v = other > v ? other : v; };
  step(__builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));
  step(__builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
  step(__builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
  step(__builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
  step(__builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));
  step(__builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(v, 63);
}
// The place of a workgroup in the row of parts: the workgroups of one XCD (numbers that are equal modulo 8) have consecutive parts, heads
// outermost, so that column tiles of the same keys meet in one L2
__device__ __forceinline__ int place_of_workgroup() {
  const int per = gridDim.x / 8;
  return gridDim.x % 8 ? blockIdx.x : blockIdx.x % 8 * per + blockIdx.x / 8;
}
// Which part this workgroup has of a batch of up to 64 PER sequences; false: none
template <int COLS, int PER>
__device__ __forceinline__ bool share_out(const PagedRows& b, int group, int least, Part& out) {
  const int lane = threadIdx.x & 63;
  SeqSpan sp[PER];                                         // of sequences PER lane .. + PER - 1
  int tiles[PER], items[PER], total = 0, longest = 0, all_items = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int seq = PER * lane + i;
    sp[i] = seq_span(b, seq < b.seqs ? seq : 0);
    const bool any = seq < b.seqs && sp[i].count;
    tiles[i] = any ? (sp[i].n + sp[i].count + 63) / 64 : 0;
    items[i] = any ? (sp[i].count * group + COLS - 1) / COLS : 0;
    longest = tiles[i] > longest ? tiles[i] : longest;
    total += items[i] * (tiles[i] + kItemTiles);                 // (at most what the host has held below 2^30)
    all_items += items[i];
  }
  total = wave_total(total);
  if (!total) return false;
  longest = wave_largest(longest);
  all_items = wave_total(all_items);
  const int room = (int)gridDim.x / b.Hkv;                 // parts of a head
  int lo = (total + room - 1) / room, hi = longest + kItemTiles;
  // (as many parts as total / T and one more of every item fit at twice the least T)
  if (2 * all_items <= room && 2 * lo < hi) hi = 2 * lo;
  lo = lo > least ? lo : least;
  int T;
  float per_T;
  auto parts_of = [&](int tiles_i) {                       // (tiles_i + kItemTiles) / T, up
    const int x = tiles_i + kItemTiles + T - 1;                  // (the quotient from the reciprocal is off by one at most: x < 2^26, T >= 4)
    int q = (int)((float)x * per_T), r = x - q * T;
    q += r >= T ? 1 : r < 0 ? -1 : 0;
    return q;
  };
  auto parts_at = [&](int at_T) {
    T = at_T;
    per_T = __builtin_amdgcn_rcpf((float)T);
    int n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) n += items[i] * parts_of(tiles[i]);
    return n;
  };
  while (lo < hi) {                                        // (at longest + kItemTiles every item is one part, and the grid holds all items)
    const int mid = (lo + hi) / 2;
    if (wave_total(parts_at(mid)) <= room) hi = mid;
    else lo = mid + 1;
  }
  const int mine = parts_at(lo), run = wave_sums(mine);
  const int of_head = __builtin_amdgcn_readlane(run, 63), w = place_of_workgroup();
  if (w >= of_head * b.Hkv) return false;
  const int hk = w / of_head, at = w - hk * of_head;
  const int who = __popcll(__ballot(run <= at));           // the lane whose sequences hold part `at`
  int rest = at - __builtin_amdgcn_readlane(run - mine, who), in_lane = 0;
  int parts = __builtin_amdgcn_readlane(parts_of(tiles[0]), who), n_tiles = __builtin_amdgcn_readlane(tiles[0], who);
  SeqSpan of{__builtin_amdgcn_readlane(sp[0].row0, who), __builtin_amdgcn_readlane(sp[0].count, who), __builtin_amdgcn_readlane(sp[0].n, who)};
  int before = __builtin_amdgcn_readlane(items[0], who) * parts;
#pragma unroll
  for (int i = 1; i < PER; ++i) {
    const int p = __builtin_amdgcn_readlane(parts_of(tiles[i]), who), n = __builtin_amdgcn_readlane(items[i], who) * p;
    if (rest >= before) {                                  // (not in the one before: the last that is taken holds it)
      rest -= before, before = n, in_lane = i, parts = p, n_tiles = __builtin_amdgcn_readlane(tiles[i], who);
      of = SeqSpan{__builtin_amdgcn_readlane(sp[i].row0, who), __builtin_amdgcn_readlane(sp[i].count, who), __builtin_amdgcn_readlane(sp[i].n, who)};
    }
  }
  const int ct = rest / parts, part = rest - ct * parts;
  int t0, t1;
  even_share(n_tiles, parts, part, t0, t1);
  out = Part{PER * who + in_lane, hk, ct, t0 * 64, t1 * 64 < of.n + of.count ? t1 * 64 : of.n + of.count, parts, part, w, of};
  return true;
}
// The same of any batch; least 0: an item to a workgroup
template <int COLS> __device__ __forceinline__ bool part_of_workgroup(const PagedRows& b, int group, int least, Part& out) {
  if (least) return b.seqs <= 64 ? share_out<COLS, 1>(b, group, least, out) : share_out<COLS, kShareSeqs / 64>(b, group, least, out);
  const SeqSpan sp = seq_span(b, blockIdx.z);
  out = Part{(int)blockIdx.z, (int)blockIdx.x, (int)blockIdx.y, 0, sp.n + sp.count, 1, 0, 0, sp};
  return (int)blockIdx.y * COLS < sp.count * group;
}
__device__ __forceinline__ void leave_note(PartNote* notes, int least, bool any, const Part& s) {
  if (threadIdx.x || !least) return;
  notes[place_of_workgroup()] = any ? PartNote{s.sp.row0, s.sp.count, s.hk, s.col_tile, s.part, s.parts, {}} : PartNote{};
}

}  // namespace

// Up to 16 columns: the four wavefronts of a workgroup take blocks of 32 keys in turn, each for itself (no barrier until the end),
// K from global memory straight into operand registers, V through 32 rows of LDS of the wavefront's own; the next block is in
// flight while one is multiplied.  Bound by what the cache streams at: one row each of 32 sequences of 200 to 2048 positions, 32
// heads of 128, 556 MB, 111 us (5.0 TB/s; all of 2048 192 us, 5.6); one of 100003 positions, 8 key/value heads, 71 us (5.8) and 5 for
// the join.  A few short sequences: 4.7 us, a chain of loads (row start, length, page, K, V).
template <int HD>
__global__ __launch_bounds__(256, 2) void paged_attn_few_kernel(PagedRows b, AttnRows a, int split_len, float* part_o, float* part_ml) {
  using Cols = Columns<HD>;
  constexpr int ES = Cols::ES, EB = Cols::EB, PIECES = HD / 8, LOADS = 32 * PIECES / 64, V_BYTES = 32 * HD * 2, STEP = 4 * 32;
  constexpr int O_FLOATS = EB * 4 * 64;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * V_BYTES > 4 * O_FLOATS * 4 ? 4 * V_BYTES : 4 * O_FLOATS * 4];
  __shared__ float lds_m[4 * 64], lds_l[4 * 64];
  const int seq = blockIdx.z, hk = blockIdx.x, group = a.Hq / b.Hkv, split = blockIdx.y;
  const SeqSpan sp = seq_span(b, seq);
  const Slice sl = slice_of(sp, split, split_len);
  if (sp.count == 0 || sl.key0 >= sl.key1) return;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r16 = lane & 15, g = lane >> 4;
  const int S = sp.n + sp.count, in_page = (1 << b.page_shift) - 1;
  const size_t page_elems = (size_t)b.Hkv * HD << b.page_shift, head_elems = (size_t)hk * HD << b.page_shift;
  const int32_t* table = b.table + (size_t)seq * b.table_width;
  const PageView view(b, a, sp, seq, hk);
  const bf16_t *kp = (const bf16_t*)a.k_pages + head_elems, *vp = (const bf16_t*)a.v_pages + head_elems;
  unsigned char* v_rows = lds + wave * V_BYTES;

  Cols cols;
  cols.start(a, sp, hk, group, r16, g);

  // the page of keys 8 (r16 / 4) .. + 7 of a block (a page holds whole eights)
  auto pages = [&](int j0) __attribute__((always_inline)) {
    const int slot = j0 + 8 * (r16 >> 2);
    return table[(slot < S ? slot : S - 1) >> b.page_shift];
  };
  constexpr int ROWS = 64 / PIECES;                        // 4 or 8 rows of V a load: within an eight
  Frag kf[2][ES];
  u32x4_t vr[LOADS];
  auto load_k = [&](Frag (&to)[2][ES], int j0, int id) __attribute__((always_inline)) {
    const int held = (unsigned)id < (unsigned)b.n_pages ? id : 0;
    const bf16_t* krow = kp + held * page_elems + (size_t)((j0 + 8 * (r16 >> 2) + (r16 & 3)) & in_page) * HD + g * 8;
#pragma unroll
    for (int bl = 0; bl < 2; ++bl)
#pragma unroll
      for (int es = 0; es < ES; ++es) to[bl][es].nat = ((const Loose16*)(krow + bl * 4 * HD + es * 32))->v;
  };
  auto load_v = [&](int j0, int id) __attribute__((always_inline)) {
    const int held = (unsigned)id < (unsigned)b.n_pages ? id : 0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int page = __builtin_amdgcn_readlane(held, i * ROWS / 8 * 4), row0 = (j0 + i * ROWS) & in_page;
      vr[i] = ((const Loose16*)(vp + page * page_elems + (size_t)row0 * HD + lane * 8))->v;
    }
  };
  auto clear_v = [&](uint32_t there) __attribute__((always_inline)) {      // as TileLoader::clear
    bool odd = false;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      if (!(there >> (i * ROWS + lane / PIECES) & 1)) vr[i] = u32x4_t{0, 0, 0, 0};
      odd |= tidy(vr[i]);
    }
    return __any(odd);
  };
  auto store_v = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = i * ROWS + lane / PIECES, piece = lane % PIECES;
      *(u32x4_t*)(v_rows + row * (HD * 2) + v_place<HD>(row, piece >> 1) + (piece & 1) * 16) = vr[i];
    }
  };
  auto there_of = [&](int j0, int id) __attribute__((always_inline)) {
    const uint64_t ok = __ballot((unsigned)id < (unsigned)b.n_pages);
    const uint32_t t = (ok & 1 ? 0xffu : 0u) | (ok & 0x10 ? 0xff00u : 0u) | (ok & 0x100 ? 0xff0000u : 0u) | (ok & 0x1000 ? 0xff000000u : 0u);
    return j0 + 32 > S ? t & ((1u << (S - j0)) - 1) : t;   // (j0 < S)
  };
  int j0 = sl.key0 + wave * 32;
  if (j0 < sl.key1) {
    int id = pages(j0), id_next = pages(j0 + STEP);
    load_k(kf, j0, id);
    load_v(j0, id);
    // a loop for the blocks that every column sees whole, and one for those behind (they hold rows of the pass; or a page is missing).
    // A block: its V goes to LDS, the next one's K and V are requested, then the products
    auto blocks = [&](auto masked) __attribute__((always_inline)) {
      constexpr bool MASKED = decltype(masked)::value;
      while (j0 < sl.key1) {
        const uint32_t there = there_of(j0, id);
        if (!MASKED && (there != 0xffffffffu || j0 + 32 > sp.n)) break;
        const int id_after = pages(j0 + 2 * STEP);
        const bool more = j0 + STEP < sl.key1;
        Frag kn[2][ES];
        if (more) load_k(kn, j0 + STEP, id_next);
        bool odd = false;
        if (MASKED) odd = clear_v(there);
        store_v();
        if (more) load_v(j0 + STEP, id_next);
        const uint64_t vis = MASKED ? seen_bits(mask_of(a, sp, cols.row), sp, cols.row, j0, there) : 0;
        cols.template multiply<1, MASKED>([&](int, int bl, int es) __attribute__((always_inline)) { return kf[bl][es]; }, v_rows, vis,
                                          a.scale_log2, r16, g);
        if (MASKED && odd) cols.add_odd_values(a, sp, view, j0, j0 + 32 < S ? j0 + 32 : S, g);
#pragma unroll
        for (int bl = 0; bl < 2; ++bl)
#pragma unroll
          for (int es = 0; es < ES; ++es) kf[bl][es] = kn[bl][es];
        id = id_next, id_next = id_after, j0 += STEP;
      }
    };
    blocks(std::false_type{});
    blocks(std::true_type{});
  }

  // ---- join the wavefronts
  float* lds_o = (float*)lds;
  __syncthreads();
  lds_m[wave * 64 + lane] = cols.m;
  lds_l[wave * 64 + lane] = sum_over_groups(cols.l);
#pragma unroll
  for (int eb = 0; eb < EB; ++eb) *(floatx4_t*)(lds_o + ((wave * EB + eb) * 64 + lane) * 4) = cols.o[eb];
  __syncthreads();
  if (cols.row >= sp.count) return;
  float top = -INFINITY, f[4], sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, lds_m[w * 64 + lane]);
  const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = __builtin_amdgcn_exp2f(lds_m[w * 64 + lane] - ref);
    sum += f[w] * lds_l[w * 64 + lane];
  }
  const size_t at = ((size_t)split * b.rows + sp.row0 + cols.row) * a.Hq + cols.head;
#pragma unroll
  for (int eb = 0; eb < EB; eb += 4) {
    if (eb + wave >= EB) continue;
    floatx4_t acc = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const floatx4_t x = *(const floatx4_t*)(lds_o + ((w * EB + eb + wave) * 64 + lane) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(f[w], x[i], acc[i]);
    }
    if (sl.count > 1) *(floatx4_t*)(part_o + at * HD + (eb + wave) * 16 + g * 4) = acc;
    else cols.finish(a, sp, acc, eb + wave, sum, g);
  }
  if (sl.count > 1 && wave == 0 && g == 0) *(float2*)(part_ml + at * 2) = make_float2(top, sum);
}

// 17 to 64 columns: every wavefront owns 16, tiles of 64 keys of K and V go through LDS for all of them, the next on its way through
// registers.  Still bound by the cache's stream where there is much of it (32 sequences of 4096, 8 key/value heads of 128: 32 columns 107 us,
// 5.0 TB/s; 64 columns 114); by the chain of starting, tiles and join where there is little (8 sequences: 32 and 35 us).
template <int HD>
__global__ __launch_bounds__(256, 2) void paged_attn_tile_kernel(PagedRows b, AttnRows a, int least, float* part_o, float* part_ml,
                                                                    PartNote* notes) {
  using Cols = Columns<HD>;
  constexpr int EB = Cols::EB, TILE = 64 * HD * 2, COLS = 64;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * TILE];   // two stages of (K tile, V tile)
  __shared__ int odd;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = a.Hq / b.Hkv;
  Part s;
  const bool any = part_of_workgroup<COLS>(b, group, least, s);
  leave_note(notes, least, any, s);
  if (!any) return;
  {
    const int r16 = lane & 15, g = lane >> 4;
    const SeqSpan sp = s.sp;
    const int col0 = s.col_tile * COLS + wave * 16;
    const bool works = col0 < sp.count * group;            // the others only bring tiles
    Cols cols;
    cols.start(a, sp, s.hk, group, col0 + r16, g);
    const TileLoader<HD> in(b, a, sp, s.seq, s.hk, wave, lane);
    const int rest = in.run(lds, &odd, s.key0, s.key1, sp.n, [&](auto masked, int j0, uint64_t there, const unsigned char* base) __attribute__((always_inline)) {
      constexpr bool MASKED = decltype(masked)::value;
      if (!works) return;
      const int krow = 8 * (r16 >> 2) + (r16 & 3);
      auto k_of = [&](int sub, int bl, int es) __attribute__((always_inline)) {
        const int row = sub * 32 + 4 * bl + krow;
        Frag f;
        f.nat = *(const u32x4_t*)(base + row * (HD * 2) + k_place<HD>(row, es * 4 + g));
        return f;
      };
      const uint64_t vis = MASKED ? seen_bits(mask_of(a, sp, cols.row), sp, cols.row, j0, there) : 0;
      cols.template multiply<2, MASKED>(k_of, base + TILE, vis, a.scale_log2, r16, g);
    });
    if (!works) return;
    if (odd) cols.add_odd_values(a, sp, in, rest, s.key1, g);
    const float sum = sum_over_groups(cols.l);
    if (s.parts == 1) {
#pragma unroll
      for (int eb = 0; eb < EB; ++eb) cols.finish(a, sp, cols.o[eb], eb, sum, g);
    } else {
      const size_t at = (size_t)s.place * COLS + wave * 16 + r16;
#pragma unroll
      for (int eb = 0; eb < EB; ++eb) *(floatx4_t*)(part_o + at * HD + eb * 16 + g * 4) = cols.o[eb];
      if (g == 0) *(float2*)(part_ml + at * 2) = make_float2(cols.m, sum);
    }
  }
}

// Many columns: 32 to a wavefront, on the 32 x 32 x 16 instructions (half as many to issue, and a column lies in two lanes instead of
// four).  Row r of a score product is key 16 (r / 16) + 8 (r / 4 % 2) + 4 (r / 8 % 2) + r % 4: the sixteen scores that a lane
// holds of 32 keys are two runs of eight, P operands again.
namespace {
typedef float floatx16_t __attribute__((ext_vector_type(16)));

template <int HD> struct WideColumns {
  static constexpr int KS = HD / 16, EB = HD / 32;
  Frag q[KS];
  floatx16_t o[EB];
  float m, l;
  int row, head;

  __device__ __forceinline__ void start(const AttnRows& a, const SeqSpan& sp, int hk, int group, int col, int half) {
    row = col / group;
    head = hk * group + col % group;
    const int r = row < sp.count ? row : sp.count - 1;
    const bf16_t* src = (const bf16_t*)a.q + (int64_t)(sp.row0 + r) * a.q_stride + (int64_t)head * HD + half * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks].nat = ((const Loose16*)(src + ks * 16))->v;
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int eb = 0; eb < EB; ++eb)
#pragma unroll
      for (int x = 0; x < 16; ++x) o[eb][x] = 0.f;
  }

  // The queries are waited for here, not at their first use inside the loop, where the wait would be for the tiles on their way too
  __device__ __forceinline__ void arrived() {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[ks].nat));
  }
  // Scores of NB blocks of 32 keys
  template <int NB> __device__ __forceinline__ void scores(const unsigned char* k_rows, float (&p)[NB][16], int lane) const {
    const int r32 = lane & 31, half = lane >> 5;
    const int krow = 16 * (r32 >> 4) + 8 * ((r32 >> 2) & 1) + 4 * ((r32 >> 3) & 1) + (r32 & 3);
    floatx16_t s[NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) s[kb][x] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
        Frag kf;
        kf.nat = *(const u32x4_t*)(k_rows + (kb * 32 + krow) * (HD * 2) + wide_k_place<HD>(krow, 2 * ks + half));
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf.v, q[ks].v, s[kb], 0, 0, 0);
      }
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) p[kb][x] = s[kb][x];
  }
  // Their probabilities; the accumulators follow the reference point
  template <bool MASKED, int NB>
  __device__ __forceinline__ void soften(float (&p)[NB][16], Frag (&pf)[2 * NB], uint64_t vis, float scale, int lane) {
    const int half = lane >> 5;
    if (MASKED) {
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
        const uint32_t word = (uint32_t)(vis >> kb * 32) >> half * 8;
#pragma unroll
        for (int x = 0; x < 16; ++x) p[kb][x] = word >> (16 * (x >> 3) + (x & 7)) & 1 ? p[kb][x] : -INFINITY;
      }
    }
    float top = p[0][0];
#pragma unroll
    for (int x = 1; x < 16 * NB; ++x) top = fmaxf(top, p[x >> 4][x & 15]);
    auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale;
    const bool grow = top > m + kRescaleStep;
    if (__any(grow)) {
      const float keep = grow ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
      l *= keep;
#pragma unroll
      for (int eb = 0; eb < EB; ++eb) o[eb] *= keep;
      m = grow ? top : m;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) {
      float w[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        w[x] = __builtin_amdgcn_exp2f(fmaf(p[t >> 1][8 * (t & 1) + x], scale, -ref));
        l += w[x];
      }
      pf[t].half[0] = pack4_bf16(w[0], w[1], w[2], w[3]);
      pf[t].half[1] = pack4_bf16(w[4], w[5], w[6], w[7]);
    }
  }
  // Operand of step i: in turn of the values (V^T, 32 columns e of 16 keys) and of the scores (K, 16 columns e of 32 keys)
  template <int NB> __device__ __forceinline__ Frag operand(const unsigned char* v_rows, const unsigned char* k_rows, int i, int lane) const {
    const int r32 = lane & 31, half = lane >> 5, r16 = lane & 15, n = i >> 1;
    Frag f;
    if (i & 1) {
      const int krow = 16 * (r32 >> 4) + 8 * ((r32 >> 2) & 1) + 4 * ((r32 >> 3) & 1) + (r32 & 3), kb = n % NB, ks = n / NB;
      f.nat = *(const u32x4_t*)(k_rows + (kb * 32 + krow) * (HD * 2) + wide_k_place<HD>(krow, 2 * ks + half));
    } else {
      const int eb = n % EB, t = n / EB;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = 8 * half + 4 * h + (r16 >> 2);
        const unsigned char* at = v_rows + (16 * t + row) * (HD * 2) + v_place<HD>(row, eb * 2 + ((lane >> 4) & 1)) + (r16 & 3) * 8;
        const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)at);
        f.half[h] = *(const uint2*)&x;
      }
    }
    return f;
  }
  // The values of one tile and the scores of the next, step by step in turn (independent sums between dependent ones), the operands of
  // AHEAD steps on their way from LDS: left to itself the compiler asks for two and waits for them (four to twelve: the same time)
  template <int NB>
  __device__ __forceinline__ void advance(const unsigned char* v_rows, const unsigned char* k_rows, const Frag (&pf)[2 * NB], float (&p)[NB][16],
                                          int lane) {
    constexpr int STEPS = 2 * KS * NB, AHEAD = 8;
    floatx16_t s[NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) s[kb][x] = 0.f;
    Frag ring[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ring[i] = operand<NB>(v_rows, k_rows, i, lane);
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD / 2 * 3, 0);          // LDS reads
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int n = i >> 1;
      if (i & 1) s[n % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % AHEAD].v, q[n / NB].v, s[n % NB], 0, 0, 0);
      else o[n % EB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % AHEAD].v, pf[n / EB].v, o[n % EB], 0, 0, 0);
      if (i + AHEAD < STEPS) ring[i % AHEAD] = operand<NB>(v_rows, k_rows, i + AHEAD, lane);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                    // a matrix instruction
      if (i + AHEAD < STEPS) {
        if (i & 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        else __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
    }
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) p[kb][x] = s[kb][x];
  }
  // The values of keys j0 .. j1 - 1 that are no numbers, to the columns that see them: rare, key by key
  __device__ __forceinline__ void add_odd_values(const AttnRows& a, const SeqSpan& sp, const PageView& in, int j0, int j1, int half) {
    for (; j0 < j1; j0 += 64) {
      const uint64_t there = in.there_at(j0), vis = seen_bits(mask_of(a, sp, row), sp, row, j0, there);
#pragma unroll 1
      for (int k = 0; k < 64 && j0 + k < j1; ++k) {
        if (!(there >> k & 1)) continue;
        const char* values = in.value_row(j0 + k, HD) + half * 8;
#pragma unroll
        for (int x = 0; x < EB * 4; ++x)                   // e = eb * 32 + 8 a4 + 4 half + i
          add_odd(values + x * 16, [&](int i, float v) __attribute__((always_inline)) {
            if (vis >> k & 1) o[x >> 2][(x & 3) * 4 + i] += v;
          });
      }
    }
  }
};
}  // namespace

// 64 x 16 bytes from `base` + off (a lane's own) to 1 KiB of LDS at `to`.  Written out because a read of LDS behind such a load, wherever it
// goes, makes the compiler wait for it; this way the waits are those of wait_then_barrier.  The load writes no register.
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(to) : "memory", "m0");
}
__device__ __forceinline__ void wait_then_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }

// Columns by the hundred.  Trees of 64 rows of 8 sequences of 400 to 4096 positions, 64 query and 8 key/value heads of 128: 59 us and 8 to 11
// for the join, 32 GFLOP; all of 4096 100 with the join, 0.69 PFLOP/s of the 1.3 that a large matrix product gets.  The exponentials take as long as
// a third of the products, and the compute units slow down under both (1.6 to 1.7 GHz in long runs).
// Four wavefronts, two workgroups to a compute unit.  A tile has two halves: the softmax (vector units), and the values of the tile with
// the scores of the next (matrix units, operands from LDS); the other workgroup is somewhere else in its tiles, so both kinds of unit
// have work.  K and V come straight to LDS, two stages of each, asked for behind barrier t (K of tile t + 2 and V of t + 1, where K of t and
// V of t - 1 were: read in front of it) and waited for in front of barrier t + 1.
template <int HD>
__global__ __launch_bounds__(256, 2) void paged_attn_wide_kernel(PagedRows b, AttnRows a, int least, float* part_o, float* part_ml, PartNote* notes) {
  using Cols = WideColumns<HD>;
  constexpr int EB = Cols::EB, TILE = 64 * HD * 2, COLS = 128, PIECES = HD / 8, ROWS = 64 / PIECES, PASS = 4 * ROWS, LOADS = 64 / PASS;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * TILE];   // K, K, V, V
  __shared__ uint64_t masks[COLS][kMaskWords];                             // of the item's rows
  __shared__ int odd, missing_from;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = a.Hq / b.Hkv;
  Part sl;
  const bool any = part_of_workgroup<COLS>(b, group, least, sl);
  leave_note(notes, least, any, sl);
  if (!any) return;
  {
    const int half = lane >> 5;
    const SeqSpan sp = sl.sp;
    const int wg_col0 = sl.col_tile * COLS;
    const bool works = wg_col0 + wave * 32 < sp.count * group;             // the others only bring tiles
    const PageView in(b, a, sp, sl.seq, sl.hk);
    const int tiles = (sl.key1 - sl.key0 + 63) / 64;

    // load i of a tile: rows i * PASS + wave * ROWS on, the lane's piece of its row where the swizzle wants it
    const int my_row = lane / PIECES, at = lane % PIECES;
    const uint32_t k_off = my_row * (HD * 2) + (wide_k_place<HD>(wave * ROWS + my_row, at));
    const uint32_t v_off = my_row * (HD * 2) + v_place<HD>(wave * ROWS + my_row, at >> 1) + (at & 1) * 16;
    const uint32_t lds0 = lds_address(lds) + wave * 1024;
    auto pages = [&](int (&x)[LOADS], int tile) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int id = in.page_at(sl.key0 + 64 * tile + i * PASS + wave * ROWS);
        x[i] = (unsigned)id < (unsigned)in.n_pages ? id : 0;
      }
    };
    auto ask = [&](const char* pool, uint32_t off, int tile, const int (&id)[LOADS], uint32_t to) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int slot = sl.key0 + 64 * tile + i * PASS + wave * ROWS;
        load_to_lds(pool + id[i] * in.page_bytes + (size_t)(slot & ((1 << in.shift) - 1)) * (HD * 2), off, to + i * 4096);
      }
    };
    int id1[LOADS], id2[LOADS];                            // pages of tiles t + 1, t + 2
    {
      int id0[LOADS];
      pages(id0, 0);
      pages(id1, 1);
      pages(id2, 2);
      ask(in.kp, k_off, 0, id0, lds0);
      if (tiles > 1) ask(in.kp, k_off, 1, id1, lds0 + TILE);
      ask(in.vp, v_off, 0, id0, lds0 + 2 * TILE);
    }
    Cols cols;
    cols.start(a, sp, sl.hk, group, wg_col0 + wave * 32 + (lane & 31), half);
    const int row0 = wg_col0 / group;
    if (threadIdx.x == 0) odd = 0, missing_from = INT32_MAX;
    // what is read once: the rows' masks, and whether pages are missing; requested together
    const int mask_words = !a.anc || sl.key1 <= sp.n ? 0 : (sp.count - row0 < COLS ? sp.count - row0 : COLS) * kMaskWords;
    uint64_t mask_word[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int w = threadIdx.x + 256 * i;
      mask_word[i] = w < mask_words ? a.anc[(size_t)(sp.row0 + row0) * kMaskWords + w] : 0ull;
    }
    const int page0 = sl.key0 >> in.shift, page1 = (sl.key1 - 1) >> in.shift;
    int missing = INT32_MAX;
    for (int i = page0 + threadIdx.x; i <= page1; i += 256)
      if ((unsigned)in.table[i] >= (unsigned)in.n_pages && i < missing) missing = i;
    wait_then_barrier();                                   // (odd, missing_from are set)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if ((int)threadIdx.x + 256 * i < mask_words) ((uint64_t*)masks)[threadIdx.x + 256 * i] = mask_word[i];
    if (missing != INT32_MAX) atomicMin(&missing_from, missing);
    cols.arrived();
    wait_then_barrier();
    // tiles in front that every column sees whole
    const int gap = __builtin_amdgcn_readfirstlane(missing_from);
    int whole = sp.n > sl.key0 ? (sp.n - sl.key0) / 64 : 0;
    whole = whole < tiles ? whole : tiles;
    if (gap != INT32_MAX) {
      const int slot = gap << in.shift, first = slot > sl.key0 ? (slot - sl.key0) / 64 : 0;
      whole = first < whole ? first : whole;
    }
    float p[2][16];
    Frag pf[4];
    if (works) cols.template scores<2>(lds, p, lane);
    auto step = [&](auto masked, int t) __attribute__((always_inline)) {
      constexpr bool MASKED = decltype(masked)::value;
      const int j0 = sl.key0 + 64 * t;
      const uint64_t there = !MASKED ? ~0ull : gap != INT32_MAX ? in.there_at(j0) : in.up_to_end(j0);
      if (works) {
        uint64_t vis = 0;
        if (MASKED) vis = seen_bits(a.anc ? masks[cols.row < sp.count ? cols.row - row0 : 0] : nullptr, sp, cols.row, j0, there);
        cols.template soften<MASKED, 2>(p, pf, vis, a.scale_log2, lane);
      }
      wait_then_barrier();
      if (t + 2 < tiles) ask(in.kp, k_off, t + 2, id2, lds0 + (t & 1) * TILE);
      if (t + 1 < tiles) ask(in.vp, v_off, t + 1, id1, lds0 + (2 + ((t + 1) & 1)) * TILE);
#pragma unroll
      for (int i = 0; i < LOADS; ++i) id1[i] = id2[i];
      pages(id2, t + 3);
      unsigned char* v_rows = lds + (2 + (t & 1)) * TILE;
      if (MASKED) {
        // values of keys that are not there become 0 (0 times what lies there is no 0), and those that are no numbers, for add_odd
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          u32x4_t* at_lds = (u32x4_t*)(v_rows + i * 4096 + wave * 1024 + lane * 16);
          u32x4_t x = *at_lds;
          if (!(there >> (i * PASS + wave * ROWS + lane / PIECES) & 1)) x = u32x4_t{0, 0, 0, 0};
          if (tidy(x)) odd = 1;
          *at_lds = x;
        }
        __syncthreads();
      }
      // (scores of a tile past the slice's last are nobody's)
      if (works) cols.template advance<2>(v_rows, lds + ((t + 1) & 1) * TILE, pf, p, lane);
    };
    int t = 0;
    for (; t < whole; ++t) step(std::false_type{}, t);
    for (; t < tiles; ++t) step(std::true_type{}, t);
    if (works && odd) cols.add_odd_values(a, sp, in, sl.key0 + 64 * whole, sl.key1, half);

    auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(cols.l), __float_as_uint(cols.l), false, false);
    const float sum = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    const bool partial = sl.parts > 1;
    const float factor = partial ? 1.0f : sum == 0.f ? 0.f : 1.0f / sum;
    // through LDS, so that a column's row is stored in one piece; 16-byte pieces of a column's HD floats, swizzled by the column
    __syncthreads();
    floatx4_t* rows = (floatx4_t*)lds + wave * 32 * (HD / 4);
    const int r32 = lane & 31;
    constexpr int QUADS = HD / 4, PER = 64 / QUADS;        // columns an instruction stores
    if (works) {
#pragma unroll
      for (int x = 0; x < EB * 4; ++x) {
        floatx4_t y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = sum == 0.f ? 0.f : cols.o[x >> 2][(x & 3) * 4 + i] * factor;
        rows[r32 * QUADS + ((2 * x + half) ^ (r32 & (QUADS - 1)))] = y;
      }
      if (partial && half == 0) *(float2*)(part_ml + ((size_t)sl.place * COLS + wave * 32 + r32) * 2) = make_float2(cols.m, sum);
#pragma unroll 4
      for (int i = 0; i < 32 / PER; ++i) {
        const int c = i * PER + lane / QUADS, quad = lane % QUADS, col = wg_col0 + wave * 32 + c, row = col / group;
        const floatx4_t y = rows[c * QUADS + (quad ^ (c & (QUADS - 1)))];
        if (partial) {
          *(floatx4_t*)(part_o + ((size_t)sl.place * COLS + wave * 32 + c) * HD + quad * 4) = y;
        } else if (row < sp.count) {
          bf16_t* out = (bf16_t*)a.out + (int64_t)(sp.row0 + row) * a.out_stride + (int64_t)(sl.hk * group + col % group) * HD + quad * 4;
          ((Loose8*)out)->v = pack4_bf16(y[0], y[1], y[2], y[3]);
        }
      }
    }
  }
}

// float32, heads of 64 and 128: the same products on the 16 x 16 x 4 instructions, 16 columns to a workgroup, whose four wavefronts take
// blocks of 16 keys in turn.  Every operand is loaded 16 bytes at a time straight into registers, because the contraction may run
// in any order and the rows of a product may stand for any e:
//   scores  lane (r16, g) holds K[r16][16 j + 4 g + i] and Q[r16][16 j + 4 g + i], i the step of four
//   values  lane (r16, g) holds V[4 g + i][64 j + 4 r16 + x] and, from the scores, P[4 g + i]: x picks which quarter of the e a product has
// One row of each of 32 sequences of 2000, 8 heads of 128: 100 us (5.2 TB/s); 64 rows of 8 sequences: 72 us, 4 GFLOP, every
// 16 columns reading the cache for themselves (from L2); trees of 8 of 8 sequences of up to 190: 8 us, the chain of loads.
template <int HD>
__global__ __launch_bounds__(256) void paged_attn_f32_kernel(PagedRows b, AttnRows a, int split_len, int col_tiles, float* part_o, float* part_ml) {
  constexpr int KJ = HD / 16, VJ = HD / 64, STEP = 4 * 16;
  __shared__ floatx4_t lds_o[4][VJ * 4][64];
  __shared__ float lds_m[4][64], lds_l[4][64];
  const int seq = blockIdx.z, hk = blockIdx.x, group = a.Hq / b.Hkv, split = blockIdx.y / col_tiles, col0 = blockIdx.y % col_tiles * 16;
  const SeqSpan sp = seq_span(b, seq);
  const Slice sl = slice_of(sp, split, split_len);
  if (col0 >= sp.count * group || sl.key0 >= sl.key1) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
  const int S = sp.n + sp.count, in_page = (1 << b.page_shift) - 1;
  const size_t page_elems = (size_t)b.Hkv * HD << b.page_shift, head_elems = (size_t)hk * HD << b.page_shift;
  const int32_t* table = b.table + (size_t)seq * b.table_width;
  const float *kp = (const float*)a.k_pages + head_elems, *vp = (const float*)a.v_pages + head_elems;
  const int col = col0 + r16, row = col / group, head = hk * group + col % group, row_here = row < sp.count ? row : sp.count - 1;
  const uint64_t* mask = mask_of(a, sp, row);
  struct __attribute__((packed, aligned(4))) Four {
    floatx4_t v;
  };

  floatx4_t q[KJ], o[VJ][4];
  const float* src = (const float*)a.q + (int64_t)(sp.row0 + row_here) * a.q_stride + (int64_t)head * HD + g * 4;
#pragma unroll
  for (int j = 0; j < KJ; ++j) q[j] = ((const Four*)(src + j * 16))->v;
#pragma unroll
  for (int j = 0; j < VJ; ++j)
#pragma unroll
    for (int x = 0; x < 4; ++x) o[j][x] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  auto page = [&](int slot) __attribute__((always_inline)) { return table[(slot < S ? slot : S - 1) >> b.page_shift]; };
  floatx4_t kf[KJ], vf[4][VJ], kn[KJ], vn[4][VJ];
  auto load = [&](floatx4_t (&k)[KJ], floatx4_t (&v)[4][VJ], int j0, int kid, int vid) __attribute__((always_inline)) {
    const float* krow = kp + ((unsigned)kid < (unsigned)b.n_pages ? kid : 0) * page_elems + (size_t)((j0 + r16) & in_page) * HD + g * 4;
    const float* vrow = vp + ((unsigned)vid < (unsigned)b.n_pages ? vid : 0) * page_elems + (size_t)((j0 + 4 * g) & in_page) * HD + r16 * 4;
#pragma unroll
    for (int j = 0; j < KJ; ++j) k[j] = ((const Four*)(krow + j * 16))->v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < VJ; ++j) v[i][j] = ((const Four*)(vrow + i * HD + j * 64))->v;
  };
  int j0 = sl.key0 + wave * 16;
  if (j0 < sl.key1) {
    int kid = page(j0 + r16), vid = page(j0 + 4 * g), kid_next = page(j0 + STEP + r16), vid_next = page(j0 + STEP + 4 * g);
    load(kf, vf, j0, kid, vid);
    for (; j0 < sl.key1; j0 += STEP) {
      const int kid_after = page(j0 + 2 * STEP + r16), vid_after = page(j0 + 2 * STEP + 4 * g);
      if (j0 + STEP < sl.key1) load(kn, vn, j0 + STEP, kid_next, vid_next);
      // keys that are there; bit 0 is key j0
      uint32_t there = (uint32_t)__ballot((unsigned)kid < (unsigned)b.n_pages && j0 + r16 < S) & 0xffffu;
      const bool masked = there != 0xffffu || j0 + 16 > sp.n;
      bool odd = false;
      if (masked) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < VJ; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const bool here = there >> (4 * g + i) & 1, number = fabsf(vf[i][j][x]) < INFINITY;
              odd |= here && !number;
              vf[i][j][x] = here && number ? vf[i][j][x] : 0.f;
            }
      }
      floatx4_t s = floatx4_t{0.f, 0.f, 0.f, 0.f}, s2 = s;               // two sums: one would wait for itself
#pragma unroll
      for (int j = 0; j < KJ; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i & 1) s2 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j][i], q[j][i], s2, 0, 0, 0);
          else s = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j][i], q[j][i], s, 0, 0, 0);
        }
      s += s2;
      uint32_t vis = 0;
      if (masked) {
        vis = (uint32_t)seen_bits(mask, sp, row, j0, there);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = vis >> (4 * g + i) & 1 ? s[i] : -INFINITY;
      }
      const float best = max_over_groups(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))) * a.scale_log2, now = fmaxf(m, best);
      const float ref = now == -INFINITY ? 0.f : now, keep = exp2f(m - ref);
      m = now;
      if (__any(keep != 1.0f)) {
        l *= keep;
#pragma unroll
        for (int j = 0; j < VJ; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[j][x] *= keep;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[i] = exp2f(fmaf(s[i], a.scale_log2, -ref));
        l += s[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < VJ; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[j][x] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i][j][x], s[i], o[j][x], 0, 0, 0);
      if (masked && __any(odd)) {                          // values that are no numbers, to the columns that see them: rare
#pragma unroll 1
        for (int key = 0; key < 16; ++key) {
          if (!(there >> key & 1)) continue;
          const int slot = j0 + key;
          const float* v = vp + page(slot) * page_elems + (size_t)(slot & in_page) * HD + g * 16;
#pragma unroll
          for (int j = 0; j < VJ; ++j)
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const float z = v[j * 64 + 4 * y + x];
                if (!(fabsf(z) < INFINITY) && (vis >> key & 1)) o[j][x][y] += z;
              }
        }
      }
#pragma unroll
      for (int j = 0; j < KJ; ++j) kf[j] = kn[j];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < VJ; ++j) vf[i][j] = vn[i][j];
      kid = kid_next, vid = vid_next, kid_next = kid_after, vid_next = vid_after;
    }
  }

  // ---- join the wavefronts
  lds_m[wave][lane] = m;
  lds_l[wave][lane] = sum_over_groups(l);
#pragma unroll
  for (int j = 0; j < VJ; ++j)
#pragma unroll
    for (int x = 0; x < 4; ++x) lds_o[wave][j * 4 + x][lane] = o[j][x];
  __syncthreads();
  float top = -INFINITY, f[4], sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, lds_m[w][lane]);
  const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = exp2f(lds_m[w][lane] - ref);
    sum = fmaf(f[w], lds_l[w][lane], sum);
  }
  if (row >= sp.count) return;
  const size_t at = (size_t)(sp.row0 + row) * a.Hq + head, rows = (size_t)b.rows * a.Hq;
  // wavefront y: e = 64 j + 16 g + 4 y + x
#pragma unroll
  for (int j = 0; j < VJ; ++j) {
    floatx4_t acc = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[x] = fmaf(f[w], lds_o[w][j * 4 + x][lane][wave], acc[x]);
    const int e0 = j * 64 + g * 16 + wave * 4;
    if (sl.count > 1) *(floatx4_t*)(part_o + (split * rows + at) * HD + e0) = acc;
    else store_four((float*)a.out + (int64_t)(sp.row0 + row) * a.out_stride + (int64_t)head * HD + e0, acc, sum);
  }
  if (sl.count > 1 && wave == 0 && g == 0) *(float2*)(part_ml + (split * rows + at) * 2) = make_float2(top, sum);
}

// out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s over the slices of a sequence, in a fixed order.  A workgroup per (row, head) and
// up to PARTS groups of HD / 4 threads that take every PARTS-th slice, four elements a thread; their sums meet in LDS.
template <typename T, int HD, int PARTS>
__global__ __launch_bounds__(PARTS * (HD / 4)) void paged_attn_join_kernel(PagedRows b, AttnRows a, int split_len, const float* part_o,
                                                                          const float* part_ml) {
  constexpr int QUADS = HD / 4;
  const SeqSpan sp = seq_span(b, blockIdx.z);
  const int count = slice_of(sp, 0, split_len).count, row = blockIdx.y, head = blockIdx.x;
  if (count <= 1 || row >= sp.count) return;
  const int part = threadIdx.x / QUADS, e = threadIdx.x % QUADS * 4;
  const size_t rows = (size_t)b.rows * a.Hq, mine = (size_t)(sp.row0 + row) * a.Hq + head;
  __shared__ float lds_o[PARTS][HD];
  __shared__ float2 lds_ml[PARTS];
  float top = -INFINITY, sum = 0.f;
  floatx4_t acc = floatx4_t{0.f, 0.f, 0.f, 0.f};
  constexpr int NS = 4;                                    // slices requested at a time
  for (int s0 = part; s0 < count; s0 += NS * PARTS) {
    float2 ml[NS];
    floatx4_t x[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int s = s0 + i * PARTS < count ? s0 + i * PARTS : s0;
      ml[i] = *(const float2*)(part_ml + (s * rows + mine) * 2);
      x[i] = *(const floatx4_t*)(part_o + (s * rows + mine) * HD + e);
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      if (s0 + i * PARTS >= count) break;
      const float now = fmaxf(top, ml[i].x), ref = now == -INFINITY ? 0.f : now;
      const float old = __builtin_amdgcn_exp2f(top - ref), f = __builtin_amdgcn_exp2f(ml[i].x - ref);
      sum = fmaf(f, ml[i].y, sum * old);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] = fmaf(f, x[i][c], acc[c] * old);
      top = now;
    }
  }
  if constexpr (PARTS > 1) {
    *(floatx4_t*)&lds_o[part][e] = acc;
    if (e == 0) lds_ml[part] = make_float2(top, sum);
    __syncthreads();
    if (part) return;
    float all = -INFINITY;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) all = fmaxf(all, lds_ml[p].x);
    const float ref = all == -INFINITY ? 0.f : all;
    sum = 0.f;
    acc = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      const float f = __builtin_amdgcn_exp2f(lds_ml[p].x - ref);
      sum = fmaf(f, lds_ml[p].y, sum);
      const floatx4_t x = *(const floatx4_t*)&lds_o[p][e];
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] = fmaf(f, x[c], acc[c]);
    }
  }
  store_four((T*)a.out + (int64_t)(sp.row0 + row) * a.out_stride + (int64_t)head * HD + e, acc, sum);
}

// The same for shared-out work.  A workgroup per part; those of an item share the item's elements out among them, four elements to a
// unit, and where that leaves fewer units than threads, the threads share the parts.  Bound by the partial results' 34 MB at 512 parts of 128
// columns of 128 (8 to 11 us).
template <int HD, int COLS>
__global__ __launch_bounds__(256) void paged_attn_share_join_kernel(PagedRows b, AttnRows a, const float* part_o, const float* part_ml,
                                                                   const PartNote* notes) {
  const PartNote n = notes[blockIdx.x];
  if (n.parts < 2) return;
  constexpr int T = HD / 4;
  const int tid = threadIdx.x, group = a.Hq / b.Hkv, left = n.count * group - n.col_tile * COLS;
  int lo, hi;
  even_share((left < COLS ? left : COLS) * T, n.parts, n.part, lo, hi);
  int width = 256, groups = 1;                             // units and shares of the parts at a time
  while (width / 2 >= hi - lo && width > 8) width /= 2, groups *= 2;
  const int share = tid / width;
  __shared__ floatx4_t lds_o[256];
  __shared__ float2 lds_ml[256];
  auto place = [&](int part) { return (size_t)(blockIdx.x - n.part + part) * COLS; };
  for (int u0 = lo; u0 < hi; u0 += width) {
    const int unit = u0 + tid % width, col = unit / T, e = unit % T * 4, c = n.col_tile * COLS + col, row = c / group;
    const bool in = unit < hi;
    float top = -INFINITY, sum = 0.f;
    floatx4_t acc = floatx4_t{0.f, 0.f, 0.f, 0.f};
    constexpr int NS = 4;                                  // requested at a time
    if (in)
      for (int p0 = share; p0 < n.parts; p0 += NS * groups) {
        float2 ml[NS];
        floatx4_t x[NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const size_t at = place(p0 + i * groups < n.parts ? p0 + i * groups : p0) + col;
          ml[i] = *(const float2*)(part_ml + at * 2);
          x[i] = *(const floatx4_t*)(part_o + at * HD + e);
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          if (p0 + i * groups >= n.parts) break;
          const float now = fmaxf(top, ml[i].x), ref = now == -INFINITY ? 0.f : now;
          const float old = __builtin_amdgcn_exp2f(top - ref), f = __builtin_amdgcn_exp2f(ml[i].x - ref);
          sum = fmaf(f, ml[i].y, sum * old);
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[k] = fmaf(f, x[i][k], acc[k] * old);
          top = now;
        }
      }
    if (groups > 1) {
      __syncthreads();
      lds_o[tid] = acc;
      lds_ml[tid] = make_float2(top, sum);
      __syncthreads();
      if (share == 0)
        for (int i = 1; i < groups; ++i) {
          const float2 ml = lds_ml[tid + i * width];
          const floatx4_t x = lds_o[tid + i * width];
          const float now = fmaxf(top, ml.x), ref = now == -INFINITY ? 0.f : now;
          const float old = __builtin_amdgcn_exp2f(top - ref), f = __builtin_amdgcn_exp2f(ml.x - ref);
          sum = fmaf(f, ml.y, sum * old);
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[k] = fmaf(f, x[k], acc[k] * old);
          top = now;
        }
    }
    if (!in || share) continue;
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    ((Loose8*)((bf16_t*)a.out + (int64_t)(n.row0 + row) * a.out_stride + (int64_t)(n.hk * group + c % group) * HD + e))->v =
        sum == 0.f ? make_uint2(0, 0) : pack4_bf16(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
  }
}

namespace {
// How a call runs: from its bounds alone, so that a captured call fits whatever its tables say later
struct AttnPlan {
  bool simple, f32, slices;
  int blocks, split_len, splits;  // slices: column blocks of 16 (a workgroup each), slices of a sequence
  int cols, workgroups, least;    // parts: columns of an item, workgroups (0: one to an item), the least tiles of one
};
AttnPlan attn_plan(int dtype, const PagedRows& b, int Hq) {
  AttnPlan p{};
  const int cols = b.max_rows * (Hq / b.Hkv), S = b.max_len + b.max_rows;
  p.simple = b.hd != 64 && b.hd != 128;
  if (p.simple) return p;
  p.f32 = dtype == 0;
  // up to 16 columns: 8 of 8 x 4096 slots 27 us, in parts on the next kernel 30; of 4 x 500 10 and 14 (ragged 32 x 4096: 58 and 54)
  p.slices = p.f32 || cols <= 16;
  if (p.slices) {
    p.blocks = (cols + 15) / 16;
    const int64_t groups = (int64_t)b.seqs * b.Hkv * p.blocks;
    // slices that all run at once, two workgroups to a compute unit (64 x 4096 slots, 8 heads: 1024 slices 195 us, 512 190; 1 x 100003: 83, 79),
    // and of float32, whose workgroups hold less, four; not below 256 slots, where the join costs what the slice saves (1 x 2000: 128 slots
    // 13.5 us, 256 11.9; float32 8 x 2000: 13.0, 12.2, 512 slots 17.9)
    const int least = 256;
    int64_t splits = p.f32 ? (1024 + groups - 1) / groups : 512 / groups;
    if (splits > S / least) splits = S / least;
    if (splits < 1) splits = 1;
    p.split_len = (int)(((S + splits - 1) / splits + 63) / 64 * 64);
    p.splits = (S + p.split_len - 1) / p.split_len;
    return p;
  }
  // 64 columns of 8 x 4096 slots: 35 us, on the kernel for more 38; of 4 x 500 18 and 22
  p.cols = cols <= 64 ? 64 : 128;
  // two workgroups to a compute unit (64-node trees of 8 ragged sequences: 512 of them 70 us, 1024 83, 256 113); a grid that holds every item,
  // or an item to a workgroup where there are many or the keys are few
  const int64_t items = (int64_t)b.seqs * b.Hkv * ((cols + p.cols - 1) / p.cols), tiles = (S + 63) / 64;
  if (b.seqs <= kShareSeqs && items <= 1024 && items * (tiles + kItemTiles) < 1 << 30 && tiles > 8) {
    p.least = 8;                                           // (one tree over 30000: 8 tiles 95 us, 4 95, 16 100; two over 1000: 34, 37, 41)
    p.workgroups = items <= 512 ? 512 : 1024;
    p.workgroups -= p.workgroups % b.Hkv;                  // (every head has room for its items: Hkv <= items)
    const int64_t most = items * ((tiles + kItemTiles + p.least - 1) / p.least);       // parts
    if (p.workgroups > most) p.workgroups = (int)most;
  }
  return p;
}
size_t part_columns(const AttnPlan& p, const PagedRows& b, int Hq) {        // columns of partial results
  return p.slices ? p.splits > 1 ? (size_t)p.splits * b.rows * Hq : 0 : (size_t)p.workgroups * p.cols;
}
template <int HD>
hipError_t launch_attn_hd(const AttnPlan& p, const PagedRows& b, const AttnRows& a, float* part_o, float* part_ml, PartNote* notes, hipStream_t s) {
  if (p.slices) {
    const dim3 grid(b.Hkv, p.splits * p.blocks, b.seqs);
    if (p.f32) hipLaunchKernelGGL(paged_attn_f32_kernel<HD>, grid, dim3(256), 0, s, b, a, p.split_len, p.blocks, part_o, part_ml);
    else hipLaunchKernelGGL(paged_attn_few_kernel<HD>, grid, dim3(256), 0, s, b, a, p.split_len, part_o, part_ml);
    if (p.splits > 1) {
      const bool many = p.splits > 4;
      auto j = p.f32 ? (many ? paged_attn_join_kernel<float, HD, 16> : paged_attn_join_kernel<float, HD, 1>)
                     : (many ? paged_attn_join_kernel<bf16_t, HD, 16> : paged_attn_join_kernel<bf16_t, HD, 1>);
      hipLaunchKernelGGL(j, dim3(a.Hq, b.max_rows, b.seqs), dim3((many ? 16 : 1) * HD / 4), 0, s, b, a, p.split_len, part_o, part_ml);
    }
    return hipGetLastError();
  }
  const int cols = b.max_rows * (a.Hq / b.Hkv);
  const dim3 grid = p.workgroups ? dim3(p.workgroups) : dim3(b.Hkv, (cols + p.cols - 1) / p.cols, b.seqs);
  auto f = p.cols == 64 ? paged_attn_tile_kernel<HD> : paged_attn_wide_kernel<HD>;
  hipLaunchKernelGGL(f, grid, dim3(256), 0, s, b, a, p.least, part_o, part_ml, notes);
  if (p.workgroups) {
    auto j = p.cols == 64 ? paged_attn_share_join_kernel<HD, 64> : paged_attn_share_join_kernel<HD, 128>;
    hipLaunchKernelGGL(j, dim3(p.workgroups), dim3(256), 0, s, b, a, part_o, part_ml, notes);
  }
  return hipGetLastError();
}
}  // namespace

size_t paged_attn_scratch_bytes(int dtype, const PagedRows& b, int Hq) {
  const AttnPlan p = attn_plan(dtype, b, Hq);
  return part_columns(p, b, Hq) * (b.hd + 2) * sizeof(float) + (size_t)p.workgroups * sizeof(PartNote);
}

hipError_t launch_paged_attn(int dtype, const PagedRows& b, const AttnRows& a, void* scratch, hipStream_t s) {
  const AttnPlan p = attn_plan(dtype, b, a.Hq);
  if (p.simple) {
    const dim3 grid(a.Hq, b.max_rows, b.seqs);
    // few heads and rows: sixteen wavefronts over the keys (64 of them: 29 us, with four 82); many: four, of which more fit a compute
    // unit (1024: 99 us, with sixteen 111; 4096: 310, with sixteen 500)
    const bool many = (int64_t)a.Hq * b.max_rows * b.seqs > 512;
    if (dtype == 0) {
      auto f = many ? paged_attn_simple_kernel<float, 4> : paged_attn_simple_kernel<float, 16>;
      hipLaunchKernelGGL(f, grid, dim3(many ? 256 : 1024), 0, s, b, a);
    } else {
      auto f = many ? paged_attn_simple_kernel<bf16_t, 4> : paged_attn_simple_kernel<bf16_t, 16>;
      hipLaunchKernelGGL(f, grid, dim3(many ? 256 : 1024), 0, s, b, a);
    }
    return hipGetLastError();
  }
  float* part_o = (float*)scratch;
  float* part_ml = part_o + part_columns(p, b, a.Hq) * b.hd;
  PartNote* notes = (PartNote*)(part_ml + part_columns(p, b, a.Hq) * 2);
  return b.hd == 64 ? launch_attn_hd<64>(p, b, a, part_o, part_ml, notes, s) : launch_attn_hd<128>(p, b, a, part_o, part_ml, notes, s);
}

}  // namespace ht
