// One token per row of logits, drawn with a given number u from the row's distribution after temperature, top-k, top-p and min-p.
//
//   e_i = exp((x_i - max x) / T)                               (1 at the maximum, 0 at -inf and NaN)
//   order: x descending, index ascending.  Each filter keeps a prefix of it: the first k; the shortest prefix of those whose mass
//   is at least p times theirs; those with e_i >= min_p.
//   token: the first i in index order whose running sum of the kept e exceeds u times their total
//
// Exponentials and sums are in 64 bits: the token must not hang on how a sum was split, and with 32 bits some row in a thousand
// of an unfiltered vocabulary falls on the other side of a border.
//
// A workgroup of 1024 threads per row, which goes over it a few times; all but the first come from L2.  (Held in registers, with every
// pass unrolled over them, the passes' own needs went to scratch memory.)  A prefix of the order ends at one element (value, index),
// so a filter is a search for that element, not a sort of the row:
//   top-k    the k-th largest of the 1024 threads' maxima is no larger than the k-th largest value, so the elements from there on hold
//            the first k; they are a few more than k, are listed and sorted, and top-p, min-p and the draw work on the list.  A larger
//            k up to 1024 is searched for as below by counts, and what it kept is listed then.
//   top-p alone, or a k that makes the list too long: a histogram of masses (or counts) over 2048 equal steps of the value finds the
//            step that holds the end, whose elements are listed and ranked; a step that holds too many becomes the next
//            histogram's range (a value far below the others, as masks leave, costs such a round).  Its masses are counted in whole
//            2^-43: sums of integers do not depend on the order of the atomics.
#include "ht_common.h"

namespace ht {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048, kList = 1024;
constexpr int kRoots = 32;                   // as many as fill the banks of LDS once: lanes on different entries do not conflict
constexpr double kNothing = 1e-300;          // e up to here is an exponential's zero
constexpr int kShort = 256;                  // list lengths whose order is counted out, not sorted: a sort's steps wait for each other

template <typename T> struct Vec16;
template <> struct Vec16<float> {
  static constexpr int N = 4;
};
template <> struct Vec16<bf16_t> {
  static constexpr int N = 8;
};
// 16 bytes from any address of the element's alignment (rows of an odd vocabulary)
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Loose16 {
  T v[Vec16<T>::N];
};
// value c of a piece held in four registers
template <typename T> __device__ inline float value_of(const uint32_t (&w)[4], int c);
template <> __device__ inline float value_of<float>(const uint32_t (&w)[4], int c) { return __uint_as_float(w[c]); }
template <> __device__ inline float value_of<bf16_t>(const uint32_t (&w)[4], int c) {
  return __uint_as_float(c & 1 ? w[c >> 1] & 0xffff0000u : w[c >> 1] << 16);
}

struct Found {
  double before, total;                      // draw: sum in front of the segment, and of all
  unsigned long long above;                  // search: weight above the crossing step
  uint32_t lo, hi;                           // search: its elements' range, as ordered keys
  int32_t bin, listed, index, seg;
};

__device__ inline uint32_t ordered(float v) {
  const uint32_t u = __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float of_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// exp of -1 <= y <= 0, for the table: the series to y^19 (the first term left out is 4e-19)
__device__ inline double exp_series(double y) {
  double e = 1.0;
#pragma unroll
  for (int i = 19; i >= 1; --i) e = fma(e, y * (1.0 / i), 1.0);
  return e;
}

// The value of lane ^ STRIDE by moves that need no LDS
template <int CTRL> __device__ inline uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false); }
template <int STRIDE> __device__ inline uint32_t of_partner(uint32_t v) {
  if constexpr (STRIDE == 1) return dpp<0xb1>(v);          // quads 1 0 3 2
  if constexpr (STRIDE == 2) return dpp<0x4e>(v);          // quads 2 3 0 1
  if constexpr (STRIDE == 4) return dpp<0x1b>(dpp<0x141>(v));          // mirrored halves of a row (^ 7), then mirrored quads (^ 3)
  if constexpr (STRIDE == 8) return dpp<0x128>(v);         // rows turned by 8
  if constexpr (STRIDE == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);         // (rows 0 0 2 2, rows 1 1 3 3)
    return threadIdx.x & 16 ? r[0] : r[1];
  }
  if constexpr (STRIDE == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  }
}
// A step of a bitonic sort between lanes STRIDE apart
template <int STRIDE> __device__ inline void sort_step(unsigned long long& key, bool up) {
  const unsigned long long other = (unsigned long long)of_partner<STRIDE>((uint32_t)(key >> 32)) << 32 | of_partner<STRIDE>((uint32_t)key);
  const bool first = (threadIdx.x & STRIDE) == 0;
  key = (other < key) == (up == first) ? other : key;
}

// Sums and extremes over a wavefront by DPP moves: lane 63 ends with all (a lane that has no partner takes `none`)
template <int CTRL, int ROWS, typename V> __device__ inline V moved(V v, V none) {
  if constexpr (sizeof(V) == 4) {
    const int r = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(V, r);
  } else {
    const uint64_t n = __builtin_bit_cast(uint64_t, none), u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp((int)n, (int)u, CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp((int)(n >> 32), (int)(u >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(V, (uint64_t)hi << 32 | lo);
  }
}
template <typename V> __device__ inline V lane_of(V v, int lane) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(V, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)u, lane));
  }
}
// Running over the lanes: lane l ends with f of lanes 0 .. l
template <typename V, typename F> __device__ inline V wave_run(V v, V none, F f) {
  v = f(moved<0x111, 0xf>(v, none), v);      // row_shr 1, 2, 4, 8; the rows' ends to the rows behind
  v = f(moved<0x112, 0xf>(v, none), v);
  v = f(moved<0x114, 0xf>(v, none), v);
  v = f(moved<0x118, 0xf>(v, none), v);
  v = f(moved<0x142, 0xa>(v, none), v);
  v = f(moved<0x143, 0xc>(v, none), v);
  return v;
}
// ... over 16 values that repeat in every row of 16 lanes: lane 15 ends with all
template <typename V, typename F> __device__ inline V row_run(V v, V none, F f) {
  v = f(moved<0x111, 0xf>(v, none), v);
  v = f(moved<0x112, 0xf>(v, none), v);
  v = f(moved<0x114, 0xf>(v, none), v);
  v = f(moved<0x118, 0xf>(v, none), v);
  return v;
}

// lower half: a there plus a 32 lanes on, upper half: the same of b; and with rows of 16, odd rows of b
__device__ inline double fold_halves(double a, double b) {
  const uint64_t x = __builtin_bit_cast(uint64_t, a), y = __builtin_bit_cast(uint64_t, b);
  const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)y, false, false);
  const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(x >> 32), (uint32_t)(y >> 32), false, false);
  return __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
}
__device__ inline double fold_rows(double a, double b) {
  const uint64_t x = __builtin_bit_cast(uint64_t, a), y = __builtin_bit_cast(uint64_t, b);
  const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)y, false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(x >> 32), (uint32_t)(y >> 32), false, false);
  return __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
}

}  // namespace

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_rows_kernel(SampleRows a) {
  constexpr int VEC = Vec16<T>::N, STRIDE = kThreads * VEC, AHEAD = 4;
  // histogram and list of the search, or the segment sums of the draw
  __shared__ __attribute__((aligned(16))) unsigned char shared_mem[32768];
  unsigned long long* hist = (unsigned long long*)shared_mem;                    // [kBins]
  double* segs = (double*)shared_mem;                                            // [4096]
  unsigned long long* loose = (unsigned long long*)(shared_mem + 16384);         // [kList] the list before it is sorted
  uint32_t* by_index = (uint32_t*)(shared_mem + 8192);                           // [kShort] the kept ones in the order of their indices
  double* by_index_e = (double*)shared_mem;
  __shared__ unsigned long long keys[kList];                                     // the sorted list: order, then index
  __shared__ double shares[kList];                                               // ... and its e
  __shared__ double roots[kRoots];                                               // 2^(j / kRoots)
  __shared__ unsigned long long fold[2][kWaves];
  __shared__ Found found;

  const int row = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, V = a.V;
  const T* z = (const T*)a.z + (size_t)row * a.stride;
  const int chunks = (V + STRIDE - 1) / STRIDE;
  bool spike = false;                                      // the maximum is +inf: those tokens share everything

  auto plain = [&](float v) __attribute__((always_inline)) { return v == v ? v : -INFINITY; };       // NaN counts as -inf
  auto piece = [&](uint32_t (&w)[4], int j) __attribute__((always_inline)) {
    const int i0 = (j * kThreads + tid) * VEC;
    if (i0 + VEC <= V) {
      const Loose16<T> raw = *(const Loose16<T>*)(z + i0);
      __builtin_memcpy(w, &raw, 16);
    } else {
      T raw[VEC];
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        raw[c] = sizeof(T) == 4 ? (T)-INFINITY : (T)0xff80;
        if (i0 + c < V) raw[c] = z[i0 + c];
      }
      __builtin_memcpy(w, raw, 16);
    }
    if (spike) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (sizeof(T) == 4) {
          w[i] = w[i] == 0x7f800000u ? 0u : 0xff800000u;
        } else {
          w[i] = ((w[i] & 0xffffu) == 0x7f80u ? 0u : 0xff80u) | (w[i] >> 16 == 0x7f80u ? 0u : 0xff800000u);
        }
      }
    }
  };
  // f(chunk, values, first index), AHEAD pieces on their way at a time
  auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll 1
    for (int j0 = 0; j0 < chunks; j0 += AHEAD) {
      uint32_t w[AHEAD][4];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (j0 + i < chunks) piece(w[i], j0 + i);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (j0 + i < chunks) {
          float x[VEC];
#pragma unroll
          for (int c = 0; c < VEC; ++c) x[c] = plain(value_of<T>(w[i], c));
          f(j0 + i, x, ((j0 + i) * kThreads + tid) * VEC);
        }
    }
  };
  // over the workgroup, one barrier (the slots take turns, so the last fold's may still be read)
  int turn = 0;
  auto block_fold = [&](auto v, auto none, auto f) __attribute__((always_inline)) {
    using W = decltype(v);
    W* slots = (W*)fold[turn];
    turn ^= 1;
    v = wave_run<W>(v, none, f);
    if (lane == 63) slots[wave] = v;
    __syncthreads();
    return lane_of(row_run<W>(slots[lane & (kWaves - 1)], none, f), 15);
  };
  auto add = [](auto x, auto y) __attribute__((always_inline)) { return x + y; };
  auto larger = [](auto x, auto y) __attribute__((always_inline)) { return x > y ? x : y; };
  auto smaller = [](auto x, auto y) __attribute__((always_inline)) { return x < y ? x : y; };
  auto count = [&](int n) __attribute__((always_inline)) -> int { return block_fold(n, 0, add); };
  // sums up to every thread
  auto block_run = [&](auto v, auto none) __attribute__((always_inline)) {
    using W = decltype(v);
    W* slots = (W*)fold[turn];
    turn ^= 1;
    v = wave_run<W>(v, none, add);
    if (lane == 63) slots[wave] = v;
    __syncthreads();
    const W ends = row_run<W>(slots[lane & (kWaves - 1)], none, add);
    return wave ? v + lane_of(ends, wave - 1) : v;
  };

  if (tid < kRoots) roots[tid] = tid ? 2.0 * exp_series((tid - kRoots) * (0.69314718055994531 / kRoots)) : 1.0;
  float best = -INFINITY, low = INFINITY;                  // this thread's largest value, the smallest one
  each([&](int, const float(&x)[VEC], int) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
      best = fmaxf(best, x[c]);
      if (x[c] > -INFINITY) low = fminf(low, x[c]);
    }
  });
  float top = block_fold(best, -INFINITY, larger);
  if (top == -INFINITY) {                                  // nothing to draw from
    if (tid == 0) {
      a.tokens[row] = -1;
      if (a.logprob) a.logprob[row] = -INFINITY;
    }
    return;
  }
  const float temp = a.temperature ? a.temperature[row] : 1.0f;
  if (!(temp > 0.f)) {
    int first = INT32_MAX;
    if (best == top)
      each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int c = VEC - 1; c >= 0; --c)
          if (x[c] == top && i0 + c < first) first = i0 + c;
      });
    first = block_fold(first, INT32_MAX, smaller);
    if (tid == 0) {
      a.tokens[row] = first;
      if (a.logprob) a.logprob[row] = 0.f;
    }
    return;
  }
  if (top == INFINITY) {
    spike = true;
    best = best == INFINITY ? 0.f : -INFINITY;
    top = low = 0.f;
  }
  // e = 2^(y / 32), y = 32 (x - top) / (T ln 2) = n + f, |f| <= 1/2: a table for n modulo 32, a power of two, and the series of 2^(f / 32) to
  // f^5 (the first term left out is 2e-15).  y is 0 at the maximum and e is 1.  With the series of the whole exponential
  // to f^13 the pass over 32000 values of one row took 16 us, now 10
  const double steepness = kRoots / 0.69314718055994531 / (double)temp;
  auto energy = [&](float x) __attribute__((always_inline)) -> double {
    constexpr double c1 = 0.69314718055994531 / kRoots, c2 = c1 * c1 / 2, c3 = c1 * c1 * c1 / 6, c4 = c2 * c2 / 6, c5 = c2 * c3 / 10;
    // n as the low bits of y + 1.5 2^52, and the power of two added to the exponent: rounding, conversion and ldexp are slow instructions
    // n as the low bits of y + 1.5 2^52, and the power of two added to the exponent: a pass is bound by the instructions it issues.
    // Below 2^-1020 (at -inf too) e stays there, which no sum notices (kNothing)
    const double y = fmax(((double)x - (double)top) * steepness, -32.0 * 1020.0), t = y + 6755399441055744.0, f = y - (t - 6755399441055744.0);
    const uint32_t k = (uint32_t)__builtin_bit_cast(uint64_t, t);
    const double root = roots[k & (kRoots - 1)], e = fma(root, f * fma(f, fma(f, fma(f, fma(f, c5, c4), c3), c2), c1), root);
    const uint64_t bits = __builtin_bit_cast(uint64_t, e);
    return __builtin_bit_cast(double, (uint64_t)((uint32_t)(bits >> 32) + ((k & ~31u) << 15)) << 32 | (uint32_t)bits);
  };
  // in whole 2^-43, up to 2^20 of them in 64 bits: the mantissa's end of e + 512
  auto whole = [&](float x) __attribute__((always_inline)) -> unsigned long long {
    return (unsigned long long)__double_as_longlong(energy(x) + 512.0) - 0x4080000000000000ull;
  };

  float cut_x = -INFINITY;                                 // kept so far: what comes before or is (cut_x, cut_i)
  int cut_i = -1;
  auto kept = [&](float x, int i) __attribute__((always_inline)) { return (x > cut_x) | ((x == cut_x) & (i <= cut_i)); };

  // `loose` (n different ones) into `keys`, ascending
  auto sort_keys = [&](int n) __attribute__((always_inline)) {
    if (n <= kShort) {
      // four threads count a quarter of the list each for an element
      const int who = tid >> 2, part = tid & 3, whole_n = (n + 31) & ~31;
      if (tid >= n && tid < whole_n) loose[tid] = ~0ull;
      __syncthreads();
      const unsigned long long key = who < n ? loose[who] : 0;
      int rank = 0;
      for (int o = part; o < whole_n; o += 32) {
#pragma unroll
        for (int i = 0; i < 32; i += 4) rank += loose[o + i] < key;
      }
      rank += __shfl_xor(rank, 1, 64);
      rank += __shfl_xor(rank, 2, 64);
      if (who < n && part == 0) keys[rank] = key;
    } else {
      // bitonic, strides below 64 inside a wavefront
      int size = 512;
      while (size < n) size *= 2;
      unsigned long long key = tid < n ? loose[tid] : ~0ull;
      for (int half = 2; half <= size; half *= 2) {
        const bool up = (tid & half) == 0;
        for (int stride = half / 2; stride >= 64; stride /= 2) {
          __syncthreads();
          if (tid < size) keys[tid] = key;
          __syncthreads();
          const unsigned long long other = tid < size ? keys[tid ^ stride] : 0;
          const bool first = (tid & stride) == 0;
          key = (other < key) == (up == first) ? other : key;
        }
        if (wave * 64 >= size) continue;
        if (half > 32) sort_step<32>(key, up);
        if (half > 16) sort_step<16>(key, up);
        if (half > 8) sort_step<8>(key, up);
        if (half > 4) sort_step<4>(key, up);
        if (half > 2) sort_step<2>(key, up);
        sort_step<1>(key, up);
      }
      __syncthreads();
      if (tid < size) keys[tid] = key;
    }
    __syncthreads();
  };
  auto key_of = [&](float x, int i) __attribute__((always_inline)) { return (unsigned long long)~ordered(x + 0.0f) << 32 | (uint32_t)i; };      // (-0 ties with 0)
  auto cut_at = [&](int i) __attribute__((always_inline)) {
    cut_x = of_ordered(~(uint32_t)(keys[i] >> 32)), cut_i = (int)(uint32_t)keys[i];
  };

  // the element of the kept ones at which the running weight reaches `need` (at least 1), or a share of all the weight from lo on where
  // `share` is not negative, becomes the cut; none if it never does.  Elements above hi or below lo are left alone
  auto search = [&](auto weight, unsigned long long need, double share, float lo, float hi) __attribute__((always_inline)) {
    unsigned long long above = 0;
    for (;;) {
      if (lo == hi) {                                      // equal values: the lowest indices, as many as it takes
        const unsigned long long w = weight(hi);
        if (share >= 0.0) {
          int all = 0;
          each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < VEC; ++c) all += x[c] == hi && kept(x[c], i0 + c);
          });
          need = (unsigned long long)ceil(share * (double)((unsigned long long)count(all) * w));
          need = need ? need : 1;
        }
        const unsigned long long r = w ? (need - above + w - 1) / w : 1;
        int at = 0, end = V;                               // smallest index with r of them up to it
        while (at < end) {
          const int mid = (at + end) / 2;
          int n = 0;
          each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < VEC; ++c) n += x[c] == hi && kept(x[c], i0 + c) && i0 + c <= mid;
          });
          if ((unsigned long long)count(n) >= r) end = mid;
          else at = mid + 1;
        }
        if (at < V) cut_x = hi, cut_i = at;
        return;
      }
      __syncthreads();
      for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
      if (tid == 0) found.bin = -1, found.listed = 0, found.lo = 0xffffffffu, found.hi = 0;
      __syncthreads();
      const double steps = kBins / ((double)hi - (double)lo);
      auto bin_of = [&](float x) __attribute__((always_inline)) {           // (of any x: within the bins)
        const int n = (int)(((double)hi - (double)x) * steps);
        return n < 0 ? 0 : n < kBins ? n : kBins - 1;
      };
      each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
        bool in[VEC], some = false;
#pragma unroll
        for (int c = 0; c < VEC; ++c) some |= in[c] = (x[c] >= lo) & (x[c] <= hi) & kept(x[c], i0 + c);
        if (!__any(some)) return;
        unsigned long long w[VEC];
        int bin[VEC];
#pragma unroll
        for (int c = 0; c < VEC; ++c) w[c] = weight(x[c]), bin[c] = bin_of(x[c]);
#pragma unroll
        for (int c = 0; c < VEC; ++c) asm volatile("" : "+v"(w[c]), "+v"(bin[c]));
#pragma unroll
        for (int c = 0; c < VEC; ++c)
          if (in[c] && w[c]) atomicAdd(&hist[bin[c]], w[c]);
      });
      __syncthreads();
      const unsigned long long h0 = hist[2 * tid], h1 = hist[2 * tid + 1];       // two steps a thread
      const unsigned long long run = block_run(h0 + h1, 0ull);
      if (share >= 0.0) {
        if (tid == kThreads - 1) found.above = run;
        __syncthreads();
        need = (unsigned long long)ceil(share * (double)found.above);
        need = need ? need : 1;
        share = -1.0;
        __syncthreads();
      }
      const unsigned long long before = above + run - h0 - h1;
      if (before < need && before + h0 >= need) found.bin = 2 * tid, found.above = before;
      else if (before + h0 < need && before + h0 + h1 >= need) found.bin = 2 * tid + 1, found.above = before + h0;
      __syncthreads();
      const int bin = found.bin;
      if (bin < 0) return;
      above = found.above;
      // its elements; a range of values a step wider on either side spares the others the 64-bit arithmetic
      const float wide_hi = (float)((double)hi - (bin - 1) / steps), wide_lo = bin == kBins - 1 ? lo : (float)((double)hi - (bin + 2) / steps);
      each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < VEC; ++c)
          if (x[c] >= wide_lo && x[c] <= wide_hi && x[c] >= lo && x[c] <= hi && bin_of(x[c]) == bin && kept(x[c], i0 + c)) {
            const int at = atomicAdd(&found.listed, 1);
            if (at < kList) loose[at] = key_of(x[c], i0 + c);
            atomicMin(&found.lo, ordered(x[c] + 0.0f));
            atomicMax(&found.hi, ordered(x[c] + 0.0f));
          }
      });
      __syncthreads();
      const int n = found.listed;
      if (n > kList) {
        lo = of_ordered(found.lo), hi = of_ordered(found.hi);
        continue;
      }
      sort_keys(n);
      const unsigned long long w = tid < n ? weight(of_ordered(~(uint32_t)(keys[tid] >> 32))) : 0, up_to = above + block_run(w, 0ull);
      if (up_to - w < need && up_to >= need) found.index = tid;
      __syncthreads();
      cut_at(found.index);
      return;
    }
  };

  // A value that at least r elements are no smaller than: the r-th largest of the threads' maxima, or a little below (-inf where there
  // are not so many maxima)
  auto floor_of = [&](int r) __attribute__((always_inline)) -> float {
    uint32_t* bins = (uint32_t*)shared_mem;                // 1024 steps
    bins[tid] = 0;
    if (tid == 0) found.bin = -1;
    const float worst = block_fold(best > -INFINITY ? best : top, top, smaller);           // (a barrier)
    const float steps = 1024.0f / (top - worst);
    auto bin_of = [&](float x) __attribute__((always_inline)) {
      const float n = (top - x) * steps;
      return n < 1023.0f ? (int)n : n >= 1023.0f ? 1023 : 0;          // (equal values, or a range past the largest float: 0)
    };
    if (best > -INFINITY) atomicAdd(&bins[bin_of(best)], 1u);
    __syncthreads();
    const int mine = (int)bins[tid], before = block_run(mine, 0) - mine;
    if (before < r && before + mine >= r) found.bin = tid;
    __syncthreads();
    const int bin = found.bin;
    // the smallest of the maxima in that step and above
    const float v = block_fold(bin >= 0 && best > -INFINITY && bin_of(best) <= bin ? best : top, top, smaller);
    return bin < 0 ? -INFINITY : v;
  };
  // The kept elements from `from` on, sorted, with their e: their number, or more than kList if they are too many to list
  auto list_from = [&](float from) __attribute__((always_inline)) -> int {
    __syncthreads();
    if (tid == 0) found.listed = 0;
    __syncthreads();
    if (best >= from)
      each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
        bool some = false;
#pragma unroll
        for (int c = 0; c < VEC; ++c) some |= x[c] >= from;
        if (!some) return;
#pragma unroll
        for (int c = 0; c < VEC; ++c)
          if (x[c] >= from && kept(x[c], i0 + c)) {
            const int at = atomicAdd(&found.listed, 1);
            if (at < kList) loose[at] = key_of(x[c], i0 + c);
          }
      });
    __syncthreads();
    const int n = found.listed;
    if (n > kList) return n;
    sort_keys(n);
    if (tid < n) shares[tid] = energy(of_ordered(~(uint32_t)(keys[tid] >> 32)));
    __syncthreads();
    return n;
  };

  const int k_in = a.top_k ? a.top_k[row] : 0, k = k_in > 0 && k_in < V ? k_in : 0;
  const float p_in = a.top_p ? a.top_p[row] : 1.0f;
  const bool cut_p = p_in < 1.0f;
  const double p = p_in > 0.f ? (double)p_in : 0.0;
  const float mp = a.min_p ? a.min_p[row] : 0.f;
  const double least = mp > 0.f ? (mp < 1.f ? (double)mp : 1.0) : 0.0;
  const float u_in = a.u[row];
  const double u = u_in > 0.f ? (double)u_in : 0.0;
  int kept_list = 0;                                       // elements of the list that are kept; 0: no list
  __syncthreads();                                         // (the table of roots)
  if (k) {
    const float from = k <= kThreads ? floor_of(k) : -INFINITY;
    const int n = k <= kList / 2 || V <= kList ? list_from(from) : kList + 1;
    if (n <= kList) {
      kept_list = k < n ? k : n;
    } else {
      low = block_fold(low, INFINITY, smaller);
      search([](float) __attribute__((always_inline)) -> unsigned long long { return 1; }, (unsigned long long)k, -1.0, fmaxf(from, low), top);
      if (k <= kList && cut_x > -INFINITY) kept_list = list_from(cut_x);         // (k of them)
    }
  }
  if (cut_p && kept_list) {
    const double mine = tid < kept_list ? shares[tid] : 0.0, run = block_run(mine, 0.0);
    if (tid == kThreads - 1) found.total = run;
    __syncthreads();
    // those whose sum in front of them does not reach p are kept, the first always
    kept_list = count(tid < kept_list && (tid == 0 || run - mine < p * found.total));
  } else if (cut_p) {
    if (!k) low = block_fold(low, INFINITY, smaller);
    // (32 temperatures below the maximum an element weighs less than half of 2^-43: nothing)
    search(whole, 0, p, fmaxf(fmaxf(cut_x, low), top - 32.0f * temp), top);
  }
  if (kept_list && least > 0.0) kept_list = count(tid < kept_list && shares[tid] >= least);
  if (kept_list && kept_list <= kShort) {
    // few are kept: brought into the order of their indices, four threads counting for an element, and one wavefront adds up
    const int who = tid >> 2, part = tid & 3;
    const uint32_t index = who < kept_list ? (uint32_t)keys[who] : 0;
    int rank = 0;
    for (int o = part; o < kept_list; o += 32) {
#pragma unroll
      for (int i = 0; i < 32; i += 4) rank += o + i < kept_list && (uint32_t)keys[o + i] < index;
    }
    rank += __shfl_xor(rank, 1, 64);
    rank += __shfl_xor(rank, 2, 64);
    __syncthreads();
    if (who < kept_list && part == 0) by_index[rank] = index, by_index_e[rank] = shares[who];
    __syncthreads();
    if (wave) return;
    constexpr int PER = kShort / 64;
    double e[PER], sum = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += e[i] = PER * lane + i < kept_list ? by_index_e[PER * lane + i] : 0.0;
    const double run = wave_run(sum, 0.0, add), total = lane_of(run, 63), target = u * total;
    const unsigned long long past = __ballot(sum > kNothing && run > target), some = __ballot(sum > kNothing);
    if (lane != (past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some))) return;
    double cum = run - sum, mine = 0.0;
    int at = 0;
    bool done = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      cum += e[i];
      if (!done && e[i] > kNothing) at = PER * lane + i, mine = e[i], done = cum > target;
    }
    a.tokens[row] = (int)by_index[at];
    if (a.logprob) a.logprob[row] = (float)log(mine / total);
    return;
  }
  if (kept_list) {
    // the same with the list sorted by index
    if (tid < kept_list) loose[tid] = (unsigned long long)(uint32_t)keys[tid] << 32 | (uint32_t)tid;
    __syncthreads();
    sort_keys(kept_list);
    const double e = tid < kept_list ? shares[(uint32_t)keys[tid]] : 0.0, run = block_run(e, 0.0);
    if (tid == kThreads - 1) found.total = run;
    __syncthreads();
    const double total = found.total, target = u * total;
    const int past = block_fold(e > kNothing && run > target ? tid : INT32_MAX, INT32_MAX, smaller);
    const int last = block_fold(e > kNothing ? tid : -1, -1, larger);
    if (tid == (past < INT32_MAX ? past : last)) {
      a.tokens[row] = (int)(keys[tid] >> 32);
      if (a.logprob) a.logprob[row] = (float)log(e / total);
    }
    return;
  }
  // min-p: what lies well below its border by value is not worth an exponential
  if (least > 0.0) {
    const float near = nextafterf((float)((double)top + (double)temp * (log(least) - 1e-3)), -INFINITY);
    if (near > cut_x) cut_x = near, cut_i = V;
  }

  // draw: sums of 64 x VEC consecutive elements, then of the segments, then inside the one that u falls into
  const bool all = cut_x == -INFINITY && least <= 0.0;
  auto drawn = [&](const float(&x)[VEC], int i0, double(&e)[VEC]) __attribute__((always_inline)) -> double {
    double sum = 0.0;
    if (!all) {
      bool some = false;
#pragma unroll
      for (int c = 0; c < VEC; ++c) some |= kept(x[c], i0 + c);
      if (!__any(some)) {
#pragma unroll
        for (int c = 0; c < VEC; ++c) e[c] = 0.0;
        return sum;
      }
    }
    // all of them, side by side: the compiler would put every exponential into a branch of its own, one latency after the other
#pragma unroll
    for (int c = 0; c < VEC; ++c) e[c] = energy(x[c]);
#pragma unroll
    for (int c = 0; c < VEC; ++c) asm volatile("" : "+v"(e[c]));
    if (!all) {
#pragma unroll
      for (int c = 0; c < VEC; ++c) e[c] = kept(x[c], i0 + c) & (e[c] >= least) ? e[c] : 0.0;
    }
#pragma unroll
    for (int c = 0; c < VEC; ++c) sum += e[c];
    return sum;
  };
  __syncthreads();
#pragma unroll 1
  for (int j0 = 0; j0 < chunks; j0 += AHEAD) {
    uint32_t w[AHEAD][4];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (j0 + i < chunks) piece(w[i], j0 + i);
    double s[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      s[i] = 0.0;
      if (j0 + i < chunks) {
        float x[VEC];
#pragma unroll
        for (int c = 0; c < VEC; ++c) x[c] = plain(value_of<T>(w[i], c));
        double e[VEC];
        s[i] = drawn(x, ((j0 + i) * kThreads + tid) * VEC, e);
      }
    }
    // four wavefront sums together: halves and rows of sixteen change places between them, and what is left is one sum over 16 lanes
    static_assert(AHEAD == 4, "four at a time");
    const double a01 = fold_halves(s[0], s[1]), a23 = fold_halves(s[2], s[3]);             // lower half: of 0 and 2, upper of 1 and 3
    const double sums = row_run(fold_rows(a01, a23), 0.0, add);                            // rows of 16: 0, 2, 1, 3
    if ((lane & 15) == 15) {
      const int i = (lane >> 5) | (lane >> 4 & 1) << 1;
      if (j0 + i < chunks) segs[(j0 + i) * kWaves + wave] = sums;
    }
  }
  __syncthreads();
  const int n_segs = chunks * kWaves;
  if (wave == 0) {
    const int per = (n_segs + 63) / 64, s0 = lane * per, s1 = s0 + per < n_segs ? s0 + per : n_segs;
    double sum = 0.0;
    for (int s = s0; s < s1; ++s) sum += segs[s];
    const double run = wave_run(sum, 0.0, add), total = lane_of(run, 63), target = u * total;
    const unsigned long long past = __ballot(sum > kNothing && run > target), some = __ballot(sum > kNothing);
    const int who = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
    if (lane == who) {
      double before = run - sum, at = 0.0;
      int seg = -1;
      for (int s = s0; s < s1; ++s) {
        if (segs[s] > kNothing) {
          seg = s, at = before;
          if (before + segs[s] > target) break;
        }
        before += segs[s];
      }
      found.seg = seg, found.before = at, found.total = total;
    }
  }
  __syncthreads();
  if (wave != found.seg % kWaves) return;
  {
    const int j = found.seg / kWaves, i0 = (j * kThreads + tid) * VEC;
    uint32_t w[4];
    piece(w, j);
    float x[VEC];
#pragma unroll
    for (int c = 0; c < VEC; ++c) x[c] = plain(value_of<T>(w, c));
    double e[VEC];
    const double sum = drawn(x, i0, e), run = wave_run(sum, 0.0, add), target = u * found.total;
    const unsigned long long past = __ballot(sum > kNothing && found.before + run > target), some = __ballot(sum > kNothing);
    const int who = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
    if (lane != who) return;
    double cum = found.before + run - sum, mine = 0.0;
    int token = -1;
    bool done = false;
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
      cum += e[c];
      if (!done && e[c] > kNothing) {
        token = i0 + c, mine = e[c];
        done = cum > target;
      }
    }
    a.tokens[row] = token;
    if (a.logprob) a.logprob[row] = (float)log(mine / found.total);
  }
}

hipError_t launch_sample_rows(int dtype, const SampleRows& a, hipStream_t s) {
  hipLaunchKernelGGL((dtype == 0 ? sample_rows_kernel<float> : sample_rows_kernel<bf16_t>), dim3(a.rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace ht
