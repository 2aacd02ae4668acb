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
// pass unrolled over them, the passes' own needs went to scratch memory.)  A prefix of the order ends at one element (value, index), so a filter is a search for that element, not a sort of the row.  The r-th largest of
// the 1024 threads' maxima is no larger than the r-th largest value, so the elements from there on hold the first r; they are a few
// more than r as a rule, are listed and sorted, and all filters work on the list.  Where the list does not reach (a large k, a flat row),
// a histogram of counts (top-k) or masses (top-p) over 2048 equal steps of the value finds the step that holds the end, whose
// elements are listed and ranked; a step that holds too many becomes the next histogram's range (a value far below the others, as masks
// leave, costs such a round).  Masses of a histogram are counted in whole 2^-43: sums of integers do not depend on the order of the
// atomics.
#include "ht_common.h"

namespace ht {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048, kList = 1024;
constexpr int kMaxima = 512;                 // maxima whose list a top-p without top-k tries first

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
__device__ inline float widen(float v) { return v; }
__device__ inline float widen(bf16_t v) { return bf16_to_float(v); }
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
  float value;
};

__device__ inline uint32_t ordered(float v) {
  const uint32_t u = __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float of_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// exp of y <= 0: y = n ln 2 + f, |f| <= ln 2 / 2, and the series to f^13 (the first term left out is 4e-18 of the result)
__device__ inline double exp_below(double y) {
  constexpr double ln2 = 0.69314718055994531, ln2_rest = 2.3190468138462996e-17, per_ln2 = 1.4426950408889634;
  y = fmax(y, -800.0);                                     // 0 from -746 on
  const double n = rint(y * per_ln2), f = fma(n, -ln2_rest, fma(n, -ln2, y));
  constexpr double c[13] = {1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040, 1.0 / 40320, 1.0 / 362880,
                            1.0 / 3628800, 1.0 / 39916800, 1.0 / 479001600};
  double e = 1.0 / 6227020800.0;
#pragma unroll
  for (int i = 12; i >= 0; --i) e = fma(e, f, c[i]);
  return ldexp(e, (int)n);
}

template <typename V> __device__ inline V wave_fold(V v, V (*f)(V, V)) {
  for (int o = 32; o; o >>= 1) v = f(v, __shfl_xor(v, o, 64));
  return v;
}
template <typename V> __device__ inline V take_sum(V a, V b) { return a + b; }
template <typename V> __device__ inline V take_max(V a, V b) { return a > b ? a : b; }
template <typename V> __device__ inline V take_min(V a, V b) { return a < b ? a : b; }

}  // namespace

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_rows_kernel(SampleRows a) {
  constexpr int VEC = Vec16<T>::N, STRIDE = kThreads * VEC, AHEAD = 4;
  // histogram and list of the search, or the segment sums of the draw
  __shared__ __attribute__((aligned(16))) unsigned char shared_mem[32768];
  unsigned long long* hist = (unsigned long long*)shared_mem;                    // [kBins]
  unsigned long long* list_w = (unsigned long long*)(shared_mem + 16384);        // [kList]
  float* list_x = (float*)(shared_mem + 24576);                                  // [kList]
  int32_t* list_i = (int32_t*)(shared_mem + 28672);                              // [kList]
  double* segs = (double*)shared_mem;                                            // [4096]
  __shared__ unsigned long long keys[kList];                                     // the sorted list: order, then index
  __shared__ double shares[kList];                                               // ... and its e
  __shared__ unsigned long long fold[kWaves];
  __shared__ Found found;

  const int row = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, V = a.V;
  const T* z = (const T*)a.z + (size_t)row * a.stride;
  const int chunks = (V + STRIDE - 1) / STRIDE;
  bool spike = false;                                      // the maximum is +inf: those tokens share everything

  // NaN counts as -inf, -0 ties with 0
  auto plain = [&](float v) __attribute__((always_inline)) {
    v = v == v ? v + 0.0f : -INFINITY;
    return !spike ? v : v == INFINITY ? 0.f : -INFINITY;
  };
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
  auto block_fold = [&](auto v, auto f) __attribute__((always_inline)) {
    using W = decltype(v);
    static_assert(sizeof(W) <= 8, "a word per wavefront");
    v = wave_fold<W>(v, f);
    __syncthreads();
    W* slots = (W*)fold;
    if (lane == 0) slots[wave] = v;
    __syncthreads();
    v = slots[lane & (kWaves - 1)];
    return wave_fold<W>(v, f);
  };
  // (a sum over all 64 lanes counts every wavefront's word four times)
  auto block_sum = [&](unsigned long long v) __attribute__((always_inline)) { return block_fold(v, take_sum<unsigned long long>) / (64 / kWaves); };

  float top = -INFINITY, low = INFINITY;
  each([&](int, const float(&x)[VEC], int) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
      top = fmaxf(top, x[c]);
      if (x[c] > -INFINITY) low = fminf(low, x[c]);
    }
  });
  const float my_top = top;
  top = block_fold(top, take_max<float>);
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
    each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
      for (int c = VEC - 1; c >= 0; --c)
        if (x[c] == top && i0 + c < first) first = i0 + c;
    });
    first = block_fold(first, take_min<int>);
    if (tid == 0) {
      a.tokens[row] = first;
      if (a.logprob) a.logprob[row] = 0.f;
    }
    return;
  }
  if (top == INFINITY) {
    spike = true;
    top = low = 0.f;
  } else {
    low = block_fold(low, take_min<float>);
  }
  const double per_temp = 1.0 / (double)temp;
  auto energy = [&](float x) __attribute__((always_inline)) -> double {
    return x == top ? 1.0 : x == -INFINITY ? 0.0 : exp_below(((double)x - (double)top) * per_temp);
  };
  // in whole 2^-43, up to 2^20 of them in 64 bits: the mantissa's end of e + 512
  auto whole = [&](float x) __attribute__((always_inline)) -> unsigned long long {
    return (unsigned long long)__double_as_longlong(energy(x) + 512.0) - 0x4080000000000000ull;
  };

  const float best = !spike ? my_top : my_top == INFINITY ? 0.f : -INFINITY;       // this thread's largest value
  float cut_x = -INFINITY;                                 // kept so far: what comes before or is (cut_x, cut_i)
  int cut_i = -1;
  auto kept = [&](float x, int i) __attribute__((always_inline)) { return x > cut_x || (x == cut_x && i <= cut_i); };

  // the element of the kept ones at which the running weight reaches `need` (at least 1) becomes the cut; none if it never does
  auto search = [&](auto weight, unsigned long long need, float floor_x) __attribute__((always_inline)) {
    float lo = fmaxf(fmaxf(cut_x, low), floor_x), hi = top;
    unsigned long long above = 0;
    for (;;) {
      if (lo == hi) {                                      // equal values: the lowest indices, as many as it takes
        const unsigned long long w = weight(hi), r = w ? (need - above + w - 1) / w : 1;
        int at = 0, end = V;                               // smallest index with r of them up to it
        while (at < end) {
          const int mid = (at + end) / 2;
          unsigned long long n = 0;
          each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < VEC; ++c) n += x[c] == hi && kept(x[c], i0 + c) && i0 + c <= mid;
          });
          if (block_sum(n) >= r) end = mid;
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
      auto bin_of = [&](float x) __attribute__((always_inline)) {
        const int n = (int)(((double)hi - (double)x) * steps);
        return n < kBins ? n : kBins - 1;
      };
      each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < VEC; ++c)
          if (x[c] >= lo && x[c] <= hi && kept(x[c], i0 + c)) atomicAdd(&hist[bin_of(x[c])], weight(x[c]));
      });
      __syncthreads();
      {                                                    // two steps a thread
        const unsigned long long h0 = hist[2 * tid], h1 = hist[2 * tid + 1];
        unsigned long long run = h0 + h1;
        for (int o = 1; o < 64; o <<= 1) {
          const unsigned long long other = __shfl_up(run, o, 64);
          if (lane >= o) run += other;
        }
        if (lane == 63) fold[wave] = run;
        __syncthreads();
        unsigned long long before = above + run - h0 - h1;
        for (int w = 0; w < wave; ++w) before += fold[w];
        if (before < need && before + h0 >= need) found.bin = 2 * tid, found.above = before;
        else if (before + h0 < need && before + h0 + h1 >= need) found.bin = 2 * tid + 1, found.above = before + h0;
      }
      __syncthreads();
      const int bin = found.bin;
      if (bin < 0) return;
      above = found.above;
      each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < VEC; ++c)
          if (x[c] >= lo && x[c] <= hi && kept(x[c], i0 + c) && bin_of(x[c]) == bin) {
            const int at = atomicAdd(&found.listed, 1);
            if (at < kList) {
              list_x[at] = x[c];
              list_i[at] = i0 + c;
              list_w[at] = weight(x[c]);
            }
            atomicMin(&found.lo, ordered(x[c]));
            atomicMax(&found.hi, ordered(x[c]));
          }
      });
      __syncthreads();
      const int n = found.listed;
      if (n > kList) {
        lo = of_ordered(found.lo), hi = of_ordered(found.hi);
        continue;
      }
      if (tid < n) {
        const float x = list_x[tid];
        const int i = list_i[tid];
        unsigned long long before = above;
        for (int o = 0; o < n; ++o) before += list_x[o] > x || (list_x[o] == x && list_i[o] < i) ? list_w[o] : 0;
        if (before < need && before + list_w[tid] >= need) found.value = x, found.index = i;
      }
      __syncthreads();
      cut_x = found.value, cut_i = found.index;
      return;
    }
  };

  // A value that no more than its own thread's larger ones can be ... : at least `r` elements are no smaller (-inf: all)
  auto floor_of = [&](int r) __attribute__((always_inline)) -> float {
    uint32_t* bins = (uint32_t*)shared_mem;                // 1024 steps
    __syncthreads();
    bins[tid] = 0;
    if (tid == 0) found.bin = -1;
    const float least_best = block_fold(best > -INFINITY ? best : top, take_min<float>);   // (barriers)
    const float steps = 1024.0f / (top - least_best);
    auto bin_of = [&](float x) __attribute__((always_inline)) {
      const float n = (top - x) * steps;
      return n < 1023.0f ? (int)n : n >= 1023.0f ? 1023 : 0;          // (equal values, or a range past the largest float: 0)
    };
    if (best > -INFINITY) atomicAdd(&bins[bin_of(best)], 1u);
    __syncthreads();
    uint32_t run = bins[tid];
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t other = __shfl_up(run, o, 64);
      if (lane >= o) run += other;
    }
    if (lane == 63) fold[wave] = run;
    __syncthreads();
    uint32_t before = run - bins[tid];
    for (int w = 0; w < wave; ++w) before += (uint32_t)fold[w];
    if (before < (uint32_t)r && before + bins[tid] >= (uint32_t)r) found.bin = tid;
    __syncthreads();
    const int bin = found.bin;
    // the smallest of the maxima in that step and above
    float v = bin >= 0 && best > -INFINITY && bin_of(best) <= bin ? best : top;
    v = block_fold(v, take_min<float>);
    return bin < 0 ? -INFINITY : v;
  };
  // The elements from `from` on, sorted: their number, or more than kList if they are too many to list
  auto list_from = [&](float from) __attribute__((always_inline)) -> int {
    __syncthreads();
    if (tid == 0) found.listed = 0;
    __syncthreads();
    each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < VEC; ++c)
        if (x[c] >= from && x[c] > -INFINITY) {
          const int at = atomicAdd(&found.listed, 1);
          if (at < kList) keys[at] = (unsigned long long)~ordered(x[c]) << 32 | (uint32_t)(i0 + c);
        }
    });
    __syncthreads();
    const int n = found.listed;
    if (n > kList) return n;
    int size = 64;
    while (size < n) size *= 2;
    unsigned long long key = tid < n ? keys[tid] : ~0ull;
    // bitonic: strides below 64 inside a wavefront
    for (int half = 2; half <= size; half *= 2)
      for (int stride = half / 2; stride; stride /= 2) {
        unsigned long long other;
        if (stride >= 64) {
          __syncthreads();
          if (tid < size) keys[tid] = key;
          __syncthreads();
          other = tid < size ? keys[tid ^ stride] : 0;
        } else {
          if (wave * 64 >= size) continue;
          other = __shfl_xor(key, stride, 64);
        }
        const bool up = (tid & half) == 0, first = (tid & stride) == 0;
        key = (other < key) == (up == first) ? other : key;
      }
    __syncthreads();
    if (tid < size) keys[tid] = key;
    if (tid < n) shares[tid] = energy(of_ordered(~(uint32_t)(key >> 32)));
    __syncthreads();
    return n;
  };
  // Sum of the list's e up to element `tid` (zeros behind the list)
  auto list_sums = [&](int n) __attribute__((always_inline)) -> double {
    double run = tid < n ? shares[tid] : 0.0;
    for (int o = 1; o < 64; o <<= 1) {
      const double other = __shfl_up(run, o, 64);
      if (lane >= o) run += other;
    }
    __syncthreads();
    double* ends = (double*)fold;
    if (lane == 63) ends[wave] = run;
    __syncthreads();
    double before = 0.0;
    for (int w = 0; w < wave; ++w) before += ends[w];
    return before + run;
  };
  auto cut_at = [&](int i) __attribute__((always_inline)) {          // element i of the list ends what is kept
    cut_x = of_ordered(~(uint32_t)(keys[i] >> 32)), cut_i = (int)(uint32_t)keys[i];
  };

  const int k_in = a.top_k ? a.top_k[row] : 0, k = k_in > 0 && k_in < V ? k_in : 0;
  const float p_in = a.top_p ? a.top_p[row] : 1.0f;
  const bool cut_p = p_in < 1.0f;
  const double p = p_in > 0.f ? (double)p_in : 0.0;
  const float mp = a.min_p ? a.min_p[row] : 0.f;
  const double least = mp > 0.f ? (mp < 1.f ? (double)mp : 1.0) : 0.0;
  int listed = 0, kept_list = 0;                           // of the list: elements, and how many of them are kept; 0: no list
  if (k) {
    const float from = k <= kThreads ? floor_of(k) : -INFINITY;
    const int n = k <= kList ? list_from(from) : kList + 1;
    if (n <= kList) {
      listed = n;
      kept_list = k < n ? k : n;
    } else {
      search([](float) __attribute__((always_inline)) -> unsigned long long { return 1; }, (unsigned long long)k, from);
    }
  }
  if (cut_p && listed) {
    const double run = list_sums(listed), before = run - (tid < listed ? shares[tid] : 0.0);
    __syncthreads();
    if (tid == kept_list - 1) found.total = run;
    __syncthreads();
    const double need = p * found.total;
    // the first element at which the sum reaches `need`: those whose sum in front of them does not are kept, the first always
    kept_list = (int)block_sum(tid < kept_list && (tid == 0 || before < need) ? 1ull : 0ull);
  } else if (cut_p) {
    // whole row (or what a long top-k has left): its mass, then the list if it holds enough of it
    double mass = 0.0;
    each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < VEC; ++c)
        if (kept(x[c], i0 + c)) mass += energy(x[c]);
    });
    mass = block_fold(mass, take_sum<double>) / (64 / kWaves);
    const double need = p * mass;
    const int n = list_from(fmaxf(floor_of(kMaxima), cut_x));
    bool enough = false;
    if (n <= kList) {
      const bool mine = tid < n && kept(of_ordered(~(uint32_t)(keys[tid < n ? tid : 0] >> 32)), (int)(uint32_t)keys[tid < n ? tid : 0]);
      const double run = list_sums(n), before = run - (tid < n ? shares[tid] : 0.0);
      const int m = (int)block_sum(mine && (tid == 0 || before < need) ? 1ull : 0ull);
      __syncthreads();
      if (tid == n - 1) found.total = run;
      __syncthreads();
      enough = m < n || found.total >= need;
      if (enough) listed = n, kept_list = m;
    }
    if (!enough) {
      const double whole_need = ceil(need * 8796093022208.0);          // 2^43
      search(whole, whole_need >= 1.0 ? (unsigned long long)whole_need : 1ull, -INFINITY);
    }
  }
  if (listed && least > 0.0) kept_list = (int)block_sum(tid < kept_list && shares[tid] >= least ? 1ull : 0ull);
  const float u_in = a.u[row];
  const double u = u_in > 0.f ? (double)u_in : 0.0;
  if (listed && kept_list <= 64) {
    // few are kept: one wavefront holds them, brings them into the order of their indices and adds up
    if (wave) return;
    uint32_t index = lane < kept_list ? (uint32_t)keys[lane] : 0xffffffffu;
    double e = lane < kept_list ? shares[lane] : 0.0;
#pragma unroll
    for (int half = 2; half <= 64; half *= 2)
#pragma unroll
      for (int stride = half / 2; stride; stride /= 2) {
        const uint32_t other = __shfl_xor(index, stride, 64);
        const double other_e = __shfl_xor(e, stride, 64);
        const bool up = (lane & half) == 0, first = (lane & stride) == 0;
        const bool take = (other < index) == (up == first) && other != index;
        index = take ? other : index, e = take ? other_e : e;
      }
    double run = e;
    for (int o = 1; o < 64; o <<= 1) {
      const double other = __shfl_up(run, o, 64);
      if (lane >= o) run += other;
    }
    const double total = __shfl(run, 63, 64), target = u * total;
    const unsigned long long past = __ballot(e > 0.0 && run > target), some = __ballot(e > 0.0);
    const int who = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
    if (lane == who) {
      a.tokens[row] = (int)index;
      if (a.logprob) a.logprob[row] = (float)log(e / total);
    }
    return;
  }
  if (listed) {
    __syncthreads();
    cut_at(kept_list - 1);
  }
  // min-p: what lies well below its border by value is not worth an exponential
  if (least > 0.0) {
    const float near = nextafterf((float)((double)top + (double)temp * (log(least) - 1e-3)), -INFINITY);
    if (near > cut_x) cut_x = near, cut_i = V;
  }

  // draw: sums of 64 x VEC consecutive elements, then of the segments, then inside the one that u falls into
  auto drawn = [&](float x, int i) __attribute__((always_inline)) -> double {
    if (!kept(x, i)) return 0.0;
    const double e = energy(x);
    return e >= least ? e : 0.0;
  };
  __syncthreads();
  each([&](int j, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
    double sum = 0.0;
#pragma unroll
    for (int c = 0; c < VEC; ++c) sum += drawn(x[c], i0 + c);
    sum = wave_fold<double>(sum, take_sum<double>);
    if (lane == 0) segs[j * kWaves + wave] = sum;
  });
  __syncthreads();
  const int n_segs = chunks * kWaves;
  if (wave == 0) {
    const int per = (n_segs + 63) / 64, s0 = lane * per, s1 = s0 + per < n_segs ? s0 + per : n_segs;
    double sum = 0.0;
    for (int s = s0; s < s1; ++s) sum += segs[s];
    double run = sum;
    for (int o = 1; o < 64; o <<= 1) {
      const double other = __shfl_up(run, o, 64);
      if (lane >= o) run += other;
    }
    const double total = __shfl(run, 63, 64), target = u * total;
    const unsigned long long past = __ballot(run > target), some = __ballot(sum > 0.0);
    const int who = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
    if (lane == who) {
      double before = run - sum;
      int seg = -1;
      double at = 0.0;
      for (int s = s0; s < s1; ++s) {
        if (segs[s] > 0.0) {
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
    double e[VEC], sum = 0.0;
#pragma unroll
    for (int c = 0; c < VEC; ++c) sum += e[c] = drawn(x[c], i0 + c);
    double run = sum;
    for (int o = 1; o < 64; o <<= 1) {
      const double other = __shfl_up(run, o, 64);
      if (lane >= o) run += other;
    }
    const double target = u * found.total;
    const unsigned long long past = __ballot(sum > 0.0 && found.before + run > target), some = __ballot(sum > 0.0);
    const int who = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
    if (lane != who) return;
    double cum = found.before + run - sum, mine = 0.0;
    int token = -1;
    bool done = false;
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
      cum += e[c];
      if (!done && e[c] > 0.0) {
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
