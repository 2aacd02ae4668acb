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
// A workgroup of 1024 threads per row.  A prefix of the order ends at one element (value, index), so a filter is a search for that
// element, not a sort: a histogram of counts (top-k) or masses (top-p) over 2048 equal steps of the value, whose crossing step
// holds a few dozen elements as a rule; they are listed and ranked against each other.  A step that holds too many becomes the next
// histogram's range (a value far below the others, as masks leave, costs such a round).  Masses are counted in whole 2^-43: sums
// of integers do not depend on the order of the atomics.
#include "ht_common.h"

namespace ht {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048, kList = 1024;

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

// CHUNKS: 16-byte pieces of the row that a thread holds; 0: the row is longer than that and read again in every pass
template <typename T, int CHUNKS>
__global__ __launch_bounds__(kThreads) void sample_rows_kernel(SampleRows a) {
  constexpr int VEC = Vec16<T>::N, STRIDE = kThreads * VEC;
  // histogram and list of the search, or the segment sums of the draw
  __shared__ __attribute__((aligned(16))) unsigned char shared_mem[32768];
  unsigned long long* hist = (unsigned long long*)shared_mem;                    // [kBins]
  unsigned long long* list_w = (unsigned long long*)(shared_mem + 16384);        // [kList]
  float* list_x = (float*)(shared_mem + 24576);                                  // [kList]
  int32_t* list_i = (int32_t*)(shared_mem + 28672);                              // [kList]
  double* segs = (double*)shared_mem;                                            // [4096]
  __shared__ unsigned long long fold[kWaves];
  __shared__ Found found;

  const int row = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, V = a.V;
  const T* z = (const T*)a.z + (size_t)row * a.stride;
  const int chunks = (V + STRIDE - 1) / STRIDE;
  bool spike = false;                                      // the maximum is +inf: those tokens share everything

  auto load = [&](float (&x)[VEC], int j) __attribute__((always_inline)) {
    const int i0 = (j * kThreads + tid) * VEC;
    if (i0 + VEC <= V) {
      const Loose16<T> raw = *(const Loose16<T>*)(z + i0);
#pragma unroll
      for (int c = 0; c < VEC; ++c) x[c] = widen(raw.v[c]);
    } else {
#pragma unroll
      for (int c = 0; c < VEC; ++c) x[c] = i0 + c < V ? widen(z[i0 + c]) : -INFINITY;
    }
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
      x[c] = x[c] == x[c] ? x[c] + 0.0f : -INFINITY;       // (-0 ties with 0)
      if (spike) x[c] = x[c] == INFINITY ? 0.f : -INFINITY;
    }
  };
  float held[CHUNKS ? CHUNKS : 1][VEC];
  if constexpr (CHUNKS > 0) {
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) load(held[j], j);
  }
  // f(chunk, values, first index).  The values pass through an empty asm, or what one pass works out from them (64-bit differences)
  // would be kept in registers for the next.
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (CHUNKS > 0) {
#pragma unroll
      for (int j = 0; j < CHUNKS; ++j)
        if (j < chunks) {
          float x[VEC];
#pragma unroll
          for (int c = 0; c < VEC; ++c) {
            x[c] = held[j][c];
            asm volatile("" : "+v"(x[c]));
          }
          f(j, x, (j * kThreads + tid) * VEC);
        }
    } else {
      for (int j = 0; j < chunks; ++j) {
        float x[VEC];
        load(x, j);
        f(j, x, (j * kThreads + tid) * VEC);
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
  top = block_fold(top, take_max<float>);
  low = block_fold(low, take_min<float>);
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
    if constexpr (CHUNKS > 0) {
#pragma unroll
      for (int j = 0; j < CHUNKS; ++j)
#pragma unroll
        for (int c = 0; c < VEC; ++c) held[j][c] = held[j][c] == INFINITY ? 0.f : -INFINITY;
    }
  }
  const double per_temp = 1.0 / (double)temp;
  auto energy = [&](float x) __attribute__((always_inline)) -> double {
    return x == top ? 1.0 : x == -INFINITY ? 0.0 : exp_below(((double)x - (double)top) * per_temp);
  };
  // in whole 2^-43, up to 2^20 of them in 64 bits: the mantissa's end of e + 512
  auto whole = [&](float x) __attribute__((always_inline)) -> unsigned long long {
    return (unsigned long long)__double_as_longlong(energy(x) + 512.0) - 0x4080000000000000ull;
  };

  float cut_x = -INFINITY;                                 // kept so far: what comes before or is (cut_x, cut_i)
  int cut_i = -1;
  auto kept = [&](float x, int i) __attribute__((always_inline)) { return x > cut_x || (x == cut_x && i <= cut_i); };

  // the element of the kept ones at which the running weight reaches `need` (at least 1) becomes the cut; none if it never does
  auto search = [&](auto weight, unsigned long long need) __attribute__((always_inline)) {
    float lo = cut_x > low ? cut_x : low, hi = top;
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

  const int k = a.top_k ? a.top_k[row] : 0;
  if (k > 0 && k < V) search([](float) __attribute__((always_inline)) -> unsigned long long { return 1; }, (unsigned long long)k);
  const float p = a.top_p ? a.top_p[row] : 1.0f;
  if (p < 1.0f) {
    unsigned long long mass = 0;
    each([&](int, const float(&x)[VEC], int i0) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < VEC; ++c)
        if (kept(x[c], i0 + c)) mass += whole(x[c]);
    });
    mass = block_sum(mass);
    const double need = ceil((double)p * (double)mass);
    search(whole, need >= 1.0 ? (unsigned long long)need : 1ull);
  }
  // min-p: what lies well below its border by value is not worth an exponential
  const float mp = a.min_p ? a.min_p[row] : 0.f;
  const double least = mp > 0.f ? (mp < 1.f ? (double)mp : 1.0) : 0.0;
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
  const float u_in = a.u[row];
  const double u = u_in > 0.f ? (double)u_in : 0.0;
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
    float x[VEC];
    load(x, j);
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
  const bool holds = a.V <= 32 * kThreads;                 // 32 values a thread
  if (dtype == 0) hipLaunchKernelGGL((holds ? sample_rows_kernel<float, 8> : sample_rows_kernel<float, 0>), dim3(a.rows), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((holds ? sample_rows_kernel<bf16_t, 4> : sample_rows_kernel<bf16_t, 0>), dim3(a.rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace ht
