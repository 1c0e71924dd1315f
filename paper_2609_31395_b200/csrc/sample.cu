// actkv_sample: a token per row of logits, from what temperature, top-k, top-p and min-p leave.
//
// Weights w = 2^(-y / 16), y = 16 log2(e) (max - z) / T, in float64: 2^(-i/16) from a table, the rest by a polynomial of degree 5 (through the values
// at the Chebyshev nodes of [-1/2, 1/2], its constant term set to 1: below 2^-46), as whole multiples of 2^-45.  Sums of integers are the same in
// every order and on every split, so that equal arguments draw equal tokens.  A weight is off by less than 2^-45 (the rounding by 2^-46, the polynomial by 2^-46.6), a sum of
// 150000 weights by less than 2^-27.8 of the largest one; as roundings go, by about 2^-36.
// (In float32 one draw in some hundred would fall on the neighbour of its token, and top-p would keep a token more or less.)
//
// A cluster holds the row in shared memory, in its own type; it is read once.  Tokens are ordered by (logit descending, token ascending), as 64-bit keys
// that are all different, and the kept ones are those that reach a border key.
//   top-k, small: the k-th largest of the maxima of 128 groups of tokens is a bound that k tokens reach; the few that reach it go to the first
// CTA, which orders them, cuts the list by k, p and m, and draws from it.
//   Otherwise top-k and top-p each ask for the key at which a count or a mass is reached: a histogram of 1024 equal steps of z, whose counts and
// masses are added up over the cluster, tells the step in which it happens.  If the tokens down to it are few, the first CTA goes on with them as above; if not,
// the tokens of the step are sorted, or, when they are more than the list holds, spread over a histogram of their keys, and so on.
//   min-p is a smallest logit, found by trying the floats around max + T ln m.
//   The draw goes over the kept tokens in the order of the vocabulary: sums per thread, per CTA, and then along the tokens of the thread in which u S falls.
//
// CTAs only write into one another's shared memory, never read there: what is written lands before a barrier of the cluster, and behind its last barrier a CTA
// can end.  (Loads from a neighbour may still be on their way when a thread has arrived.)
//
// What bounds it.  Few rows: the chain of passes and barriers: at 152K float32 tokens loading takes 2.0 us, a barrier of the cluster 0.7, the
// weights of a CTA's 19000 tokens 3.4.  Many rows: loading and barriers (1024 bf16 rows of 152K, T = 0: 140 us
// where reading takes 48), the weights (11 float64 operations a token: 150 us more), and, in histograms, shared memory's atomics (about 16 cycles per
// warp, one for a count, two for a mass).
// Measured, us: 16 rows of 152K float32: T = 0 7.2, the whole distribution 14.6, k = 20 13.0, k = 1000 30, p = 0.95 43; 64 rows 20, 34, 35, 69, 91; 1024 bf16
// rows 140, 290, 212, 567, 916.
// Tried: a persistent grid of clusters (321 instead of 288 for the last whole ones); a bound from 2048 groups for k up to 1280 (27 instead of 24, one row);
// the upper word of a mass only where it is not 0 (908 -> 944); a step's tokens ordered by counting (p = 0.95, 64 rows: 89 -> 101).
#include <cooperative_groups.h>

#include <algorithm>
#include <cfloat>

#include "common.cuh"

namespace actkv {
namespace sa {

namespace cg = cooperative_groups;

constexpr int LOG_NB = 10, NB = 1 << LOG_NB;          // steps of a histogram
constexpr int CAP = 1024;                  // tokens that are sorted
constexpr int MAX_CLUSTER = 8;
constexpr int MAX_SLICE = 43008;           // tokens of a CTA
constexpr double MAGIC = 6755399441055744.0;          // 1.5 * 2^52: adding it rounds to a whole number in the low bits
constexpr float OCTAVES = 47.f;                       // weights below 2^-47 are 0
constexpr int NT = 512, NW = NT / 32, BPT = NB / NT;
// The bound of a small top-k, from maxima of 128 groups: at k = 20 about 22 tokens reach it, at k = 120 some 350 (16 rows of 152K: 13.3 and 18.1 us, by the
// histogram 20.5 and 22.9); with fewer groups left over than eight it may lie anywhere.
constexpr int GROUPS = 128, SMALL_K = 120;
constexpr int FEW = NT / 4;                // tokens of a short list, by counting: k = 20, 16 rows of 152K 13.3 us, by sorting 15.1

// 2^(-i / 16)
__constant__ double ROOTS[16] = {
    0x1.0000000000000p+0, 0x1.ea4afa2a490dap-1, 0x1.d5818dcfba487p-1, 0x1.c199bdd85529cp-1,
    0x1.ae89f995ad3adp-1, 0x1.9c49182a3f090p-1, 0x1.8ace5422aa0dbp-1, 0x1.7a11473eb0187p-1,
    0x1.6a09e667f3bcdp-1, 0x1.5ab07dd485429p-1, 0x1.4bfdad5362a27p-1, 0x1.3dea64c123422p-1,
    0x1.306fe0a31b715p-1, 0x1.2387a6e756238p-1, 0x1.172b83c7d517bp-1, 0x1.0b5586cf9890fp-1};

struct Args {
  const void* logits;
  int64_t row_stride;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* token;
  float* logprob;
  int32_t* kept;
  int32_t* status;
  int32_t vocab, slice;
};

__device__ __forceinline__ uint32_t okey(float x) {
  uint32_t b = __float_as_uint(x);
  if (b == 0x80000000u) b = 0u;                                            // -0 and +0 are equal
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float okey_inv(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token) { return ((uint64_t)okey(x) << 32) | (0xffffffffu - token); }
__device__ __forceinline__ float logit_of(uint64_t key) { return okey_inv((uint32_t)(key >> 32)); }

// Parts that are not live together share their place.  What another CTA writes may arrive as soon as this one has joined the barrier before; so
// over the own histogram, which is given away before the barrier in front of them, lies what comes with or behind the lists; over the inbox,
// read before the barrier behind it, the own list, given away before its barrier, and the last sums; over the joint histogram, written behind a
// barrier, what comes with the first one.
struct Hist {
  uint32_t cnt[NB], lo[NB], hi[NB];        // tokens, mass in two words
};
struct Shared {
  union {
    Hist own;                              // this CTA's tokens
    uint64_t all[CAP];                     // written by the others
    int32_t group[GROUPS];                 // (before any histogram) the groups' maxima, written by the others
  };
  union {
    Hist inbox;                            // [CTA][its share of the steps], written by the others
    uint64_t list[CAP];
    ulonglong2 end[MAX_CLUSTER][NW];       // mass and number of every warp's kept tokens, written by the others
  };
  union {
    Hist sum;                              // all tokens, written by the others
    struct {
      int2 ends[MAX_CLUSTER][NW];          // largest and smallest logit of every warp as ordered(), written by the others
      uint64_t sent[CAP];                  // short lists, written by the others (perhaps while the ends are read)
    };
    uint64_t mass[2][FEW];                 // of a short list
    uint64_t weight[CAP];                  // of a stretch of a longer one
  };
  double tab[16][16];                      // 2^(-i/16), sixteen times, so that no two lanes of a half warp meet on a bank
  uint64_t scan[2][NW];
  uint64_t found[4];
  uint64_t range[MAX_CLUSTER][2];          // written by the others
  uint32_t few[MAX_CLUSTER];
  uint32_t n_list, n_all;
};

// (a subnormal number too, which the library's float32 arithmetic takes for 0)
__device__ __forceinline__ double exact_double(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x7f800000u) != 0 ? (double)x : (b & 0x80000000u ? -1.0 : 1.0) * (double)(int)(b & 0x7fffffu) * 0x1p-149;
}

// 0 (of either sign) <= x <= most (false for NaN), and x > 0 where x is no NaN, by the bits: float32 comparisons take a subnormal number for 0.
__device__ __forceinline__ bool from_zero_to(float x, float most) {
  return __float_as_uint(x) <= __float_as_uint(most) || __float_as_uint(x) == 0x80000000u;
}
__device__ __forceinline__ bool positive(float x) { return __float_as_int(x) > 0; }

// Order of the logits as signed integers (-0 just below +0).  NaN lie outside the infinities.
__device__ __forceinline__ int32_t ordered(float x) {
  const int32_t b = __float_as_int(x);
  return b ^ ((b >> 31) & 0x7fffffff);
}
constexpr int32_t POS_INF = 0x7f800000, NEG_INF = (int32_t)0x807fffff;

struct Scale {                             // of a row
  double top, c;                           // largest logit; 16 log2(e) / T
  int limit;                               // high word of a gap of 47 octaves and a little, whose weight rounds to 0
};
// top - z, at most a limit (its high word) and a little.
__device__ __forceinline__ double gap_of(float z, double top, int limit) {
  const double d = top - (double)z;
  return __hiloint2double(min(__double2hiint(d), limit), __double2loint(d));
}
// onto + 2^(-d c / 16), d c in [0, 2^14]
__device__ __forceinline__ double power(double d, double c, double onto, const double (*tab)[16]) {
  const double k = fma(d, c, MAGIC), r = fma(d, c, MAGIC - k);
  const int ki = __double2loint(k);
  double p = fma(r, -0x1.5d897e525c216p-30, 0x1.3b2c9b8a6caeap-23);
  p = fma(p, r, -0x1.c6b08d6f2a289p-17);
  p = fma(p, r, 0x1.ebfbdff555824p-11);
  p = fma(p, r, -0x1.62e42fefa39f3p-5);
  p = fma(p, r, 1.0);
  const double t = tab[ki & 15][threadIdx.x & 15];
  return fma(__hiloint2double(__double2hiint(t) - (ki & ~15) * 65536, __double2loint(t)), p, onto);
}
// Between 128 and 256 a float64 goes in steps of 2^-45: what is added to it is rounded to them, and up to 127 weights can be.
constexpr double SUM45 = 128.0;
__device__ __forceinline__ double add45(double sum, float z, const Scale& s, const double (*tab)[16]) {
  return power(gap_of(z, s.top, s.limit), s.c, sum, tab);
}
__device__ __forceinline__ uint64_t of_sum45(double sum) { return (uint64_t)__double_as_longlong(sum) - 0x4060000000000000ull; }
__device__ __forceinline__ uint64_t weight45(float z, const Scale& s, const double (*tab)[16]) { return of_sum45(add45(SUM45, z, s, tab)); }

__device__ __forceinline__ uint64_t warp_scan(uint64_t v) {                 // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
  return v;
}
__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Sums of two numbers over the threads before this one, and of all.
__device__ __forceinline__ void block_before(Shared& sh, uint64_t& a, uint64_t& b, uint64_t& all_a, uint64_t& all_b) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t ia = warp_scan(a), ib = warp_scan(b);
  __syncthreads();
  if (lane == 31) sh.scan[0][warp] = ia, sh.scan[1][warp] = ib;
  __syncthreads();
  uint64_t ta = lane < NT / 32 ? sh.scan[0][lane] : 0, tb = lane < NT / 32 ? sh.scan[1][lane] : 0;
  const uint64_t sa = warp_scan(ta), sb = warp_scan(tb);
  all_a = __shfl_sync(0xffffffffu, sa, 31);
  all_b = __shfl_sync(0xffffffffu, sb, 31);
  a = ia - a + __shfl_sync(0xffffffffu, sa - ta, warp);
  b = ib - b + __shfl_sync(0xffffffffu, sb - tb, warp);
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// All threads of the cluster, whatever came before; what a CTA has written into another one's shared memory is there.  (Nothing is read from another
// CTA: behind its last barrier a CTA can end.)
__device__ __forceinline__ void cluster_barrier() {
  __syncthreads();
  cluster_arrive();
  cluster_wait();
}

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void open(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void open(const uint4& v, float (&x)[8]) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
};
__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
// The largest and the smallest of three, subnormal ones too; the largest is NaN if one is.
__device__ __forceinline__ float larger(float x, float y, float z) {
  float v;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(v) : "f"(x), "f"(y), "f"(z));
  return v;
}
__device__ __forceinline__ float smaller(float x, float y, float z) {
  float v;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(v) : "f"(x), "f"(y), "f"(z));
  return v;
}
template <typename T>
__device__ __forceinline__ void see(T x, float& most, float& least) {
  most = larger(most, to_f(x), to_f(x));
  least = smaller(least, to_f(x), to_f(x));
}

// Tokens that reach a key in order: by the logit as a number, and where that is equal by the key.
struct Border {
  uint64_t key;
  float at;                                // (comparisons take a subnormal logit for 0: among these, too, the key tells)
  __device__ __forceinline__ explicit Border(uint64_t k) : key(k), at(k != 0 ? logit_of(k) : -FLT_MAX) {}
  __device__ __forceinline__ bool keeps(float x, uint32_t token) const { return x > at || (x >= at && key_of(x, token) >= key); }
};
// (Lists are as long as a histogram has counted, if a token's step comes out the same each time it is formed; their places are bounded all the same.)
// The step of a histogram in which a token falls, -1: none.  First equal steps of z, of the tokens that a border keeps; then equal steps of the
// keys from hi down to lo.
struct Where {
  bool linear;
  float top, scale;
  uint64_t lo, hi;
  int shift;
  // Smallest and largest z of the steps a .. b, and a little more.
  __device__ __forceinline__ float2 around(int a, int b) const {
    if (!linear) return make_float2(logit_of(lo), logit_of(hi));
    if (scale == 0.f) return make_float2(-FLT_MAX, top);
    const float from = b == NB - 1 ? -FLT_MAX : top - (float)(b + 1) / scale, to = top - (float)a / scale, slack = 1e-6f * fmaxf(fabsf(from), fabsf(to)) + 1e-30f;
    return make_float2(fmaxf(from - slack - 1e-5f * (float)(b + 1) / scale, -FLT_MAX), to + slack + 1e-5f * (float)a / scale);
  }
  __device__ __forceinline__ int by_logit(float z) const { return (int)fminf((top - z) * scale, (float)(NB - 1)); }
  __device__ __forceinline__ int by_logit(float z, uint32_t token, const Border& border) const {
    return border.keeps(z, token) ? by_logit(z) : -1;
  }
  __device__ __forceinline__ int by_key(float z, uint32_t token) const {
    const uint64_t k = key_of(z, token);
    return k < lo || k > hi ? -1 : (int)((hi - k) >> shift);
  }
  __device__ __forceinline__ int operator()(float z, uint32_t token, const Border& border) const {
    return linear ? by_logit(z, token, border) : by_key(z, token);
  }
};

__device__ __forceinline__ void add_mass(Hist& h, uint32_t b, uint64_t w) {
  const uint32_t lo = (uint32_t)w, old = atomicAdd(&h.lo[b], lo);
  atomicAdd(&h.hi[b], (uint32_t)(w >> 32) + (old + lo < old ? 1u : 0u));
}
__device__ __forceinline__ uint64_t lds64(const uint64_t* p) {
  uint64_t v;
  asm volatile("ld.shared.u64 %0, [%1];" : "=l"(v) : "r"((uint32_t)__cvta_generic_to_shared(p)) : "memory");
  return v;
}
__device__ __forceinline__ void sts64(uint64_t* p, uint64_t v) {
  asm volatile("st.shared.u64 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(p)), "l"(v) : "memory");
}
__device__ __forceinline__ void larger_first(uint64_t& x, uint64_t& y, bool descending) {
  if ((x < y) == descending) {
    const uint64_t t = x;
    x = y;
    y = t;
  }
}
// a[0 .. n) in shared memory, different and not 0, into descending order; a has CAP places.  Bitonic: a warp has 64 places in registers, and what lies further
// apart is exchanged in shared memory.
__device__ __noinline__ void sort_descending(uint64_t* a, int n) {
  static_assert(CAP == NT * 2, "64 places per warp");
  const int tid = threadIdx.x, lane = tid & 31, base = tid / 32 * 64;
  int size = 64;
  while (size < n) size *= 2;
  const bool mine = base < size;                                           // (of the warp)
  uint64_t x = base + lane < n ? lds64(a + base + lane) : 0, y = base + 32 + lane < n ? lds64(a + base + 32 + lane) : 0;
  auto inside = [&](int len) {                                             // distances up to 32
    if (len >= 64) larger_first(x, y, ((base + lane) & len) == 0);
#pragma unroll
    for (int d = 16; d >= 1; d /= 2) {
      if (d >= len) continue;
      const uint64_t ox = __shfl_xor_sync(0xffffffffu, x, d), oy = __shfl_xor_sync(0xffffffffu, y, d);
      const bool first = (lane & d) == 0;
      x = (x > ox) == (first == (((base + lane) & len) == 0)) ? x : ox;
      y = (y > oy) == (first == (((base + 32 + lane) & len) == 0)) ? y : oy;
    }
  };
  if (mine)
    for (int len = 2; len <= 64; len *= 2) inside(len);
  for (int len = 128; len <= size; len *= 2) {
    if (mine) {
      sts64(a + base + lane, x);
      sts64(a + base + 32 + lane, y);
    }
    for (int d = len / 2; d >= 64; d /= 2) {
      __syncthreads();
      if (tid < size / 2) {
        const int i = 2 * tid - (tid & (d - 1));
        uint64_t u = lds64(a + i), v = lds64(a + i + d);
        if ((u < v) == ((i & len) == 0)) {
          sts64(a + i, v);
          sts64(a + i + d, u);
        }
      }
    }
    __syncthreads();
    if (mine) {
      x = lds64(a + base + lane);
      y = lds64(a + base + 32 + lane);
      inside(len);
    }
  }
  __syncthreads();
  if (mine) {
    sts64(a + base + lane, x);
    sts64(a + base + 32 + lane, y);
  }
  __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(NT, 2) sample_kernel(const __grid_constant__ Args a) {
  pdl_begin();
  extern __shared__ __align__(16) uint8_t sa_smem[];
  Shared& sh = *reinterpret_cast<Shared*>(sa_smem);
  T* buf = reinterpret_cast<T*>(sa_smem + (sizeof(Shared) + 15) / 16 * 16);
  cg::cluster_group cl = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int64_t r = blockIdx.x / C;
  const float t = a.temperature != nullptr ? a.temperature[r] : 1.f, p = a.top_p != nullptr ? a.top_p[r] : 1.f;
  const float m = a.min_p != nullptr ? a.min_p[r] : 0.f, u = a.u[r];
  const int k = a.top_k != nullptr ? a.top_k[r] : 0;
  auto result = [&](int32_t token, float logprob, int32_t kept) {
    a.token[r] = token;
    if (a.logprob != nullptr) a.logprob[r] = logprob;
    if (a.kept != nullptr) a.kept[r] = kept;
  };
  if (!from_zero_to(t, FLT_MAX) || !(p == p) || !(m == m) || !from_zero_to(u, 1.f)) {          // (the whole cluster)
    if (rank == 0 && tid == 0) {
      report(a.status, ACTKV_E_INVALID, (int)r, k);
      result(-1, -INFINITY, 0);
    }
    return;
  }

  cluster_arrive();                                                        // (nothing is written into a CTA that has not begun)

  // ---- the row into shared memory, and its largest and smallest logit ----
  const int first = min(a.vocab, rank * a.slice), n_own = min(a.vocab - first, a.slice);
  const T* src = (const T*)a.logits + r * a.row_stride + first;
  constexpr int N = Vec<T>::N;
  const int off = (int)(((uintptr_t)src & 15) / sizeof(T));                 // as far off a vector's beginning as in memory
  T* row = buf + off;
  auto z = [&](int i) { return to_f(row[i]); };
  const int head = min(n_own, (N - off) % N), vecs = (n_own - head) / N;
  float most = -INFINITY, least = INFINITY;                                 // NaN: there is one
  if (tid < head) see(row[tid] = src[tid], most, least);
#pragma unroll 4                                                             // (eight: 72 us instead of 62 for 1024 rows of 32003 tokens, T = 0)
  for (int i = tid; i < vecs; i += NT) {
    const uint4 v = *reinterpret_cast<const uint4*>(src + head + i * N);
    *reinterpret_cast<uint4*>(row + head + i * N) = v;
    float x[N];
    Vec<T>::open(v, x);
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      most = larger(most, x[e], x[e + 1]);
      least = smaller(least, x[e], x[e + 1]);
    }
  }
  {
    const int i = head + vecs * N + tid;
    if (i < n_own) see(row[i] = src[i], most, least);
  }
  int32_t high = ordered(most), low = ordered(least);
  if (tid < 256) sh.tab[tid >> 4][tid & 15] = ROOTS[tid >> 4];
  if (tid == 0) sh.n_list = sh.n_all = 0;
  const bool greedy = __float_as_uint(t) << 1 == 0u || k == 1, by_k = k > 0 && k < a.vocab, by_p = p < 1.f;
  const bool bounded = by_k && k <= SMALL_K;                               // a bound for the k-th largest
  double temp = 1.0, below = 0.0;                                          // temperature, and how far below the largest logit m reaches
  Scale scale;
  if (!greedy) {
    temp = exact_double(t);
    if (positive(m) && m < 1.f) below = temp * log(exact_double(m));
    scale.c = 16.0 * 1.4426950408889634074 / temp;
    scale.limit = __double2hiint(temp * (47.0 * 0.69314718055994530942)) + 1;
  }
  cluster_wait();
  if (bounded && !greedy) {                                                // maxima of 4 C lanes, GROUPS over the cluster
    int32_t g = high;
    for (int o = 1; o < 4 * C; o <<= 1) g = max(g, __shfl_xor_sync(0xffffffffu, g, o));
    g = __shfl_sync(0xffffffffu, g, lane / C * 4 * C);
    if (lane < 8) cl.map_shared_rank(&sh, lane % C)->group[rank * (GROUPS / C) + warp * (8 / C) + lane / C] = g;
  }
  {
    const int32_t h = __reduce_max_sync(0xffffffffu, high), l = __reduce_min_sync(0xffffffffu, low);
    if (lane < C) cl.map_shared_rank(&sh, lane)->ends[rank][warp] = make_int2(h, l);
  }
  cluster_barrier();
  high = INT32_MIN, low = INT32_MAX;
  for (int i = lane; i < C * NW; i += 32) {
    const int2 v = (&sh.ends[0][0])[i];
    high = max(high, v.x);
    low = min(low, v.y);
  }
  high = __reduce_max_sync(0xffffffffu, high);
  low = __reduce_min_sync(0xffffffffu, low);
  if (high == -1) high = 0;                                                // (-0 and +0 are equal)
  if (high >= POS_INF || high <= NEG_INF || low < NEG_INF) {
    if (rank == 0 && tid == 0) result(-1, -INFINITY, 0);
    return;
  }
  const float top = __int_as_float(high ^ ((high >> 31) & 0x7fffffff));
  if (greedy) {
    // the first CTA that has the largest logit looks for it
    int leader = C * NW;
    for (int i = lane; i < C * NW; i += 32) {
      const int32_t h = (&sh.ends[0][0])[i].x;
      if ((h == -1 ? 0 : h) == high) leader = min(leader, i);
    }
    if (rank != __reduce_min_sync(0xffffffffu, leader) / NW) return;
    uint32_t at = ~0u;
    const uint32_t want = okey(top);
    for (int i = tid; i < n_own; i += NT)
      if (okey(z(i)) == want) at = min(at, (uint32_t)i);
    at = __reduce_min_sync(0xffffffffu, at);
    if (lane == 0) sh.scan[0][warp] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < NW; ++w) at = min(at, (uint32_t)sh.scan[0][w]);
      result(first + (int)at, 0.f, 1);
    }
    return;
  }
  scale.top = (double)top;
  auto log_of = [&](float x, uint64_t S) { return (float)(((double)x - scale.top) / temp - log((double)S * 0x1p-45)); };
  uint64_t by_m = 0;                                                       // key of the smallest logit with w >= m
  if (positive(m)) {
    const uint32_t near = okey((float)(scale.top + below));
    const uint32_t mine = near + lane < 16u ? 0u : near + lane - 16u;
    const float x = okey_inv(mine);
    const double w = power(gap_of(x <= top ? x : top, scale.top, __double2hiint(temp * 690.0)), scale.c, 0.0, sh.tab);
    const uint32_t hit = __ballot_sync(0xffffffffu, x == x && x >= -FLT_MAX && w >= exact_double(m));
    // (near a logit of 0 floats lie closer than weights are told apart: any of these is right to 2^-46)
    by_m = (uint64_t)(hit == 0 ? near : near + (uint32_t)__ffs((int)hit) - 17u) << 32;
    by_m = min(m < 1.f ? by_m : ~(uint64_t)0, (uint64_t)okey(top) << 32);   // (1: the largest and its equals, however close others come)
  }

  // All that can be kept is a list of nn tokens in the first CTA, which sorts it, cuts it and draws from it.  cut: the list is to be cut to k; then
  // the mass that p is a part of is the list's.
  auto draw_from_list = [&](int nn, bool cut, uint64_t target) {
    if (nn <= FEW) {                                                       // by counting, four threads a token
      const int i = tid >> 2, q = tid & 3;
      const uint64_t key = i < nn ? sh.all[i] : 0;
      if (tid < nn) sh.mass[0][tid] = weight45(logit_of(sh.all[tid]), scale, sh.tab);
      __syncthreads();
      const uint64_t w = i < nn ? sh.mass[0][i] : 0;
      int place = 0;                                                       // in order, and the mass in front
      uint64_t front = 0;
      for (int o = q; o < nn; o += 4)
        if (sh.all[o] > key) ++place, front += sh.mass[0][o];
      front += __shfl_xor_sync(0xffffffffu, front, 1);
      front += __shfl_xor_sync(0xffffffffu, front, 2);
      place += __shfl_xor_sync(0xffffffffu, place, 1);
      place += __shfl_xor_sync(0xffffffffu, place, 2);
      bool keep = i < nn && (!cut || place < k) && key >= by_m;
      if (by_p) {
        if (cut) {
          // (the last of the first k knows their mass)
          if (q == 0 && i < nn && place == min(k, nn) - 1) sh.found[0] = front + w;
          __syncthreads();
          target = p > 0.f ? max((uint64_t)1, (uint64_t)ceil((double)p * (double)sh.found[0])) : 1;
        }
        keep = keep && front < target;
      }
      if (q == 0 && i < nn) sh.mass[1][i] = keep ? w : 0;
      const int nk = __syncthreads_count(keep && q == 0);
      uint64_t at = 0, S = 0;                                              // in the order of the vocabulary (the lower half: 2^32 - 1 - token)
      for (int o = q; o < nn; o += 4) {
        const uint64_t v = sh.mass[1][o];
        S += v;
        if ((uint32_t)sh.all[o] > (uint32_t)key) at += v;
      }
      at += __shfl_xor_sync(0xffffffffu, at, 1);
      at += __shfl_xor_sync(0xffffffffu, at, 2);
      S += __shfl_xor_sync(0xffffffffu, S, 1);
      S += __shfl_xor_sync(0xffffffffu, S, 2);
      const uint64_t goal = min((uint64_t)((double)u * (double)S), S - 1);
      if (q == 0 && keep && goal >= at && goal < at + w) result((int32_t)(0xffffffffu - (uint32_t)key), log_of(logit_of(key), S), nk);
      return;
    }
    sort_descending(sh.all, nn);
    constexpr int PER = CAP / NT;
    const int most = cut ? min(nn, k) : nn;
    uint64_t w[PER], mine = 0, ones = 0, all, none;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
      w[e] = i < most ? weight45(logit_of(sh.all[i]), scale, sh.tab) : 0;
      mine += w[e];
    }
    block_before(sh, mine, ones, all, none);
    if (cut && by_p) target = p > 0.f ? max((uint64_t)1, (uint64_t)ceil((double)p * (double)all)) : 1;
    // kept: in front of the target, and not too small (a prefix both)
    uint64_t run = mine, kept = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
      if (i < most && (!by_p || run < target) && sh.all[i] >= by_m) ++kept;
      run += w[e];
    }
    uint64_t before_kept = kept, all_kept_n, zero = 0, zeros;
    block_before(sh, before_kept, zero, all_kept_n, zeros);
    const int nk = (int)all_kept_n;
    // in the order of the vocabulary: the masses of stretches of tokens, then the tokens of the one in which u S falls
    const int stretch = max(0, 32 - __clz(a.vocab - 1) - LOG_NB);
    for (int i = tid; i < NB; i += NT) sh.sum.lo[i] = sh.sum.hi[i] = 0;
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    auto token_at = [&](int i) { return 0xffffffffu - (uint32_t)sh.all[i]; };
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
      if (i < nk) add_mass(sh.sum, token_at(i) >> stretch, w[e]);
    }
    __syncthreads();
    uint64_t part[BPT], at = 0, S;
#pragma unroll
    for (int e = 0; e < BPT; ++e) {
      part[e] = ((uint64_t)sh.sum.hi[tid * BPT + e] << 32) + sh.sum.lo[tid * BPT + e];
      at += part[e];
    }
    zero = 0;
    block_before(sh, at, zero, S, zeros);
    const uint64_t goal = min((uint64_t)((double)u * (double)S), S - 1);
#pragma unroll
    for (int e = 0; e < BPT; ++e) {
      if (goal >= at && goal < at + part[e]) sh.found[0] = tid * BPT + e, sh.found[1] = at;
      at += part[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
      if (i < nk && token_at(i) >> stretch == (uint32_t)sh.found[0]) {
        const uint32_t to = atomicAdd(&sh.n_list, 1u);
        sh.list[to] = sh.all[i];
        sh.weight[to] = w[e];
      }
    }
    __syncthreads();
    const int members = (int)sh.n_list;
    for (int i = tid; i < members; i += NT) {
      const uint64_t key = sh.list[i];
      uint64_t before = sh.found[1];
      for (int o = 0; o < members; ++o)
        if ((uint32_t)sh.list[o] > (uint32_t)key) before += sh.weight[o];  // (the lower half: 2^32 - 1 - token)
      if (goal >= before && goal < before + sh.weight[i]) result((int32_t)(0xffffffffu - (uint32_t)key), log_of(logit_of(key), S), nk);
    }
  };

  // ---- the border: tokens that reach it in order are kept ----
  Where where;
  where.top = top;
  const float range = fminf(top - __int_as_float(low ^ ((low >> 31) & 0x7fffffff)), OCTAVES * kLn2 * t);
  Border border(0);
  int listed = -1;                                                         // all that can be kept: so many tokens in the first CTA's list, to be cut to k or not,
  bool cut_k = false;                                                      // and the mass that p asks for
  uint64_t list_target = 0;
  if (bounded) {
    // the smallest of the groups' maxima that fewer than k exceed: the k-th largest
    if (tid == 0) sh.found[0] = 0x7fffffff;
    {
      const int32_t g = sh.group[tid >> 2];
      int over = 0;
#pragma unroll 2
      for (int o = 0; o < GROUPS / 4; o += 4) {
        const int4 x = *reinterpret_cast<const int4*>(sh.group + (tid & 3) * (GROUPS / 4) + o);
        over += (x.x > g ? 1 : 0) + (x.y > g ? 1 : 0) + (x.z > g ? 1 : 0) + (x.w > g ? 1 : 0);
      }
      over += __shfl_xor_sync(0xffffffffu, over, 1);
      over += __shfl_xor_sync(0xffffffffu, over, 2);
      const int32_t least = __reduce_min_sync(0xffffffffu, over < k ? g : INT32_MAX);
      __syncthreads();
      if (lane == 0) atomicMin((int32_t*)&sh.found[0], least);
    }
    __syncthreads();
    // (as a number; of subnormal ones all may pass for 0 and so for as large as the bound, and none is lost)
    const int32_t b = (int32_t)(uint32_t)sh.found[0];
    const float bound = b <= NEG_INF ? -FLT_MAX : __int_as_float(b ^ ((b >> 31) & 0x7fffffff));
    auto take = [&](int i) {
      const uint32_t at = atomicAdd(&sh.n_list, 1u);
      if (at < CAP) sh.list[at] = key_of(z(i), first + i);
    };
    int i = tid;
    for (; i + 3 * NT < n_own; i += 4 * NT) {
      const float x0 = z(i), x1 = z(i + NT), x2 = z(i + 2 * NT), x3 = z(i + 3 * NT);
      if (x0 >= bound || x1 >= bound || x2 >= bound || x3 >= bound) {
        if (x0 >= bound) take(i);
        if (x1 >= bound) take(i + NT);
        if (x2 >= bound) take(i + 2 * NT);
        if (x3 >= bound) take(i + 3 * NT);
      }
    }
    for (; i < n_own; i += NT)
      if (z(i) >= bound) take(i);
    __syncthreads();
    const int room = CAP / C, own = (int)sh.n_list;
    if (tid < C) cl.map_shared_rank(&sh, tid)->few[rank] = own;
    if (own <= room) {
      Shared* to = cl.map_shared_rank(&sh, 0);
      for (int o = tid; o < own; o += NT) to->sent[rank * room + o] = sh.list[o];
    }
    cluster_barrier();
    int n = 0;
    bool fits = true;
    for (int c = 0; c < C; ++c) {
      fits = fits && (int)sh.few[c] <= room;
      n += sh.few[c];
    }
    if (fits) {
      if (rank != 0) return;
      for (int o = tid; o < CAP; o += NT) {
        const int c = o / room, i = o % room;
        if (i >= (int)sh.few[c]) continue;
        int at = i;
        for (int x = 0; x < c; ++x) at += sh.few[x];
        sh.all[at] = sh.sent[o];
      }
      __syncthreads();
      listed = n;
      cut_k = true;
    } else {
      __syncthreads();
      if (tid == 0) sh.n_list = 0;                                         // (many equal logits, or the largest ones in few groups)
      __syncthreads();
    }
  }
#pragma unroll 1
  for (int pass = by_k ? 0 : 1; pass < (by_p ? 2 : 1) && listed < 0; ++pass) {
    const bool mass = pass == 1;
    uint64_t target = (uint64_t)k, above = 0, total = 0;                   // above: what lies over the steps
    int step = 0;
    uint32_t n = 0;
    bool all_kept = false;
    where.linear = true;
    // (the tokens below (1 - p) / vocab have less than 1 - p together, so that the last one to be kept is none of them)
    const float reach = mass ? fminf(range, t * (__logf((float)a.vocab / (1.f - p)) + 0.1f)) : range;
    where.scale = reach > 1e-30f ? (float)NB / reach : 0.f;
#pragma unroll 1
    for (;;) {
      // the joint histogram
      for (int i = tid; i < NB; i += NT) sh.own.cnt[i] = sh.own.lo[i] = sh.own.hi[i] = 0;
      __syncthreads();
      // four at a time, so that they do not wait for one another; the mass of the last step, where p leaves most tokens, is added up here
      uint64_t rest = 0;
      auto count = [&](auto&& step_of) {
        for (int i = tid; i < n_own; i += 4 * NT) {
          int b[4];
          uint64_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = i + e * NT < n_own ? z(i + e * NT) : -INFINITY;
            b[e] = step_of(x, first + i + e * NT);
            w[e] = mass ? weight45(x, scale, sh.tab) : 0;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (b[e] >= 0) atomicAdd(&sh.own.cnt[b[e]], 1u);
            if (b[e] == NB - 1) rest += w[e];
            if (mass && (uint32_t)b[e] < NB - 1) add_mass(sh.own, b[e], w[e]);
          }
        }
      };
      if (!where.linear) count([&](float x, uint32_t token) { return where.by_key(x, token); });
      else count([&](float x, uint32_t token) { return where.by_logit(x, token, border); });
      if (mass) {
        rest = warp_sum(rest);
        if (lane == 0) add_mass(sh.own, NB - 1, rest);
      }
      __syncthreads();
      const int share = NB / C;
      for (int b = tid; b < NB; b += NT) {
        Hist& to = cl.map_shared_rank(&sh, b / share)->inbox;
        const int at = rank * share + b % share;
        to.cnt[at] = sh.own.cnt[b];
        if (mass) {
          to.lo[at] = sh.own.lo[b];
          to.hi[at] = sh.own.hi[b];
        }
      }
      cluster_barrier();
      for (int i = tid; i < share; i += NT) {
        uint32_t nn = 0;
        uint64_t mm = 0;
        for (int c = 0; c < C; ++c) {
          nn += sh.inbox.cnt[c * share + i];
          if (mass) mm += ((uint64_t)sh.inbox.hi[c * share + i] << 32) + sh.inbox.lo[c * share + i];
        }
        for (int c = 0; c < C; ++c) {
          Hist& to = cl.map_shared_rank(&sh, c)->sum;
          to.cnt[rank * share + i] = nn;
          to.lo[rank * share + i] = (uint32_t)mm;
          to.hi[rank * share + i] = (uint32_t)(mm >> 32);
        }
      }
      cluster_barrier();
      // the step in which the target is reached
      uint64_t vn[BPT], vm[BPT], sn = 0, sm = 0, all_n, all_m;
#pragma unroll
      for (int e = 0; e < BPT; ++e) {
        const int b = tid * BPT + e;
        vn[e] = sh.sum.cnt[b];
        vm[e] = ((uint64_t)sh.sum.hi[b] << 32) + sh.sum.lo[b];
        sn += vn[e];
        sm += vm[e];
      }
      block_before(sh, sn, sm, all_n, all_m);
      if (where.linear && mass) {
        total = all_m;
        target = p > 0.f ? max((uint64_t)1, min(total, (uint64_t)ceil((double)p * (double)total))) : 1;
      }
      if (above + (mass ? all_m : all_n) < target) {                       // (fewer tokens than k)
        all_kept = true;
        break;
      }
#pragma unroll
      for (int e = 0; e < BPT; ++e) {
        const uint64_t v = mass ? vm[e] : vn[e], at = above + (mass ? sm : sn);
        if (at < target && at + v >= target) {
          sh.found[0] = tid * BPT + e;
          sh.found[1] = at;
          sh.found[2] = vn[e];
          sh.found[3] = sn + vn[e];                                        // tokens up to the end of the step
        }
        sn += vn[e];
        sm += vm[e];
      }
      __syncthreads();
      step = (int)sh.found[0];
      above = sh.found[1];
      n = (uint32_t)sh.found[2];
      const uint32_t upto = (uint32_t)sh.found[3];
      __syncthreads();

      if (where.linear && upto <= CAP) {
        // All that can be kept is a short list: the first CTA sorts it, cuts it and draws from it.
        Shared* to = cl.map_shared_rank(&sh, 0);
        const float2 near = where.around(0, step);
#pragma unroll 4
        for (int i = tid; i < n_own; i += NT) {
          if (z(i) < near.x) continue;
          const int b = where(z(i), first + i, border);
          if (b < 0 || b > step) continue;
          const uint32_t at = atomicAdd(&to->n_all, 1u);
          if (at < CAP) to->all[at] = key_of(z(i), first + i);
        }
        cluster_barrier();
        if (rank != 0) return;
        listed = (int)upto;
        cut_k = pass == 0;
        list_target = target;
        break;
      }
      if (n <= CAP) break;
      if (where.linear) {                                                  // the keys between which the step's tokens lie
        uint64_t lo = ~0ull, hi = 0;
        for (int i = tid; i < n_own; i += NT) {
          if (where(z(i), first + i, border) == step) {
            const uint64_t key = key_of(z(i), first + i);
            lo = min(lo, key);
            hi = max(hi, key);
          }
        }
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) {
          lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
          hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
        __syncthreads();
        if (lane == 0) sh.scan[0][warp] = lo, sh.scan[1][warp] = hi;
        __syncthreads();
        if (tid < C) {
          for (int w = 0; w < NW; ++w) lo = min(lo, sh.scan[0][w]), hi = max(hi, sh.scan[1][w]);
          uint64_t* to = cl.map_shared_rank(&sh, tid)->range[rank];
          to[0] = lo;
          to[1] = hi;
        }
        cluster_barrier();
        lo = ~0ull, hi = 0;
        for (int c = 0; c < C; ++c) lo = min(lo, sh.range[c][0]), hi = max(hi, sh.range[c][1]);
        where.linear = false;
        where.lo = lo;
        where.hi = hi;
      } else {                                                             // the keys of the step
        const uint64_t hi = where.hi - ((uint64_t)step << where.shift), span = (1ull << where.shift) - 1;
        where.hi = hi;
        where.lo = max(where.lo, hi >= span ? hi - span : (uint64_t)0);
      }
      // (a step of more than one token spans more than one key: they are all different)
      where.shift = max(0, 64 - __clzll((long long)(where.hi - where.lo)) - LOG_NB);
    }
    if (all_kept || listed >= 0) continue;
    // the step's tokens, in every CTA, and sorted
    const float2 near = where.around(step, step);
#pragma unroll 4
    for (int i = tid; i < n_own; i += NT) {
      if (!(z(i) >= near.x && z(i) <= near.y && where(z(i), first + i, border) == step)) continue;
      const uint32_t at = atomicAdd(&sh.n_list, 1u);
      if (at < CAP) sh.list[at] = key_of(z(i), first + i);
    }
    __syncthreads();
    {
      const int own = min((int)sh.n_list, CAP);
      for (int c = warp; c < C; c += NW) {
        Shared* to = cl.map_shared_rank(&sh, c);
        uint32_t at = 0;
        if (lane == 0) at = atomicAdd(&to->n_all, (uint32_t)own);
        at = __shfl_sync(0xffffffffu, at, 0);
        for (int i = lane; i < own && at + i < CAP; i += 32) to->all[at + i] = sh.list[i];
      }
    }
    cluster_barrier();
    sort_descending(sh.all, (int)n);
    constexpr int PER = CAP / NT;
    uint64_t w[PER], at = 0, zero = 0, all, zeros;                       // (one each where k asks)
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
      w[e] = i >= (int)n ? 0 : mass ? weight45(logit_of(sh.all[i]), scale, sh.tab) : 1;
      at += w[e];
    }
    block_before(sh, at, zero, all, zeros);
    at += above;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      if (at < target && at + w[e] >= target) sh.found[0] = sh.all[tid * PER + e];
      at += w[e];
    }
    if (tid == 0) sh.n_list = sh.n_all = 0;
    __syncthreads();
    border = Border(max(border.key, sh.found[0]));
    __syncthreads();
  }

  if (listed >= 0) {
    draw_from_list(listed, cut_k, list_target);
    return;
  }

  // ---- the draw, in the order of the vocabulary ----
  border = Border(max(border.key, by_m));
  const int words = 4 / (int)sizeof(T);                                    // tokens of a bank's word
  const int sub = ((n_own + NT * words - 1) / (NT * words) | 1) * words, i0 = min(n_own, tid * sub), i1 = min(n_own, i0 + sub);   // (an odd number of words: no two lanes on one bank)
  double sum[4] = {SUM45, SUM45, SUM45, SUM45};
  uint32_t kept = i1 - i0;
  const bool some = border.key != 0 || low <= NEG_INF;                     // not all tokens
  if (some) kept = 0;
  if (!some) {
    int i = i0;
    for (; i + 3 < i1; i += 4) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = add45(sum[e], z(i + e), scale, sh.tab);
    }
    for (; i < i1; ++i) sum[0] = add45(sum[0], z(i), scale, sh.tab);
  } else {
    for (int base = i0; base < i1; base += 32) {                           // which are kept, then their weights
      uint32_t bits = 0;
#pragma unroll 4
      for (int i = min(base + 32, i1) - 1; i >= base; --i) bits = bits * 2 + (border.keeps(z(i), first + i) ? 1 : 0);
      kept += __popc(bits);
      while (bits != 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sum[e] = add45(sum[e], bits != 0 ? z(base + __ffs((int)bits) - 1) : -INFINITY, scale, sh.tab);
          bits &= bits - 1;
        }
      }
    }
  }
  static_assert(MAX_SLICE / NT + 4 < 127, "a thread's sum stays below 128");
  const uint64_t mine = of_sum45(sum[0]) + of_sum45(sum[1]) + of_sum45(sum[2]) + of_sum45(sum[3]), upto = warp_scan(mine);
  kept = __reduce_add_sync(0xffffffffu, kept);
  {
    const uint64_t all = __shfl_sync(0xffffffffu, upto, 31);
    if (lane < C) cl.map_shared_rank(&sh, lane)->end[rank][warp] = make_ulonglong2(all, kept);
  }
  cluster_barrier();
  uint64_t S = 0, run = 0;
  uint32_t n_kept = 0;
  for (int i = lane; i < C * NW; i += 32) {
    const ulonglong2 v = (&sh.end[0][0])[i];
    S += v.x;
    run += i < rank * NW + warp ? v.x : 0;
    n_kept += (uint32_t)v.y;
  }
  S = warp_sum(S);
  run = warp_sum(run) + upto - mine;
  n_kept = __reduce_add_sync(0xffffffffu, n_kept);
  const uint64_t goal = min((uint64_t)((double)u * (double)S), S - 1);
  const uint32_t here = __ballot_sync(0xffffffffu, goal >= run && goal < run + mine);
  if (here != 0) {                                                         // one warp of the cluster, along the tokens of one of its lanes
    const int lead = __ffs((int)here) - 1, j1 = __shfl_sync(0xffffffffu, i1, lead);
    uint64_t at = __shfl_sync(0xffffffffu, run, lead);
    for (int j = __shfl_sync(0xffffffffu, i0, lead); j < j1; j += 32) {
      const int i = j + lane;
      const float x = i < j1 ? z(i) : -INFINITY;
      const uint64_t w = border.keeps(x, first + i) ? weight45(x, scale, sh.tab) : 0, up = at + warp_scan(w);
      if (goal < up && goal >= up - w) result(first + i, log_of(x, S), (int32_t)n_kept);
      at = __shfl_sync(0xffffffffu, up, 31);
    }
  }
}

}  // namespace sa
}  // namespace actkv

extern "C" int actkv_sample(const void* logits, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t row_stride, const float* u,
                            const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, int32_t* token,
                            float* logprob, int32_t* kept, int32_t* status, actkv_stream_t stream) {
  using namespace actkv;
  using namespace actkv::sa;
  if ((dtype != ACTKV_F32 && dtype != ACTKV_BF16) || n_rows < 0 || vocab <= 0 || (n_rows > 1 && row_stride < vocab)) return ACTKV_E_INVALID;
  if (n_rows == 0) return ACTKV_OK;
  if (!logits || !u || !token || (uintptr_t)logits % (dtype == ACTKV_BF16 ? 2 : 4) != 0) return ACTKV_E_INVALID;
  static_assert(ACTKV_SAMPLE_MAX_VOCAB == MAX_CLUSTER * MAX_SLICE, "the largest vocabulary");
  if (vocab > ACTKV_SAMPLE_MAX_VOCAB || n_rows > (1 << 27)) return ACTKV_E_TOOBIG;
  Args a = {};
  a.logits = logits;
  a.row_stride = row_stride;
  a.u = u;
  a.temperature = temperature;
  a.top_p = top_p;
  a.min_p = min_p;
  a.top_k = top_k;
  a.token = token;
  a.logprob = logprob;
  a.kept = kept;
  a.status = status;
  a.vocab = vocab;
  // CTAs of a row: so many that two fit on an SM (with half as many and one on an SM: 300 float32 rows of 152K 146 us instead of 137, 64 rows with p = 0.95 98
  // instead of 90, 1024 bf16 rows 318 instead of 290, but 64 whole rows 32.7 instead of 34.7), more while there are CTAs for less than half of the SMs (one row of
  // 32003: 9.2 us with two, 6.5 with eight)
  const int bytes = dtype == ACTKV_BF16 ? 2 : 4;
  int C = 1;
  while (C < MAX_CLUSTER && ((int64_t)vocab * bytes > C * 76032 || (int64_t)n_rows * C * 2 <= 148)) C *= 2;
  a.slice = ((vocab + C - 1) / C + 7) / 8 * 8;
  cudaStream_t s = (cudaStream_t)stream;
  auto go = [&](auto kernel) {
    const size_t smem = (sizeof(Shared) + 15) / 16 * 16 + (size_t)(a.slice + 8) * bytes;
    if (ensure_dyn_smem(kernel, smem) != cudaSuccess) return ACTKV_E_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n_rows * C));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = C;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    (void)cudaLaunchKernelEx(&cfg, kernel, a);
    ACTKV_CHECK_LAUNCH();
    return ACTKV_OK;
  };
  return dtype == ACTKV_BF16 ? go(sample_kernel<__nv_bfloat16>) : go(sample_kernel<float>);
}
