// actkv_sample: a token per row of logits, from what temperature, top-k, top-p and min-p leave.
//
// Weights w = 2^(-y / 16), y = 16 log2(e) (max - z) / T, in float64: 2^(-i/16) from a table, the rest by a polynomial of degree 5 (through the values
// at the Chebyshev nodes of [-1/2, 1/2], its constant term set to 1: below 2^-46), as whole multiples of 2^-45.  Sums of integers are the same in
// every order and on every split, so that equal arguments draw equal tokens, and a sum of 150000 weights is off by less than 2^-36 of the largest one.
// (In float32 one draw in some hundred would fall on the neighbour of its token, and top-p would keep a token more or less.)
//
// A cluster holds the row in shared memory; it is read once.  Tokens are ordered by (logit descending, token ascending), as 64-bit keys that are all
// different, and the kept ones are those that reach a border key.
//   top-k, small: the k-th largest of the maxima of 256 groups of tokens is a bound that k tokens reach; the few that reach it go to the first
// CTA, which sorts them, cuts the list by k, p and m, and draws from it.
//   Otherwise top-k and top-p each ask for the key at which a count or a mass is reached: a histogram of 1024 equal steps of z, whose counts and
// masses are added up over the cluster, tells the step in which it happens.  If the tokens down to it are few, the first CTA goes on with them as above; if not, the
// tokens of the step are sorted, or, when they are more than the list holds, spread over a histogram of their keys, and so on.
//   min-p is a smallest logit, found by trying the floats around max + T ln m.
//   The draw goes over the kept tokens in the order of the vocabulary: sums per thread, per CTA, and then along the tokens of the thread in which u S falls.
//
// What bounds it: few rows: the chain of passes and cluster barriers; many rows: the float64 unit (11 operations a token at 64 a clock
// and SM), beside reading the logits.
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
constexpr double MAGIC45 = 192.0;                     // 1.5 * 2^7: the same in steps of 2^-45
constexpr float OCTAVES = 47.f;                       // weights below 2^-47 are 0
constexpr int NT = 512, NW = NT / 32, BPT = NB / NT;
constexpr int GROUPS = 256;                // of a row's tokens, for the bound of a small top-k
constexpr int SMALL_K = GROUPS / 2;

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

// Parts that are not live together share their place.  What another CTA writes may arrive as soon as this one has joined the barrier before: the
// joint list lies over the own histogram (given away before the barrier in front of the list), the own list over the inbox, the sorted list over the joint
// histogram.
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
  };
  union {
    Hist sum;                              // all tokens, written by the others
    uint64_t sorted[CAP];
  };
  double tab[16][16];                      // 2^(-i/16), sixteen times, so that no two lanes of a half warp meet on a bank
  uint64_t scan[2][NW];
  uint64_t found[4];
  int32_t high[MAX_CLUSTER], low[MAX_CLUSTER];         // largest and smallest logit as ordered(), written by the others
  uint64_t total[MAX_CLUSTER], range[MAX_CLUSTER][2];
  uint32_t kept[MAX_CLUSTER], few[MAX_CLUSTER];
  uint32_t n_list, n_all;
};

// (a subnormal number too, which the library's float32 arithmetic takes for 0)
__device__ __forceinline__ double exact_double(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x7f800000u) != 0 ? (double)x : (b & 0x80000000u ? -1.0 : 1.0) * (double)(int)(b & 0x7fffffu) * 0x1p-149;
}

// Order of the logits as signed integers (-0 just below +0).  NaN lie outside the infinities.
__device__ __forceinline__ int32_t ordered(float x) {
  const int32_t b = __float_as_int(x);
  return b ^ ((b >> 31) & 0x7fffffff);
}
constexpr int32_t POS_INF = 0x7f800000, NEG_INF = (int32_t)0x807fffff;

struct Scale {                             // of a row
  double top, c;                           // largest logit; 16 log2(e) / T
};
// 2^(-y / 16) for y in [0, 2^14], scaled and shifted into the low bits of `onto`.
__device__ __forceinline__ double power(double y, double onto, const double (*tab)[16]) {
  const double k = y + MAGIC, r = y - (k - MAGIC);
  const int ki = __double2loint(k);
  double p = fma(r, -0x1.5d897e525c216p-30, 0x1.3b2c9b8a6caeap-23);
  p = fma(p, r, -0x1.c6b08d6f2a289p-17);
  p = fma(p, r, 0x1.ebfbdff555824p-11);
  p = fma(p, r, -0x1.62e42fefa39f3p-5);
  p = fma(p, r, 1.0);
  const double t = tab[ki & 15][threadIdx.x & 15];
  return fma(__hiloint2double(__double2hiint(t) - ((ki >> 4) << 20), __double2loint(t)), p, onto);
}
// y of a logit, at most `most` (the high word of a limit) and a little.
__device__ __forceinline__ double steps_below(float z, const Scale& s, int most) {
  const double y = (s.top - (double)z) * s.c;
  return __hiloint2double(min(__double2hiint(y), most), __double2loint(y));
}
// The weight in steps of 2^-45.  From y = 752 on it rounds to 0.
__device__ __forceinline__ uint64_t weight45(float z, const Scale& s, const double (*tab)[16]) {
  return (uint64_t)__double_as_longlong(power(steps_below(z, s, 0x40878000), MAGIC45, tab)) - 0x4068000000000000ull;
}

__device__ __forceinline__ uint64_t warp_scan(uint64_t v) {                 // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
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

// The step of a histogram in which a token falls, -1: none.  First equal steps of z, of the tokens that reach `border`; then equal steps of the
// keys from hi down to lo.
struct Where {
  bool linear;
  float top, scale;
  uint64_t border, lo, hi;
  int shift;
  __device__ __forceinline__ int operator()(float z, uint32_t token) const {
    const uint64_t k = key_of(z, token);
    if (linear) return z == -INFINITY || k < border ? -1 : (int)fminf((top - z) * scale, (float)(NB - 1));
    return k < lo || k > hi ? -1 : (int)((hi - k) >> shift);
  }
};

template <typename T>
__global__ void __launch_bounds__(NT, 2) sample_kernel(const __grid_constant__ Args a) {
  pdl_begin();
  extern __shared__ __align__(16) uint8_t sa_smem[];
  Shared& sh = *reinterpret_cast<Shared*>(sa_smem);
  float* buf = reinterpret_cast<float*>(sa_smem + (sizeof(Shared) + 15) / 16 * 16);
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
  if (!(t >= 0.f && t < INFINITY) || !(p == p) || !(m == m) || !(u >= 0.f && u <= 1.f)) {      // (the whole cluster)
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
  float* z = buf + off;
  const int head = min(n_own, (N - off) % N), vecs = (n_own - head) / N;
  int32_t high = INT32_MIN, low = INT32_MAX;
  auto see = [&](float x) {
    const int32_t o = ordered(x);
    high = max(high, o);
    low = min(low, o);
  };
  if (tid < head) see(z[tid] = to_f(src[tid]));
#pragma unroll 4
  for (int i = tid; i < vecs; i += NT) {
    float x[N];
    Vec<T>::open(*reinterpret_cast<const uint4*>(src + head + i * N), x);
#pragma unroll
    for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(z + head + i * N + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
#pragma unroll
    for (int e = 0; e < N; ++e) see(x[e]);
  }
  {
    const int i = head + vecs * N + tid;
    if (i < n_own) see(z[i] = to_f(src[i]));
  }
  if (tid < 256) sh.tab[tid >> 4][tid & 15] = exp2(-(tid >> 4) / 16.0);
  if (tid == 0) sh.n_list = sh.n_all = 0;
  const bool greedy = __float_as_uint(t) << 1 == 0u || k == 1, by_k = k > 0 && k < a.vocab, by_p = p < 1.f;
  const bool bounded = by_k && k <= SMALL_K;                               // a bound for the k-th largest
  cluster_wait();
  if (bounded && !greedy) {                                                // maxima of 2 C lanes, GROUPS over the cluster
    int32_t g = high;
    for (int o = 1; o < 2 * C; o <<= 1) g = max(g, __shfl_xor_sync(0xffffffffu, g, o));
    if (lane % (2 * C) == 0)
      for (int c = 0; c < C; ++c) cl.map_shared_rank(&sh, c)->group[rank * (GROUPS / C) + tid / (2 * C)] = g;
  }
  {
    const int32_t h = __reduce_max_sync(0xffffffffu, high), l = __reduce_min_sync(0xffffffffu, low);
    if (lane == 0) sh.scan[0][warp] = ((uint64_t)(uint32_t)h << 32) | (uint32_t)l;
    __syncthreads();
    if (warp == 0) {
      const uint64_t v = sh.scan[0][lane & (NW - 1)];
      high = __reduce_max_sync(0xffffffffu, (int32_t)(v >> 32));
      low = __reduce_min_sync(0xffffffffu, (int32_t)(uint32_t)v);
      if (lane < C) {
        Shared* to = cl.map_shared_rank(&sh, lane);
        to->high[rank] = high;
        to->low[rank] = low;
      }
    }
  }
  cluster_barrier();
  high = INT32_MIN, low = INT32_MAX;
  int leader = 0;                                                          // the first CTA that has the largest logit
  for (int c = C - 1; c >= 0; --c) {
    const int32_t h = sh.high[c] == -1 ? 0 : sh.high[c];                   // (-0 and +0 are equal)
    if (h >= high) high = h, leader = c;
    low = min(low, sh.low[c]);
  }
  if (high >= POS_INF || high <= NEG_INF || low < NEG_INF) {
    if (rank == 0 && tid == 0) result(-1, -INFINITY, 0);
    return;
  }
  const float top = __int_as_float(high ^ ((high >> 31) & 0x7fffffff));
  if (greedy) {
    if (rank != leader) return;
    uint32_t at = ~0u;
    const uint32_t want = okey(top);
    for (int i = tid; i < n_own; i += NT)
      if (okey(z[i]) == want) at = min(at, (uint32_t)i);
    at = __reduce_min_sync(0xffffffffu, at);
    if (lane == 0) sh.scan[0][warp] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < NW; ++w) at = min(at, (uint32_t)sh.scan[0][w]);
      result(first + (int)at, 0.f, 1);
    }
    return;
  }
  Scale scale;
  scale.top = (double)top;
  const double temp = exact_double(t);
  scale.c = 16.0 * 1.4426950408889634074 / temp;
  auto log_of = [&](float x, uint64_t S) { return (float)(((double)x - scale.top) / temp - log((double)S * 0x1p-45)); };
  uint64_t by_m = 0;                                                       // key of the smallest logit with w >= m
  if (m > 0.f) {
    const uint32_t near = okey((float)(scale.top + (m < 1.f ? temp * log(exact_double(m)) : 0.0)));
    const uint32_t mine = near + lane < 16u ? 0u : near + lane - 16u;
    const float x = okey_inv(mine);
    const double w = power(steps_below(x <= top ? x : top, scale, 0x40d00000), 0.0, sh.tab);
    const uint32_t hit = __ballot_sync(0xffffffffu, x == x && x >= -FLT_MAX && w >= (m < 1.f ? exact_double(m) : 1.0));
    // (near a logit of 0 floats lie closer than weights are told apart: any of these is right to 2^-46)
    by_m = (uint64_t)(hit == 0 ? near : near + (uint32_t)__ffs((int)hit) - 17u) << 32;
    by_m = min(by_m, (uint64_t)okey(top) << 32);
  }

  // All that can be kept is a list of nn tokens in the first CTA, which sorts it, cuts it and draws from it.  cut_k: the list is to be cut to k; then
  // the mass that p is a part of is the list's.
  auto draw_from_list = [&](int nn, bool cut_k, uint64_t target) {
    for (int i = tid; i < nn; i += NT) {
      const uint64_t key = sh.all[i];
      int before = 0;
#pragma unroll 4
      for (int o = 0; o < nn; ++o) before += sh.all[o] > key ? 1 : 0;
      sh.sorted[before] = key;
    }
    __syncthreads();
    constexpr int PER = CAP / NT;
    const int most = cut_k ? min(nn, k) : nn;
    uint64_t w[PER], mine = 0, ones = 0, all, none;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
      w[e] = i < most ? weight45(logit_of(sh.sorted[i]), scale, sh.tab) : 0;
      mine += w[e];
    }
    block_before(sh, mine, ones, all, none);
    if (cut_k && by_p) target = p > 0.f ? max((uint64_t)1, (uint64_t)ceil((double)p * (double)all)) : 1;
    // kept: in front of the target, and not too small (a prefix both)
    uint64_t run = mine, kept = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
      if (i < most && (!by_p || run < target) && sh.sorted[i] >= by_m) ++kept;
      run += w[e];
    }
    uint64_t before_kept = kept, all_kept_n, zero = 0, zeros;
    block_before(sh, before_kept, zero, all_kept_n, zeros);
    const int nk = (int)all_kept_n;
    // in the order of the vocabulary
    for (int i = tid; i < nk; i += NT) {
      const uint64_t key = sh.sorted[i];
      const uint32_t token = (uint32_t)key;
      int before = 0;
#pragma unroll 4
      for (int o = 0; o < nk; ++o) before += (uint32_t)sh.sorted[o] > token ? 1 : 0;    // (the lower half: 2^32 - 1 - token)
      sh.all[before] = key;
    }
    __syncthreads();
    mine = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid * PER + e;
      w[e] = i < nk ? weight45(logit_of(sh.all[i]), scale, sh.tab) : 0;
      mine += w[e];
    }
    uint64_t at = mine, S;
    zero = 0;
    block_before(sh, at, zero, S, zeros);
    const uint64_t goal = min((uint64_t)((double)u * (double)S), S - 1);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      if (goal >= at && goal < at + w[e]) {
        const uint64_t key = sh.all[tid * PER + e];
        result((int32_t)(0xffffffffu - (uint32_t)key), log_of(logit_of(key), S), nk);
      }
      at += w[e];
    }
  };

  // ---- the border: tokens that reach it in order are kept ----
  Where where;
  where.top = top;
  const float range = fminf(top - __int_as_float(low ^ ((low >> 31) & 0x7fffffff)), OCTAVES * kLn2 * t);
  where.scale = range > 1e-30f ? (float)NB / range : 0.f;
  where.border = 0;
  if (bounded) {
    if (tid < GROUPS) {
      const int32_t g = sh.group[tid];
      int before = 0;
#pragma unroll 8
      for (int o = 0; o < GROUPS; ++o) {
        const int32_t x = sh.group[o];
        before += x > g || (x == g && o < tid) ? 1 : 0;
      }
      if (before == k - 1) sh.found[0] = (uint32_t)(g == 0 ? -1 : g);       // (-0 is as large as +0)
    }
    __syncthreads();
    const int32_t bound = (int32_t)(uint32_t)sh.found[0];
    for (int i = tid; i < n_own; i += NT) {
      const int32_t o = ordered(z[i]);
      if (o >= bound && o > NEG_INF) {
        const uint32_t at = atomicAdd(&sh.n_list, 1u);
        if (at < CAP) sh.list[at] = key_of(z[i], first + i);
      }
    }
    __syncthreads();
    if (tid < C) cl.map_shared_rank(&sh, tid)->few[rank] = sh.n_list;
    cluster_barrier();
    uint32_t at = 0, n = 0;
    for (int c = 0; c < C; ++c) {
      at += c < rank ? sh.few[c] : 0;
      n += sh.few[c];
    }
    if (n <= CAP) {
      Shared* to = cl.map_shared_rank(&sh, 0);
      for (int i = tid; i < (int)sh.n_list; i += NT) to->all[at + i] = sh.list[i];
      cluster_barrier();
      if (rank == 0) draw_from_list((int)n, true, 0);
      return;
    }
    __syncthreads();
    if (tid == 0) sh.n_list = 0;                                           // (many equal logits, or the largest ones in few groups)
    __syncthreads();
  }
#pragma unroll 1
  for (int pass = by_k ? 0 : 1; pass < (by_p ? 2 : 1); ++pass) {
    const bool mass = pass == 1;
    uint64_t target = (uint64_t)k, above = 0, total = 0;                   // above: what lies over the steps
    int step = 0;
    uint32_t n = 0;
    bool all_kept = false;
    where.linear = true;
#pragma unroll 1
    for (;;) {
      // the joint histogram
      for (int i = tid; i < NB; i += NT) sh.own.cnt[i] = sh.own.lo[i] = sh.own.hi[i] = 0;
      __syncthreads();
      for (int i = tid; i < n_own; i += NT) {
        const float x = z[i];
        const int b = where(x, first + i);
        if (b >= 0) {
          atomicAdd(&sh.own.cnt[b], 1u);
          if (mass) {
            const uint64_t w = weight45(x, scale, sh.tab);
            const uint32_t wl = (uint32_t)w, old = atomicAdd(&sh.own.lo[b], wl);
            atomicAdd(&sh.own.hi[b], (uint32_t)(w >> 32) + (old + wl < old ? 1u : 0u));
          }
        }
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
        for (int i = tid; i < n_own; i += NT) {
          const int b = where(z[i], first + i);
          if (b >= 0 && b <= step) {
            Shared* to = cl.map_shared_rank(&sh, 0);
            to->all[atomicAdd(&to->n_all, 1u)] = key_of(z[i], first + i);
          }
        }
        cluster_barrier();
        if (rank == 0) draw_from_list((int)upto, pass == 0, target);
        return;
      }
      if (n <= CAP) break;
      if (where.linear) {                                                  // the keys between which the step's tokens lie
        uint64_t lo = ~0ull, hi = 0;
        for (int i = tid; i < n_own; i += NT) {
          if (where(z[i], first + i) == step) {
            const uint64_t key = key_of(z[i], first + i);
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
    if (all_kept) continue;
    // the step's tokens, in every CTA, and sorted
    for (int i = tid; i < n_own; i += NT)
      if (where(z[i], first + i) == step) sh.list[atomicAdd(&sh.n_list, 1u)] = key_of(z[i], first + i);
    __syncthreads();
    {
      const int own = (int)sh.n_list;
      for (int c = warp; c < C; c += NW) {
        Shared* to = cl.map_shared_rank(&sh, c);
        uint32_t at = 0;
        if (lane == 0) at = atomicAdd(&to->n_all, (uint32_t)own);
        at = __shfl_sync(0xffffffffu, at, 0);
        for (int i = lane; i < own; i += 32) to->all[at + i] = sh.list[i];
      }
    }
    cluster_barrier();
    for (int i = tid; i < (int)n; i += NT) {
      const uint64_t key = sh.all[i];
      int before = 0;
#pragma unroll 4
      for (int o = 0; o < (int)n; ++o) before += sh.all[o] > key ? 1 : 0;
      sh.sorted[before] = key;
    }
    __syncthreads();
    if (!mass) {
      if (tid == 0) sh.found[0] = sh.sorted[target - above - 1];
    } else {
      constexpr int PER = CAP / NT;
      uint64_t w[PER], at = 0, zero = 0, all, zeros;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int i = tid * PER + e;
        w[e] = i < (int)n ? weight45(logit_of(sh.sorted[i]), scale, sh.tab) : 0;
        at += w[e];
      }
      block_before(sh, at, zero, all, zeros);
      at += above;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        if (at < target && at + w[e] >= target) sh.found[0] = sh.sorted[tid * PER + e];
        at += w[e];
      }
    }
    if (tid == 0) sh.n_list = sh.n_all = 0;
    __syncthreads();
    where.border = max(where.border, sh.found[0]);
    __syncthreads();
  }

  // ---- the draw, in the order of the vocabulary ----
  where.border = max(where.border, by_m);
  const int sub = ((n_own + NT - 1) / NT) | 1, i0 = min(n_own, tid * sub), i1 = min(n_own, i0 + sub);   // (odd: no two lanes on one bank)
  uint64_t mine = 0, kept = 0, own, own_kept;
  if (where.border == 0) {
    int n = 0;
#pragma unroll 4
    for (int i = i0; i < i1; ++i) {
      const float x = z[i];
      mine += weight45(x, scale, sh.tab);                                  // (0 for -inf)
      n += x != -INFINITY ? 1 : 0;
    }
    kept = n;
  } else {
    for (int i = i0; i < i1; ++i) {
      const float x = z[i];
      if (key_of(x, first + i) >= where.border && x != -INFINITY) mine += weight45(x, scale, sh.tab), ++kept;
    }
  }
  uint64_t run = mine;
  block_before(sh, run, kept, own, own_kept);
  if (tid < C) {
    Shared* to = cl.map_shared_rank(&sh, tid);
    to->total[rank] = own;
    to->kept[rank] = (uint32_t)own_kept;
  }
  cluster_barrier();
  uint64_t S = 0;
  uint32_t n_kept = 0;
  for (int c = 0; c < C; ++c) {
    run += c < rank ? sh.total[c] : 0;
    S += sh.total[c];
    n_kept += sh.kept[c];
  }
  const uint64_t goal = min((uint64_t)((double)u * (double)S), S - 1);
  const uint32_t here = __ballot_sync(0xffffffffu, goal >= run && goal < run + mine);
  if (here != 0) {                                                         // one warp of the cluster, along the tokens of one of its lanes
    const int lead = __ffs((int)here) - 1, j1 = __shfl_sync(0xffffffffu, i1, lead);
    uint64_t at = __shfl_sync(0xffffffffu, run, lead);
    for (int j = __shfl_sync(0xffffffffu, i0, lead); j < j1; j += 32) {
      const int i = j + lane;
      const float x = i < j1 ? z[i] : -INFINITY;
      const uint64_t w = x != -INFINITY && key_of(x, first + i) >= where.border ? weight45(x, scale, sh.tab) : 0, up = at + warp_scan(w);
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
  // CTAs of a row: so many that two fit on an SM, more while the SMs have not two each
  int C = 1;
  while (C < MAX_CLUSTER && (vocab > C * 19008 || (int64_t)n_rows * C * 2 <= 148)) C *= 2;
  a.slice = ((vocab + C - 1) / C + 7) / 8 * 8;
  cudaStream_t s = (cudaStream_t)stream;
  auto go = [&](auto kernel) {
    const size_t smem = (sizeof(Shared) + 15) / 16 * 16 + (size_t)(a.slice + 8) * 4;
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
