// actkv_sample: a token per row of logits, from what temperature, top-k, top-p and min-p leave.
//
// Weights w = 2^-y, y = (max - z) log2(e) / T, in float64 (a table of 2^(-i/256) and a polynomial of degree 4 in the rest, error below 2^-50), as
// whole multiples of 2^-45: sums of integers are the same in every order and on every split, so that equal arguments draw equal
// tokens, and a sum of 150000 weights is off by less than 2^-36 of the largest one.  (In float32 one draw in some hundred would fall on the
// neighbour of its token, and top-p would keep a token more or less.)
//
// A cluster holds the row in shared memory; it is read once.  Tokens are ordered by (logit descending, token ascending), as 64-bit keys that are all
// different.  Top-k and top-p each ask for the key at which a count or a mass is reached: a histogram of 1024 equal steps of z, whose counts and
// masses are added up over the cluster, tells the step in which it happens; the tokens of the step are sorted, or, when they are more than
// the list holds, spread over a histogram of their keys, and so on.  The draw goes over the kept tokens in the order of the vocabulary: sums per
// thread, per CTA, and then along the thread in which u S falls.
//
// What bounds it: reading the logits; few rows: the chain of passes and cluster barriers.
#include <cooperative_groups.h>

#include <algorithm>

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
template <int NT>
struct Shared {
  union {
    Hist own;                              // this CTA's tokens
    uint64_t all[CAP];                     // written by the others
  };
  union {
    Hist inbox;                            // [CTA][its share of the steps], written by the others
    uint64_t list[CAP];
  };
  union {
    Hist sum;                              // all tokens, written by the others
    uint64_t sorted[CAP];
  };
  double tab[256];
  uint64_t scan[2][32];
  uint64_t found[4];
  struct Part {
    uint64_t best;
    float low;
    uint32_t odd;
  } part[MAX_CLUSTER];                     // written by the others
  uint64_t total[MAX_CLUSTER], range[MAX_CLUSTER][2];
  uint32_t kept[MAX_CLUSTER];
  uint32_t n_list, n_all;
};

// (a subnormal number too, which the library's float32 arithmetic takes for 0)
__device__ __forceinline__ double exact_double(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x7f800000u) != 0 ? (double)x : (b & 0x80000000u ? -1.0 : 1.0) * (double)(int)(b & 0x7fffffu) * 0x1p-149;
}

struct Scale {                             // of a row
  double top, c;                           // largest logit; 256 log2(e) / T
};
// The weight as a float64 (0 below 2^-47).
__device__ __forceinline__ double weight_of(float z, const Scale& s, const double* tab) {
  const double y = (s.top - (double)z) * s.c;
  if (!(y < 256.0 * OCTAVES)) return 0.0;
  const double k = y + MAGIC, r = y - (k - MAGIC);
  const int ki = __double2loint(k);
  constexpr double L = -0.69314718055994530942 / 256.0;
  double p = fma(r, L * L * L * L / 24.0, L * L * L / 6.0);
  p = fma(p, r, L * L / 2.0);
  p = fma(p, r, L);
  p = fma(p, r, 1.0);
  const double m = tab[ki & 255] * p;
  return __hiloint2double(__double2hiint(m) - ((ki >> 8) << 20), __double2loint(m));
}
__device__ __forceinline__ uint64_t fixed45(double w) {
  return (uint64_t)__double_as_longlong(w + MAGIC45) - 0x4068000000000000ull;
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
template <int NT>
__device__ __forceinline__ void block_before(Shared<NT>& sh, uint64_t& a, uint64_t& b, uint64_t& all_a, uint64_t& all_b) {
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
  static __device__ __forceinline__ void put(float* dst, const uint4& v) { *reinterpret_cast<uint4*>(dst) = v; }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void put(float* dst, const uint4& v) {
    reinterpret_cast<uint4*>(dst)[0] = make_uint4(v.x << 16, v.x & 0xffff0000u, v.y << 16, v.y & 0xffff0000u);
    reinterpret_cast<uint4*>(dst)[1] = make_uint4(v.z << 16, v.z & 0xffff0000u, v.w << 16, v.w & 0xffff0000u);
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

template <typename T, int NT>
__global__ void __launch_bounds__(NT) sample_kernel(const __grid_constant__ Args a) {
  pdl_begin();
  constexpr int NW = NT / 32, BPT = NB / NT;
  extern __shared__ __align__(16) uint8_t sa_smem[];
  Shared<NT>& sh = *reinterpret_cast<Shared<NT>*>(sa_smem);
  float* buf = reinterpret_cast<float*>(sa_smem + (sizeof(Shared<NT>) + 15) / 16 * 16);
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

  // ---- the row into shared memory ----
  const int first = min(a.vocab, rank * a.slice), n_own = min(a.vocab - first, a.slice);
  const T* src = (const T*)a.logits + r * a.row_stride + first;
  constexpr int N = Vec<T>::N;
  const int off = (int)(((uintptr_t)src & 15) / sizeof(T));                 // as far off a vector's beginning as in memory
  float* z = buf + off;
  const int head = min(n_own, (N - off) % N), vecs = (n_own - head) / N;
  if (tid < head) z[tid] = to_f(src[tid]);
#pragma unroll 4
  for (int i = tid; i < vecs; i += NT) Vec<T>::put(z + head + i * N, *reinterpret_cast<const uint4*>(src + head + i * N));
  {
    const int i = head + vecs * N + tid;
    if (i < n_own) z[i] = to_f(src[i]);
  }
  for (int i = tid; i < 256; i += NT) sh.tab[i] = exp2(-i / 256.0);
  if (tid == 0) sh.n_list = sh.n_all = 0;
  __syncthreads();
  float low = INFINITY;
  uint64_t best = 0;
  {
    uint32_t high = okey(-INFINITY);                                       // (keys: subnormal logits are told apart)
    int at = 0;
    bool odd = false;
    for (int i = tid; i < n_own; i += NT) {
      const float x = z[i];
      odd |= !(x < INFINITY);
      const uint32_t k32 = okey(x);
      if (k32 > high) high = k32, at = i;
      if (x > -INFINITY) low = fminf(low, x);
    }
    if (high > okey(-INFINITY)) best = ((uint64_t)high << 32) | (0xffffffffu - (uint32_t)(first + at));
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
      best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
      low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    }
    odd = __any_sync(0xffffffffu, odd);
    if (lane == 0) {
      sh.scan[0][warp] = best;
      sh.scan[1][warp] = ((uint64_t)(odd ? 1u : 0u) << 32) | __float_as_uint(low);
    }
    __syncthreads();
    cluster_wait();
    if (warp == 0) {
      const uint64_t v = lane < NW ? sh.scan[1][lane] : (uint64_t)__float_as_uint(INFINITY);
      best = lane < NW ? sh.scan[0][lane] : 0;
      low = __uint_as_float((uint32_t)v);
      odd = __any_sync(0xffffffffu, (v >> 32) != 0);
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) {
        best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
      }
      if (lane < C) {
        auto* to = &cl.map_shared_rank(&sh, lane)->part[rank];
        to->best = best;
        to->low = low;
        to->odd = odd ? 1u : 0u;
      }
    }
    cluster_barrier();
    best = 0;
    low = INFINITY;
    uint32_t any = 0;
    for (int c = 0; c < C; ++c) {
      best = max(best, sh.part[c].best);
      low = fminf(low, sh.part[c].low);
      any |= sh.part[c].odd;
    }
    if (any != 0 || best == 0) {
      if (rank == 0 && tid == 0) result(-1, -INFINITY, 0);
      return;
    }
    if (__float_as_uint(t) << 1 == 0u) {
      if (rank == 0 && tid == 0) result((int32_t)(0xffffffffu - (uint32_t)best), 0.f, 1);
      return;
    }
  }
  const float top = logit_of(best);
  Scale scale;
  scale.top = (double)top;
  const double temp = exact_double(t), least = m < 1.f ? exact_double(m) : 1.0;
  scale.c = 256.0 * 1.4426950408889634074 / temp;
  auto log_of = [&](float x, uint64_t S) { return (float)(((double)x - scale.top) / temp - log((double)S * 0x1p-45)); };

  // ---- the border: tokens that reach it in order are kept ----
  Where where;
  where.top = top;
  const float range = fminf(top - low, OCTAVES * kLn2 * t);
  where.scale = range > 1e-30f ? (float)NB / range : 0.f;
  where.border = 0;
  const bool by_k = k > 0 && k < a.vocab, by_p = p < 1.f;
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
            const uint64_t w = fixed45(weight_of(x, scale, sh.tab));
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
            Shared<NT>* to = cl.map_shared_rank(&sh, 0);
            to->all[atomicAdd(&to->n_all, 1u)] = key_of(z[i], first + i);
          }
        }
        cluster_barrier();
        if (rank != 0) return;
        const int nn = (int)upto;
        for (int i = tid; i < nn; i += NT) {
          const uint64_t key = sh.all[i];
          int before = 0;
#pragma unroll 4
          for (int o = 0; o < nn; ++o) before += sh.all[o] > key ? 1 : 0;
          sh.sorted[before] = key;
        }
        __syncthreads();
        constexpr int PER = CAP / NT;
        const int most = pass == 0 ? min(nn, k) : nn;
        uint64_t w[PER], mine = 0, ones = 0, all, none;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int i = tid * PER + e;
          w[e] = i < most ? fixed45(weight_of(logit_of(sh.sorted[i]), scale, sh.tab)) : 0;
          mine += w[e];
        }
        block_before(sh, mine, ones, all, none);
        if (pass == 0 && by_p) target = p > 0.f ? max((uint64_t)1, (uint64_t)ceil((double)p * (double)all)) : 1;
        // kept: in front of the target, and not too small (a prefix both)
        uint64_t run = mine, kept = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int i = tid * PER + e;
          if (i < most && (!by_p || run < target) && (weight_of(logit_of(sh.sorted[i]), scale, sh.tab) >= least)) ++kept;
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
          w[e] = i < nk ? fixed45(weight_of(logit_of(sh.all[i]), scale, sh.tab)) : 0;
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
        Shared<NT>* to = cl.map_shared_rank(&sh, c);
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
        w[e] = i < (int)n ? fixed45(weight_of(logit_of(sh.sorted[i]), scale, sh.tab)) : 0;
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
  const int sub = ((n_own + NT - 1) / NT) | 1, i0 = min(n_own, tid * sub), i1 = min(n_own, i0 + sub);   // (odd: no two lanes on one bank)
  auto weight = [&](int i, uint64_t& w) {
    const float x = z[i];
    if (x == -INFINITY || key_of(x, first + i) < where.border) return false;
    const double d = weight_of(x, scale, sh.tab);
    w = fixed45(d);
    return d >= least;
  };
  uint64_t mine = 0, kept = 0, own, own_kept;
  for (int i = i0; i < i1; ++i) {
    uint64_t w;
    if (weight(i, w)) mine += w, ++kept;
  }
  uint64_t run = mine;
  block_before(sh, run, kept, own, own_kept);
  if (tid < C) {
    Shared<NT>* to = cl.map_shared_rank(&sh, tid);
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
  if (goal >= run && goal < run + mine) {
    for (int i = i0; i < i1; ++i) {
      uint64_t w;
      if (!weight(i, w)) continue;
      run += w;
      if (run > goal) {
        result(first + i, log_of(z[i], S), (int32_t)n_kept);
        break;
      }
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
  a.slice = ((vocab + C - 1) / C + 31) / 32 * 32;
  cudaStream_t s = (cudaStream_t)stream;
  auto go = [&](auto kernel, int nt, size_t fixed) {
    const size_t smem = (fixed + 15) / 16 * 16 + (size_t)(a.slice + 8) * 4;
    if (ensure_dyn_smem(kernel, smem) != cudaSuccess) return ACTKV_E_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n_rows * C));
    cfg.blockDim = dim3(nt);
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
  // one CTA on an SM: as many threads as two have
  if ((int64_t)n_rows * C <= 148)
    return dtype == ACTKV_BF16 ? go(sample_kernel<__nv_bfloat16, 1024>, 1024, sizeof(Shared<1024>)) : go(sample_kernel<float, 1024>, 1024, sizeof(Shared<1024>));
  return dtype == ACTKV_BF16 ? go(sample_kernel<__nv_bfloat16, 512>, 512, sizeof(Shared<512>)) : go(sample_kernel<float, 512>, 512, sizeof(Shared<512>));
}
