// actkv_logprob: log probabilities of given tokens, entropy and the top alternatives of every logits row, in one sweep.
//
// Per thread, with m the largest logit it has met, c = log2 e and r = c m rounded: y = c x - r (one fused operation), S = sum 2^y,
// T = sum 2^y y; when r moves by d, S' = S 2^-d and T' = (T - d S) 2^-d.  Behind the sweep both are taken from r to c m itself (by the
// remainder c m - r), so that nothing is lost to the size of the logits, and joined over the row: s = ln 2 log2 S, lse = m + s,
// log P(t) = (x_t - m) - s, entropy = s - ln 2 T / S.  Sums go in pairs (two-lane instructions), 3.5 instructions a logit instead of 7 (1500 rows,
// 20 alternatives: 172 -> 166 us).  Logits beyond 10^37 and -inf take a longer way to the same sums.
//
// Top alternatives.  While it streams, a thread notes the maximum of every 16 logits (a slot).  Behind the sweep the CTA has 128
// groups of threads; the top_k-th largest of the groups' maxima is a bound that top_k logits reach, so only they and the few
// others that reach it (64: about 25 more, in random order) can be among the top_k.  The slots that reach
// the bound are read again, a thread per logit, and the candidates are ranked by counting, as 64-bit keys (order-preserving image of
// the logit, then the token, lower ones first), so that ties need no further rule.  No barrier and no shared counter while
// the row is read: with candidates gathered on the way, under a bound from the row's beginning, 1500 rows of 152K took 278 us
// at top_k 8, of which 126 went to that.  Rows with more candidates than the list holds (long ties, a row in an order
// that puts its largest logits into few threads) are read a second time, step by step, with the list cut to top_k whenever it fills.
//
// What bounds it: reading the logits once.  Few rows: a cluster of CTAs per row, joined through distributed shared memory.
#include <cooperative_groups.h>

#include "common.cuh"

namespace actkv {
namespace lp {

constexpr int GROUPS = 128;               // groups of threads whose maxima give the bound
constexpr int PER = 16;                   // logits of a thread per step
constexpr int SLOTS = 24;                 // maxima that a thread notes, at most (longer rows: of several steps each)
constexpr int LIST = 1024;                // candidates kept
constexpr int TIGHT = 256;                // second reading: candidates that stay between two steps, at most
constexpr float NO_REF = -3.402823466e38f;
constexpr float FAR = -1e4f;              // 2 to its power is 0
constexpr float HUGE_LOGIT = 1e37f;

struct Args {
  const void* logits;
  int64_t row_stride;
  const int32_t* given;
  float *logprob, *entropy, *lse, *top_logprob;
  int32_t* top_index;
  int32_t* status;
  int32_t vocab, n_given, top_k;
};

__device__ __forceinline__ uint32_t okey(float x) {
  uint32_t b = __float_as_uint(x);
  if (b == 0x80000000u) b = 0u;                                            // -0 and +0 are equal
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
constexpr uint32_t LEAST_ZERO = ~0x807fffffu;                              // okey of the negative subnormal furthest from 0
__device__ __forceinline__ float okey_inv(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token) { return ((uint64_t)okey(x) << 32) | (0xffffffffu - token); }

__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b0, float b1, float c0, float c1) {
  uint64_t a, b, c, d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(a) : "f"(a0), "f"(a1));
  asm("mov.b64 %0, {%1, %2};" : "=l"(b) : "f"(b0), "f"(b1));
  asm("mov.b64 %0, {%1, %2};" : "=l"(c) : "f"(c0), "f"(c1));
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(d0), "=f"(d1) : "l"(d));
}
__device__ __forceinline__ void add2(float& s0, float& s1, float a0, float a1) {
  uint64_t s, a;
  asm("mov.b64 %0, {%1, %2};" : "=l"(s) : "f"(s0), "f"(s1));
  asm("mov.b64 %0, {%1, %2};" : "=l"(a) : "f"(a0), "f"(a1));
  asm("add.rn.f32x2 %0, %0, %1;" : "+l"(s) : "l"(a));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(s0), "=f"(s1) : "l"(s));
}

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }   // -inf
  static __device__ __forceinline__ void open(const uint4& v, float* x) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
  static __device__ __forceinline__ void open(const uint4& v, float* x) {
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

template <int NT>
struct Smem {
  static constexpr int CAP = NT * 8 + TIGHT;   // second reading: candidates with those of a step (one vector per thread)
  union {
    float slot[SLOTS][NT];
    uint64_t cand[CAP];
  };
  uint64_t list[LIST];                    // candidates; then the CTA's top k, descending
  float4 red[NT / 32];                     // (m, S, T) of the warps
  float group[GROUPS];
  uint32_t hist[256];
  float4 mst;                             // (m, S, T) of the CTA
  int n_best;
  uint32_t item[LIST];                    // slots that are read again
  uint32_t n_cand, n_item, thr;
  uint32_t pick[3];
};

template <int NT, int W>
__device__ __forceinline__ void rank_few(uint64_t* cand, int n, int k) {
  const int tid = threadIdx.x, i = tid / W;
  const uint64_t a = i < n ? cand[i] : 0;
  int r = 0;
#pragma unroll 4
  for (int o = tid % W; o < n; o += W) r += cand[o] > a ? 1 : 0;
#pragma unroll
  for (int d = 1; d < W; d <<= 1) r += __shfl_xor_sync(0xffffffffu, r, d);
  __syncthreads();
  if (i < n && tid % W == 0 && r < k) cand[r] = a;
  __syncthreads();
}

// The k largest of cand[0 .. n) in descending order into cand[0 .. min(n, k)).  All threads call it, between barriers.
template <int NT>
__device__ __noinline__ void cut(Smem<NT>* sm, uint64_t* cand, int n, int k) {
  constexpr int CAP = Smem<NT>::CAP;
  const int tid = threadIdx.x;
  if (n > NT / 2 && n > k) {
    // the k-th largest key, digit by digit, until what shares its digits is wanted whole; then only what is not smaller stays (all keys are
    // different).  (1009 candidates of a short, masked row: ranked against each other 30 us.)
    uint64_t prefix = 0;
    uint32_t left = (uint32_t)k;
    int shift = 56;
    for (;; shift -= 8) {
      for (int i = tid; i < 256; i += NT) sm->hist[i] = 0;
      __syncthreads();
      for (int i = tid; i < n; i += NT) {
        const uint64_t key = cand[i];
        if (shift == 56 || (key >> (shift + 8)) == prefix) atomicAdd(&sm->hist[(uint32_t)(key >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (tid < 32) {                                          // lane t has digits 255 - 8 t downwards
        uint32_t h[8], mine = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          h[j] = sm->hist[255 - 8 * tid - j];
          mine += h[j];
        }
        uint32_t incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const uint32_t t = __shfl_up_sync(0xffffffffu, incl, d);
          if (tid >= d) incl += t;
        }
        uint32_t above = incl - mine;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (above < left && above + h[j] >= left) {
            sm->pick[0] = (uint32_t)(255 - 8 * tid - j);
            sm->pick[1] = left - above;
            sm->pick[2] = h[j];
          }
          above += h[j];
        }
      }
      __syncthreads();
      prefix = (prefix << 8) | sm->pick[0];
      left = sm->pick[1];
      const bool done = sm->pick[2] == left || shift == 0;
      __syncthreads();
      if (done) break;
    }
    const uint64_t least = prefix << shift;
    uint64_t mine[(CAP + NT - 1) / NT];
#pragma unroll
    for (int j = 0; j < (CAP + NT - 1) / NT; ++j) {
      const int i = tid + j * NT;
      mine[j] = i < n ? cand[i] : 0;
      if (!(i < n && mine[j] >= least)) mine[j] = 0;                       // (no key is 0: a token is below 2^31)
    }
    if (tid == 0) sm->pick[0] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < (CAP + NT - 1) / NT; ++j)
      if (mine[j] != 0) cand[atomicAdd(&sm->pick[0], 1u)] = mine[j];
    __syncthreads();
    n = (int)sm->pick[0];
    __syncthreads();
  }
  // ranks by counting; with few candidates several lanes share one
  if (n <= NT / 8) return rank_few<NT, 8>(cand, n, k);
  if (n <= NT / 4) return rank_few<NT, 4>(cand, n, k);
  rank_few<NT, 2>(cand, n, k);
}

__device__ __forceinline__ float4 join(float4 a, float4 b) {               // (m, S, T)
  const float m = fmaxf(a.x, b.x);
  // (distances of up to 2^128 are cut where the power is 0 long since: no infinity meets that 0)
  const float da = fmaxf((a.x - m) * kLog2e, FAR), db = fmaxf((b.x - m) * kLog2e, FAR);
  const float fa = exp2f(da), fb = exp2f(db);
  return make_float4(m, a.y * fa + b.y * fb, (a.z + da * a.y) * fa + (b.z + db * b.y) * fb, 0.f);
}

// Second reading of a row's part, for the top k of rows whose candidates do not fit the list: the logits of a vector per thread and step,
// one by one, the list cut to the k largest whenever more than TIGHT are in it.  Logits below the image `thr` are none of them.
template <int NT, typename T>
__device__ __noinline__ int top_again(Smem<NT>* sm, const T* z, int mis, int vocab, int v0, int v1, int k, uint32_t thr) {
  constexpr int VE = Vec<T>::N;
  const int tid = threadIdx.x;
  static_assert(NT * VE + TIGHT <= Smem<NT>::CAP, "a step fits");
  __syncthreads();
  if (tid == 0) sm->n_cand = 0;
  __syncthreads();
  for (int vb = v0; vb < v1; vb += NT) {
    const int v = vb + tid;
    int over = 0;
    for (int e = 0; e < VE; ++e) {
      const int64_t t = (int64_t)v * VE + e - mis;
      if (v >= v1 || t < 0 || t >= vocab) continue;
      const float x = to_f(z[t]);
      if (okey(x) < thr) continue;
      const uint32_t at = atomicAdd(&sm->n_cand, 1u);
      sm->cand[at] = key_of(x, (uint32_t)t);                               // (at most TIGHT before the step: it fits)
      over |= at >= TIGHT;
    }
    if (__syncthreads_or(over)) {
      cut<NT>(sm, sm->cand, (int)sm->n_cand, k);
      if (tid == 0) sm->n_cand = (uint32_t)k;                              // (more than TIGHT >= k there were)
      // what comes later is larger as a token: an equal logit no longer counts
      thr = (uint32_t)(sm->cand[k - 1] >> 32);
      thr = thr == 0xffffffffu ? thr : thr + 1;
      __syncthreads();
    }
  }
  const int n = (int)sm->n_cand;
  cut<NT>(sm, sm->cand, n, k);
  for (int i = tid; i < min(n, k); i += NT) sm->list[i] = sm->cand[i];
  __syncthreads();
  return min(n, k);
}

template <typename T, int NT, int C>
__global__ void __launch_bounds__(NT, 1024 / NT) logprob_kernel(const Args a) {
  const void* logits = a.logits;
  pdl_begin(logits);
  extern __shared__ __align__(16) uint8_t lp_smem[];
  Smem<NT>* sm = reinterpret_cast<Smem<NT>*>(lp_smem);
  constexpr int VE = Vec<T>::N, U = PER / VE;                              // vectors of a thread per step
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / C, part = blockIdx.x % C;
  const int vocab = a.vocab, k = a.top_k;
  const T* z = reinterpret_cast<const T*>(logits) + (int64_t)row * a.row_stride;
  const int mis = (int)(((uintptr_t)z & 15) / sizeof(T));                  // logits of the first vector that belong to others
  const uint4* zv = reinterpret_cast<const uint4*>(z - mis);
  const int nv = (int)(((int64_t)mis + vocab + VE - 1) / VE);
  const int v0 = (int)((int64_t)nv * part / C), v1 = (int)((int64_t)nv * (part + 1) / C);
  // vectors of which all logits are the row's own; the others (at most one at each end) are read one by one
  const int in0 = mis > 0 ? 1 : 0, in1 = (int)(((int64_t)mis + vocab) / VE);
  auto read = [&](int v) {
    uint4 r = Vec<T>::none();
    if (v < v1) {
      if (v >= in0 && v < in1) {
        r = __ldg(zv + v);
      } else {
        T* one = reinterpret_cast<T*>(&r);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const int64_t t = (int64_t)v * VE + e - mis;
          if (t >= 0 && t < vocab) one[e] = z[t];
        }
      }
    }
    return r;
  };
  uint4 next[U];
#pragma unroll
  for (int u = 0; u < U; ++u) next[u] = read(v0 + u * NT + tid);
  int32_t tok = -1;
  float ztok = 0.f;
  if (part == 0 && tid < a.n_given) {                                      // (early: beside the row's own loads)
    tok = a.given[(int64_t)row * a.n_given + tid];
    if (tok >= 0 && tok < vocab) ztok = to_f(z[tok]);
  }

  const int steps = (v1 - v0 + NT * U - 1) / (NT * U), per_slot = (steps + SLOTS - 1) / SLOTS;
  float m = NO_REF, r = 0.f, S0 = 0.f, S1 = 0.f, T0 = 0.f, T1 = 0.f;
  bool big = true;                                                         // m is too large for r
  float tm = -INFINITY, slot_max = -INFINITY;                              // of the thread's logits, of the slot's
  int slot = 0, in_slot = 0;
  for (int vb = v0; vb < v1; vb += NT * U) {
    float x[PER];
#pragma unroll
    for (int u = 0; u < U; ++u) Vec<T>::open(next[u], x + u * VE);
    if (vb + NT * U < v1) {                                                // (in flight while this step is worked on)
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = read(vb + NT * U + u * NT + tid);
    }
    float mx = x[0], mn = x[0];
#pragma unroll
    for (int e = 1; e < PER; ++e) {
      mx = fmaxf(mx, x[e]);
      mn = fminf(mn, x[e]);
    }
    slot_max = fmaxf(slot_max, mx);
    if (++in_slot == per_slot) {
      sm->slot[slot++][tid] = slot_max;
      tm = fmaxf(tm, slot_max);
      slot_max = -INFINITY;
      in_slot = 0;
    }
    if (mx > m) {
      const bool far = fabsf(mx) > HUGE_LOGIT;
      const float to = mx * kLog2e, d = fmaxf(far || big ? (m - mx) * kLog2e : r - to, FAR), f = exp2f(d);
      T0 = (T0 + d * S0) * f;
      T1 = (T1 + d * S1) * f;
      S0 *= f;
      S1 *= f;
      m = mx;
      r = to;
      big = far;
    }
    if (!big && mn > -HUGE_LOGIT) {
#pragma unroll
      for (int e = 0; e < PER; e += 2) {
        float y0, y1;
        fma2(y0, y1, x[e], x[e + 1], kLog2e, kLog2e, -r, -r);
        const float p0 = exp2f(y0), p1 = exp2f(y1);
        add2(S0, S1, p0, p1);
        fma2(T0, T1, p0, p1, y0, y1, T0, T1);
      }
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const float y = big ? (x[e] - m) * kLog2e : fmaf(x[e], kLog2e, -r), p = exp2f(y);
        S0 += p;
        T0 = fmaf(p, fmaxf(y, FAR), T0);                                   // (p is 0 long before; -inf must not meet it)
      }
    }
  }
  if (in_slot > 0) {
    sm->slot[slot++][tid] = slot_max;
    tm = fmaxf(tm, slot_max);
  }

  // ---- (m, S, T) of the warps; maxima of the groups ----
  float4 mst;
  {
    const float S = S0 + S1, rest = big ? 0.f : fmaf(m, kLog2e, -r), f = exp2f(-rest);
    mst = make_float4(m, S * f, (T0 + T1 - rest * S) * f, 0.f);
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    const float4 b = make_float4(__shfl_xor_sync(0xffffffffu, mst.x, o), __shfl_xor_sync(0xffffffffu, mst.y, o),
                                 __shfl_xor_sync(0xffffffffu, mst.z, o), 0.f);
    mst = (lane & o) ? join(b, mst) : join(mst, b);
  }
  if (lane == 0) sm->red[warp] = mst;
  constexpr int TG = NT / GROUPS;                                          // threads of a group
  float gm = tm;
#pragma unroll
  for (int d = 1; d < TG; d <<= 1) gm = fmaxf(gm, __shfl_xor_sync(0xffffffffu, gm, d));
  if (tid % TG == 0) sm->group[tid / TG] = gm;
  if (tid == 0) sm->n_cand = sm->n_item = 0;
  __syncthreads();
  mst = sm->red[0];
#pragma unroll
  for (int w = 1; w < NT / 32; ++w) mst = join(mst, sm->red[w]);

  int n_top = 0;
  if (k > 0) {
    // the bound: the k-th largest of the groups' maxima (the threads of a group count its rank)
    {
      const int c = tid / TG;
      const float v = sm->group[c];
      int rank = 0;
#pragma unroll 8
      for (int o = tid % TG; o < GROUPS; o += TG) {
        const float w = sm->group[o];
        rank += w > v || (w == v && o < c) ? 1 : 0;
      }
#pragma unroll
      for (int d = 1; d < TG; d <<= 1) rank += __shfl_xor_sync(0xffffffffu, rank, d);
      // (maxima are flushed: one that is 0 may stand for any subnormal logit, while candidates are compared by their bits)
      if (rank == k - 1 && tid % TG == 0) sm->thr = v == -INFINITY ? 0u : v == 0.f ? LEAST_ZERO : okey(v);
    }
    __syncthreads();
    const uint32_t thr = sm->thr;
    const float bound = thr == 0 ? -INFINITY : okey_inv(thr);
    // slots that reach it, then their logits, spread over all threads: one round trip to memory
    if (tm >= bound)
      for (int sl = 0; sl < slot; ++sl)
        if (sm->slot[sl][tid] >= bound) {
          const uint32_t at = atomicAdd(&sm->n_item, 1u);
          if (at < LIST) sm->item[at] = (uint32_t)(sl * NT + tid);
        }
    __syncthreads();
    const uint32_t items = sm->n_item;
    if (items <= LIST) {
      const int per_item = per_slot * PER;
      for (int i = tid; i < (int)items * per_item; i += NT) {
        const int it = i / per_item, in = i - it * per_item, st = in / PER, e = in % PER;
        const int sl = (int)(sm->item[it] / NT), who = (int)(sm->item[it] % NT), step = sl * per_slot + st;
        const int v = v0 + (step * U + e / VE) * NT + who;
        const int64_t t = (int64_t)v * VE + e % VE - mis;
        if (step >= steps || v >= v1 || t < 0 || t >= vocab) continue;
        const float x = to_f(z[t]);
        if (okey(x) >= thr) {
          const uint32_t at = atomicAdd(&sm->n_cand, 1u);
          if (at < LIST) sm->list[at] = key_of(x, (uint32_t)t);
        }
      }
    }
    __syncthreads();
    const uint32_t n = sm->n_cand;
    if (items <= LIST && n <= LIST) {
      cut<NT>(sm, sm->list, (int)n, k);
      n_top = min((int)n, k);
    } else {
      n_top = top_again<NT, T>(sm, z, mis, vocab, v0, v1, k, thr);
    }
  }
  if constexpr (C > 1) {
    namespace cg = cooperative_groups;
    cg::cluster_group cl = cg::this_cluster();
    if (tid == 0) {
      sm->mst = mst;
      sm->n_best = n_top;
    }
    cl.sync();
    if (part == 0) {
      // the others' parts: every thread one key, all reads in flight at once
      int n = n_top;
      int from[C];
#pragma unroll
      for (int c = 1; c < C; ++c) {
        from[c] = n;
        n += cl.map_shared_rank(sm, c)->n_best;
      }
#pragma unroll
      for (int c = 1; c < C; ++c) {
        const Smem<NT>* other = cl.map_shared_rank(sm, c);
        mst = join(mst, other->mst);
      }
      from[0] = 0;
      auto list_of = [&](int i) {
        int c = 0;
#pragma unroll
        for (int d = 1; d < C; ++d) c = i >= from[d] ? d : c;
        return c;
      };
      auto start_of = [&](int c) {
        int at = 0;
#pragma unroll
        for (int d = 1; d < C; ++d) at = c >= d ? from[d] : at;
        return at;
      };
      for (int i = n_top + tid; i < n; i += NT) {
        const int c = list_of(i);
        sm->list[i] = cl.map_shared_rank(sm, c)->list[i - start_of(c)];
      }
      __syncthreads();
      // every part is sorted: a key's rank is its place in its own part and, by bisection, those of the others
      static_assert(C * ACTKV_LOGPROB_MAX_TOP <= NT, "one key per thread");
      const uint64_t mine = tid < n ? sm->list[tid] : 0;
      int rank = 0;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        int lo = from[c], hi = c + 1 < C ? from[c + 1] : n;
        const int begin = lo;
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (sm->list[mid] > mine) lo = mid + 1;
          else hi = mid;
        }
        rank += lo - begin;
      }
      __syncthreads();
      if (tid < n && rank < k) sm->list[rank] = mine;
      __syncthreads();
      n_top = min(n, k);
    }
    cl.sync();                                                             // (the others' shared memory has been read)
    if (part != 0) return;
  }

  // ---- results ----
  const bool none = mst.y == 0.f;
  const float ls = kLn2 * log2f(mst.y);
  auto lp_of = [&](float v) { return none ? -INFINITY : (v - mst.x) - ls; };
  if (tid == 0) {
    if (a.lse != nullptr) a.lse[row] = none ? -INFINITY : mst.x + ls;
    if (a.entropy != nullptr) a.entropy[row] = none ? 0.f : ls - kLn2 * (mst.z / mst.y);
  }
  for (int j = tid; j < k; j += NT) {
    const uint64_t key = j < n_top ? sm->list[j] : 0;
    a.top_index[(int64_t)row * k + j] = j < n_top ? (int32_t)(0xffffffffu - (uint32_t)key) : -1;
    a.top_logprob[(int64_t)row * k + j] = j < n_top ? lp_of(okey_inv((uint32_t)(key >> 32))) : -INFINITY;
  }
  for (int j = tid; j < a.n_given; j += NT) {
    if (j != tid) {
      tok = a.given[(int64_t)row * a.n_given + j];
      if (tok >= 0 && tok < vocab) ztok = to_f(z[tok]);
    }
    float v = 0.f;
    if (tok >= vocab) {
      report(a.status, ACTKV_E_BADINDEX, row, tok);
      v = __uint_as_float(0x7fc00000u);
    } else if (tok >= 0) {
      v = lp_of(ztok);
    }
    a.logprob[(int64_t)row * a.n_given + j] = v;
  }
}

template <typename T, int NT, int C>
int launch(const Args& a, int n_rows, cudaStream_t s) {
  if (ensure_dyn_smem(logprob_kernel<T, NT, C>, sizeof(Smem<NT>)) != cudaSuccess) return ACTKV_E_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_rows * C);
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = sizeof(Smem<NT>);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = C;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = C > 1 ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, logprob_kernel<T, NT, C>, a);
  ACTKV_CHECK_LAUNCH();
  return ACTKV_OK;
}

template <typename T>
int dispatch(const Args& a, int n_rows, cudaStream_t s) {
  // CTAs per row: up to 4 while every CTA has an SM to itself and at least 4096 logits.  (Rows of 152K, 20 alternatives, us at 1 / 2 / 4 / 8
  // CTAs: 16 rows 18.7 / 14.0 / 10.9 / 14.8, 64 rows 18.8 / 14.2 / 16.4 / 29.8, 100 rows 19.0 / 21.8 / 24.4 / 45.3.)
  int c = 1;
  while (c < 4 && (int64_t)n_rows * 2 * c <= 148 && a.vocab / (2 * c) >= 4096) c *= 2;
  if (c == 4) return launch<T, 512, 4>(a, n_rows, s);
  if (c == 2) return launch<T, 512, 2>(a, n_rows, s);
  // Many rows: four CTAs of 256 threads per SM hide the selection of one behind the reading of the others (1500 rows: 165 us, with two of
  // 512 175); fewer rows than they need to fill the SMs are read faster by 512 threads (296 rows: 43.5 and 35.3).
  return n_rows >= 512 ? launch<T, 256, 1>(a, n_rows, s) : launch<T, 512, 1>(a, n_rows, s);
}

}  // namespace lp
}  // namespace actkv

extern "C" int actkv_logprob(const void* logits, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t row_stride,
                             const int32_t* given, int32_t n_given, int32_t top_k, float* logprob, float* entropy, float* lse,
                             float* top_logprob, int32_t* top_index, int32_t* status, actkv_stream_t stream) {
  using namespace actkv;
  using namespace actkv::lp;
  if (dtype != ACTKV_F32 && dtype != ACTKV_BF16) return ACTKV_E_INVALID;
  if (n_rows < 0 || vocab <= 0 || row_stride < vocab || n_given < 0 || top_k < 0 || top_k > ACTKV_LOGPROB_MAX_TOP) return ACTKV_E_INVALID;
  if (n_rows == 0) return ACTKV_OK;
  if (!logits || ((uintptr_t)logits & (dtype == ACTKV_F32 ? 3 : 1))) return ACTKV_E_INVALID;
  if (n_given > 0 && (!given || !logprob)) return ACTKV_E_INVALID;
  if (top_k > 0 && (!top_logprob || !top_index)) return ACTKV_E_INVALID;
  if (n_rows > 0x7fffffff / 8) return ACTKV_E_TOOBIG;
  Args a{logits, row_stride, given, logprob, entropy, lse, top_logprob, top_index, status, vocab, n_given, top_k};
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == ACTKV_F32 ? dispatch<float>(a, n_rows, s) : dispatch<__nv_bfloat16>(a, n_rows, s);
}
