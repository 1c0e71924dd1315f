// actkv_penalize: biases, penalties for tokens that the history holds, and masks on logits, before a token is drawn.
//
// A CTA has a slice of the vocabulary and some consecutive rows of one request.  It keeps a word per token of the slice in shared memory
// (bit 31: has a bias, bit 30: in the prompt, below: how often it was generated), counts the history into it once, and adds the one token by
// which each further row has seen more.  Integer counts: the same in every order.  Then it goes over the slice: in place, only tokens whose word is set are
// read, and what the mask takes away is written without being read; out of place every logit is read and written once.
//
// What bounds it: in place without masks the history (4 bytes a token, from L2 for all but the first CTA of a request; every CTA looks at all of it), else
// writing, or reading and writing, the logits; in small calls the chain of loads and instructions that are not in the cache yet.
// Measured: 16 requests of 2000-34000 tokens, in place, 152K: 11.4 us (the longest history: 17 vectors a thread, in five rounds of four); 64 requests, three quarters
// with masks: 38; 4-8 bf16 rows for each of 16 requests, out of place: 32.7; 6 x 200-300 rows out of place, a third with masks: 382, 70 % of the rate of a copy; 15 x 25-37
// rows out of place, histories up to 9000 tokens, without masks and biases: 109, 80 %; up to 34000 tokens and biases: 125, 70 %.
// Tried: tokens dealt to the CTAs of a cluster, counted through distributed shared memory (25 us instead of 14 for the first case); three CTAs on an SM (registers spill: 19
// and 666 instead of 14 and 437); 1024 threads and one CTA (11.7 and 458 instead of 13.3 and 442); slices chosen so that the last wave of CTAs is full
// (single large rows 4 to 7 % faster, drafts and small ones 2 to 4 % slower).
#include <algorithm>

#include "common.cuh"

namespace actkv {
namespace pn {

constexpr int NT = 512;
constexpr uint32_t BIAS = 1u << 31, PROMPT = 1u << 30, COUNT = PROMPT - 1;
constexpr int MAX_SLICE = 24576;           // tokens of a CTA: 96 KB, two CTAs on an SM

struct Args {
  const void* logits;
  void* out;
  int64_t in_stride, out_stride;
  const int32_t* win_indptr;
  actkv_logit_rules_t q;
  int32_t* status;
  int32_t vocab, n_req, sum_win, max_win, max_hist;
  int32_t slice, n_slices, groups, rows_per, alike;              // alike: all rows begin at the same place of a vector
};

struct Rules {                             // of one request
  float theta, inverse, freq, pres;        // (z / theta as a product: a rounding more)
};

// Penalties by a token's word, 0 where none; no branches.
__device__ __forceinline__ float penalty(float z, uint32_t word, const Rules& q) {
  const float turned = z * (z > 0.f ? q.inverse : q.theta);
  z = word & ~BIAS ? turned : z;
  const uint32_t n = word & COUNT;
  const float less = z - fmaf(q.freq, __uint_as_float(0x4b000000u | n) - 8388608.f, q.pres);         // (n below 2^23 as a float32)
  return n != 0 ? less : z;
}

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// 16 bytes of logits.  rules: tokens with a bias are left as they are.
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
  static __device__ __forceinline__ void rules(uint4& v, const uint32_t (&w)[4], const Rules& q) {
    v.x = (int32_t)w[0] > 0 ? __float_as_uint(penalty(__uint_as_float(v.x), w[0], q)) : v.x;
    v.y = (int32_t)w[1] > 0 ? __float_as_uint(penalty(__uint_as_float(v.y), w[1], q)) : v.y;
    v.z = (int32_t)w[2] > 0 ? __float_as_uint(penalty(__uint_as_float(v.z), w[2], q)) : v.z;
    v.w = (int32_t)w[3] > 0 ? __float_as_uint(penalty(__uint_as_float(v.w), w[3], q)) : v.w;
  }
  static __device__ __forceinline__ void mask(uint4& v, uint32_t bits) {
    v.x = bits & 1u ? v.x : 0xff800000u;
    v.y = bits & 2u ? v.y : 0xff800000u;
    v.z = bits & 4u ? v.z : 0xff800000u;
    v.w = bits & 8u ? v.w : 0xff800000u;
  }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
  static __device__ __forceinline__ uint32_t two_rules(uint32_t v, uint32_t w0, uint32_t w1, const Rules& q) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(penalty(__uint_as_float(v << 16), w0, q), penalty(__uint_as_float(v & 0xffff0000u), w1, q));
    const uint32_t n = *reinterpret_cast<const uint32_t*>(&r);
    return ((int32_t)w0 > 0 ? n & 0xffffu : v & 0xffffu) | ((int32_t)w1 > 0 ? n & 0xffff0000u : v & 0xffff0000u);
  }
  static __device__ __forceinline__ void rules(uint4& v, const uint32_t (&w)[8], const Rules& q) {
    v.x = two_rules(v.x, w[0], w[1], q);
    v.y = two_rules(v.y, w[2], w[3], q);
    v.z = two_rules(v.z, w[4], w[5], q);
    v.w = two_rules(v.w, w[6], w[7], q);
  }
  static __device__ __forceinline__ uint32_t two(uint32_t v, uint32_t bits) {
    v = bits & 1u ? v : (v & 0xffff0000u) | 0xff80u;
    return bits & 2u ? v : (v & 0xffffu) | 0xff800000u;
  }
  static __device__ __forceinline__ void mask(uint4& v, uint32_t bits) {
    v.x = two(v.x, bits);
    v.y = two(v.y, bits >> 2);
    v.z = two(v.z, bits >> 4);
    v.w = two(v.w, bits >> 6);
  }
};

constexpr int READ = 4;                    // vectors of the history that a thread has in flight (eight: 1 us more in every small call)
// Vectors of logits in flight.  Out of place without masks: 15 x 25-37 rows 108 us, with two 125.  With masks, 6 x 200-300 rows: 383, with one 437, with four, whose
// registers spill, 405.  In place few vectors are read at all: 4.6 us in the smallest calls, with four 5.1.
template <bool MASKED, bool IN_PLACE> constexpr int BATCH = !MASKED && !IN_PLACE ? 4 : 2;

// How a row's logits of tokens [v0, v1) are walked over: vectors a0 .. a1 of N, and single tokens at the ends (all of them when in and out begin at
// different places of a vector).
template <typename T>
struct Walk {
  static constexpr int N = Vec<T>::N;
  int head, vecs;
  __device__ __forceinline__ Walk(const T* in, const T* out, int n) {      // (of the slice's first token)
    const bool whole = (((uintptr_t)in ^ (uintptr_t)out) & 15) == 0;
    head = whole ? min(n, (N - (int)(((uintptr_t)in & 15) / sizeof(T))) % N) : 0;
    vecs = whole ? (n - head) / N : 0;
  }
  __device__ __forceinline__ int thread_of(int at) const {                 // which thread has the slice's token `at`
    const int in = at - head, end = vecs * N;
    return in < 0 ? at : in < end ? in / N % NT : (head + in - end) % NT;
  }
};

template <typename T>
struct Row {
  const T* in;                             // of token 0
  T* out;
  const uint32_t* allow;                   // null: no mask
  Walk<T> walk;
};

// The words of the mask that hold a thread's next batch of vectors.
template <int B>
struct Masks {
  uint32_t lo[B], hi[B];
};
template <typename T, int B>
__device__ __forceinline__ void load_masks(const uint32_t* allow, const Walk<T>& walk, int base, int v0, int last_word, Masks<B>& m) {
#pragma unroll
  for (int u = 0; u < B; ++u) {
    const int i = base + u * NT, at = (v0 + walk.head + i * Vec<T>::N) >> 5;
    const bool some = allow != nullptr && i < walk.vecs;
    m.lo[u] = some ? allow[at] : ~0u;
    m.hi[u] = some ? allow[min(at + 1, last_word)] : ~0u;
  }
}

// Batches of vectors, whose loads stand before any store (the compiler cannot know that out is not read again); ahead: the masks of the first batch, in the end those
// of the next row's first, which like those of every next batch are on their way meanwhile.  Logits of tokens with a bias are carried over, if they are allowed.
template <bool MASKED, bool IN_PLACE, typename T, typename Next>
__device__ __forceinline__ void sweep(const Row<T>& row, Next&& next, const uint32_t* word, bool words, int last_word, int v0, int v1,
                                      const Rules& q, Masks<BATCH<MASKED, IN_PLACE>>& ahead) {
  const T* in = row.in;
  T* out = row.out;
  const uint32_t* allow = MASKED ? row.allow : nullptr;
  constexpr int N = Vec<T>::N, B = BATCH<MASKED, IN_PLACE>;
  constexpr uint32_t ALL = (1u << N) - 1;
  const int tid = threadIdx.x, head = row.walk.head, vecs = row.walk.vecs, a0 = v0 + head, a1 = a0 + vecs * N;
  auto one = [&](int v) {
    const uint32_t w = words ? word[v - v0] : 0u;
    if (allow != nullptr && !(allow[v >> 5] >> (v & 31) & 1u)) store1(out + v, -INFINITY);
    else if ((int32_t)w > 0) store1(out + v, penalty(load1(in + v), w, q));
    else if (!IN_PLACE) out[v] = in[v];
  };
  // the words of a vector, and what they have set
  auto words_of = [&](int v, uint32_t (&w)[N]) {
    uint32_t any = 0;
    if (head % 4 == 0) {
#pragma unroll
      for (int e = 0; e < N; e += 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(word + (v - v0) + e);
        w[e] = x.x, w[e + 1] = x.y, w[e + 2] = x.z, w[e + 3] = x.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) w[e] = word[v - v0 + e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) any |= w[e];
    return any;
  };
  int base = tid;
#pragma unroll 1
  for (bool more = true; more;) {
    uint4 raw[B];
    uint32_t hit[B], bits[B];
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const int i = base + u * NT, v = a0 + i * N;
      bits[u] = MASKED ? __funnelshift_r(ahead.lo[u], ahead.hi[u], v & 31) & ALL : ALL;
      hit[u] = 0;
      if (i >= vecs) continue;
      uint32_t w[N];
      if (IN_PLACE && words && bits[u] != 0) hit[u] = words_of(v, w);
      if (bits[u] != 0 && (hit[u] != 0 || !IN_PLACE)) raw[u] = *reinterpret_cast<const uint4*>(in + v);
    }
    more = base + B * NT < vecs;
    if (MASKED && more) load_masks(allow, row.walk, base + B * NT, v0, last_word, ahead);
    else if (MASKED) next();
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const int i = base + u * NT, v = a0 + i * N;
      const uint32_t now = bits[u];
      if (i >= vecs) continue;
      if (now == 0) {
        *reinterpret_cast<uint4*>(out + v) = Vec<T>::none();
      } else if (hit[u] != 0 || !IN_PLACE) {
        uint32_t w[N];
        if (IN_PLACE || (words && words_of(v, w) != 0)) {
          if (IN_PLACE) (void)words_of(v, w);
          Vec<T>::rules(raw[u], w, q);
        }
        if (now != ALL) Vec<T>::mask(raw[u], now);
        *reinterpret_cast<uint4*>(out + v) = raw[u];
      } else if (now != ALL) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (!(now >> e & 1u)) store1(out + v + e, -INFINITY);
      }
    }
    base += B * NT;
  }
#pragma unroll 1
  for (int i = tid; i < head + v1 - a1; i += NT) one(i < head ? v0 + i : a1 + i - head);
}

// n tokens of the rows from, from + step, ... below to; out: of row 0.  (A call, so that the kernels carry little of it.)
template <typename T>
__device__ __noinline__ void forbid(T* out, int64_t stride, int from, int to, int step, int n) {
  for (int i = from; i < to; i += step)
    for (int v = threadIdx.x; v < n; v += NT) store1(out + i * stride + v, -INFINITY);
}

// MASKED: there are masks.
template <typename T, bool MASKED, bool IN_PLACE>
__global__ void __launch_bounds__(NT, 2) penalize_kernel(const __grid_constant__ Args a) {
  pdl_begin();
  extern __shared__ __align__(16) uint32_t s_word[];
  const int tid = threadIdx.x;
  const int sl = blockIdx.x % a.n_slices, unit = blockIdx.x / a.n_slices, grp = unit % a.groups, r = unit / a.groups;
  const bool first = sl == 0 && grp == 0 && tid == 0;
  // (all loads that hang on nothing else before the first look at one)
  const bool has_history = a.q.tokens != nullptr, has_bias = a.q.bias_indptr != nullptr;
  const int w0 = a.win_indptr[r], w1 = a.win_indptr[r + 1], W = w1 - w0;
  Rules q;
  q.theta = a.q.repetition != nullptr ? a.q.repetition[r] : 1.f;
  q.freq = a.q.frequency != nullptr ? a.q.frequency[r] : 0.f;
  q.pres = a.q.presence != nullptr ? a.q.presence[r] : 0.f;
  const int hist = has_history ? a.q.hist_len[r] : 0;
  const int prompt = has_history && a.q.prompt_len != nullptr ? a.q.prompt_len[r] : 0;
  const int b0 = has_bias ? a.q.bias_indptr[r] : 0, b1 = has_bias ? a.q.bias_indptr[r + 1] : 0, n_bias = b1 - b0;
  const int v0 = sl * a.slice, v1 = min(a.vocab, v0 + a.slice);
  // Out of place nothing may be drawn from rows that are refused: what the buffer holds is of another step, and without the rules.
  auto refuse = [&](int from, int to, int step) {
    if (!IN_PLACE) forbid((T*)a.out + v0, a.out_stride, from, to, step, v1 - v0);
  };
  if (w0 < 0 || w1 < w0 || w1 > a.sum_win || W > a.max_win) {
    if (first) report(a.status, ACTKV_E_INVALID, r, W);
    refuse(max(w0, 0) + grp, min(w1, a.sum_win), a.groups);
    return;
  }
  const int i0 = grp * a.rows_per, i1 = min(W, i0 + a.rows_per);
  if (i0 >= i1) return;
  if (!(q.theta >= 0x1p-126f && q.theta <= 0x1p126f) || !(fabsf(q.freq) < INFINITY) || !(fabsf(q.pres) < INFINITY) || hist < 0 || hist > a.max_hist ||
      hist > a.q.token_stride || b0 < 0 || b1 < b0 || b1 > a.q.n_bias) {
    if (first) report(a.status, ACTKV_E_INVALID, r, hist);
    refuse(w0 + i0, w0 + i1, 1);
    return;
  }
  q.inverse = __frcp_rn(q.theta);                                          // (in its range a normal number: a subnormal one would be taken for 0)
  const bool counts = hist > 0 && (q.theta != 1.f || q.freq != 0.f || q.pres != 0.f), words = counts || n_bias > 0;
  const int32_t* tokens = a.q.tokens + (int64_t)r * a.q.token_stride;
  // f of the slice's tokens among the history's [lo, hi), by their place in the slice
  auto history = [&](int lo, int hi, auto&& f) {
    auto see = [&](int32_t token) {
      const uint32_t v = (uint32_t)token - (uint32_t)v0;
      if (v < (uint32_t)(v1 - v0)) f(v);
    };
    const int head = min(hi - lo, (int)((0u - (uint32_t)(uintptr_t)(tokens + lo) & 15u) / 4)), vecs = (hi - lo - head) / 4;
    if (tid < head) see(tokens[lo + tid]);
    for (int base = tid; base < vecs; base += READ * NT) {
      int4 t[READ];
#pragma unroll
      for (int u = 0; u < READ; ++u)
        t[u] = base + u * NT < vecs ? *reinterpret_cast<const int4*>(tokens + lo + head + (base + u * NT) * 4) : make_int4(-1, -1, -1, -1);
#pragma unroll
      for (int u = 0; u < READ; ++u) {
        see(t[u].x);
        see(t[u].y);
        see(t[u].z);
        see(t[u].w);
      }
    }
    const int at = lo + head + vecs * 4 + tid;
    if (at < hi) see(tokens[at]);
  };
  // the row of allow for a row, -1: none, -2: there is no such row
  auto mask_of = [&](int i) {
    if (!MASKED || i >= i1) return -1;
    const int m = a.q.allow_row != nullptr ? a.q.allow_row[w0 + i] : w0 + i;
    if (m < a.q.n_allow) return max(m, -1);
    if (sl == 0 && tid == 0) report(a.status, ACTKV_E_BADINDEX, r, m);
    return -2;
  };
  auto allow_of = [&](int m) { return m >= 0 ? a.q.allow + (int64_t)m * a.q.allow_stride : nullptr; };
  auto walk_of = [&](int i) {
    return Walk<T>((const T*)a.logits + (int64_t)(w0 + i) * a.in_stride + v0, (const T*)a.out + (int64_t)(w0 + i) * a.out_stride + v0, v1 - v0);
  };
  const int last_word = (a.vocab - 1) >> 5;
  int mask = mask_of(i0);
  Masks<BATCH<MASKED, IN_PLACE>> masks;
  if (MASKED) load_masks<T>(allow_of(mask), walk_of(i0), tid, v0, last_word, masks);
  int seen = max(0, hist - (W - 1 - i0));                                  // tokens that the row stands behind
  if (words) {
    for (int i = tid * 4; i < v1 - v0; i += NT * 4) *reinterpret_cast<uint4*>(s_word + i) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    bool bad = false;
    if (counts) {
      const int mid = min(max(prompt, 0), seen);
      if (mid > 0) {
        history(0, mid, [&](uint32_t v) { s_word[v] = PROMPT; });          // (the same from whichever thread)
        __syncthreads();
      }
      history(mid, seen, [&](uint32_t v) { atomicAdd(&s_word[v], 1u); });
    }
    for (int i = tid; i < n_bias; i += NT) {
      const int32_t t = a.q.bias_token[b0 + i];
      bad |= (uint32_t)t >= (uint32_t)a.vocab || (i > 0 && a.q.bias_token[b0 + i - 1] >= t);
      if (t >= v0 && t < v1) atomicOr(&s_word[t - v0], BIAS);
    }
    if (__syncthreads_or(bad)) {
      if (first) report(a.status, ACTKV_E_BADINDEX, r, b0);
      refuse(w0 + i0, w0 + i1, 1);
      return;
    }
  }
  for (int i = i0; i < i1; ++i) {
    const Row<T> row = {(const T*)a.logits + (int64_t)(w0 + i) * a.in_stride, (T*)a.out + (int64_t)(w0 + i) * a.out_stride, allow_of(mask), walk_of(i)};
    const bool skip = mask == -2;
    mask = mask_of(i + 1);
    auto next = [&] {
      if (MASKED) load_masks<T>(allow_of(mask), a.alike ? row.walk : walk_of(i + 1), tid, v0, last_word, masks);
    };
    if (!skip && (words || row.allow != nullptr || !IN_PLACE)) sweep<MASKED, IN_PLACE>(row, next, s_word, words, last_word, v0, v1, q, masks);
    else {
      next();
      if (!IN_PLACE) {                                                     // (skipped)
#pragma unroll 1
        for (int v = v0 + tid; v < v1; v += NT) store1(row.out + v, -INFINITY);
      }
    }
    if (n_bias > 0 && !skip) {
      __syncthreads();                                                     // (what the sweep carried over is there)
      for (int k = tid; k < n_bias; k += NT) {
        const int32_t t = a.q.bias_token[b0 + k];
        if (t < v0 || t >= v1 || (row.allow != nullptr && !(row.allow[t >> 5] >> (t & 31) & 1u))) continue;
        store1(row.out + t, penalty(load1(row.in + t) + a.q.bias_value[b0 + k], s_word[t - v0], q));
      }
    }
    if (counts && i + 1 < i1) {
      // One token more for the next row, counted by the thread that alone looks at its word; with biases, or rows that lie differently, in between.
      const int next = max(0, hist - (W - 2 - i));
      const bool apart = n_bias > 0 || !a.alike;
      if (apart) __syncthreads();
      if (next > seen) {
        const int32_t token = tokens[seen];
        if (token >= v0 && token < v1 && tid == row.walk.thread_of(token - v0)) {
          if (seen < prompt) s_word[token - v0] |= PROMPT;
          else s_word[token - v0] += 1;
        }
      }
      seen = next;
      if (apart) __syncthreads();
    }
  }
}

}  // namespace pn
}  // namespace actkv

extern "C" int actkv_penalize(const void* logits, int32_t dtype, int32_t vocab, int64_t row_stride, const int32_t* win_indptr, int32_t n_req,
                              int32_t sum_win, int32_t max_win, int32_t max_hist, const actkv_logit_rules_t* rules, void* out,
                              int64_t out_stride, int32_t* status, actkv_stream_t stream) {
  using namespace actkv;
  using namespace actkv::pn;
  if (!rules || (dtype != ACTKV_F32 && dtype != ACTKV_BF16) || vocab <= 0 || n_req < 0 || sum_win < 0 || max_win < 0 || max_hist < 0)
    return ACTKV_E_INVALID;
  if (sum_win > 1 && (row_stride < vocab || out_stride < vocab)) return ACTKV_E_INVALID;
  if (rules->tokens && (!rules->hist_len || rules->token_stride < 0)) return ACTKV_E_INVALID;
  if (rules->bias_indptr && (rules->n_bias < 0 || (rules->n_bias > 0 && (!rules->bias_token || !rules->bias_value)))) return ACTKV_E_INVALID;
  if (rules->allow && (rules->n_allow < 0 || rules->allow_stride < ((int64_t)vocab + 31) / 32)) return ACTKV_E_INVALID;
  if (n_req == 0 || sum_win == 0) return ACTKV_OK;
  const int item = dtype == ACTKV_BF16 ? 2 : 4;
  if (!logits || !out || !win_indptr || max_win == 0 || ((uintptr_t)logits | (uintptr_t)out) % item != 0) return ACTKV_E_INVALID;
  if (logits == out && sum_win > 1 && row_stride != out_stride) return ACTKV_E_INVALID;
  if (max_hist >= (1 << 23) || vocab > (1 << 30)) return ACTKV_E_TOOBIG;                        // (counts as float32)
  Args a = {};
  a.logits = logits;
  a.out = out;
  a.in_stride = row_stride;
  a.out_stride = out_stride;
  a.win_indptr = win_indptr;
  a.q = *rules;
  a.status = status;
  a.vocab = vocab;
  a.n_req = n_req;
  a.sum_win = sum_win;
  a.max_win = std::min(max_win, sum_win);
  a.max_hist = max_hist;
  a.alike = row_stride * item % 16 == 0 && out_stride * item % 16 == 0;
  // slices: at least as many as shared memory asks for, more while the SMs have not two CTAs each; rows of a request apart for the same reason
  const int64_t want = 148 * 2, least = (vocab + MAX_SLICE - 1) / MAX_SLICE;
  const int64_t rows = (int64_t)n_req * a.max_win, slices = std::max(least, std::min<int64_t>((want + rows - 1) / rows, (vocab + 4095) / 4096));
  a.slice = (int32_t)(((vocab + slices - 1) / slices + 31) / 32 * 32);
  a.n_slices = (vocab + a.slice - 1) / a.slice;
  const int64_t groups = std::max<int64_t>(1, std::min<int64_t>(a.max_win, 2 * want / ((int64_t)n_req * a.n_slices)));
  a.rows_per = (int32_t)((a.max_win + groups - 1) / groups);
  a.groups = (a.max_win + a.rows_per - 1) / a.rows_per;
  const int64_t ctas = (int64_t)n_req * a.groups * a.n_slices;
  if (ctas > 0x7fffffff) return ACTKV_E_TOOBIG;
  const size_t smem = (size_t)a.slice * 4;
  cudaStream_t s = (cudaStream_t)stream;
  auto go = [&](auto kernel) {
    if (ensure_dyn_smem(kernel, smem) != cudaSuccess) return ACTKV_E_CUDA;
    launch_pdl(kernel, (unsigned)ctas, NT, smem, s, a);
    ACTKV_CHECK_LAUNCH();
    return ACTKV_OK;
  };
  auto typed = [&](auto type) {
    using T = decltype(type);
    if (a.q.allow != nullptr) return logits == out ? go(penalize_kernel<T, true, true>) : go(penalize_kernel<T, true, false>);
    return logits == out ? go(penalize_kernel<T, false, true>) : go(penalize_kernel<T, false, false>);
  };
  return dtype == ACTKV_BF16 ? typed(__nv_bfloat16{}) : typed(0.f);
}
