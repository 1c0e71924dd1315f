// actkv_penalize: biases, penalties for tokens that the history holds, and masks on logits, before a token is drawn.
//
// A CTA has a slice of the vocabulary and some consecutive rows of one request.  It keeps a word per token of the slice in shared memory
// (bit 31: in the prompt, bit 30: has a bias, below: how often it was generated), counts the history into it once, and adds the one token by
// which each further row has seen more.  Integer counts: the same in every order.  Then it goes over the slice: in place, only tokens whose word is set are
// read, and what the mask takes away is written without being read; out of place every logit is read and written once.
//
// What bounds it: in place without masks the history (4 bytes a token, from L2 for all but the first CTA of a request), else writing, or reading and
// writing, the logits.
#include <algorithm>

#include "common.cuh"

namespace actkv {
namespace pn {

constexpr int NT = 512;
constexpr uint32_t PROMPT = 1u << 31, BIAS = 1u << 30, COUNT = BIAS - 1;
constexpr int MAX_SLICE = 24576;           // tokens of a CTA: 96 KB, two CTAs on an SM

struct Args {
  const void* logits;
  void* out;
  int64_t in_stride, out_stride;
  const int32_t* win_indptr;
  actkv_logit_rules_t q;
  int32_t* status;
  int32_t vocab, n_req, sum_win, max_win, max_hist;
  int32_t slice, n_slices, groups, rows_per, in_place;
};

struct Rules {                             // of one request
  float theta, freq, pres;
  const int32_t* bias_token;
  const float* bias_value;
  int n_bias;
};

__device__ __forceinline__ float apply(float z, uint32_t word, int token, const Rules& q) {
  if (word & BIAS) {
    int lo = 0, hi = q.n_bias - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (q.bias_token[mid] < token) lo = mid + 1;
      else hi = mid;
    }
    z += q.bias_value[lo];
  }
  if (word & ~BIAS) z = z > 0.f ? __fdiv_rn(z, q.theta) : z * q.theta;
  if (word & COUNT) z -= q.freq * (float)(word & COUNT) + q.pres;
  return z;
}

template <typename T> struct Io;
template <> struct Io<float> {
  using V4 = float4;
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ void store(float* p, float x) { *p = x; }
  static __device__ __forceinline__ void open(const V4& v, float (&x)[4]) { x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
  static __device__ __forceinline__ V4 close(const float (&x)[4]) { return make_float4(x[0], x[1], x[2], x[3]); }
};
template <> struct Io<__nv_bfloat16> {
  using V4 = uint2;
  static __device__ __forceinline__ float load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
  static __device__ __forceinline__ void open(const V4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
  }
  static __device__ __forceinline__ V4 close(const float (&x)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
};

// One token.  word: 0 where no rule but the mask looks at it.
template <typename T>
__device__ __forceinline__ void one(const T* in, T* out, int v, uint32_t word, bool allowed, bool in_place, const Rules& q) {
  if (!allowed) Io<T>::store(out + v, -INFINITY);
  else if (word) Io<T>::store(out + v, apply(Io<T>::load(in + v), word, v, q));
  else if (!in_place) out[v] = in[v];
}

// The row's logits of tokens [v0, v1).
template <typename T>
__device__ __forceinline__ void sweep(const T* in, T* out, const uint32_t* word, bool words, const uint32_t* allow, int v0, int v1, bool in_place,
                                      const Rules& q) {
  using V4 = typename Io<T>::V4;
  const int tid = threadIdx.x;
  const bool whole = (((uintptr_t)(in + v0) | (uintptr_t)(out + v0)) & (sizeof(V4) - 1)) == 0;
  int v = v0;
  if (whole) {
    const int end = v0 + ((v1 - v0) & ~3);
#pragma unroll 4
    for (v = v0 + tid * 4; v < end; v += NT * 4) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (words) w = *reinterpret_cast<const uint4*>(word + (v - v0));
      const uint32_t nib = allow != nullptr ? allow[v >> 5] >> (v & 31) & 15u : 15u;
      const uint32_t any = w.x | w.y | w.z | w.w;
      if (in_place && nib == 15u && any == 0u) continue;
      if (nib == 0u) {
        const float none[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        *reinterpret_cast<V4*>(out + v) = Io<T>::close(none);
      } else if (!in_place) {
        const V4 raw = *reinterpret_cast<const V4*>(in + v);
        if (nib == 15u && any == 0u) {
          *reinterpret_cast<V4*>(out + v) = raw;
          continue;
        }
        float x[4];
        Io<T>::open(raw, x);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (ww[e]) x[e] = apply(x[e], ww[e], v + e, q);
          if (!(nib >> e & 1u)) x[e] = -INFINITY;
        }
        *reinterpret_cast<V4*>(out + v) = Io<T>::close(x);
      } else {
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) one(in, out, v + e, ww[e], nib >> e & 1u, true, q);
      }
    }
    v = end;
  }
  for (v += tid; v < v1; v += NT) {
    const bool allowed = allow == nullptr || (allow[v >> 5] >> (v & 31) & 1u);
    one(in, out, v, words ? word[v - v0] : 0u, allowed, in_place, q);
  }
}

template <typename T>
__global__ void __launch_bounds__(NT) penalize_kernel(const __grid_constant__ Args a) {
  pdl_begin();
  extern __shared__ __align__(16) uint32_t s_word[];
  const int tid = threadIdx.x;
  const int sl = blockIdx.x % a.n_slices, unit = blockIdx.x / a.n_slices, grp = unit % a.groups, r = unit / a.groups;
  const bool first = sl == 0 && grp == 0 && tid == 0;
  const int w0 = a.win_indptr[r], w1 = a.win_indptr[r + 1], W = w1 - w0;
  if (w0 < 0 || w1 < w0 || w1 > a.sum_win || W > a.max_win) {
    if (first) report(a.status, ACTKV_E_INVALID, r, W);
    return;
  }
  const int i0 = grp * a.rows_per, i1 = min(W, i0 + a.rows_per);
  if (i0 >= i1) return;
  Rules q;
  q.theta = a.q.repetition != nullptr ? a.q.repetition[r] : 1.f;
  q.freq = a.q.frequency != nullptr ? a.q.frequency[r] : 0.f;
  q.pres = a.q.presence != nullptr ? a.q.presence[r] : 0.f;
  const int hist = a.q.tokens != nullptr ? a.q.hist_len[r] : 0;
  const int b0 = a.q.bias_indptr != nullptr ? a.q.bias_indptr[r] : 0, b1 = a.q.bias_indptr != nullptr ? a.q.bias_indptr[r + 1] : 0;
  if (!(q.theta > 0.f && q.theta < INFINITY) || !(fabsf(q.freq) < INFINITY) || !(fabsf(q.pres) < INFINITY) || hist < 0 || hist > a.max_hist ||
      hist > a.q.token_stride || b0 < 0 || b1 < b0 || b1 > a.q.n_bias) {
    if (first) report(a.status, ACTKV_E_INVALID, r, hist);
    return;
  }
  q.bias_token = a.q.bias_token + b0;
  q.bias_value = a.q.bias_value + b0;
  q.n_bias = b1 - b0;
  const int v0 = sl * a.slice, v1 = min(a.vocab, v0 + a.slice);
  const bool counts = hist > 0 && (q.theta != 1.f || q.freq != 0.f || q.pres != 0.f), words = counts || q.n_bias > 0;
  const int32_t* tokens = a.q.tokens + (int64_t)r * a.q.token_stride;
  const int prompt = counts && a.q.prompt_len != nullptr ? a.q.prompt_len[r] : 0;
  auto count = [&](int at, int32_t token) {
    const uint32_t v = (uint32_t)token - (uint32_t)v0;
    if (v < (uint32_t)(v1 - v0)) {
      if (at < prompt) atomicOr(&s_word[v], PROMPT);
      else atomicAdd(&s_word[v], 1u);
    }
  };
  int seen = max(0, hist - (W - 1 - i0));                                  // tokens that the row stands behind
  if (words) {
    for (int i = tid * 4; i < v1 - v0; i += NT * 4) *reinterpret_cast<uint4*>(s_word + i) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    bool bad = false;
    for (int i = tid; i < q.n_bias; i += NT) {
      const int32_t t = q.bias_token[i];
      bad |= (uint32_t)t >= (uint32_t)a.vocab || (i > 0 && q.bias_token[i - 1] >= t);
      if (t >= v0 && t < v1) atomicOr(&s_word[t - v0], BIAS);
    }
    if (counts) {
      const int head = min(seen, (int)((0u - (uint32_t)(uintptr_t)tokens & 15u) / 4)), vecs = (seen - head) / 4;
      if (tid < head) count(tid, tokens[tid]);
#pragma unroll 4
      for (int i = tid; i < vecs; i += NT) {
        const int at = head + i * 4;
        const int4 t = *reinterpret_cast<const int4*>(tokens + at);
        count(at, t.x);
        count(at + 1, t.y);
        count(at + 2, t.z);
        count(at + 3, t.w);
      }
      const int at = head + vecs * 4 + tid;
      if (at < seen) count(at, tokens[at]);
    }
    if (__syncthreads_or(bad)) {
      if (first) report(a.status, ACTKV_E_BADINDEX, r, b0);
      return;
    }
  }
  for (int i = i0; i < i1; ++i) {
    const int64_t row = w0 + i;
    const uint32_t* allow = nullptr;
    bool skip = false;
    if (a.q.allow != nullptr) {
      const int m = a.q.allow_row != nullptr ? a.q.allow_row[row] : (int)row;
      if (m >= a.q.n_allow) {
        if (sl == 0 && tid == 0) report(a.status, ACTKV_E_BADINDEX, r, m);
        skip = true;
      } else if (m >= 0) {
        allow = a.q.allow + (int64_t)m * a.q.allow_stride;
      }
    }
    if (!skip && (words || allow != nullptr || !a.in_place))
      sweep<T>((const T*)a.logits + row * a.in_stride, (T*)a.out + row * a.out_stride, s_word, words, allow, v0, v1, a.in_place != 0, q);
    if (counts && i + 1 < i1) {
      const int next = max(0, hist - (W - 2 - i));
      __syncthreads();
      if (tid == 0 && next > seen) count(seen, tokens[seen]);
      seen = next;
      __syncthreads();
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
  if (max_hist >= (int32_t)BIAS) return ACTKV_E_TOOBIG;
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
  a.in_place = logits == out;
  // slices: at least as many as shared memory asks for, more while the SMs have not two CTAs each; rows of a request apart for the same reason
  const int64_t want = 148 * 2, least = (vocab + MAX_SLICE - 1) / MAX_SLICE;
  const int64_t slices = std::max(least, std::min<int64_t>((want + n_req - 1) / n_req, (vocab + 4095) / 4096));
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
  return dtype == ACTKV_BF16 ? go(penalize_kernel<__nv_bfloat16>) : go(penalize_kernel<float>);
}
