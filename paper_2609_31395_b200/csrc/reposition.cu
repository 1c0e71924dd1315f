// actkv_reposition: cached keys carried from one position to another, or from one table of rotary frequencies to another, in
// place in their pages (Section 2.5 for the pages; the paper leaves positions to the model).
//
// A key cached at position p is R(p f) k, with the rotation R acting on pairs of dims.  Rotations add, so what the key is at position p' under
// frequencies f' is R(p' f' - p f) of what lies in the page: one turn per pair, k itself is not needed.  The angle is formed in turns, as
// 64-bit fixed point: F = f / 2 pi modulo 1 in steps of 2^-64 (float64 product, error 2^-56), phase = p' F' - p F modulo 2^64, which is
// exact however far the positions are apart; its upper 32 bits, rounded to 23, go to sine and cosine in float32.
//
// What bounds it: reading and writing the turned dims of every key that moves once, 4 rotary_dim bytes per (key, head, layer), and 4
// bytes per position.  A thread has the same dims of every key that it turns (its frequencies stay in registers), and the keys of its next heads or token in
// flight while it turns these.  Positions that all heads share are turned to sine and cosine once per token.
// Measured: 8 x 9100 keys of 4 heads of 128 dims, positions per head, 6 layers: 148 us, 91 % of the rate of a copy; 8 x 20000-35000 keys to other frequencies,
// 2 layers: 149 us, 93 %; 16 x 500-6000 keys of 8 heads, 32 of 64 dims, three axes, 2 layers: 50 us, 30 %: bound by instructions (320 a key and lane: three
// positions read, three that are the index, an axis to choose for each pair on both sides; with both given on every axis 53); 1000 keys: 5.5 us, two launches.
// Without the copies ahead 183, 158 and 72 us.
//
// A key in place cannot be turned twice, so the call is all or nothing: a first kernel looks over the lengths and pages, the second does nothing
// when status is set.
#include <algorithm>

#include "common.cuh"

namespace actkv {
namespace rp {

constexpr int NT = 256;
constexpr int MAX_PAIRS = 128;
constexpr int UNROLL = 4;                  // heads of a token that a thread has in flight

struct Positions {
  const int32_t* base;                     // null: the token's index
  int64_t stride_axis, stride_unit;
  __device__ __forceinline__ int32_t at(int axis, int64_t unit, int64_t off, int j) const {
    return base == nullptr ? j : base[axis * stride_axis + unit * stride_unit + off];
  }
};
struct Args {
  PoolView pool;
  TablesView tab;
  Positions from, to;
  const float *freq, *to_freq;             // to_freq null: the same
  const int32_t* tok_indptr;
  int32_t* status;
  int32_t layer_begin, sum_tok, max_tok, pairs, n_axes, interleaved, sec_end[4];
  int32_t lanes, lane_step, second;        // lanes of a key, elements from one to the next, and from the first dims of its pairs to the second
  int32_t steps, head_groups, heads_per, shared;
};

__device__ __forceinline__ bool bad_request(const Args& a, int r, int32_t& n) {
  const int32_t t0 = a.tok_indptr[r], t1 = a.tok_indptr[r + 1], L = a.tab.seq_len[r];
  n = t1 - t0;
  return t0 < 0 || t1 < t0 || t1 > a.sum_tok || n > a.max_tok || n > L || ((int64_t)n + a.pool.page_size - 1) / a.pool.page_size > a.tab.max_pages;
}

// Lengths and pages of all requests.
__global__ void __launch_bounds__(NT) check_kernel(const Args a) {
  pdl_begin();
  for (int r = blockIdx.y; r < a.tab.n_req; r += gridDim.y) {
    int32_t n;
    if (bad_request(a, r, n)) {
      if (blockIdx.x == 0 && threadIdx.x == 0) report(a.status, ACTKV_E_INVALID, r, n);
      continue;
    }
    const int pages = (int)(((int64_t)n + a.pool.page_size - 1) / a.pool.page_size);
    for (int p = blockIdx.x * NT + threadIdx.x; p < pages; p += gridDim.x * NT) (void)page_or_neg(a.tab, a.pool.n_pages, r, p, a.status);
  }
}

__device__ __forceinline__ uint64_t turns64(float f) {                      // f / 2 pi modulo 1, in steps of 2^-64
  double t = (double)f * 0.15915494309189533577;
  t -= floor(t);
  return __double2ull_rz(t * 18446744073709551616.0);
}
// The upper half of p F modulo 2^64: a position times the frequency, in steps of 2^-32 turns.
__device__ __forceinline__ uint32_t phase_of(uint32_t p, uint64_t F) { return p * (uint32_t)(F >> 32) + __umulhi(p, (uint32_t)F); }
__device__ __forceinline__ uint32_t phase_of(int32_t p, uint64_t F) { return phase_of((uint32_t)p, F) - (p < 0 ? (uint32_t)F : 0u); }
// (The phase rounded to its upper 23 bits, as a float32 in [1, 2) without a conversion: those share the special function units with sine and cosine, 24 operations
// of a lane's 8 pairs, and 16 so.  Half a step is 2^-21.4 rad; with the rounding of the product and of 2 pi the angle is off by 2^-20.7 at most, to both sides alike, and
// sine and cosine by 2^-21.1 of their own: 2^-19.9 in all.)
__device__ __forceinline__ void sincos_of(uint32_t phase, float& sn, float& cs) {
  const float t = (__uint_as_float(((phase + 0x100u) >> 9 ^ 0x400000u) | 0x3f800000u) - 1.5f) * 6.283185307179586f;      // in [-pi, pi)
  sn = __sinf(t);
  cs = __cosf(t);
}
__device__ __forceinline__ float bf1(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float2 bf2(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// a == b ? x : y, as an instruction: of a chain of them the compiler makes an array in local memory
__device__ __forceinline__ int32_t where_equal(int32_t a, int32_t b, int32_t x, int32_t y) {
  int32_t v;
  asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\tselp.s32 %0, %3, %4, p;\n\t}" : "=r"(v) : "r"(a), "r"(b), "r"(x), "r"(y));
  return v;
}

// Where the token's keys lie, within a layer and head 0; -1: nowhere.
__device__ __forceinline__ int64_t place_of(const Args& a, int r, int j) {
  const int P = a.pool.page_size;
  const int32_t page = a.tab.page_table[(int64_t)r * a.tab.max_pages + j / P];
  return (uint32_t)page < (uint32_t)a.pool.n_pages ? (int64_t)page * a.pool.stride_page + (int64_t)(j % P) * a.pool.stride_slot : -1;
}

template <int BYTES> struct Raw;
template <> struct Raw<16> { using T = uint4; };
template <> struct Raw<8> { using T = uint2; };
template <> struct Raw<4> { using T = uint32_t; };
template <> struct Raw<2> { using T = uint16_t; };
template <int N> union Elems {             // N bf16
  typename Raw<2 * N>::T raw;
  uint16_t e[N];
  uint32_t pair[(N + 1) / 2];
};

template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  static_assert(BYTES == 4 || BYTES == 8 || BYTES == 16, "");
  const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(d), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait_one() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

// A lane has E pairs: HALF: E dims and as many `second` elements further on; else 2 E dims side by side.  TWO: the frequencies
// may change.  AXES: there may be more than one axis.  (E below a whole vector: only with both.)
// A thread goes through items of U heads of one token: it turns the keys of one while those of the next are on their way into shared memory (places that
// only this thread reads) and the positions and the page of the one behind that into registers.
template <bool HALF, int E, bool TWO, bool AXES>
struct Shape {
  static constexpr int V = HALF ? 2 : 1, W = HALF ? E : 2 * E, NA = AXES ? 4 : 1;           // vectors, elements of one, axes
  static constexpr int U = AXES ? UNROLL / 2 : UNROLL;
  static constexpr int CTAS = 2;                                           // (three, 80 registers: 194 us instead of 148)
  using Vec = typename Raw<2 * W>::T;
  static constexpr size_t SMEM = W > 1 ? (size_t)2 * U * V * NT * sizeof(Vec) : 16;
};
template <bool HALF, int E, bool TWO, bool AXES>
__global__ void __launch_bounds__(NT, (Shape<HALF, E, TWO, AXES>::CTAS)) turn_kernel(const __grid_constant__ Args a) {
  using S = Shape<HALF, E, TWO, AXES>;
  constexpr int V = S::V, W = S::W, NA = S::NA, U = S::U;
  using Vec = typename S::Vec;
  pdl_begin();
  extern __shared__ __align__(16) uint8_t rp_smem[];
  __shared__ __align__(16) uint64_t s_turns[TWO ? 2 : 1][MAX_PAIRS];
  Vec* buf = reinterpret_cast<Vec*>(rp_smem) + threadIdx.x;                // [stage][head][vector][thread]
  const int tid = threadIdx.x, per = NT / a.lanes, slot = tid / a.lanes, c = tid - slot * a.lanes;
  const int r = blockIdx.y, layer = blockIdx.z / a.head_groups, hg = blockIdx.z - layer * a.head_groups;
  const bool same = !TWO || a.to_freq == nullptr;
  int32_t n;
  const bool stop = status_set(a.status);
  const int tok0 = blockIdx.x * per * a.steps;
  if (bad_request(a, r, n) || stop || tok0 >= n) return;                   // (all threads)
  for (int p = tid; p < a.pairs; p += NT) {
    s_turns[0][p] = turns64(a.freq[p]);
    if (TWO) s_turns[TWO ? 1 : 0][p] = turns64(same ? a.freq[p] : a.to_freq[p]);
  }
  __syncthreads();
  if (slot >= per) return;
  const int t0 = a.tok_indptr[r], H = a.pool.n_kv_heads, h0 = hg * a.heads_per, h1 = min(H, h0 + a.heads_per);
  uint64_t F[E], G[TWO ? E : 1];
  int axis[AXES ? E : 1];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    F[e] = s_turns[0][c * E + e];
    if (TWO) G[e] = s_turns[TWO ? 1 : 0][c * E + e];
    if (AXES) {
      int x = 0;
      while (c * E + e >= a.sec_end[x]) ++x;
      axis[e] = x;
    }
  }
  __nv_bfloat16* base = const_cast<__nv_bfloat16*>(a.pool.base) + (int64_t)(a.layer_begin + layer) * a.pool.stride_layer + c * a.lane_step;
  const int end = min(n, tok0 + a.steps * per);

  struct Item {
    int64_t place;                         // of the token's keys, with the item's first head
    int32_t f[U][NA], t[U][NA];
    uint32_t move;                         // heads whose key moves
    bool first;                            // ... of the token
  };
  int j = tok0 + slot, h = h0;                                             // the next item to fetch
  // positions and page of the next item; no heads left: move stays 0
  auto fetch = [&](Item& it) {
    it.move = 0;
    it.place = -1;
    it.first = h == h0;
    if (j >= end) return;
    const int64_t off = (int64_t)t0 + j, place = place_of(a, r, j);
    it.place = place < 0 ? -1 : place + (int64_t)h * a.pool.stride_head;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t unit = (int64_t)layer * H + min(h + u, h1 - 1);
#pragma unroll
      for (int x = 0; x < NA; ++x) {
        it.f[u][x] = it.t[u][x] = 0;
        if (AXES && x >= a.n_axes) continue;
        it.f[u][x] = a.from.at(x, unit, off, j);
        it.t[u][x] = a.to.at(x, unit, off, j);
      }
      if (h + u < h1) it.move |= 1u << u;
    }
    h += U;
    if (h >= h1) {
      h = h0;
      j += per;
    }
  };
  // which keys move, and these on their way
  auto issue = [&](Item& it, int stage) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      bool move = !same;
#pragma unroll
      for (int x = 0; x < NA; ++x) move |= it.f[u][x] != it.t[u][x];
      if (it.place < 0 || !move) it.move &= ~(1u << u);
      if constexpr (W > 1) {
        if (it.move >> u & 1u) {
          const __nv_bfloat16* src = base + it.place + (int64_t)u * a.pool.stride_head;
#pragma unroll
          for (int x = 0; x < V; ++x) copy_async<2 * W>(buf + ((stage * U + u) * V + x) * NT, src + x * a.second);
        }
      }
    }
    copy_commit();
  };
  Item now, next, later;
  fetch(now);
  fetch(next);
  issue(now, 0);
  float cs[E], sn[E];
  int stage = 0;
#pragma unroll 1
  while (now.place != -1 || next.place != -1 || j < end) {
    issue(next, stage ^ 1);
    fetch(later);
    copy_wait_one();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!(now.move >> u & 1u)) continue;
      __nv_bfloat16* key = base + now.place + (int64_t)u * a.pool.stride_head;
      Elems<W> v[V];
#pragma unroll
      for (int x = 0; x < V; ++x) {
        if constexpr (W > 1) v[x].raw = buf[((stage * U + u) * V + x) * NT];
        else v[x].raw = *reinterpret_cast<const Vec*>(key + x * a.second);
      }
      if (!a.shared || (now.first && u == 0)) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          int32_t f = now.f[u][0], t = now.t[u][0];
          if (AXES) {
#pragma unroll
            for (int x = 1; x < NA; ++x)
              f = where_equal(axis[e], x, now.f[u][x], f), t = where_equal(axis[e], x, now.t[u][x], t);
          }
          // (one table: the positions' distance, which fits 32 bits beside its sign)
          const uint32_t up = phase_of((uint32_t)t - (uint32_t)f, F[e]), ph = TWO ? phase_of(t, G[TWO ? e : 0]) - phase_of(f, F[e]) : t >= f ? up : up - (uint32_t)F[e];
          sincos_of(ph, sn[e], cs[e]);
        }
      }
      if (HALF && E == 1) {
        const float x = bf1(v[0].e[0]), y = bf1(v[V - 1].e[0]);
        v[0].pair[0] = pack2(x * cs[0] - y * sn[0], 0.f);
        v[V - 1].pair[0] = pack2(y * cs[0] + x * sn[0], 0.f);
      } else if (HALF) {
#pragma unroll
        for (int e = 0; e + 1 < E; e += 2) {
          const float2 x = bf2(v[0].pair[e / 2]), y = bf2(v[V - 1].pair[e / 2]);
          v[0].pair[e / 2] = pack2(x.x * cs[e] - y.x * sn[e], x.y * cs[e + 1] - y.y * sn[e + 1]);
          v[V - 1].pair[e / 2] = pack2(y.x * cs[e] + x.x * sn[e], y.y * cs[e + 1] + x.y * sn[e + 1]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float2 x = bf2(v[0].pair[e]);
          v[0].pair[e] = pack2(x.x * cs[e] - x.y * sn[e], x.y * cs[e] + x.x * sn[e]);
        }
      }
#pragma unroll
      for (int x = 0; x < V; ++x) *reinterpret_cast<Vec*>(key + x * a.second) = v[x].raw;
    }
    now = next;
    next = later;
    stage ^= 1;
  }
}

template <bool HALF, int E, bool TWO, bool AXES>
struct Kernel {
  static constexpr auto kernel = turn_kernel<HALF, E, TWO, AXES>;
  static constexpr size_t smem = Shape<HALF, E, TWO, AXES>::SMEM;
};

}  // namespace rp
}  // namespace actkv

extern "C" int actkv_reposition(const actkv_pool_t* pool, const actkv_tables_t* tables, int32_t layer_begin, int32_t layer_end,
                                const actkv_rope_t* rope, const float* to_inv_freq, const actkv_positions_t* from,
                                const actkv_positions_t* to, const int32_t* tok_indptr, int32_t sum_tok, int32_t max_tok,
                                int32_t* status, actkv_stream_t stream) {
  using namespace actkv;
  using namespace actkv::rp;
  if (!pool || !tables || !pool->base || !rope) return ACTKV_E_INVALID;
  if (layer_begin < 0 || layer_end > pool->n_layers || layer_begin > layer_end) return ACTKV_E_INVALID;
  const int D = pool->head_dim, H = pool->n_kv_heads, R = tables->n_req, nls = layer_end - layer_begin;
  if (D <= 0 || D % 8 != 0 || D > 256 || H <= 0 || pool->page_size <= 0 || pool->n_pages <= 0 || R < 0 || sum_tok < 0 || max_tok < 0) return ACTKV_E_INVALID;
  if (rope->rotary_dim < 0 || rope->rotary_dim % 2 != 0 || rope->rotary_dim > D || rope->n_axes < 1 || rope->n_axes > 4) return ACTKV_E_INVALID;
  Args a = {};
  a.pairs = rope->rotary_dim / 2;
  a.interleaved = rope->interleaved ? 1 : 0;
  a.n_axes = rope->n_axes;
  int64_t end = 0;
  for (int x = 0; x < 4; ++x) {
    if (x < rope->n_axes) {
      if (rope->section[x] < 0) return ACTKV_E_INVALID;
      end += rope->section[x];
    }
    a.sec_end[x] = (int32_t)(end < D ? end : D);
  }
  if (end != a.pairs) return ACTKV_E_INVALID;
  if (R == 0 || nls == 0 || max_tok == 0 || a.pairs == 0) return ACTKV_OK;
  if (!rope->inv_freq || !tok_indptr || !tables->page_table || !tables->seq_len || tables->max_pages < 0) return ACTKV_E_INVALID;
  a.from = from ? Positions{from->base, from->stride_axis, from->stride_unit} : Positions{nullptr, 0, 0};
  a.to = to ? Positions{to->base, to->stride_axis, to->stride_unit} : Positions{nullptr, 0, 0};
  if (!to_inv_freq && !a.from.base && !a.to.base) return ACTKV_OK;           // nothing moves
  if (R > 65535 || (int64_t)nls * H > 65535 || max_tok > (1 << 30)) return ACTKV_E_TOOBIG;
  a.pool = make_view(pool);
  a.tab = make_view(tables);
  a.freq = rope->inv_freq;
  a.to_freq = to_inv_freq;
  a.tok_indptr = tok_indptr;
  a.status = status;
  a.layer_begin = layer_begin;
  a.sum_tok = sum_tok;
  a.max_tok = max_tok;
  a.shared = (!a.from.base || a.from.stride_unit == 0) && (!a.to.base || a.to.stride_unit == 0);
  cudaStream_t s = (cudaStream_t)stream;
  const int64_t pages = ((int64_t)max_tok + pool->page_size - 1) / pool->page_size;
  launch_pdl(check_kernel, dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(16, (pages + NT - 1) / NT)), (unsigned)R), NT, 0, s, a);
  ACTKV_CHECK_LAUNCH();
  // pairs of a lane: as many as make a vector of up to 16 bytes on which all rows, heads and halves begin
  int per_lane = a.interleaved ? 4 : 8;
  const int64_t all = (int64_t)((uintptr_t)pool->base / 2) | pool->stride_layer | pool->stride_page | pool->stride_slot | pool->stride_head;
  while (per_lane > 1 && (a.pairs % per_lane != 0 || all % (a.interleaved ? 2 * per_lane : per_lane) != 0)) per_lane /= 2;
  const bool side_by_side = a.interleaved && all % 2 == 0;                  // (else element by element)
  a.lanes = a.pairs / per_lane;
  a.lane_step = a.interleaved ? 2 * per_lane : per_lane;
  a.second = a.interleaved ? 1 : a.pairs;
  const int per = NT / a.lanes;
  // heads apart while there are few tokens, together (and several steps per CTA, for whose sake a thread forms its frequencies once) when
  // there are CTAs enough for every SM to have eight (at most 8 steps: 148 and 149 us in the two large cases above; at most 4: 154 and 147, 16: 150 and 155;
  // a quarter of the steps: 179 in the first of them, and 64 instead of 50 with three axes)
  const int64_t blocks = (int64_t)R * nls * ((max_tok + per - 1) / per);
  a.heads_per = blocks * ((H + UNROLL - 1) / UNROLL) < 148 * 4 ? 1 : UNROLL;
  if (a.shared && blocks >= 148 * 8) a.heads_per = H;
  a.head_groups = (H + a.heads_per - 1) / a.heads_per;
  a.steps = (int32_t)std::max<int64_t>(1, std::min<int64_t>(8, blocks * a.head_groups / (148 * 8)));
  const dim3 grid((unsigned)((max_tok + per * a.steps - 1) / (per * a.steps)), (unsigned)R, (unsigned)(nls * a.head_groups));
  const bool two = to_inv_freq != nullptr, axes = a.n_axes > 1;
  auto go = [&](auto shape) {
    using S = decltype(shape);
    if (ensure_dyn_smem(S::kernel, S::smem) != cudaSuccess) return ACTKV_E_CUDA;
    launch_pdl(S::kernel, grid, NT, S::smem, s, a);
    ACTKV_CHECK_LAUNCH();
    return ACTKV_OK;
  };
  if (!side_by_side) {
    if (per_lane == 8) return two ? (axes ? go(Kernel<true, 8, true, true>{}) : go(Kernel<true, 8, true, false>{}))
                                  : (axes ? go(Kernel<true, 8, false, true>{}) : go(Kernel<true, 8, false, false>{}));
    return per_lane == 4 ? go(Kernel<true, 4, true, true>{}) : per_lane == 2 ? go(Kernel<true, 2, true, true>{}) : go(Kernel<true, 1, true, true>{});
  }
  if (per_lane == 4) return two ? (axes ? go(Kernel<false, 4, true, true>{}) : go(Kernel<false, 4, true, false>{}))
                                : (axes ? go(Kernel<false, 4, false, true>{}) : go(Kernel<false, 4, false, false>{}));
  return per_lane == 2 ? go(Kernel<false, 2, true, true>{}) : go(Kernel<false, 1, true, true>{});
}
