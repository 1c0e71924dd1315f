// actkv_reposition: cached keys carried from one position to another, or from one table of rotary frequencies to another, in
// place in their pages (Section 2.5 for the pages; the paper leaves positions to the model).
//
// A key cached at position p is R(p f) k, with the rotation R acting on pairs of dims.  Rotations add, so what the key is at position p' under
// frequencies f' is R(p' f' - p f) of what lies in the page: one turn per pair, k itself is not needed.  The angle is formed in turns, as
// 64-bit fixed point: F = f / 2 pi modulo 1 in steps of 2^-64 (float64 product, error 2^-56), phase = p' F' - p F modulo 2^64, which is
// exact however far the positions are apart; its upper 32 bits go to sine and cosine in float32.
//
// What bounds it: reading and writing the turned dims of every key that moves once, 4 rotary_dim bytes per (key, head, layer), and 4
// bytes per position.  A thread has the same dims of every key that it turns (its frequencies stay in registers), and four heads of a token in
// flight.  Positions that all heads share are turned to sine and cosine once per token.
//
// A key in place cannot be turned twice, so the call is all or nothing: a first kernel looks over the lengths and pages, the second does nothing
// when status is set.
#include <algorithm>

#include "common.cuh"

namespace actkv {
namespace rp {

constexpr int NT = 256;
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
  int32_t lanes, steps, head_groups, heads_per, shared;
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
__device__ __forceinline__ void sincos_of(uint64_t phase, float& sn, float& cs) {
  const float t = (float)(int32_t)(phase >> 32) * 1.4629180792671596e-9f;   // 2 pi 2^-32: in [-pi, pi)
  sn = __sinf(t);
  cs = __cosf(t);
}
__device__ __forceinline__ float2 bf2(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Where the token's keys lie, within a layer and head 0; -1: nowhere.
__device__ __forceinline__ int64_t place_of(const Args& a, int r, int j) {
  const int P = a.pool.page_size;
  const int32_t page = a.tab.page_table[(int64_t)r * a.tab.max_pages + j / P];
  return (uint32_t)page < (uint32_t)a.pool.n_pages ? (int64_t)page * a.pool.stride_page + (int64_t)(j % P) * a.pool.stride_slot : -1;
}

// HALF: a lane has 8 pairs, dims 8 c .. 8 c + 7 and those half a turned part further on; else 4 pairs side by side, dims 8 c .. 8 c + 7.
// TWO: the frequencies change.  AXES: more than one axis.
template <bool HALF, bool TWO, bool AXES>
__global__ void __launch_bounds__(NT) turn_kernel(const __grid_constant__ Args a) {
  pdl_begin();
  constexpr int E = HALF ? 8 : 4, V = HALF ? 2 : 1, U = AXES ? 1 : UNROLL, NA = AXES ? 4 : 1;
  const int tid = threadIdx.x, per = NT / a.lanes, slot = tid / a.lanes, c = tid - slot * a.lanes;
  const int r = blockIdx.y, layer = blockIdx.z / a.head_groups, hg = blockIdx.z - layer * a.head_groups;
  int32_t n;
  const bool stop = status_set(a.status);
  if (bad_request(a, r, n) || stop) return;
  const int tok0 = blockIdx.x * per * a.steps;
  if (tok0 >= n || slot >= per) return;
  const int t0 = a.tok_indptr[r], H = a.pool.n_kv_heads, h0 = hg * a.heads_per, h1 = min(H, h0 + a.heads_per);
  uint64_t F[E], G[TWO ? E : 1];
  int axis[AXES ? E : 1];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int p = c * E + e;
    F[e] = turns64(a.freq[p]);
    if (TWO) G[e] = turns64(a.to_freq[p]);
    if (AXES) {
      axis[e] = 0;
      while (p >= a.sec_end[axis[e]]) ++axis[e];
    }
  }
  __nv_bfloat16* base = const_cast<__nv_bfloat16*>(a.pool.base) + (int64_t)(a.layer_begin + layer) * a.pool.stride_layer + c * 8;
  const int dv = a.pairs;
#pragma unroll 1
  for (int st = 0; st < a.steps; ++st) {
    const int j = tok0 + st * per + slot;
    if (j >= n) return;
    const int64_t place = place_of(a, r, j), off = (int64_t)t0 + j;
    if (place < 0) continue;
    float cs[E], sn[E];
#pragma unroll 1
    for (int hb = h0; hb < h1; hb += U) {
      int32_t pf[U][NA], pt[U][NA];
      bool move[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t unit = (int64_t)layer * H + min(hb + u, h1 - 1);
        move[u] = false;
#pragma unroll
        for (int x = 0; x < NA; ++x) {
          if (AXES && x >= a.n_axes) {
            pf[u][x] = pt[u][x] = 0;
            continue;
          }
          pf[u][x] = a.from.at(x, unit, off, j);
          pt[u][x] = a.to.at(x, unit, off, j);
          move[u] |= TWO || pf[u][x] != pt[u][x];
        }
        move[u] = move[u] && hb + u < h1;
      }
      uint4 v[U][V];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (move[u]) {
          const uint4* src = reinterpret_cast<const uint4*>(base + place + (int64_t)(hb + u) * a.pool.stride_head);
          v[u][0] = src[0];
          if (HALF) v[u][V - 1] = *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(src) + dv);
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!move[u]) continue;
        if (!a.shared || (hb == h0 && u == 0)) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            int32_t f = pf[u][0], t = pt[u][0];
            if (AXES) {
#pragma unroll
              for (int x = 1; x < NA; ++x)
                if (axis[e] == x) f = pf[u][x], t = pt[u][x];
            }
            const uint64_t ph = TWO ? (uint64_t)(int64_t)t * G[TWO ? e : 0] - (uint64_t)(int64_t)f * F[e] : (uint64_t)((int64_t)t - f) * F[e];
            sincos_of(ph, sn[e], cs[e]);
          }
        }
        uint4* dst = reinterpret_cast<uint4*>(base + place + (int64_t)(hb + u) * a.pool.stride_head);
        if (HALF) {
          uint32_t *ua = reinterpret_cast<uint32_t*>(&v[u][0]), *ub = reinterpret_cast<uint32_t*>(&v[u][V - 1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 x = bf2(ua[e]), y = bf2(ub[e]);
            ua[e] = pack2(x.x * cs[2 * e] - y.x * sn[2 * e], x.y * cs[(2 * e + 1) % E] - y.y * sn[(2 * e + 1) % E]);
            ub[e] = pack2(y.x * cs[2 * e] + x.x * sn[2 * e], y.y * cs[(2 * e + 1) % E] + x.y * sn[(2 * e + 1) % E]);
          }
          dst[0] = v[u][0];
          *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(dst) + dv) = v[u][V - 1];
        } else {
          uint32_t* ua = reinterpret_cast<uint32_t*>(&v[u][0]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 x = bf2(ua[e]);
            ua[e] = pack2(x.x * cs[e] - x.y * sn[e], x.y * cs[e] + x.x * sn[e]);
          }
          dst[0] = v[u][0];
        }
      }
    }
  }
}

// The same, a pair at a time, for strides and halves that are not whole 16-byte vectors.
__global__ void __launch_bounds__(NT) turn_pairs_kernel(const __grid_constant__ Args a) {
  pdl_begin();
  const int r = blockIdx.y, layer = blockIdx.z;
  int32_t n;
  const bool stop = status_set(a.status);
  if (bad_request(a, r, n) || stop) return;
  const int t0 = a.tok_indptr[r], H = a.pool.n_kv_heads, j0 = blockIdx.x * a.steps, j1 = min(n, j0 + a.steps);
  __nv_bfloat16* base = const_cast<__nv_bfloat16*>(a.pool.base) + (int64_t)(a.layer_begin + layer) * a.pool.stride_layer;
  const int items = (j1 - j0) * H * a.pairs;
  for (int i = threadIdx.x; i < items; i += NT) {
    const int p = i % a.pairs, row = i / a.pairs, h = row % H, j = j0 + row / H;
    const int64_t place = place_of(a, r, j);
    if (place < 0) continue;
    bool move = a.to_freq != nullptr;
    const int64_t unit = (int64_t)layer * H + h, off = (int64_t)t0 + j;
    for (int x = 0; x < a.n_axes; ++x) move |= a.from.at(x, unit, off, j) != a.to.at(x, unit, off, j);
    if (!move) continue;
    int axis = 0;
    while (p >= a.sec_end[axis]) ++axis;
    const uint64_t F = turns64(a.freq[p]), G = a.to_freq != nullptr ? turns64(a.to_freq[p]) : F;
    const uint64_t ph = (uint64_t)(int64_t)a.to.at(axis, unit, off, j) * G - (uint64_t)(int64_t)a.from.at(axis, unit, off, j) * F;
    float sn, cs;
    sincos_of(ph, sn, cs);
    __nv_bfloat16* k = base + place + (int64_t)h * a.pool.stride_head;
    const int da = a.interleaved ? 2 * p : p, db = a.interleaved ? 2 * p + 1 : p + a.pairs;
    const float x = __bfloat162float(k[da]), y = __bfloat162float(k[db]);
    k[da] = __float2bfloat16_rn(x * cs - y * sn);
    k[db] = __float2bfloat16_rn(y * cs + x * sn);
  }
}

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
  const bool vec = a.pairs % (a.interleaved ? 4 : 8) == 0 && ((uintptr_t)pool->base & 15) == 0 && pool->stride_layer % 8 == 0 &&
                   pool->stride_page % 8 == 0 && pool->stride_slot % 8 == 0 && pool->stride_head % 8 == 0;
  if (!vec) {
    a.steps = std::max(1, 4096 / (H * a.pairs));
    launch_pdl(turn_pairs_kernel, dim3((unsigned)((max_tok + a.steps - 1) / a.steps), (unsigned)R, (unsigned)nls), NT, 0, s, a);
    ACTKV_CHECK_LAUNCH();
    return ACTKV_OK;
  }
  a.lanes = a.interleaved ? a.pairs / 4 : a.pairs / 8;
  const int per = NT / a.lanes;
  // heads apart while there are few tokens, together (and several steps per CTA, for whose sake a thread forms its frequencies once) when
  // there are CTAs enough for every SM to have eight
  const int64_t blocks = (int64_t)R * nls * ((max_tok + per - 1) / per);
  a.heads_per = blocks * ((H + UNROLL - 1) / UNROLL) < 148 * 4 ? 1 : UNROLL;
  if (a.shared && blocks >= 148 * 8) a.heads_per = H;
  a.head_groups = (H + a.heads_per - 1) / a.heads_per;
  a.steps = (int32_t)std::max<int64_t>(1, std::min<int64_t>(4, blocks * a.head_groups / (148 * 8)));
  const dim3 grid((unsigned)((max_tok + per * a.steps - 1) / (per * a.steps)), (unsigned)R, (unsigned)(nls * a.head_groups));
  const bool two = to_inv_freq != nullptr, axes = a.n_axes > 1;
  auto go = [&](auto kernel) { launch_pdl(kernel, grid, NT, 0, s, a); };
  if (!a.interleaved) {
    if (two) axes ? go(turn_kernel<true, true, true>) : go(turn_kernel<true, true, false>);
    else axes ? go(turn_kernel<true, false, true>) : go(turn_kernel<true, false, false>);
  } else {
    if (two) axes ? go(turn_kernel<false, true, true>) : go(turn_kernel<false, true, false>);
    else axes ? go(turn_kernel<false, false, true>) : go(turn_kernel<false, false, false>);
  }
  ACTKV_CHECK_LAUNCH();
  return ACTKV_OK;
}
