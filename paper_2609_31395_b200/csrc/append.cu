// actkv_append: the new tokens' keys and values into their slots, queries and keys turned to their positions (rotary, up to
// four axes) on the way (Section 2.5).
//
// One CTA per (token row, layer).  x' = x cos t - y sin t, y' = y cos t + x sin t per pair; the angle position * inv_freq is formed
// and reduced to half turns in float64 (a position of 10^6 leaves a float32 angle 0.06 rad of rounding), its sine and cosine
// are taken in float32 once per CTA and shared by all heads.  A thread turns two 16-byte vectors at a time.
//
// What bounds it: decode steps by latency, a chain of three reads (request of the row, its length, its page) beside the
// loads of the row itself; chunks of many tokens by reading and writing every row once.
#include "common.cuh"

namespace actkv {
namespace ap {

constexpr int NT = 128;
constexpr int MAX_PAIRS = 128;

struct Rows {
  const __nv_bfloat16* base;
  int64_t stride_layer, stride_row, stride_head;
};
struct Args {
  PoolView pool;
  TablesView tab;
  Rows q, k, v;
  const int32_t* win_indptr;
  const int32_t* positions;
  const float* inv_freq;
  __nv_bfloat16* q_out;
  int32_t* status;
  int32_t layer_begin, n_q_heads, sum_win;
  int32_t pairs, interleaved, n_axes, sec_end[4];
};

// Where row i goes: element offset of its K slot within a layer and head 0, -1 when it is dropped, NO_ROW for a row of no request.
// One warp calls it.
constexpr int64_t NO_ROW = -2;
__device__ __forceinline__ int64_t place_of(const Args& a, int i) {
  const int lane = threadIdx.x & 31, R = a.tab.n_req;
  const int32_t stop = refused(a.status);
  int n = 0;                                     // requests 1 .. R - 1 that begin at or before the row (empty ones among them)
  for (int r = 1 + lane; r < R; r += 32) n += a.win_indptr[r] <= i ? 1 : 0;
  const int r = (int)__reduce_add_sync(0xffffffffu, (uint32_t)n);
  const int w0 = a.win_indptr[r], w1 = a.win_indptr[r + 1], L = a.tab.seq_len[r];
  if (i < w0 || i >= w1) return NO_ROW;
  const int64_t j = (int64_t)L - w1 + i;
  const int P = a.pool.page_size;
  const bool out = j < 0 || j / P >= a.tab.max_pages;
  const int32_t page = out ? -1 : a.tab.page_table[(int64_t)r * a.tab.max_pages + (int)(j / P)];
  if (stop) return -1;                           // (L does not count the new tokens)
  if ((uint32_t)page >= (uint32_t)a.pool.n_pages) {
    if (lane == 0) report(a.status, out ? ACTKV_E_INVALID : ACTKV_E_BADPAGE, r, out ? L : page);
    return -1;
  }
  return (int64_t)page * a.pool.stride_page + (j % P) * a.pool.stride_slot;
}

__device__ __forceinline__ float2 bf2(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ uint32_t turn_pair(uint32_t v, float cs, float sn) {
  const float2 x = bf2(v);
  return pack2(x.x * cs - x.y * sn, x.y * cs + x.x * sn);
}

// VEC: every row and head begins on 16 bytes and the halves of the turned dims are whole vectors.
template <bool VEC>
__global__ void __launch_bounds__(NT) append_kernel(const Args a) {
  pdl_begin();
  __shared__ __align__(16) float s_cos[MAX_PAIRS], s_sin[MAX_PAIRS];       // (apart: a thread reads those of 8 pairs as vectors)
  __shared__ int64_t s_place;
  const int i = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x;
  const int D = a.pool.head_dim, Hkv = a.pool.n_kv_heads, Hq = a.q_out != nullptr ? a.n_q_heads : 0;
  if (tid >= NT - 32) {
    const int64_t at = place_of(a, i);
    if ((tid & 31) == 0) s_place = at;
  }
  for (int p = tid; p < a.pairs; p += NT) {
    int axis = 0;
    while (p >= a.sec_end[axis]) ++axis;
    // in half turns, reduced to [-1, 1]
    double t = (double)a.positions[(int64_t)axis * a.sum_win + i] * (double)a.inv_freq[p] * 0.31830988618379067154;
    t -= 2.0 * rint(0.5 * t);
    float sn, cs;
    sincospif((float)t, &sn, &cs);
    s_cos[p] = cs;
    s_sin[p] = sn;
  }
  __syncthreads();
  const int64_t place = s_place;
  if (place == NO_ROW) return;
  const __nv_bfloat16* qr = a.q.base + (int64_t)layer * a.q.stride_layer + (int64_t)i * a.q.stride_row;
  const __nv_bfloat16* kr = a.k.base + (int64_t)layer * a.k.stride_layer + (int64_t)i * a.k.stride_row;
  const __nv_bfloat16* vr = a.v.base + (int64_t)layer * a.v.stride_layer + (int64_t)i * a.v.stride_row;
  __nv_bfloat16* qo = a.q_out + ((int64_t)layer * a.sum_win + i) * a.n_q_heads * D;
  __nv_bfloat16* kv = const_cast<__nv_bfloat16*>(a.pool.base) + (int64_t)(a.layer_begin + layer) * a.pool.stride_layer + place;
  const int heads = Hq + (place >= 0 ? Hkv : 0);
  auto src_of = [&](int h) { return h < Hq ? qr + (int64_t)h * a.q.stride_head : kr + (int64_t)(h - Hq) * a.k.stride_head; };
  auto dst_of = [&](int h) { return h < Hq ? qo + (int64_t)h * D : kv + (int64_t)(h - Hq) * a.pool.stride_head; };
  if (VEC) {
    // items of a head: turned pairs of vectors (or, interleaved, turned vectors), then vectors that pass
    const int turn = a.interleaved ? a.pairs / 4 : a.pairs / 8, pass = (D - 2 * a.pairs) / 8, per = turn + pass;
    const int dh = NT / per, dc = NT - dh * per;               // from one item of a thread to its next
    for (int h = tid / per, c = tid - h * per; h < heads;) {
      const __nv_bfloat16* src = src_of(h);
      __nv_bfloat16* dst = dst_of(h);
      if (c >= turn) {
        const int d = 2 * a.pairs + (c - turn) * 8;
        *reinterpret_cast<uint4*>(dst + d) = *reinterpret_cast<const uint4*>(src + d);
      } else if (a.interleaved) {
        uint4 v = *reinterpret_cast<const uint4*>(src + c * 8);
        const float4 cs = *reinterpret_cast<const float4*>(&s_cos[c * 4]), sn = *reinterpret_cast<const float4*>(&s_sin[c * 4]);
        v.x = turn_pair(v.x, cs.x, sn.x);
        v.y = turn_pair(v.y, cs.y, sn.y);
        v.z = turn_pair(v.z, cs.z, sn.z);
        v.w = turn_pair(v.w, cs.w, sn.w);
        *reinterpret_cast<uint4*>(dst + c * 8) = v;
      } else {
        uint4 va = *reinterpret_cast<const uint4*>(src + c * 8), vb = *reinterpret_cast<const uint4*>(src + a.pairs + c * 8);
        uint32_t *ua = reinterpret_cast<uint32_t*>(&va), *ub = reinterpret_cast<uint32_t*>(&vb);
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const float4 cs = *reinterpret_cast<const float4*>(&s_cos[c * 8 + 2 * e]), sn = *reinterpret_cast<const float4*>(&s_sin[c * 8 + 2 * e]);
          float2 x = bf2(ua[e]), y = bf2(ub[e]);
          ua[e] = pack2(x.x * cs.x - y.x * sn.x, x.y * cs.y - y.y * sn.y);
          ub[e] = pack2(y.x * cs.x + x.x * sn.x, y.y * cs.y + x.y * sn.y);
          x = bf2(ua[e + 1]), y = bf2(ub[e + 1]);
          ua[e + 1] = pack2(x.x * cs.z - y.x * sn.z, x.y * cs.w - y.y * sn.w);
          ub[e + 1] = pack2(y.x * cs.z + x.x * sn.z, y.y * cs.w + x.y * sn.w);
        }
        *reinterpret_cast<uint4*>(dst + c * 8) = va;
        *reinterpret_cast<uint4*>(dst + a.pairs + c * 8) = vb;
      }
      h += dh;
      c += dc;
      if (c >= per) {
        c -= per;
        ++h;
      }
    }
    if (place >= 0)
      for (int it = tid; it < Hkv * (D / 8); it += NT) {
        const int h = it / (D / 8), d = (it - h * (D / 8)) * 8;
        *reinterpret_cast<uint4*>(kv + a.pool.stride_kv + (int64_t)h * a.pool.stride_head + d) =
            *reinterpret_cast<const uint4*>(vr + (int64_t)h * a.v.stride_head + d);
      }
  } else {
    // one pair, or one dim that passes, at a time
    const int per = a.pairs + (D - 2 * a.pairs);
    for (int it = tid; it < heads * per; it += NT) {
      const int h = it / per, c = it - h * per;
      const __nv_bfloat16* src = src_of(h);
      __nv_bfloat16* dst = dst_of(h);
      if (c >= a.pairs) {
        dst[a.pairs + c] = src[a.pairs + c];
      } else {
        const int da = a.interleaved ? 2 * c : c, db = a.interleaved ? 2 * c + 1 : c + a.pairs;
        const float x = __bfloat162float(src[da]), y = __bfloat162float(src[db]);
        const float cs = s_cos[c], sn = s_sin[c];
        dst[da] = __float2bfloat16_rn(x * cs - y * sn);
        dst[db] = __float2bfloat16_rn(y * cs + x * sn);
      }
    }
    if (place >= 0)
      for (int it = tid; it < Hkv * D; it += NT) {
        const int h = it / D, d = it - h * D;
        kv[a.pool.stride_kv + (int64_t)h * a.pool.stride_head + d] = vr[(int64_t)h * a.v.stride_head + d];
      }
  }
}

inline bool whole_vectors(const actkv_rows_t* r) {
  return ((uintptr_t)r->base & 15) == 0 && r->stride_layer % 8 == 0 && r->stride_row % 8 == 0 && r->stride_head % 8 == 0;
}

}  // namespace ap
}  // namespace actkv

extern "C" int actkv_append(const actkv_pool_t* pool, const actkv_tables_t* tables, int32_t layer_begin, int32_t layer_end,
                            const actkv_rows_t* q, const actkv_rows_t* k, const actkv_rows_t* v, const int32_t* win_indptr,
                            int32_t n_q_heads, const actkv_rope_t* rope, const int32_t* positions, void* q_out, int32_t sum_win,
                            int32_t* status, actkv_stream_t stream) {
  using namespace actkv;
  using namespace actkv::ap;
  if (!pool || !tables || !pool->base || !k || !v) return ACTKV_E_INVALID;
  if (layer_begin < 0 || layer_end > pool->n_layers || layer_begin > layer_end) return ACTKV_E_INVALID;
  const int D = pool->head_dim, Hkv = pool->n_kv_heads, R = tables->n_req;
  if (D <= 0 || D % 8 != 0 || D > 256 || Hkv <= 0 || pool->page_size <= 0 || pool->n_pages <= 0) return ACTKV_E_INVALID;
  if (R < 0 || sum_win < 0 || n_q_heads < 0 || (q != nullptr && (n_q_heads == 0 || !q_out))) return ACTKV_E_INVALID;
  const int nls = layer_end - layer_begin;
  Args a = {};
  if (rope != nullptr) {
    if (rope->rotary_dim < 0 || rope->rotary_dim % 2 != 0 || rope->rotary_dim > D || rope->n_axes < 1 || rope->n_axes > 4)
      return ACTKV_E_INVALID;
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
    if (a.pairs > 0 && sum_win > 0 && R > 0 && nls > 0 && (!rope->inv_freq || !positions)) return ACTKV_E_INVALID;
    a.inv_freq = rope->inv_freq;
  }
  if (R == 0 || nls == 0 || sum_win == 0) return ACTKV_OK;
  if (!win_indptr || !k->base || !v->base || (q && !q->base) || !tables->page_table || !tables->seq_len || tables->max_pages < 0)
    return ACTKV_E_INVALID;
  if (nls > 65535) return ACTKV_E_TOOBIG;
  a.pool = make_view(pool);
  a.tab = make_view(tables);
  a.k = Rows{(const __nv_bfloat16*)k->base, k->stride_layer, k->stride_row, k->stride_head};
  a.v = Rows{(const __nv_bfloat16*)v->base, v->stride_layer, v->stride_row, v->stride_head};
  if (q) a.q = Rows{(const __nv_bfloat16*)q->base, q->stride_layer, q->stride_row, q->stride_head};
  a.win_indptr = win_indptr;
  a.positions = positions;
  a.q_out = q ? (__nv_bfloat16*)q_out : nullptr;
  a.status = status;
  a.layer_begin = layer_begin;
  a.n_q_heads = n_q_heads;
  a.sum_win = sum_win;
  const bool vec = a.pairs % (a.interleaved ? 4 : 8) == 0 && whole_vectors(k) && whole_vectors(v) && (!q || whole_vectors(q)) &&
                   ((uintptr_t)a.q_out & 15) == 0 && ((uintptr_t)pool->base & 15) == 0 && pool->stride_layer % 8 == 0 &&
                   pool->stride_kv % 8 == 0 && pool->stride_page % 8 == 0 && pool->stride_slot % 8 == 0 && pool->stride_head % 8 == 0;
  const dim3 grid((unsigned)sum_win, (unsigned)nls);
  launch_pdl(vec ? append_kernel<true> : append_kernel<false>, grid, NT, 0, (cudaStream_t)stream, a);
  ACTKV_CHECK_LAUNCH();
  return ACTKV_OK;
}
