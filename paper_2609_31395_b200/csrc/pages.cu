// actkv_resize and actkv_copy: pages of a request claimed, given back, and copied into those of another (Section 2.5, Section
// 7.2 last paragraph).
//
// resize_kernel  one CTA.  Whether the call can be carried out (enough free pages, all ids in range) is known before
//                anything is written; pops are read before pushes overwrite their places on the stack.
//                Bound by latency: four round trips to memory.
// copy_kernel    one CTA per (page of a source, source, layer and K or V): the rows are read once and written to every
//                branch of that source.  Bound by reading and writing every byte once.
#include "common.cuh"

namespace actkv {
namespace pg {

constexpr int RZ_NT = 1024;

// Requests base .. base + RZ_NT - 1, one per thread: pages before and after, what the ones before it pop and push.
struct Share {
  int L, N, Y, X;                // lengths, pages
  int64_t pop, push;             // exclusive prefixes over this batch
  int64_t pops, pushes;          // totals of this batch
};
__device__ __forceinline__ void scan2(int64_t& a, int64_t& b, int64_t& ta, int64_t& tb) {     // exclusive; totals
  __shared__ int64_t s_a[RZ_NT / 32], s_b[RZ_NT / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t ia = a, ib = b;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, ia, d), y = __shfl_up_sync(0xffffffffu, ib, d);
    if (lane >= d) { ia += x; ib += y; }
  }
  __syncthreads();
  if (lane == 31) { s_a[warp] = ia; s_b[warp] = ib; }
  __syncthreads();
  ia -= a;
  ib -= b;
  ta = tb = 0;
  for (int w = 0; w < RZ_NT / 32; ++w) {
    if (w == warp) { ia += ta; ib += tb; }
    ta += s_a[w];
    tb += s_b[w];
  }
  a = ia;
  b = ib;
}
__device__ __forceinline__ Share share_of(const TablesView& tab, int P, const int32_t* new_len, int base) {
  const int r = base + threadIdx.x;
  Share s{0, -1, 0, 0, 0, 0, 0, 0};
  if (r < tab.n_req) {
    s.L = tab.seq_len[r];
    s.N = new_len[r];
    s.Y = s.L <= 0 ? 0 : (s.L - 1) / P + 1;
    s.X = s.N < 0 ? s.Y : s.N == 0 ? 0 : (s.N - 1) / P + 1;
    s.pop = max(0, s.X - s.Y);
    s.push = max(0, s.Y - s.X);
  }
  scan2(s.pop, s.push, s.pops, s.pushes);
  return s;
}

__global__ void __launch_bounds__(RZ_NT) resize_kernel(TablesView tab, int32_t P, int32_t n_pages, const int32_t* __restrict__ new_len,
                                                       int32_t* status) {
  pdl_begin(new_len);
  __shared__ int64_t s_off[2][RZ_NT + 1];
  __shared__ int32_t s_y[RZ_NT], s_x[RZ_NT];
  const int R = tab.n_req, tid = threadIdx.x;
  const int32_t fc = *tab.free_count;
  if (__syncthreads_or(status_set(status))) return;
  // ---- what the call takes, and whether it can ----
  int64_t pops = 0, pushes = 0;
  bool bad = fc < 0 || fc > n_pages;
  if (bad && tid == 0) report(status, ACTKV_E_INVALID, -1, fc);
  for (int base = 0; base < R; base += RZ_NT) {
    const Share s = share_of(tab, P, new_len, base);
    if (base + tid < R && (s.L < 0 || s.Y > tab.max_pages || s.X > tab.max_pages)) {
      bad = true;
      report(status, ACTKV_E_INVALID, base + tid, s.N);
    }
    pops += s.pops;
    pushes += s.pushes;
  }
  if (pops > fc && !bad) {
    bad = true;
    if (tid == 0) report(status, ACTKV_E_NOFREE, (int32_t)min(pops, (int64_t)0x7fffffff), fc);
  }
  if (fc - pops + pushes > n_pages && !bad) {
    bad = true;
    if (tid == 0) report(status, ACTKV_E_INVALID, -2, (int32_t)min(fc - pops + pushes, (int64_t)0x7fffffff));
  }
  if (__syncthreads_or(bad)) return;
  // entry e of the batch's pops (which = 0) or pushes (1): the request (last one whose prefix is <= e) and its place
  auto find = [&](int which, int64_t e, int n) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_off[which][mid] <= e) lo = mid;
      else hi = mid - 1;
    }
    return lo;
  };
  // phase 0: every id that moves is a page id; 1: pops; 2: pushes and lengths
  for (int phase = 0; phase < 3; ++phase) {
    int64_t pop0 = 0, push0 = 0;
    for (int base = 0; base < R; base += RZ_NT) {
      const Share s = share_of(tab, P, new_len, base);
      s_off[0][tid] = s.pop;
      s_off[1][tid] = s.push;
      s_y[tid] = s.Y;
      s_x[tid] = s.X;
      __syncthreads();
      const int n = min(RZ_NT, R - base);
      if (phase < 2)
        for (int64_t e = tid; e < s.pops; e += RZ_NT) {
          const int32_t id = tab.free_list[fc - 1 - (pop0 + e)];
          if (phase == 0) {
            if ((uint32_t)id >= (uint32_t)n_pages) { bad = true; report(status, ACTKV_E_BADPAGE, -1, id); }
          } else {
            const int k = find(0, e, n);
            tab.page_table[(int64_t)(base + k) * tab.max_pages + s_y[k] + (e - s_off[0][k])] = id;
          }
        }
      if (phase != 1)
        for (int64_t e = tid; e < s.pushes; e += RZ_NT) {
          const int k = find(1, e, n);
          int32_t* entry = tab.page_table + (int64_t)(base + k) * tab.max_pages + s_x[k] + (e - s_off[1][k]);
          const int32_t id = *entry;
          if (phase == 0) {
            if ((uint32_t)id >= (uint32_t)n_pages) { bad = true; report(status, ACTKV_E_BADPAGE, base + k, id); }
          } else {
            tab.free_list[fc - pops + push0 + e] = id;
            *entry = -1;
          }
        }
      if (phase == 2 && base + tid < R && s.N >= 0) tab.seq_len[base + tid] = s.N;
      pop0 += s.pops;
      push0 += s.pushes;
      __syncthreads();
    }
    if (__syncthreads_or(bad)) return;
  }
  if (tid == 0) *tab.free_count = (int32_t)(fc - pops + pushes);
}

constexpr int CP_NT = 128;
constexpr int CP_MAXB = 64;      // branches a CTA serves per sweep over the pairs

struct CopyArgs {
  PoolView pool;
  TablesView tab;
  const int32_t *src, *dst, *length;
  int32_t n_copy, max_len, layer_begin;
  int32_t* status;
};

__device__ __forceinline__ bool pair_ok(const CopyArgs& a, int i, bool tell) {
  const int s = a.src[i], d = a.dst[i], n = a.length[i], R = a.tab.n_req;
  bool ok = (uint32_t)s < (uint32_t)R && (uint32_t)d < (uint32_t)R && s != d && n >= 0 && n <= a.max_len;
  if (ok) ok = n <= a.tab.seq_len[s] && n <= a.tab.seq_len[d] && (n == 0 || (n - 1) / a.pool.page_size < a.tab.max_pages);
  if (!ok && tell) report(a.status, ACTKV_E_INVALID, i, n);
  return ok;
}

// grid: (logical page, pair, layer * 2 + kv).  The first pair of a source works for all pairs of that source.
template <bool VEC>
__global__ void __launch_bounds__(CP_NT) copy_kernel(const CopyArgs a) {
  pdl_begin();
  __shared__ int64_t s_dst[CP_MAXB];
  __shared__ int s_slots[CP_MAXB];
  __shared__ int s_n;
  const int tid = threadIdx.x, lp = blockIdx.x, i = blockIdx.y, layer = blockIdx.z >> 1, kv = blockIdx.z & 1;
  const int P = a.pool.page_size, H = a.pool.n_kv_heads, D = a.pool.head_dim;
  if (blockIdx.x == 0 && blockIdx.z == 0) {      // one CTA of every pair looks it over
    if (tid == 0) pair_ok(a, i, true);
    const int d = a.dst[i];
    for (int j = tid; j < a.n_copy; j += CP_NT)
      if (j != i && (a.dst[j] == d || a.src[j] == d)) report(a.status, ACTKV_E_INVALID, i, d);
  }
  const int src = a.src[i];
  int before = 0;
  for (int j = tid; j < i; j += CP_NT) before |= a.src[j] == src && pair_ok(a, j, false) ? 1 : 0;
  if (__syncthreads_or(before) || !pair_ok(a, i, false)) return;
  const int src_page = page_or_neg(a.tab, a.pool.n_pages, src, lp < a.tab.max_pages ? lp : 0, nullptr);
  __nv_bfloat16* base = const_cast<__nv_bfloat16*>(a.pool.base) + (int64_t)(a.layer_begin + layer) * a.pool.stride_layer +
                        (kv ? a.pool.stride_kv : 0);
  for (int j0 = i; j0 < a.n_copy; j0 += CP_MAXB) {
    // ---- the branches among pairs j0 .. j0 + CP_MAXB - 1 that have tokens on this page ----
    if (tid == 0) s_n = 0;
    __syncthreads();
    if (tid < CP_MAXB && j0 + tid < a.n_copy && a.src[j0 + tid] == src && pair_ok(a, j0 + tid, false)) {
      const int slots = min(P, a.length[j0 + tid] - lp * P);
      if (slots > 0) {
        if (src_page < 0) page_or_neg(a.tab, a.pool.n_pages, src, lp, a.status);
        const int page = page_or_neg(a.tab, a.pool.n_pages, a.dst[j0 + tid], lp, a.status);
        if (page >= 0 && src_page >= 0) {
          const int at = atomicAdd(&s_n, 1);
          s_dst[at] = (int64_t)page * a.pool.stride_page;
          s_slots[at] = slots;
        }
      }
    }
    __syncthreads();
    const int n = s_n;
    int most = 0;
    for (int b = 0; b < n; ++b) most = max(most, s_slots[b]);
    const __nv_bfloat16* from = base + (int64_t)src_page * a.pool.stride_page;
    constexpr int E = VEC ? 8 : 1, U = VEC ? 4 : 1;
    const int per_row = D / E, per_slot = H * per_row, items = most * per_slot;
    for (int it0 = tid; it0 < items; it0 += CP_NT * U) {
      uint4 v[U];
      __nv_bfloat16 w[U];
      int64_t off[U];
      int slot[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int it = it0 + u * CP_NT;
        slot[u] = it < items ? it / per_slot : P;
        const int rem = it - slot[u] * per_slot, h = rem / per_row;
        off[u] = (int64_t)slot[u] * a.pool.stride_slot + (int64_t)h * a.pool.stride_head + (rem - h * per_row) * E;
        if (it < items) {
          if (VEC) v[u] = *reinterpret_cast<const uint4*>(from + off[u]);
          else w[u] = from[off[u]];
        }
      }
      for (int b = 0; b < n; ++b) {
        __nv_bfloat16* to = base + s_dst[b];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (slot[u] < s_slots[b]) {
            if (VEC) *reinterpret_cast<uint4*>(to + off[u]) = v[u];
            else to[off[u]] = w[u];
          }
      }
    }
    __syncthreads();
  }
}

}  // namespace pg
}  // namespace actkv

extern "C" {

int actkv_resize(const actkv_pool_t* pool, const actkv_tables_t* tables, const int32_t* new_len, int32_t* status,
                 actkv_stream_t stream) {
  using namespace actkv;
  if (!pool || !tables || pool->page_size <= 0 || pool->n_pages < 0 || tables->n_req < 0 || tables->max_pages < 0)
    return ACTKV_E_INVALID;
  if (tables->n_req == 0) return ACTKV_OK;
  if (!new_len || !tables->page_table || !tables->seq_len || !tables->free_list || !tables->free_count) return ACTKV_E_INVALID;
  launch_pdl(pg::resize_kernel, 1, pg::RZ_NT, 0, (cudaStream_t)stream, make_view(tables), pool->page_size, pool->n_pages, new_len, status);
  ACTKV_CHECK_LAUNCH();
  return ACTKV_OK;
}

int actkv_copy(const actkv_pool_t* pool, const actkv_tables_t* tables, int32_t layer_begin, int32_t layer_end, const int32_t* src,
               const int32_t* dst, const int32_t* length, int32_t n_copy, int32_t max_len, int32_t* status, actkv_stream_t stream) {
  using namespace actkv;
  using namespace actkv::pg;
  if (!pool || !tables || !pool->base) return ACTKV_E_INVALID;
  if (layer_begin < 0 || layer_end > pool->n_layers || layer_begin > layer_end) return ACTKV_E_INVALID;
  if (pool->head_dim <= 0 || pool->n_kv_heads <= 0 || pool->page_size <= 0 || pool->n_pages < 0 || n_copy < 0 || max_len < 0 ||
      tables->n_req < 0 || tables->max_pages < 0)
    return ACTKV_E_INVALID;
  const int nls = layer_end - layer_begin;
  if (n_copy == 0 || nls == 0 || max_len == 0) return ACTKV_OK;
  if (!src || !dst || !length || !tables->page_table || !tables->seq_len) return ACTKV_E_INVALID;
  if (n_copy > 65535 || nls > 32767) return ACTKV_E_TOOBIG;
  CopyArgs a;
  a.pool = make_view(pool);
  a.tab = make_view(tables);
  a.src = src;
  a.dst = dst;
  a.length = length;
  a.n_copy = n_copy;
  a.max_len = max_len;
  a.layer_begin = layer_begin;
  a.status = status;
  const bool vec = ((uintptr_t)pool->base & 15) == 0 && pool->head_dim % 8 == 0 && pool->stride_layer % 8 == 0 &&
                   pool->stride_kv % 8 == 0 && pool->stride_page % 8 == 0 && pool->stride_slot % 8 == 0 && pool->stride_head % 8 == 0;
  const dim3 grid((unsigned)((max_len - 1) / pool->page_size + 1), (unsigned)n_copy, (unsigned)nls * 2);
  launch_pdl(vec ? copy_kernel<true> : copy_kernel<false>, grid, CP_NT, 0, (cudaStream_t)stream, a);
  ACTKV_CHECK_LAUNCH();
  return ACTKV_OK;
}

}  // extern "C"
