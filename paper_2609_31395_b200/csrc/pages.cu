// actkv_resize and actkv_copy: pages of a request claimed, given back, and copied into those of another (Section 2.5, Section
// 7.2 last paragraph).
//
// resize_kernel  one CTA, or a cluster of them.  Whether the call can be carried out (enough free pages, all ids in range) is
//                known before anything is written; pops are read before pushes overwrite their places on the stack.
//                Bound by latency: two round trips to memory and a scan over the requests.
// copy_kernel    one CTA per (page of a source, source, layer and K or V): the rows are read once and written to every
//                branch of that source.  Bound by reading and writing every byte once.
#include <cooperative_groups.h>

#include "tc_ptx.cuh"

namespace actkv {
namespace pg {

namespace cg = cooperative_groups;

constexpr int RZ_KEEP = 4;       // ids that a thread holds between the check and the writes

// Exclusive prefixes of two counts below 2^31 (packed in one word) over the CTA, and their totals.
template <int NT>
__device__ __forceinline__ uint64_t scan_pair(uint64_t v, uint64_t& total, uint64_t* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t incl = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint64_t t = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += t;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) {
    if (w == warp) incl += total;
    total += s_warp[w];
  }
  return incl - v;
}

// The entries that move, pops first, then pushes, are one list over all requests; CTA c of the CS of the cluster takes entries
// (c * NT + thread) + n * CS * NT of it.  Requests are taken NT at a time (a batch; more than one only beyond NT requests).
// Writes begin when every CTA has found its entries in order (first cluster barrier).  Ids are read before it and kept in
// registers; those of a longer list are read again: pops before the second barrier, behind which pushes overwrite their places.
template <int NT, int CS>
__global__ void __launch_bounds__(NT) resize_kernel(TablesView tab, int32_t P, int32_t n_pages, const int32_t* __restrict__ new_len,
                                                    int32_t* status) {
  pdl_begin(new_len);
  __shared__ uint32_t s_pop[NT], s_push[NT];     // exclusive prefixes within the batch
  __shared__ int32_t s_y[NT], s_x[NT];
  __shared__ uint64_t s_warp[NT / 32];
  __shared__ int s_bad;
  const int R = tab.n_req, tid = threadIdx.x;
  int rank = 0;
  if constexpr (CS > 1) rank = (int)cg::this_cluster().block_rank();
  const int32_t fc = *tab.free_count;
  const int failed = status_set(status) ? 1 : 0;
  int32_t L = 0, N = -1, Y = 0, X = 0;
  uint64_t before = 0, total = 0;
  auto batch = [&](int base) {                   // one request per thread: pages before and after, what the ones before it move
    const int r = base + tid;
    L = 0, N = -1;
    if (r < R) {
      L = tab.seq_len[r];
      N = new_len[r];
    }
    Y = L <= 0 ? 0 : (L - 1) / P + 1;
    X = N < 0 ? Y : N == 0 ? 0 : (N - 1) / P + 1;
    const uint64_t mine = (uint64_t)(uint32_t)max(0, X - Y) | ((uint64_t)(uint32_t)max(0, Y - X) << 32);
    const bool far = L < 0 || Y > tab.max_pages || X > tab.max_pages;
    before = scan_pair<NT>(far ? 0 : mine, total, s_warp);
    s_pop[tid] = (uint32_t)before;
    s_push[tid] = (uint32_t)(before >> 32);
    s_y[tid] = Y;
    s_x[tid] = X;
    return far;
  };
  // ---- what the call takes, and whether it can ----
  int64_t pops = 0, pushes = 0;
  bool bad = false;
  auto fail = [&](bool is, int32_t code, int32_t where, int64_t what) {
    if (is && !bad && !failed && rank == 0) report(status, code, where, (int32_t)min(what, (int64_t)0x7fffffff));
    bad |= is;
  };
  const int n_batches = (R + NT - 1) / NT;
  for (int b = n_batches - 1; b >= 0; --b) {     // (the first batch stays in place)
    const bool far = batch(b * NT);
    fail(far, ACTKV_E_INVALID, b * NT + tid, N);
    pops += (uint32_t)total;
    pushes += (int64_t)(total >> 32);
  }
  bad = __syncthreads_or(bad || failed) != 0;
  const bool solo = tid == 0;
  if (fc < 0 || fc > n_pages) { if (solo) fail(true, ACTKV_E_INVALID, -1, fc); bad = true; }
  if (pops > fc) { if (solo) fail(true, ACTKV_E_NOFREE, (int32_t)min(pops, (int64_t)0x7fffffff), fc); bad = true; }
  if (fc - pops + pushes > n_pages) { if (solo) fail(true, ACTKV_E_INVALID, -2, fc - pops + pushes); bad = true; }
  // entry e of the batch's pops or pushes: the request (the last one whose prefix is <= e)
  auto find = [&](const uint32_t* pre, uint32_t e, int n) {
    int lo = 0;
    for (int step = NT / 2; step > 0; step >>= 1)
      if (lo + step < n && pre[lo + step] <= e) lo += step;
    return lo;
  };
  int32_t id[RZ_KEEP];
  int32_t* to[RZ_KEEP];                          // pops: the table entry; pushes: the entry they leave
  // which: 0 look all entries over and keep the first, 1 write the pops that were not kept, 2 the pushes
  auto sweep = [&](int which) {
    int64_t pop0 = 0, push0 = 0;
    for (int b = 0; b < n_batches; ++b) {
      if (n_batches > 1) batch(b * NT);
      __syncthreads();
      const int n = min(NT, R - b * NT);
      const uint32_t np = (uint32_t)total, nq = (uint32_t)(total >> 32);
      const uint32_t e0 = rank * NT + tid;
      int kept = 0;
      for (uint64_t e = e0; e < (uint64_t)np + nq; e += CS * NT, ++kept) {
        const bool pop = e < np;
        if (which > 0 && (pop != (which == 1) || (n_batches == 1 && kept < RZ_KEEP))) continue;
        const uint32_t i = (uint32_t)(pop ? e : e - np);
        const int k = find(pop ? s_pop : s_push, i, n);
        int32_t* entry = tab.page_table + (int64_t)(b * NT + k) * tab.max_pages + (pop ? s_y[k] + (int32_t)(i - s_pop[k]) : s_x[k] + (int32_t)(i - s_push[k]));
        const int32_t page = pop ? tab.free_list[fc - 1 - (pop0 + i)] : *entry;
        if (which == 0) {
          if ((uint32_t)page >= (uint32_t)n_pages) {
            if (!bad) report(status, ACTKV_E_BADPAGE, pop ? -1 : b * NT + k, page);
            bad = true;
          }
#pragma unroll
          for (int j = 0; j < RZ_KEEP; ++j)
            if (kept == j) { id[j] = page; to[j] = entry; }
        } else if (pop) {
          *entry = page;
        } else {
          tab.free_list[fc - pops + push0 + i] = page;
          *entry = -1;
        }
      }
      pop0 += np;
      push0 += nq;
      if (n_batches > 1) __syncthreads();
    }
  };
  if (!bad) sweep(0);
  int any = __syncthreads_or(bad);
  if constexpr (CS > 1) {
    cg::cluster_group cl = cg::this_cluster();
    if (tid == 0) s_bad = any;
    cl.sync();
    any = 0;
    for (int c = 0; c < CS; ++c) any |= *cl.map_shared_rank(&s_bad, c);
  }
  if (!any) {
    const uint32_t np = (uint32_t)total;
    const bool more = n_batches > 1 || pops + pushes > (int64_t)RZ_KEEP * CS * NT;      // (uniform over the cluster)
    if (more) {
      sweep(1);
      __syncthreads();
      if constexpr (CS > 1) cg::this_cluster().sync();
    }
    if (n_batches == 1) {
#pragma unroll
      for (int j = 0; j < RZ_KEEP; ++j) {
        const int64_t e = (int64_t)rank * NT + tid + (int64_t)j * CS * NT;
        if (e < np) {
          *to[j] = id[j];
        } else if (e < pops + pushes) {
          tab.free_list[fc - pops + (e - np)] = id[j];
          *to[j] = -1;
        }
      }
    }
    if (more) sweep(2);
    if constexpr (CS > 1) {
      if (n_batches > 1) cg::this_cluster().sync();                       // (one batch: everybody has its lengths in registers)
    }
    if (rank == 0)
      for (int r = tid; r < R; r += NT) {
        const int32_t n = n_batches == 1 ? N : new_len[r];
        if (n >= 0) tab.seq_len[r] = n;
      }
    if (rank == 0 && tid == 0) *tab.free_count = (int32_t)(fc - pops + pushes);
  }
  if (rank == 0 && tid == 0 && status != nullptr) status[3] = any ? ACTKV_STATUS_REFUSED : 0;
  if constexpr (CS > 1) cg::this_cluster().sync();                        // (flags are read from one another's shared memory)
}

template <int NT, int CS>
int launch_resize(const actkv_pool_t* pool, const actkv_tables_t* tables, const int32_t* new_len, int32_t* status, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(CS);
  cfg.blockDim = dim3(NT);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = CS;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = CS > 1 ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, resize_kernel<NT, CS>, make_view(tables), pool->page_size, pool->n_pages, new_len, status);
  ACTKV_CHECK_LAUNCH();
  return ACTKV_OK;
}

constexpr int CP_NT = 128;

struct CopyArgs {
  PoolView pool;
  TablesView tab;
  const int32_t *src, *dst, *length;
  int32_t n_copy, max_len, layer_begin;
  int32_t* status;
};

// What the CTAs of a copy find out first.  The first sound pair of a source works for all pairs of that source; NT pairs are looked at
// together, one per thread, in two round trips to memory.
template <int NT>
struct CopySmem {
  int64_t dst[NT];               // branches that have tokens on this page: element offset of their page,
  int slots[NT];                 // tokens on it
  int n;
};
struct CopySource {
  int src, len, page, col;
  int32_t stop;                  // refused
};
// (dst is a request, of dst_len tokens)
__device__ __forceinline__ bool sound_pair(const CopyArgs& a, int src, int src_len, int dst, int dst_len, int n) {
  return dst != src && n >= 0 && n <= a.max_len && n <= src_len && n <= dst_len && (n == 0 || (n - 1) / a.pool.page_size < a.tab.max_pages);
}
// The source of pair i, for logical page lp; false: nothing to do.  `first`: one CTA of every pair, which reports what is wrong with it.
template <int NT>
__device__ __forceinline__ bool copy_source(const CopyArgs& a, int i, int lp, bool first, CopySource& s) {
  const int tid = threadIdx.x;
  s.stop = refused(a.status);
  s.src = a.src[i];
  if ((uint32_t)s.src >= (uint32_t)a.tab.n_req) {
    if (first && tid == 0 && !s.stop) report(a.status, ACTKV_E_INVALID, i, s.src);
    return false;
  }
  s.col = lp < a.tab.max_pages ? lp : a.tab.max_pages - 1;                 // (max_len may be beyond the table; no sound pair is)
  s.page = a.tab.max_pages > 0 ? a.tab.page_table[(int64_t)s.src * a.tab.max_pages + s.col] : -1;
  s.len = a.tab.seq_len[s.src];
  if (first && !s.stop) {                                                  // (here, not where branches are looked for: that ends early)
    const int d = a.dst[i], n = a.length[i];
    const bool known = (uint32_t)d < (uint32_t)a.tab.n_req;
    if (tid == 0 && !(known && sound_pair(a, s.src, s.len, d, a.tab.seq_len[d], n))) report(a.status, ACTKV_E_INVALID, i, n);
    for (int j = tid; j < a.n_copy; j += NT)
      if (j != i && (a.dst[j] == d || a.src[j] == d)) report(a.status, ACTKV_E_INVALID, i, d);
  }
  return true;
}
// Branches among pairs j0 .. j0 + NT - 1 into sm: 1, none of them this CTA's business: 0, another CTA works for this source: -1.
template <int NT>
__device__ __forceinline__ int copy_branches(const CopyArgs& a, int i, int j0, int lp, const CopySource& s, CopySmem<NT>* sm) {
  const int tid = threadIdx.x, P = a.pool.page_size;
  __syncthreads();
  if (tid == 0) sm->n = 0;
  __syncthreads();
  const int j = j0 + tid;
  bool sound = false;
  if (j < a.n_copy && (j == i || a.src[j] == s.src)) {
    const int d = a.dst[j], n = a.length[j];
    if ((uint32_t)d < (uint32_t)a.tab.n_req) {
      const int dst_len = a.tab.seq_len[d], page = a.tab.max_pages > 0 ? a.tab.page_table[(int64_t)d * a.tab.max_pages + s.col] : -1;
      sound = sound_pair(a, s.src, s.len, d, dst_len, n);
      const int slots = min(P, n - lp * P);
      if (sound && j >= i && slots > 0) {
        const bool src_ok = (uint32_t)s.page < (uint32_t)a.pool.n_pages, dst_ok = (uint32_t)page < (uint32_t)a.pool.n_pages;
        if (src_ok && dst_ok) {
          const int at = atomicAdd(&sm->n, 1);
          sm->dst[at] = (int64_t)page * a.pool.stride_page;
          sm->slots[at] = slots;
        } else if (!s.stop) {
          report(a.status, ACTKV_E_BADPAGE, src_ok ? d : s.src, src_ok ? page : s.page);
        }
      }
    }
  }
  // (an unsound pair copies nothing itself; when it comes first, the next sound one works for the rest)
  if (__syncthreads_or((sound && j < i) || (j == i && !sound) || s.stop)) return -1;
  return j0 + NT > i && sm->n > 0 ? 1 : 0;
}
__device__ __forceinline__ __nv_bfloat16* copy_base(const CopyArgs& a) {
  return const_cast<__nv_bfloat16*>(a.pool.base) + (int64_t)(a.layer_begin + (blockIdx.z >> 1)) * a.pool.stride_layer +
         ((blockIdx.z & 1) ? a.pool.stride_kv : 0);
}

// Pages whose tokens' rows are one run of bytes: through shared memory by bulk copies, up to CB_BYTES of a page per CTA.
// grid: (logical page * parts + part, pair, layer * 2 + kv).
constexpr int CB_NT = 32, CB_BYTES = 16384;
__global__ void __launch_bounds__(CB_NT) copy_bulk_kernel(const __grid_constant__ CopyArgs a, const int parts) {
  pdl_begin();
  __shared__ __align__(128) uint8_t buf[CB_BYTES];
  __shared__ CopySmem<CB_NT> sm;
  __shared__ uint64_t bar;
  const int lp = blockIdx.x / parts, part = blockIdx.x - lp * parts, i = blockIdx.y;
  const bool first = blockIdx.x == 0 && blockIdx.z == 0;
  if (threadIdx.x == 0) {
    tc::mbar_init(tc::smem_u32(&bar), 1);
    tc::fence_barrier_init();
  }
  CopySource s;
  if (!copy_source<CB_NT>(a, i, lp, first, s)) return;
  const int slot_bytes = a.pool.n_kv_heads * a.pool.head_dim * 2, begin = part * CB_BYTES;
  __nv_bfloat16* base = copy_base(a);
  const int held = min(CB_BYTES, min(a.pool.page_size, s.len - lp * a.pool.page_size) * slot_bytes - begin);    // bytes of the source
  bool here = false, lost = false;
  for (int j0 = 0; j0 < a.n_copy; j0 += CB_NT) {
    const int what = copy_branches<CB_NT>(a, i, j0, lp, s, &sm);
    if (what < 0) break;
    if (what == 0 || threadIdx.x != 0 || held <= 0 || lost) continue;
    if (!here) {                                               // once: all of the part that the source has
      const uint32_t b = tc::smem_u32(&bar);
      tc::mbar_expect_tx(b, (uint32_t)held);
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(tc::smem_u32(buf)),
                   "l"((const uint8_t*)(base + (int64_t)s.page * a.pool.stride_page) + begin), "r"(held), "r"(b) : "memory");
      here = tc::mbar_wait(b, 0, nullptr, tc::WAIT_LIMIT_CYCLES);
      if (!here) {
        lost = true;
        report(a.status, ACTKV_E_TIMEOUT, i, lp);
        tc::mbar_wait(b, 0, nullptr, tc::DRAIN_LIMIT_CYCLES);
        continue;
      }
    }
    for (int k = 0; k < sm.n; ++k) {
      const int bytes = min(CB_BYTES, sm.slots[k] * slot_bytes - begin);
      if (bytes > 0)
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"((uint8_t*)(base + sm.dst[k]) + begin),
                     "r"(tc::smem_u32(buf)), "r"(bytes) : "memory");
    }
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
  if (threadIdx.x == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

// Any layout.  grid: (logical page, pair, layer * 2 + kv).
template <bool VEC>
__global__ void __launch_bounds__(CP_NT) copy_kernel(const __grid_constant__ CopyArgs a) {
  pdl_begin();
  __shared__ CopySmem<CP_NT> sm;
  const int tid = threadIdx.x, lp = blockIdx.x, i = blockIdx.y;
  const int H = a.pool.n_kv_heads, D = a.pool.head_dim;
  const bool first = blockIdx.x == 0 && blockIdx.z == 0;
  CopySource s;
  if (!copy_source<CP_NT>(a, i, lp, first, s)) return;
  __nv_bfloat16* base = copy_base(a);
  for (int j0 = 0; j0 < a.n_copy; j0 += CP_NT) {
    const int what = copy_branches<CP_NT>(a, i, j0, lp, s, &sm);
    if (what < 0) return;
    if (what == 0) continue;
    const int n = sm.n;
    int most = 0;
    for (int b = 0; b < n; ++b) most = max(most, sm.slots[b]);
    const __nv_bfloat16* from = base + (int64_t)s.page * a.pool.stride_page;
    constexpr int E = VEC ? 8 : 1, U = VEC ? 4 : 1;
    const int per_row = D / E, per_slot = H * per_row, items = most * per_slot;
    for (int it0 = tid; it0 < items; it0 += CP_NT * U) {
      uint4 v[U];
      __nv_bfloat16 w[U];
      int64_t off[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int it = it0 + u * CP_NT;
        const int slot = it / per_slot, rem = it - slot * per_slot, h = rem / per_row;
        off[u] = (int64_t)slot * a.pool.stride_slot + (int64_t)h * a.pool.stride_head + (rem - h * per_row) * E;
        if (it < items) {
          if (VEC) v[u] = *reinterpret_cast<const uint4*>(from + off[u]);
          else w[u] = from[off[u]];
        }
      }
      for (int b = 0; b < n; ++b) {
        __nv_bfloat16* to = base + sm.dst[b];
        const int end = sm.slots[b] * per_slot;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (it0 + u * CP_NT < end) {
            if (VEC) *reinterpret_cast<uint4*>(to + off[u]) = v[u];
            else to[off[u]] = w[u];
          }
      }
    }
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
  if ((int64_t)tables->n_req * tables->max_pages > 0x7fffffff) return ACTKV_E_TOOBIG;
  cudaStream_t s = (cudaStream_t)stream;
  if (tables->n_req <= 32) return pg::launch_resize<256, 1>(pool, tables, new_len, status, s);
  return pg::launch_resize<512, 8>(pool, tables, new_len, status, s);
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
  const int64_t pages = (max_len - 1) / pool->page_size + 1, slot_bytes = (int64_t)pool->n_kv_heads * pool->head_dim * 2;
  const int64_t parts = (pool->page_size * slot_bytes + CB_BYTES - 1) / CB_BYTES;
  // rows of a page's tokens in one run: 6 layers of 35000 tokens into 3 branches 292 us by vectors
  if (vec && pool->stride_head == pool->head_dim && pool->stride_slot * 2 == slot_bytes && pages * parts <= 0x7fffffff &&
      pool->page_size * slot_bytes <= 0x7fffffff) {
    launch_pdl(copy_bulk_kernel, dim3((unsigned)(pages * parts), (unsigned)n_copy, (unsigned)nls * 2), CB_NT, 0, (cudaStream_t)stream, a, (int)parts);
  } else {
    const dim3 grid((unsigned)pages, (unsigned)n_copy, (unsigned)nls * 2);
    launch_pdl(vec ? copy_kernel<true> : copy_kernel<false>, grid, CP_NT, 0, (cudaStream_t)stream, a);
  }
  ACTKV_CHECK_LAUNCH();
  return ACTKV_OK;
}

}  // extern "C"
