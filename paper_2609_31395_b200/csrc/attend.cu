// actkv_attend: attention of the newest tokens over the paged cache (Section 2.3), with the LSE that Section 7.1 takes from
// the attention backend.
//
// One pass over K and V.  Keys come in tiles of 16; a warp forms the logits of a tile, D[key, row] = K Q^T, keeps a running
// reference m and a running sum l of exp2(t - m) per row (t in log2 units), and accumulates O^T[dim, row] += V^T P^T.  With
// the keys on the long side of the matrix instruction (m16n8k16) 8 rows fill it, the usual number of query heads per KV head;
// with the rows on that side half of every product would be padding.
//   The reference moves only when a logit exceeds it by more than 8 (a factor of 256 in a probability: nothing in float32),
// so that most tiles need no maximum over the lanes and no rescaling.
//   P enters the second product as two bf16 summands, p truncated to bf16 and the rest: with one, the rounding of P is as
// large as that of the output (together 1.4 times the error of a float32 computation).  The tensor pipe has the room.
//
// What bounds it: reading K and V, 4 D bytes a key and KV head.
//
// Work.  For every KV head all (layer, request, block of rows) units in one line, each as long as its key tiles; the head's CTAs take
// equal pieces of the line, from the lengths on the device, so that ragged requests are balanced and a captured graph follows
// growing caches.  CTAs that follow one another have the same piece of different heads: what they read lies in the same pages
// (head_dim 64, 8 heads: 137 us with one line through all heads, 100 so).
// A unit that lies in several pieces leaves (m, l, O) partials, joined by attend_join_kernel in piece order.  (Joined by the CTA that finishes
// last instead, found by marks in the workspace, a launch fewer: 10.1 us against 8.3 for 1000 tokens, 21.7 against 15.1 for 8000; a chain
// of fences and reads by one CTA takes longer than a launch whose start is already behind it.)  Short and few requests: launch_cluster.
// Within a CTA the groups of RG warps take the tiles of a piece in turn; the warps of a group share a ring of tiles
// in shared memory and have 8 NT rows each.
#include <cooperative_groups.h>

#include <algorithm>

#include "attend_tc.cuh"

namespace actkv {
namespace at {

constexpr int KT = 16;                    // keys per tile
constexpr int MIN_TILES = 4;              // fewest tiles of a CTA's piece

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {     // the rest of 16 is zeroed
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}

// What a launch variant is made of.  NT: row tiles of 8 per warp; RG: warps that share a ring (and have different rows).
// PER_SM, WARPS: 0 for the usual numbers.
template <int DP, int NT, int RG, int PER_SM = 0, int WARPS = 0>
struct Cfg {
  static constexpr int NW = WARPS > 0 ? WARPS : 4, NTH = NW * 32;
  static constexpr int NG = NW / RG;
  static constexpr int RB = 8 * NT * RG;                                   // rows of a block
  static constexpr int TILE = KT * DP * 2 * 2;                             // bytes: K and V
  // CTAs per SM, as many as registers allow (the variants of 32 rows a warp at 128 dims, and of 16 at 256, spill 20 to 44 bytes at the
  // 255 that a thread has at most); they share what the rings may take.  (8 rows, 35000 x 8 tokens of 128 dims:
  // 98.8 us with two, 95 with three; 16000 x 16 of 64 dims: 121 with two, 94 with four.)
  static constexpr int CTAS = PER_SM > 0 ? PER_SM : DP > 128 ? 1 : NT > 1 ? 2 : DP == 64 ? 4 : 3;
  static constexpr int RING_MAX = 192 / CTAS * 1024;
  static constexpr int STAGES = RING_MAX / (NG * TILE) > 16 ? 16 : RING_MAX / (NG * TILE);
  static constexpr int RING = NG * STAGES * TILE;
  static constexpr int RED = NW * 8 * (DP + 4) * 4;
  static_assert(RED <= RING, "the join of the warps reuses the ring");
};

template <int DP, int NT, int RG, int CL, int PER_SM = 0, int WARPS = 0>
__global__ void __launch_bounds__((Cfg<DP, NT, RG, PER_SM, WARPS>::NTH), (Cfg<DP, NT, RG, PER_SM, WARPS>::CTAS))
    attend_kernel(const __grid_constant__ Args a) {
  using C = Cfg<DP, NT, RG, PER_SM, WARPS>;
  constexpr int NW = C::NW, NTH = C::NTH;
  pdl_begin();
  extern __shared__ __align__(128) uint8_t at_smem[];
  __shared__ float2 s_ml[NW][8 * NT];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int grp = warp / RG, part = warp % RG;
  const int G = a.group, D = a.pool.head_dim, P = a.pool.page_size;

  using L1 = Line<KT, C::RB, MIN_TILES>;
  Seg sg;
  int h;
  if constexpr (CL > 1) {                                                  // a cluster per unit, equal shares of its tiles
    const int unit = blockIdx.x / CL, rank = blockIdx.x % CL, lr = unit / a.rb_max, Hkv = a.pool.n_kv_heads;
    sg.rb = unit - lr * a.rb_max;
    sg.r = lr % a.tab.n_req;
    sg.layer = lr / a.tab.n_req / Hkv;
    h = lr / a.tab.n_req - sg.layer * Hkv;
    sg.q = load_req<KT>(a, sg.r, unit < a.tab.n_req * a.rb_max && sg.rb == 0 && rank == 0 && warp == 0);
    if (sg.rb * C::RB >= sg.q.W * G) return;                               // (the whole cluster)
    const int share = (sg.q.tiles + CL - 1) / CL;
    sg.t_in = rank * share;
    sg.n_tiles = max(0, min(share, sg.q.tiles - sg.t_in));
  }
  std::conditional_t<(CL > 1), int, L1> line = [&]() {
    if constexpr (CL > 1) return 0;
    else return L1(a, blockIdx.x == 0 && warp == 0);
  }();
  if constexpr (CL == 1) {
    if (line.x >= line.x1) return;
    h = line.h;
  }

  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(at_smem) + grp * C::STAGES * C::TILE;
  const int g = lane >> 2, t2 = (lane & 3) * 2;
  const int nch = D / 8;                                                   // 16-byte chunks of a row
  if (D < DP) {                                                            // dims past head_dim: zeros, never written again
    const int spare = DP / 8 - nch;
    for (int i = tid; i < C::RING / (DP * 2) * spare; i += NTH) {
      const int row = i / spare, c = nch + i % spare;
      *reinterpret_cast<uint4*>(at_smem + row * DP * 2 + ((c ^ (row & 7)) << 4)) = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
  }
  auto group_sync = [&]() {
    if (RG == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + grp), "n"(RG * 32) : "memory");
  };

  bool more = true;
  auto next = [&]() {
    if constexpr (CL > 1) {
      const bool now = more;
      more = false;
      return now;
    } else {
      return line.next(sg);
    }
  };
  while (next()) {
    const Req& q = sg.q;
    const int r = sg.r, rb = sg.rb, t_in = sg.t_in, n_tiles = sg.n_tiles, layer = sg.layer;
    const int L = q.L, rows = q.W * G;

    // ---- the stream of this group's tiles ----
    const __nv_bfloat16* kbase = a.pool.base + (int64_t)(a.layer_begin + layer) * a.pool.stride_layer + (int64_t)h * a.pool.stride_head;
    const int first = q.lo_tile + t_in + grp, end = q.lo_tile + t_in + n_tiles;
    auto page_of = [&](int tile) -> int {                                  // page of key tile * 16 + lane % 16, -1 behind the end
      const int key = tile * KT + (lane & 15);
      if (tile >= end || key >= L) return -1;
      const int lp = a.page_shift >= 0 ? key >> a.page_shift : key / P;
      return checked_page(a.tab, a.pool.n_pages, r, lp, a.status);
    };
    auto issue = [&](int tile, int stage, int page) {
      if (tile < end) {
        const int key = tile * KT + (lane & 15);
        const int slot = a.page_shift >= 0 ? key & (P - 1) : key % P;
        const int64_t koff = page >= 0 ? (int64_t)page * a.pool.stride_page + (int64_t)slot * a.pool.stride_slot : -1;
        constexpr int CH = DP / 8, RPI = 32 / CH;                          // chunks of a row, rows per step of the warp
        constexpr int MINE = KT / RG;                                      // rows of the tile that this warp loads
        const int c = lane % CH;
#pragma unroll
        for (int i = 0; i < MINE / RPI; ++i) {
          const int row = part * MINE + i * RPI + lane / CH;
          const int64_t o = __shfl_sync(0xffffffffu, koff, row);
          const uint32_t dst = ring + stage * C::TILE + row * DP * 2 + ((c ^ (row & 7)) << 4);
          const __nv_bfloat16* src = kbase + (o < 0 ? 0 : o + c * 8);
          if (c < nch) {
            cp_async16(dst, src, o < 0 ? 0 : 16);
            cp_async16(dst + C::TILE / 2, o < 0 ? src : src + a.pool.stride_kv, o < 0 ? 0 : 16);
          }
        }
      }
      cp_commit();
    };
    int pages[C::STAGES];                                                  // (all looked up before the first is used)
#pragma unroll
    for (int i = 0; i < C::STAGES; ++i) pages[i] = page_of(first + i * C::NG);
#pragma unroll
    for (int i = 0; i < C::STAGES - 1; ++i) issue(first + i * C::NG, i, pages[i]);
    int page_next = pages[C::STAGES - 1];

    // ---- rows of this warp ----
    const int row0 = rb * C::RB + part * 8 * NT;
    const bool active = row0 < rows;
    const int64_t qrow = (int64_t)layer * a.sum_win + q.win0;
    uint32_t qf[DP / 16][NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int rho = row0 + n * 8 + g;
      const int w = rho / G;
      const __nv_bfloat16* src = a.q + ((qrow + w) * a.n_q_heads + h * G + (rho - w * G)) * D + t2;
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          qf[ks][n][c] = (rho < rows && 2 * ks + c < nch) ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + c * 8) : 0u;
    }
    // keys that all rows of this warp see
    const int pos0 = a.causal ? L - q.W : L - 1;                           // position of window row 0
    const int step = a.causal ? 1 : 0;
    const int w_lo = row0 / G, w_hi = min(row0 + 8 * NT, rows) - 1;
    const int all_hi = pos0 + step * w_lo;
    const int all_lo = a.win_left > 0 ? pos0 + step * (w_hi / G) - a.win_left + 1 : 0;

    float acc[DP / 16][NT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int mt = 0; mt < DP / 16; ++mt)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[mt][n][c] = 0.f;
      m[n][0] = m[n][1] = NO_REF;
      l[n][0] = l[n][1] = 0.f;
    }

    int stage = 0, stage_w = C::STAGES - 1;
#pragma unroll 1
    for (int tile = first; tile < end; tile += C::NG) {
      cp_wait<C::STAGES - 2>();
      group_sync();                                                        // the tile is here; the previous one has been read
      issue(tile + (C::STAGES - 1) * C::NG, stage_w, page_next);
      page_next = page_of(tile + C::STAGES * C::NG);
      const uint32_t ks_addr = ring + stage * C::TILE;
      stage = stage + 1 == C::STAGES ? 0 : stage + 1;
      stage_w = stage_w + 1 == C::STAGES ? 0 : stage_w + 1;
      if (!active) continue;

      // logits of 16 keys
      float s[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[n][c] = 0.f;
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) {
        uint32_t kf[4];
        const int row = lane & 15, c = 2 * ks + (lane >> 4);
        ldsm4(kf, ks_addr + row * DP * 2 + ((c ^ (row & 7)) << 4));
#pragma unroll
        for (int n = 0; n < NT; ++n) mma16816(s[n], kf, qf[ks][n][0], qf[ks][n][1]);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[n][c] *= a.scale_log2;
      const int key0 = tile * KT;
      const bool masked = key0 + KT - 1 > all_hi || key0 < all_lo;
      uint32_t hidden = 0;                                                 // bit 4 n + c: s[n][c] is of a key that its row does not see
      if (masked) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int key = key0 + g + (c >> 1) * 8;
            const int pos = pos0 + step * ((row0 + n * 8 + t2 + (c & 1)) / G);
            if (key > pos || (a.win_left > 0 && key <= pos - a.win_left)) {
              s[n][c] = -INFINITY;
              hidden |= 1u << (4 * n + c);
            }
          }
      }
      // the references, when some logit has left them behind
      bool beyond = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) beyond |= s[n][c] > m[n][c & 1] + REF_SLACK;
      if (__any_sync(0xffffffffu, beyond)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float v = fmaxf(fmaxf(s[n][c], s[n][c + 2]), m[n][c]);
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
            const float f = exp2f(m[n][c] - v);
            m[n][c] = v;
            l[n][c] *= f;
#pragma unroll
            for (int mt = 0; mt < DP / 16; ++mt) {
              acc[mt][n][c] *= f;
              acc[mt][n][c + 2] *= f;
            }
          }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s[n][c] = exp2f(s[n][c] - m[n][c & 1]);
          l[n][c & 1] += s[n][c];
        }
      // V of a tile that not every row sees whole: an infinity or NaN there must not meet a hidden key's 0 in a product.  (A row that
      // sees the key takes it whatever its probability: one that is 0 in float32 makes a NaN, as it does in every other tile.)
      const uint32_t vs_addr = ks_addr + C::TILE / 2;
      if (masked) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
          uint4 v;
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(vs_addr + (i * 32 + lane) * 16) : "memory");
          for (uint32_t u : {v.x, v.y, v.z, v.w}) odd |= (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u;
        }
        if (__any_sync(0xffffffffu, odd)) {
#pragma unroll 1
          for (int kk = 0; kk < KT; ++kk) {
            const uint32_t hid = __shfl_sync(0xffffffffu, hidden, (kk & 7) * 4 + (lane & 3)) >> (kk < 8 ? 0 : 2);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const float p0 = __shfl_sync(0xffffffffu, kk < 8 ? s[n][0] : s[n][2], (kk & 7) * 4 + (lane & 3));
              const float p1 = __shfl_sync(0xffffffffu, kk < 8 ? s[n][1] : s[n][3], (kk & 7) * 4 + (lane & 3));
#pragma unroll
              for (int mt = 0; mt < DP / 16; ++mt)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                  uint16_t raw;
                  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(raw) : "r"(vs_addr + kk * DP * 2 + (((2 * mt + hf) ^ (kk & 7)) << 4) + g * 2) : "memory");
                  const float v = __uint_as_float((uint32_t)raw << 16);
                  if (!(hid >> (4 * n) & 1u)) acc[mt][n][2 * hf] = fmaf(p0, v, acc[mt][n][2 * hf]);
                  if (!(hid >> (4 * n) & 2u)) acc[mt][n][2 * hf + 1] = fmaf(p1, v, acc[mt][n][2 * hf + 1]);
                }
            }
          }
          continue;
        }
      }
      uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint32_t u0 = __float_as_uint(s[n][2 * c]), u1 = __float_as_uint(s[n][2 * c + 1]);
          const float r0 = s[n][2 * c] - __uint_as_float(u0 & 0xffff0000u), r1 = s[n][2 * c + 1] - __uint_as_float(u1 & 0xffff0000u);
          uint32_t lo;
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(lo) : "f"(r1), "f"(r0));
          ph[n][c] = transpose8(__byte_perm(u0, u1, 0x7632));
          pl[n][c] = transpose8(lo);
        }
#pragma unroll
      for (int mt = 0; mt < DP / 16; ++mt) {
        uint32_t vf[4];
        const int row = (lane & 7) + ((lane >> 4) << 3), c = 2 * mt + ((lane >> 3) & 1);
        ldsm4t(vf, vs_addr + row * DP * 2 + ((c ^ (row & 7)) << 4));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma16816(acc[mt][n], vf, ph[n][0], ph[n][1]);
          mma16816(acc[mt][n], vf, pl[n][0], pl[n][1]);
        }
      }
    }
    cp_wait<0>();

    // ---- the groups' shares of the piece together ----
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], 4);
        l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], 8);
        l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], 16);
        if (lane < 4) s_ml[warp][n * 8 + t2 + c] = make_float2(m[n][c], l[n][c]);
      }
    __syncthreads();                                                       // ... and nobody reads the rings any more
    bool whole = false;
    int64_t slot = 0;
    if constexpr (CL == 1) {
      whole = sg.b0 == sg.b1;
      slot = line.slot(sg);
      if (t_in == 0 && tid == 0) a.desc[line.unit(sg)] = make_int2(sg.b0, sg.b1);
    }
    float* red = reinterpret_cast<float*>(at_smem);
    // (a cluster: the CTA's share of the unit's rows, for the others to read)
    float* mine = reinterpret_cast<float*>(at_smem + C::RED);
    float2* mine_ml = reinterpret_cast<float2*>(mine + C::RB * DP);
    constexpr int RS = DP + 4;
#pragma unroll 1
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int nn = 0; nn < NT; ++nn) {
        if (nn != n) continue;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int row = t2 + c;
          float M = NO_REF;
#pragma unroll
          for (int k = 0; k < C::NG; ++k) M = fmaxf(M, s_ml[k * RG + part][nn * 8 + row].x);
          const float f = exp2f(m[nn][c] - M);
          float* dst = red + (warp * 8 + row) * RS + g;
#pragma unroll
          for (int mt = 0; mt < DP / 16; ++mt) {
            dst[mt * 16] = acc[mt][nn][c] * f;
            dst[mt * 16 + 8] = acc[mt][nn][c + 2] * f;
          }
        }
      }
      __syncthreads();
      for (int i = tid; i < RG * 8 * (DP / 4); i += NTH) {
        const int d = (i % (DP / 4)) * 4, row = i / (DP / 4) % 8, pt = i / (DP / 4 * 8);
        const int in_block = (pt * NT + n) * 8 + row, rho = rb * C::RB + in_block;
        if (rho >= rows) continue;
        float M = NO_REF, sum = 0.f;
#pragma unroll
        for (int k = 0; k < C::NG; ++k) M = fmaxf(M, s_ml[k * RG + pt][n * 8 + row].x);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < C::NG; ++k) {
          const float2 ml = s_ml[k * RG + pt][n * 8 + row];
          sum = fmaf(ml.y, exp2f(ml.x - M), sum);
          const float4 v = *reinterpret_cast<const float4*>(red + ((k * RG + pt) * 8 + row) * RS + d);
          o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
        }
        if (CL > 1) {
          *reinterpret_cast<float4*>(mine + in_block * DP + d) = o;
          if (d == 0) mine_ml[in_block] = make_float2(M, sum);
        } else if (whole) {
          const int w = rho / G;
          const int64_t at = (qrow + w) * a.n_q_heads + h * G + (rho - w * G);
          store_row(a, at, d, o, sum, M, D);
        } else {
          *reinterpret_cast<float4*>(a.part + (slot * C::RB + in_block) * DP + d) = o;
          if (d == 0) a.part_ml[slot * C::RB + in_block] = make_float2(M, sum);
        }
      }
      __syncthreads();
    }
    if constexpr (CL > 1) {
      static_assert(C::RED + C::RB * (DP * 4 + 8) <= C::RING, "the shares fit behind the join of the warps");
      namespace cg = cooperative_groups;
      cg::cluster_group cl = cg::this_cluster();
      cl.sync();
      for (int row = (int)cl.block_rank(); row < C::RB; row += CL) {
        const int rho = rb * C::RB + row;
        if (rho >= rows) break;
        float M = NO_REF, sum = 0.f, f[CL];
        float2 ml[CL];
#pragma unroll
        for (int c = 0; c < CL; ++c) ml[c] = cl.map_shared_rank(mine_ml, c)[row];
#pragma unroll
        for (int c = 0; c < CL; ++c) M = fmaxf(M, ml[c].x);
#pragma unroll
        for (int c = 0; c < CL; ++c) {
          f[c] = exp2f(ml[c].x - M);
          sum = fmaf(ml[c].y, f[c], sum);
        }
        const int w = rho / G;
        const int64_t at = (qrow + w) * a.n_q_heads + h * G + (rho - w * G);
        for (int d = tid * 4; d < DP; d += NTH * 4) {
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int c = 0; c < CL; ++c) {
            const float4 v = *reinterpret_cast<const float4*>(cl.map_shared_rank(mine, c) + row * DP + d);
            o.x = fmaf(v.x, f[c], o.x);
            o.y = fmaf(v.y, f[c], o.y);
            o.z = fmaf(v.z, f[c], o.z);
            o.w = fmaf(v.w, f[c], o.w);
          }
          store_row(a, at, d, o, sum, M, D);
        }
      }
      cl.sync();                                                           // (the others' shares have been read)
      return;
    }
    // (dims past head_dim: the join has written over their zeros)
    if (D < DP) {
      const int spare = DP / 8 - nch;
      for (int i = tid; i < C::RING / (DP * 2) * spare; i += NTH) {
        const int row = i / spare, c = nch + i % spare;
        *reinterpret_cast<uint4*>(at_smem + row * DP * 2 + ((c ^ (row & 7)) << 4)) = make_uint4(0, 0, 0, 0);
      }
      __syncthreads();
    }
  }
}

// The partials of one row of a unit that lies in several pieces, in piece order.  One CTA per (row, unit).
constexpr int JN = 256;
template <int DP>
__global__ void __launch_bounds__(JN) attend_join_kernel(const __grid_constant__ Args a, int32_t RB) {
  // (no early start of the next kernel: 8000 x 1 14.8 us with it, 13.6 without; see below)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ float2 s_ml[MAX_CTAS];
  __shared__ float s_red[JN / 32][DP];
  __shared__ float s_r[JN / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t unit = blockIdx.x;
  const int rb = (int)(unit % a.rb_max);
  const int64_t lr = unit / a.rb_max;
  const int r = (int)(lr % a.tab.n_req), lh = (int)(lr / a.tab.n_req);
  const int rho = rb * RB + blockIdx.y, G = a.group, D = a.pool.head_dim;
  const int2 b = a.desc[unit];                                             // (read beside the request's: not valid where W = 0)
  const Req q = load_req<KT>(a, r, false);
  if (rho >= q.W * G || b.x == b.y) return;
  const int n = b.y - b.x + 1, row = blockIdx.y;
  const int Hkv = a.pool.n_kv_heads, layer = lh / Hkv, h = lh - layer * Hkv;
  auto slot = [&](int i) { return slot_of(i, b.x, h, Hkv); };
  // the first partials of this warp are on their way while the weights are formed
  constexpr int E = DP / 32, AHEAD = 4;
  float ahead[AHEAD][E];
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) {
    const int i = warp + k * (JN / 32);
#pragma unroll
    for (int e = 0; e < E; ++e) ahead[k][e] = i < n ? a.part[(slot(i) * RB + row) * DP + e * 32 + lane] : 0.f;
  }
  float M = NO_REF;
  for (int i = tid; i < n; i += JN) {
    const float2 v = a.part_ml[slot(i) * RB + row];
    s_ml[i] = v;
    M = fmaxf(M, v.x);
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  if (lane == 0) s_r[warp] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < JN / 32; ++w) M = fmaxf(M, s_r[w]);
  // (every warp forms the sum by itself, in the same order)
  float sum = 0.f;
  for (int i = lane; i < n; i += 32) sum = fmaf(s_ml[i].y, exp2f(s_ml[i].x - M), sum);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  float o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) {
    const int i = warp + k * (JN / 32);
    const float f = i < n ? exp2f(s_ml[i].x - M) : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(ahead[k][e], f, o[e]);
  }
#pragma unroll 4
  for (int i = warp + AHEAD * (JN / 32); i < n; i += JN / 32) {
    const float* src = a.part + (slot(i) * RB + row) * DP;
    const float f = exp2f(s_ml[i].x - M);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(src[e * 32 + lane], f, o[e]);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) s_red[warp][e * 32 + lane] = o[e];
  __syncthreads();
  const int w = rho / G;
  const int64_t at = ((int64_t)layer * a.sum_win + q.win0 + w) * a.n_q_heads + h * G + (rho - w * G);
  if (tid < D) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < JN / 32; ++k) v += s_red[k][tid];
    a.out[at * D + tid] = __float2bfloat16_rn(sum == 0.f ? v * 0.f : v / sum);    // (0, or NaN where V has it)
  }
  if (tid == 0 && a.lse != nullptr) a.lse[at] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
}

// The same with a warp per row, eight rows of a unit per CTA: for launches with more rows than CTAs of the kernel above fit on the SMs.
template <int DP>
__global__ void __launch_bounds__(JN) attend_join_rows_kernel(const __grid_constant__ Args a, int32_t RB) {
  // (The next kernel may start when this one has ended, not before: with CTAs of the next call placed among those of this kernel,
  // calls one behind another took 474 us, so 366: 64 requests of 8K-32K.)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, row = blockIdx.y * (JN / 32) + (threadIdx.x >> 5);
  const int64_t unit = blockIdx.x;
  const int rb = (int)(unit % a.rb_max);
  const int64_t lr = unit / a.rb_max;
  const int r = (int)(lr % a.tab.n_req), lh = (int)(lr / a.tab.n_req);
  const int rho = rb * RB + row, G = a.group, D = a.pool.head_dim;
  const int2 b = a.desc[unit];
  const Req q = load_req<KT>(a, r, false);
  if (rho >= q.W * G || b.x == b.y) return;
  const int n = b.y - b.x + 1, Hkv = a.pool.n_kv_heads, layer = lh / Hkv, h = lh - layer * Hkv;
  auto slot = [&](int i) { return slot_of(i, b.x, h, Hkv); };
  constexpr int E = DP / 32;
  float M = NO_REF, sum = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int i0 = 0; i0 < n; i0 += 32) {                                     // 32 pieces at a time, one per lane
    const float2 ml = i0 + lane < n ? a.part_ml[slot(i0 + lane) * RB + row] : make_float2(NO_REF, 0.f);
    float top = ml.x;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    top = fmaxf(top, M);
    const float f = exp2f(M - top), w = exp2f(ml.x - top);
    M = top;
    float s = ml.y * w;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    sum = fmaf(sum, f, s);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= f;
    const int m = min(32, n - i0);
#pragma unroll 8
    for (int i = 0; i < m; ++i) {
      const float wi = __shfl_sync(0xffffffffu, w, i);
      const float* src = a.part + (slot(i0 + i) * RB + row) * DP + lane;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = fmaf(src[e * 32], wi, o[e]);
    }
  }
  const int w = rho / G;
  const int64_t at = ((int64_t)layer * a.sum_win + q.win0 + w) * a.n_q_heads + h * G + (rho - w * G);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e * 32 + lane < D) a.out[at * D + e * 32 + lane] = __float2bfloat16_rn(o[e] * inv);
  if (lane == 0 && a.lse != nullptr) a.lse[at] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
}

// The tensor-core kernel takes more rows than one instruction of the warp-level one holds, its loads are boxes of a page's rows (pages of 16
// to 128 tokens), and its start and end (12 us of a call at 32 rows, 27 at 64, most of it code that is run once) want work to stand against.
// By rows and (key, KV head) pairs of the launch, as the host bounds them; us with the warp-level and the tensor-core kernel, 4 heads:
//   16 rows, 128 dims:  1 x 8000 14.6 15.8, 8 x 8000 38.2 40.8, 16 x 16000 105 100;
//   32 rows, 128 dims:  8 x 500 17.8 17.5, 1 x 8000 18.4 15.9, 8 x 2000 31.6 22.7, 16 x 16000 153 101; 64 dims: 8 x 500 14.2 16.3, 1 x 8000 15.6 15.3;
//   64 rows, 128 dims:  1 x 8000 23.0 31.3, 8 x 2000 42.4 31.1, 16 x 16000 248 129; 64 dims: 1 x 8000 18.5 30.0, 8 x 2000 27.7 26.2.
inline bool use_tc(int D, int P, int64_t rows, int64_t pairs) {
  if ((D != 64 && D != 128) || (P != 16 && P != 32 && P != 64 && P != 128) || rows <= 8) return false;
  return rows <= 16 ? pairs >= (512 << 10) : rows <= 32 ? pairs >= (24 << 10) : pairs * ((rows + 63) / 64) >= (64 << 10);
}
// rows of a block for this many rows per request at most: the smallest variant that holds them
inline int block_rows(int D, int64_t rows, bool tc) {
  if (tc) return rows <= 32 ? 32 : 64;
  if (D > 128) return rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  return rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
}
inline int padded_dim(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

struct WsLayout {
  size_t desc_off, ml_off, part_off, total;
  int RB, DP;
  int64_t rb_max, units;
};
inline WsLayout ws_layout(int Hkv, int D, int64_t n_req, int64_t nls, int G, int64_t max_win, bool tc) {
  WsLayout l;
  l.RB = block_rows(D, max_win * G, tc);
  l.DP = padded_dim(D);
  l.rb_max = std::max<int64_t>(1, (max_win * G + l.RB - 1) / l.RB);
  l.units = nls * Hkv * n_req * l.rb_max;
  l.desc_off = 0;
  l.ml_off = align_up((size_t)l.units * sizeof(int2), 256);
  l.part_off = l.ml_off + align_up((size_t)2 * MAX_CTAS * l.RB * sizeof(float2), 256);
  l.total = l.part_off + (size_t)2 * MAX_CTAS * l.RB * l.DP * 4;
  return l;
}

template <int DP>
int launch_join(const Args& a, int64_t pieces, int64_t units, int RB, cudaStream_t s) {
  if (pieces == 1) return ACTKV_OK;
  // (64 rows, 128 units of two pieces: a CTA per row 120 us, a warp per row 6)
  if (units * RB <= SMS * (2048 / JN)) launch_pdl(attend_join_kernel<DP>, dim3((unsigned)units, RB), JN, 0, s, a, (int32_t)RB);
  else launch_pdl(attend_join_rows_kernel<DP>, dim3((unsigned)units, (RB + JN / 32 - 1) / (JN / 32)), JN, 0, s, a, (int32_t)RB);
  ACTKV_CHECK_LAUNCH();
  return ACTKV_OK;
}
// CTAs of a head's line when the SMs take `per_sm` each
inline int64_t pieces_of(int64_t tiles_bound, int Hkv, int per_sm, int min_tiles) {
  return std::max<int64_t>(1, std::min<int64_t>(SMS * per_sm / Hkv, (tiles_bound / Hkv + min_tiles - 1) / min_tiles));
}
// Requests that are short and few: a cluster of CLUSTER CTAs per unit, joined through distributed shared memory, one launch; while all CTAs fit
// on the SMs at once, and up to CLUSTER_TOKENS.  Measured, us with a line per head and with clusters, 4 heads of 128 dims and 8 rows, 1, 3,
// 6 and 12 requests: 500 tokens 7.9 8.4 9.1 11.2, 6.2 6.7 6.6 7.6; 2000 tokens 8.5 12.7 15.0 21.0, 7.7 8.3 10.2 14.2; 4000 tokens
// 10.9 14.5 19.8 27.9, 9.3 10.2 17.3 21.9; 8000 tokens 13.6 19.5 26.7 41.8, 14.3 16.4 29.1 36.6 (and unequal lengths are the line's).
constexpr int CLUSTER = 8, CLUSTER_TOKENS = 4096;
template <int DP, int PER_SM, int WARPS>
int launch_cluster(const Args& a, int64_t units, cudaStream_t s) {
  using C = Cfg<DP, 1, 1, PER_SM, WARPS>;
  auto kernel = attend_kernel<DP, 1, 1, CLUSTER, PER_SM, WARPS>;
  if (ensure_dyn_smem(kernel, C::RING) != cudaSuccess) return ACTKV_E_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)units * CLUSTER);
  cfg.blockDim = dim3(C::NTH);
  cfg.dynamicSmemBytes = C::RING;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = CLUSTER;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, kernel, a);
  ACTKV_CHECK_LAUNCH();
  return ACTKV_OK;
}
template <int DP, int NT, int RG>
int launch(const Args& a, int64_t tiles_bound, int64_t units, cudaStream_t s) {
  using C = Cfg<DP, NT, RG>;
  if constexpr (NT == 1 && RG == 1) {
    if (a.max_tok <= CLUSTER_TOKENS && units * CLUSTER <= SMS * C::CTAS) {
      // one CTA per SM: as many warps as three (head_dim 64: four) small ones would have
      if constexpr (DP <= 128) {
        if (units * CLUSTER <= SMS) return launch_cluster<DP, 1, DP == 64 ? 16 : 12>(a, units, s);
      }
      return launch_cluster<DP, C::CTAS, C::NW>(a, units, s);
    }
  }
  if (ensure_dyn_smem(attend_kernel<DP, NT, RG, 1>, C::RING) != cudaSuccess) return ACTKV_E_CUDA;
  const int64_t pieces = pieces_of(tiles_bound, a.pool.n_kv_heads, C::CTAS, MIN_TILES);
  launch_pdl(attend_kernel<DP, NT, RG, 1>, (unsigned)(pieces * a.pool.n_kv_heads), C::NTH, C::RING, s, a);
  ACTKV_CHECK_LAUNCH();
  return launch_join<DP>(a, pieces, units, C::RB, s);
}
template <int D>
int launch_wide(const Args& a, const actkv_pool_t* pool, int64_t max_tok, int64_t tiles_bound, int64_t units, int RB, cudaStream_t s) {
  CUtensorMap kmap, vmap;
  if (!tcx::make_maps(pool, &kmap, &vmap))
    return RB == 32 ? launch<D, 4, 1>(a, tiles_bound, units, s) : launch<D, 4, 2>(a, tiles_bound, units, s);
  const int64_t bound = units * std::max<int64_t>(1, (max_tok + tcx::TKEYS - 1) / tcx::TKEYS);
  const int64_t pieces = pieces_of(bound, a.pool.n_kv_heads, 1, tcx::MIN_TILES_TC);
  const int rc = RB == 32 ? tcx::launch_tc<D, 32>(a, pool, kmap, vmap, pieces, s) : tcx::launch_tc<D, 64>(a, pool, kmap, vmap, pieces, s);
  return rc != ACTKV_OK ? rc : launch_join<D>(a, pieces, units, RB, s);
}

}  // namespace at
}  // namespace actkv

extern "C" {

size_t actkv_attend_workspace_bytes(const actkv_pool_t* pool, int32_t n_req, int32_t n_layers_sub, int32_t n_q_heads,
                                    int32_t max_win, int32_t max_tok) {
  if (!pool || pool->n_kv_heads <= 0 || pool->head_dim <= 0 || n_req < 0 || n_layers_sub < 0 || n_q_heads <= 0 ||
      max_win < 0 || max_tok < 0)
    return 0;
  // (either kernel: a call on fewer layers, or with a smaller bound, may take the other one)
  size_t most = 0;
  for (bool tc : {false, true})
    most = std::max(most, actkv::at::ws_layout(pool->n_kv_heads, pool->head_dim, n_req, n_layers_sub, n_q_heads / pool->n_kv_heads, max_win, tc).total);
  return most;
}

int actkv_attend(const actkv_pool_t* pool, const actkv_tables_t* tables, int32_t layer_begin, int32_t layer_end, const void* q,
                 const int32_t* win_indptr, int32_t n_q_heads, float sm_scale, int32_t causal, int32_t window_left, void* out,
                 float* lse_out, int32_t sum_win, int32_t max_win, int32_t max_tok, void* ws, size_t ws_bytes, int32_t* status,
                 actkv_stream_t stream) {
  using namespace actkv;
  using namespace actkv::at;
  if (!pool || !tables || !pool->base) return ACTKV_E_INVALID;
  if (layer_begin < 0 || layer_end > pool->n_layers || layer_begin > layer_end) return ACTKV_E_INVALID;
  const int D = pool->head_dim, Hkv = pool->n_kv_heads, R = tables->n_req;
  if (D <= 0 || D % 8 != 0 || D > 256 || Hkv <= 0 || pool->page_size <= 0 || pool->n_pages <= 0) return ACTKV_E_INVALID;
  if (n_q_heads <= 0 || n_q_heads % Hkv != 0) return ACTKV_E_INVALID;
  const int G = n_q_heads / Hkv;
  if (G > MAX_GROUP || R < 0 || sum_win < 0 || max_win < 0 || max_tok < 0 || window_left < 0) return ACTKV_E_INVALID;
  if (((uintptr_t)pool->base & 15) || pool->stride_layer % 8 || pool->stride_kv % 8 || pool->stride_page % 8 ||
      pool->stride_slot % 8 || pool->stride_head % 8 || ((uintptr_t)q & 15) || ((uintptr_t)out & 15))
    return ACTKV_E_INVALID;
  const int nls = layer_end - layer_begin;
  if (R == 0 || nls == 0 || sum_win == 0) return ACTKV_OK;
  if (!q || !win_indptr || !out || max_win == 0 || !tables->seq_len) return ACTKV_E_INVALID;
  if (!tables->page_table || tables->max_pages < 0) return ACTKV_E_INVALID;
  if (q == out) return ACTKV_E_INVALID;
  if (max_tok > (1 << 30) || (int64_t)max_win * G > (1 << 24)) return ACTKV_E_TOOBIG;
  const bool tc = use_tc(D, pool->page_size, (int64_t)max_win * G, (int64_t)R * nls * Hkv * max_tok);
  const WsLayout lay = ws_layout(Hkv, D, R, nls, G, max_win, tc);
  if (!ws || ws_bytes < lay.total) return ACTKV_E_WORKSPACE;
  if (lay.units > 0x7fffffff || (int64_t)R * lay.rb_max * std::max<int64_t>(1, ((int64_t)max_tok + KT - 1) / KT) > 0x7fffffff)
    return ACTKV_E_TOOBIG;
  Args a;
  a.pool = make_view(pool);
  a.tab = make_view(tables);
  a.q = (const __nv_bfloat16*)q;
  a.win_indptr = win_indptr;
  a.out = (__nv_bfloat16*)out;
  a.lse = lse_out;
  a.desc = (int2*)((char*)ws + lay.desc_off);
  a.part_ml = (float2*)((char*)ws + lay.ml_off);
  a.part = (float*)((char*)ws + lay.part_off);
  a.status = status;
  a.layer_begin = layer_begin;
  a.nls = nls;
  a.n_q_heads = n_q_heads;
  a.group = G;
  a.sum_win = sum_win;
  a.max_win = max_win;
  a.max_tok = max_tok;
  a.rb_max = (int32_t)lay.rb_max;
  a.page_shift = (pool->page_size & (pool->page_size - 1)) == 0 ? __builtin_ctz((unsigned)pool->page_size) : -1;
  a.scale_log2 = sm_scale * kLog2e;
  a.causal = causal;
  a.win_left = std::min(window_left, max_tok + max_win);                   // (no row looks back further, and positions minus this stay in 32 bits)
  const int64_t bound = lay.units * std::max<int64_t>(1, ((int64_t)max_tok + KT - 1) / KT);
  cudaStream_t s = (cudaStream_t)stream;
  if (tc)
    return D == 64 ? launch_wide<64>(a, pool, max_tok, bound, lay.units, lay.RB, s) : launch_wide<128>(a, pool, max_tok, bound, lay.units, lay.RB, s);
  if (lay.DP == 256) {
    switch (lay.RB) {
      case 8: return launch<256, 1, 1>(a, bound, lay.units, s);
      case 16: return launch<256, 2, 1>(a, bound, lay.units, s);
      case 32: return launch<256, 2, 2>(a, bound, lay.units, s);
      default: return launch<256, 2, 4>(a, bound, lay.units, s);
    }
  }
  if (lay.DP == 128) {
    switch (lay.RB) {
      case 8: return launch<128, 1, 1>(a, bound, lay.units, s);
      case 16: return launch<128, 2, 1>(a, bound, lay.units, s);
      case 32: return launch<128, 4, 1>(a, bound, lay.units, s);
      case 64: return launch<128, 4, 2>(a, bound, lay.units, s);
      default: return launch<128, 4, 4>(a, bound, lay.units, s);
    }
  }
  switch (lay.RB) {
    case 8: return launch<64, 1, 1>(a, bound, lay.units, s);
    case 16: return launch<64, 2, 1>(a, bound, lay.units, s);
    case 32: return launch<64, 4, 1>(a, bound, lay.units, s);
    case 64: return launch<64, 4, 2>(a, bound, lay.units, s);
    default: return launch<64, 4, 4>(a, bound, lay.units, s);
  }
}

}  // extern "C"
