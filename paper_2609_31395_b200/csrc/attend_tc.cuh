// actkv_attend on the tensor cores of the fifth generation (tcgen05): 9 and more rows per request and KV head (drafted tokens, chunks,
// large groups), head_dim 64 or 128, and work enough (use_tc in attend.cu).
//
// Why a second kernel.  Of every key the warp-level kernel loads fragments for each 8 rows and carries every instruction of the softmax
// in the warps that feed the matrix pipe: 32 rows took 1.8 times, 64 rows 3.0 times what 8 rows take (16 requests of 16000 tokens, 4 heads of
// 128 dims: 89 us with 8 rows; 32: 153, 64: 248).  Here a tile of 128 keys is one operand:
//   S[key, row] = K Q^T       M = 128 keys, N = NR rows, both operands K-major in shared memory, S in tensor memory;
//   P = exp2(S - reference)   a thread per key; bf16 summands (p truncated, and the rest) of all rows into shared memory;
//   O^T[dim, row] += V^T P    M = head_dim, N = 2 NR: the two summands side by side, so that V is read once; both operands lie with the
//                             long side contiguous (V as the pool has it: [key][dim], P as its thread writes it: [key][row]).
// Two warpgroups take the tiles in turn, each with references, sums and an O of its own, joined at the end of a stretch (one warpgroup for all
// tiles, 64 rows: 160 us at 128 dims, where its 3100 cycles a tile were the longest chain).  Sums of P are kept per thread and row in
// registers.  The references live in shared memory and move (then O is rescaled) only when a logit exceeds one by more than 8: in
// the first tile, hardly ever after.
//
// Roles of a CTA (one per SM): warps 0-7 softmax and epilogue, warp 8 issues the products for S, warp 9
// those for O, warps 12-15 load.  K and V have a ring each, S and P two buffers, one for each warpgroup; S runs ahead of the softmax by up
// to two tiles.  All waits are bounded; one that gives up raises a flag that ends every role (ACTKV_E_TIMEOUT).
//
// What bounds it: reading K and V up to 32 rows (128 dims: 101 us where 8 rows in the other kernel take 89); beyond, the softmax: a warpgroup
// takes 4250 cycles for a tile of 64 columns, 2100 with two of them, against 1425 (64 dims) that the tile's bytes take to arrive.  8192
// exponentials are 512 of those cycles; the columns behind the last row of a block are computed all the same (a block of 33 rows costs
// as much as one of 64), and the 64-row variants spill (412 to 420 bytes stored, 244 to 248 loaded per thread; 32 rows: none).
#pragma once

#include "attend_line.cuh"
#include "pool_map.cuh"
#include "ring.cuh"
#include "stall_hook.cuh"

namespace actkv {
namespace at {
namespace tcx {

using namespace actkv::tc;

constexpr int TKEYS = 128;
// (warps 10 and 11 only fill up the third warpgroup, as registers are handed round by warpgroups)
constexpr int SOFT = 128, S_WARP = 8, O_WARP = 9, LOAD_WARP = 12, THREADS = 512;
constexpr int SOFT_REGS = 184, REST_REGS = 72;                 // 128 each at launch: 256 * 184 + 256 * 72 = 512 * 128
constexpr int MIN_TILES_TC = 1;

template <int D, int NR>
struct Tc {
  static constexpr int UNIT = TKEYS * D * 2;                   // bytes of a K or V tile: halves of 64 dims, rows of 128 bytes
  static constexpr int PBUF = TKEYS * 2 * NR * 2;              // bytes of a P buffer: [key] rows of 128 bytes; 64 rows: summands apart
  static constexpr int QBYTES = NR * D * 2;
  static constexpr int STAGES = 64 * 1024 / UNIT;              // of the K ring, and of the V ring: 2 or 4
  static constexpr int TM_COLS = 8 * NR;                       // S, two buffers; O, one per softmax warpgroup, twice as wide (6 NR in all)
  static constexpr int V_OFF = STAGES * UNIT, P_OFF = 2 * V_OFF, Q_OFF = P_OFF + 2 * PBUF, CTL_OFF = Q_OFF + QBYTES;
};

template <int D, int NR>
struct Ctl {
  uint64_t full[2][4], empty[2][4];        // K ring, V ring
  uint64_t s_full[2], s_empty[2], p_full[2], p_empty[2];
  uint64_t q_full, o_full, o_empty, drained;
  uint32_t tmem;
  int abort;
  int stop[2][2];
  unsigned last[2][4];                     // parity of the last load into each entry
  int poisoned;
  alignas(16) float ref[2][NR];            // per softmax warpgroup (read as vectors)
  float fac[2][NR];
  float col[2][4][NR];                     // maxima or sums of the columns, per warp
  int pos[NR];
  int64_t at[NR];                          // output row
  uint32_t poison[2][NR][D / 32];          // (row, dim) that met +infinity / -infinity in a tile not every row sees whole (NaN: both)
};
template <int D, int NR>
constexpr size_t smem_bytes() { return Tc<D, NR>::CTL_OFF + sizeof(Ctl<D, NR>) + 1024; }       // (the ring begins on 1024 bytes)

// barriers 1 and 2: one softmax warpgroup; 3: both
__device__ __forceinline__ void soft_sync(int wg) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(1 + wg) : "memory"); }
__device__ __forceinline__ void both_sync() { asm volatile("barrier.cta.sync 3, 256;" ::: "memory"); }
__device__ __forceinline__ bool soft_any(int wg, bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r) : "r"(v ? 1u : 0u), "r"(1 + wg) : "memory");
  return r != 0;
}
// Sums (or maxima) over the 32 lanes of N values each, by halves: a lane ends up with N / 32 columns, the first of which is returned.
template <int N, bool MAX>
__device__ __forceinline__ int across(float* v, int lane) {
  int first = 0;
#pragma unroll
  for (int d = 16, n = N / 2; d >= 1; d >>= 1, n >>= 1) {
    const bool up = lane & d;
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
      if (k >= n) break;
      const float mine = up ? v[n + k] : v[k], other = __shfl_xor_sync(0xffffffffu, up ? v[k] : v[n + k], d);
      v[k] = MAX ? fmaxf(mine, other) : mine + other;
    }
    first += up ? n : 0;
  }
  return first;
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float* v) {
  const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Operand with the long side (M or N) contiguous, 128-byte swizzle: rows of 64 bf16, one per k; eight rows of k are 1024 bytes,
// the next 64 of the long side `lead` bytes away.
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr, uint32_t lead) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)2 << 61);
}
template <int D, int NR>
__global__ void __launch_bounds__(THREADS, 1) attend_tc_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap kmap,
                                                               const __grid_constant__ CUtensorMap vmap, const int k5,
                                                               const long long limit, const int stall) {
  using T = Tc<D, NR>;
  using CT = Ctl<D, NR>;
  pdl_begin();
  extern __shared__ uint8_t tcx_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(tcx_raw) + 1023) & ~(uintptr_t)1023);
  CT* ctl = reinterpret_cast<CT*>(base + T::CTL_OFF);
  const uint32_t sbase = smem_u32(base);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = a.group;
  volatile int* abort_flag = &ctl->abort;

  if (tid == 0) {
    for (int kv = 0; kv < 2; ++kv)
      for (int i = 0; i < T::STAGES; ++i) {
        mbar_init(smem_u32(&ctl->full[kv][i]), 1);
        mbar_init(smem_u32(&ctl->empty[kv][i]), 1);
        ctl->last[kv][i] = RING_UNUSED;
      }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&ctl->s_full[i]), 1);
      mbar_init(smem_u32(&ctl->s_empty[i]), SOFT);
      mbar_init(smem_u32(&ctl->p_full[i]), SOFT);
      mbar_init(smem_u32(&ctl->p_empty[i]), 1);
      ctl->stop[i][0] = ctl->stop[i][1] = 0;
    }
    mbar_init(smem_u32(&ctl->q_full), 2 * SOFT);
    mbar_init(smem_u32(&ctl->o_full), 1);
    mbar_init(smem_u32(&ctl->o_empty), 2 * SOFT);
    mbar_init(smem_u32(&ctl->drained), 2);
    ctl->abort = 0;
    ctl->poisoned = 0;
    fence_barrier_init();
  }
  for (int i = tid; i < 2 * NR * (D / 32); i += THREADS) (&ctl->poison[0][0][0])[i] = 0;
  if (warp == S_WARP) {
    tmem_alloc(smem_u32(&ctl->tmem), T::TM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem, tm_o = tmem + 2 * NR;
  Line<TKEYS, NR, MIN_TILES_TC> line(a, blockIdx.x == 0 && warp == 0);
  Seg sg;

  if (warp < S_WARP) {
    reg_inc<SOFT_REGS>();
    // ================================ softmax: two warpgroups take the tiles in turn; thread = key of the tile ================================
    const int wg = warp >> 2, kt = tid & 127;
    uint32_t t0 = 0, seg = 0;                                  // tiles, stretches before this stretch
    bool dead = false;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16, to = tm_o + wg * 2 * NR + lane_off;
    float* ref = ctl->ref[wg];
    float* fac = ctl->fac[wg];
    while (line.next(sg)) {
      const Req& q = sg.q;
      const int L = q.L, rows = q.W * G, row0 = sg.rb * NR, n_rows = min(NR, rows - row0);
      const int pos0 = a.causal ? L - q.W : L - 1, step = a.causal ? 1 : 0;
      const int all_hi = pos0 + step * (row0 / G);
      const int all_lo = a.win_left > 0 ? pos0 + step * ((row0 + n_rows - 1) / G) - a.win_left + 1 : 0;
      const int64_t qrow = (int64_t)sg.layer * a.sum_win + q.win0;
      // Q of the stretch (every product of the one before is complete: o_full has been waited for)
#pragma unroll
      for (int i = tid; i < NR * (D / 8); i += 2 * SOFT) {
        const int row = i / (D / 8), c = i % (D / 8), rho = row0 + row, w = rho / G;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < n_rows)
          v = *reinterpret_cast<const uint4*>(a.q + ((qrow + w) * a.n_q_heads + line.h * G + (rho - w * G)) * D + c * 8);
        *reinterpret_cast<uint4*>(base + T::Q_OFF + (c >> 3) * (NR * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = v;
      }
      if (kt < NR) {
        ref[kt] = NO_REF;
        if (wg == 0) {
          const int rho = row0 + min(kt, n_rows - 1), w = rho / G;
          ctl->pos[kt] = pos0 + step * w;
          ctl->at[kt] = (qrow + w) * a.n_q_heads + line.h * G + (rho - w * G);
        }
      }
      fence_proxy_async();
      mbar_arrive(smem_u32(&ctl->q_full));
      both_sync();
      float l[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n) l[n] = 0.f;

      const int i_first = (int)((wg - t0) & 1);
      for (int i = i_first; i < sg.n_tiles; i += 2) {
        const uint32_t t = t0 + i;
        const int b = wg;                                      // (= t & 1)
        const uint32_t use = t >> 1;
        if (!mbar_wait_warp(smem_u32(&ctl->s_full[b]), use & 1, abort_flag, limit)) dead = true;
        tc_fence_after();
        const uint32_t ts = tmem + b * NR + lane_off;
        const int key = (q.lo_tile + sg.t_in + i) * TKEYS + kt;
        const bool masked = key - kt + TKEYS - 1 > all_hi || key - kt < all_lo;
        float x[NR];
        auto load = [&]() {
#pragma unroll
          for (int c = 0; c < NR; c += 32) tmem_ld32(ts + c, x + c);
          tmem_ld_wait();
#pragma unroll
          for (int n = 0; n < NR; ++n) x[n] *= a.scale_log2;
          if (masked) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              const int pos = ctl->pos[n];
              if (key > pos || (a.win_left > 0 && key <= pos - a.win_left)) x[n] = -INFINITY;
            }
          }
        };
        load();
        float over = -INFINITY;
#pragma unroll
        for (int n = 0; n < NR; n += 4) {
          const float4 r = *reinterpret_cast<const float4*>(&ref[n]);
          x[n] -= r.x;
          x[n + 1] -= r.y;
          x[n + 2] -= r.z;
          x[n + 3] -= r.w;
          over = fmaxf(over, fmaxf(fmaxf(x[n], x[n + 1]), fmaxf(x[n + 2], x[n + 3])));
        }
        if (dead) ctl->stop[wg][use & 1] = 1;
        const bool move = soft_any(wg, over > REF_SLACK);
        if (*reinterpret_cast<volatile int*>(&ctl->stop[wg][use & 1])) break;      // (the same answer for all four warps)
        if (move) {
          // new references: the columns' maxima over the tile
          load();
          {
            const int first = across<NR, true>(x, lane);
#pragma unroll
            for (int n = 0; n < NR / 32; ++n) ctl->col[wg][warp & 3][first + n] = x[n];
          }
          soft_sync(wg);
          if (kt < NR) {
            const float old = ref[kt];
            const float top = fmaxf(fmaxf(fmaxf(ctl->col[wg][0][kt], ctl->col[wg][1][kt]), fmaxf(ctl->col[wg][2][kt], ctl->col[wg][3][kt])), old);
            ref[kt] = top;
            fac[kt] = exp2f(old - top);
          }
          soft_sync(wg);
#pragma unroll
          for (int n = 0; n < NR; ++n) l[n] *= fac[n];
          if (i >= 2) {
            // O so far, when the product of this warpgroup's last tile is complete (this tile's waits for P)
            if (!mbar_wait_warp(smem_u32(&ctl->p_empty[b]), (use & 1) ^ 1, abort_flag, limit)) dead = true;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 2 * NR; c += 32) {
              float o[32];
              tmem_ld32(to + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int n = 0; n < 32; ++n) o[n] *= fac[(c + n) % NR];
              tmem_st32(to + c, o);
            }
            tmem_st_wait();
          }
          load();
#pragma unroll
          for (int n = 0; n < NR; ++n) x[n] -= ref[n];
        }
        tc_fence_before();
        mbar_arrive(smem_u32(&ctl->s_empty[b]));
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          x[n] = exp2f(x[n]);
          l[n] += x[n];
        }
        if (masked) {
          // V of a key that some row must not see, or of a slot behind the end: infinities and NaN leave the product; what they make of the
          // rows that do see the key, whatever its probability there, is noted
          const uint32_t sl = t % T::STAGES;
          // (unguarded by the others: a wait of this thread alone; the entry stays until this tile's product)
          if (!mbar_wait(smem_u32(&ctl->full[1][sl]), (t / T::STAGES) & 1, abort_flag, limit)) dead = true;
          for (int c = 0; c < D / 8; ++c) {
            uint8_t* at = base + T::V_OFF + sl * T::UNIT + (c >> 3) * 16384 + kt * 128 + (((c & 7) ^ (kt & 7)) << 4);
            const uint4 v = *reinterpret_cast<const uint4*>(at);
            bool odd = false;
            for (uint32_t u : {v.x, v.y, v.z, v.w}) odd |= (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u;
            if (!odd) continue;
            for (int k = 0; k < 8; ++k) {
              uint16_t* el = reinterpret_cast<uint16_t*>(at) + k;
              const uint32_t bits = *el;
              if ((bits & 0x7f80u) != 0x7f80u) continue;
              *el = 0;
              const bool nan = (bits & 0x7fu) != 0, neg = (bits & 0x8000u) != 0;
              const int d = c * 8 + k;
#pragma unroll 1
              for (int n = 0; n < NR; ++n) {
                const int pos = ctl->pos[n];
                if (key > pos || (a.win_left > 0 && key <= pos - a.win_left)) continue;
                if (nan || !neg) atomicOr(&ctl->poison[0][n][d >> 5], 1u << (d & 31));
                if (nan || neg) atomicOr(&ctl->poison[1][n][d >> 5], 1u << (d & 31));
                ctl->poisoned = 1;
              }
            }
          }
        }
        if (!mbar_wait_warp(smem_u32(&ctl->p_empty[b]), (use & 1) ^ 1, abort_flag, limit)) dead = true;
        uint8_t* pr = base + T::P_OFF + b * T::PBUF + kt * 128;
#pragma unroll
        for (int c = 0; c < NR / 8; ++c) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float p0 = x[c * 8 + 2 * k], p1 = x[c * 8 + 2 * k + 1];
            const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
            const float r0 = p0 - __uint_as_float(u0 & 0xffff0000u), r1 = p1 - __uint_as_float(u1 & 0xffff0000u);
            hi[k] = __byte_perm(u0, u1, 0x7632);
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(lo[k]) : "f"(r1), "f"(r0));
          }
          // rows of 128 bytes: 64 rows: one summand each, 16 KB apart; 32 rows: both
          uint8_t* ph = pr + ((c ^ (kt & 7)) << 4);
          uint8_t* pl = NR == 64 ? ph + 16384 : pr + (((c + 4) ^ (kt & 7)) << 4);
          *reinterpret_cast<uint4*>(ph) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(pl) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        fence_proxy_async();
        mbar_arrive(smem_u32(&ctl->p_full[b]));
      }
      // ---- the stretch's rows: the two warpgroups' shares together, each puts out half of the rows ----
      {
        const int first = across<NR, false>(l, lane);
#pragma unroll
        for (int n = 0; n < NR / 32; ++n) ctl->col[wg][warp & 3][first + n] = l[n];
      }
      if (!mbar_wait_warp(smem_u32(&ctl->o_full), seg & 1, abort_flag, limit)) dead = true;
      tc_fence_after();
      both_sync();
      const bool whole = sg.b0 == sg.b1;
      const int64_t slot = line.slot(sg);
      const bool mine_too = i_first < sg.n_tiles;              // (a stretch of one tile: one warpgroup has none)
      const bool theirs_too = (i_first ^ 1) < sg.n_tiles;
      if (sg.t_in == 0 && tid == 0) a.desc[line.unit(sg)] = make_int2(sg.b0, sg.b1);
      if (kt < NR) {
        float M[2], sum[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          M[g] = ctl->ref[g][kt];
          sum[g] = ctl->col[g][0][kt] + ctl->col[g][1][kt] + ctl->col[g][2][kt] + ctl->col[g][3][kt];
        }
        const float top = fmaxf(M[0], M[1]), f0 = exp2f(M[0] - top), f1 = exp2f(M[1] - top), all = sum[0] * f0 + sum[1] * f1;
        fac[kt] = (wg == 0 ? f0 : f1) * (!whole ? 1.f : all == 0.f ? 0.f : 1.f / all);
        if (wg == 0 && kt < n_rows) {
          if (!whole) a.part_ml[slot * NR + kt] = make_float2(top, all);
          else if (a.lse != nullptr) a.lse[ctl->at[kt]] = all == 0.f ? -INFINITY : (top + log2f(all)) * kLn2;
        }
      }
      both_sync();
      {
        // M = 128: dim = lane of tensor memory; M = 64: 16 dims in the first 16 lanes of every warp
        const int d = D == 128 ? kt : (warp & 3) * 16 + lane;
        const bool mine = D == 128 || lane < 16;
        const bool poisoned = ctl->poisoned != 0;
        float* swap = reinterpret_cast<float*>(base + T::P_OFF);               // [row][dim] (P is no longer needed)
        static_assert(NR * D * 4 <= 2 * T::PBUF, "O of all rows fits where P was");
        auto half = [&](int h, float* o) {                                     // this warpgroup's O of rows h * NR / 2 ..
          float o2[NR / 2];
          if constexpr (NR == 64) {
            tmem_ld32(to + h * 32, o);
            tmem_ld32(to + NR + h * 32, o2);
          } else {
            tmem_ld16(to + h * 16, o);
            tmem_ld16(to + NR + h * 16, o2);
          }
          tmem_ld_wait();
#pragma unroll
          for (int n = 0; n < NR / 2; ++n) o[n] = (o[n] + o2[n]) * fac[h * (NR / 2) + n];
        };
        float o[NR / 2];
        if (mine_too) {
          half(wg ^ 1, o);
          if (mine) {
#pragma unroll
            for (int n = 0; n < NR / 2; ++n) swap[((wg ^ 1) * (NR / 2) + n) * D + d] = o[n];
          }
          half(wg, o);
        }
        tc_fence_before();
        mbar_arrive(smem_u32(&ctl->o_empty));
        both_sync();
        if (mine) {
#pragma unroll
          for (int n = 0; n < NR / 2; ++n) {
            const int row = wg * (NR / 2) + n;
            if (row >= n_rows) continue;
            float v = (mine_too ? o[n] : 0.f) + (theirs_too ? swap[row * D + d] : 0.f);
            if (poisoned) {
              const uint32_t up = ctl->poison[0][row][d >> 5] >> (d & 31) & 1u, down = ctl->poison[1][row][d >> 5] >> (d & 31) & 1u;
              if (up) v += INFINITY;
              if (down) v += -INFINITY;
            }
            if (whole) a.out[ctl->at[row] * D + d] = __float2bfloat16_rn(v);
            else a.part[(slot * NR + row) * D + d] = v;
          }
        }
        both_sync();                                           // references, poison and P's place are rewritten
        if (poisoned) {
          for (int i = tid; i < 2 * NR * (D / 32); i += 2 * SOFT) (&ctl->poison[0][0][0])[i] = 0;
          if (tid == 0) ctl->poisoned = 0;
          both_sync();
        }
      }
      t0 += (uint32_t)sg.n_tiles;
      ++seg;
    }
  } else if (warp < LOAD_WARP) {
    reg_dec<REST_REGS>();
    if (warp > O_WARP) goto out;
    // ================================ MMA issuers: one for S, which runs ahead as its buffers allow, one for O ================================
    constexpr uint32_t IDESC_S = idesc_bf16(128, NR), IDESC_O = idesc_bf16(D, 2 * NR) | (1u << 15) | (1u << 16);
    const uint64_t qd = smem_desc_sw128(sbase + T::Q_OFF);
    const bool for_s = warp == S_WARP;
    uint32_t t = 0, seg = 0;
    bool ok = true;
    while (ok && line.next(sg)) {
      const int n = sg.n_tiles;
      if (for_s) ok = mbar_wait_warp(smem_u32(&ctl->q_full), seg & 1, abort_flag, limit);
      else ok = mbar_wait_warp(smem_u32(&ctl->o_empty), (seg & 1) ^ 1, abort_flag, limit);
      for (int i = 0; ok && i < n; ++i, ++t) {
        const uint32_t b = t & 1, use = t >> 1, sl = t % T::STAGES, ph = (t / T::STAGES) & 1;
        if (for_s) {
          ok = mbar_wait_warp(smem_u32(&ctl->full[0][sl]), ph, abort_flag, limit) &&
               mbar_wait_warp(smem_u32(&ctl->s_empty[b]), (use & 1) ^ 1, abort_flag, limit);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t kd = smem_desc_sw128(sbase + sl * T::UNIT);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              umma_bf16(tmem + b * NR, kd + (uint64_t)(((k >> 2) * 16384 + (k & 3) * 32) >> 4),
                        qd + (uint64_t)(((k >> 2) * (NR * 128) + (k & 3) * 32) >> 4), IDESC_S, k > 0 ? 1u : 0u);
            umma_commit(smem_u32(&ctl->s_full[b]));
            umma_commit(smem_u32(&ctl->empty[0][sl]));
          }
        } else {
          ok = mbar_wait_warp(smem_u32(&ctl->full[1][sl]), ph, abort_flag, limit) &&
               mbar_wait_warp(smem_u32(&ctl->p_full[b]), use & 1, abort_flag, limit);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t vd = smem_desc_mn(sbase + T::V_OFF + sl * T::UNIT, 16384), pd = smem_desc_mn(sbase + T::P_OFF + b * T::PBUF, 16384);
#pragma unroll
            for (int k = 0; k < TKEYS / 16; ++k)
              umma_bf16(tm_o + b * 2 * NR, vd + (uint64_t)((k * 2048) >> 4), pd + (uint64_t)((k * 2048) >> 4), IDESC_O,
                        (i > 1 || k > 0) ? 1u : 0u);           // (the first two tiles begin a warpgroup's O each)
            umma_commit(smem_u32(&ctl->p_empty[b]));
            umma_commit(smem_u32(&ctl->empty[1][sl]));
            if (i == n - 1) umma_commit(smem_u32(&ctl->o_full));
          }
        }
        __syncwarp();
      }
      ++seg;
    }
    // everything issued has retired before tensor memory is freed
    if (elect_one()) umma_commit(smem_u32(&ctl->drained));
    __syncwarp();
    if (for_s) mbar_wait_warp(smem_u32(&ctl->drained), 0, nullptr, DRAIN_LIMIT_CYCLES);
  } else {
    reg_dec<REST_REGS>();
    // ================================ loaders: two warps for K, two for V, on tiles in turn ================================
    const int kv = (warp - LOAD_WARP) >> 1, ps = a.pool.page_size, ppt = TKEYS / ps, lp_shift = 31 - __clz(ppt);
    constexpr int NH = D / 64;
    const CUtensorMap* map = kv ? &vmap : &kmap;
    uint32_t t0 = 0;
    bool ok = true;
    while (ok && line.next(sg)) {
      const int L = sg.q.L, n = sg.n_tiles, n_lp = (L + ps - 1) / ps;
      for (int i = (int)((warp - t0) & 1); i < n; i += 2) {
        const uint32_t t = t0 + i, sl = t % T::STAGES, ph = (t / T::STAGES) & 1;
        if (stall >= 0 && i >= stall) { ok = false; break; }   // injected fault: this and all later tiles never arrive
        // lane j < ppt NH: page j % ppt, half j / ppt.  Pages past the end: the last one again (their keys are masked)
        int pid = 0;
        if (lane < ppt && n_lp > 0)
          pid = checked_page(a.tab, a.pool.n_pages, sg.r, min((sg.q.lo_tile + sg.t_in + i) * ppt + lane, n_lp - 1), a.status);
        int got = 1;
        if (lane == 0) {
          got = mbar_wait(smem_u32(&ctl->empty[kv][sl]), ph ^ 1, abort_flag, limit) ? 1 : 0;
          if (got) {
            ctl->last[kv][sl] = ph;
            if (n_lp > 0) mbar_expect_tx(smem_u32(&ctl->full[kv][sl]), T::UNIT);
            else mbar_arrive(smem_u32(&ctl->full[kv][sl]));    // an empty request: every key is masked
          }
        }
        ok = __shfl_sync(0xffffffffu, got, 0) != 0;
        if (!ok) break;
        pid = __shfl_sync(0xffffffffu, pid, lane & (ppt - 1));
        if (lane < ppt * NH && n_lp > 0) {
          const int half = lane >> lp_shift;
          const uint32_t dst = sbase + kv * T::V_OFF + sl * T::UNIT + half * 16384 + (lane & (ppt - 1)) * ps * 128;
          const uint32_t bar = smem_u32(&ctl->full[kv][sl]);
          if (k5) tma_load_5d(dst, map, bar, half * 64, 0, line.h, pid, a.layer_begin + sg.layer);
          else tma_load_4d(dst, map, bar, half * 64, line.h, pid * ps, a.layer_begin + sg.layer);
        }
      }
      t0 += (uint32_t)n;
    }
  }
out:
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (*abort_flag && tid == 0) {
    report(a.status, ACTKV_E_TIMEOUT, (int)blockIdx.x, line.h);
    // loads still in flight land in this CTA's shared memory: waited for, with a limit
    for (int i = 0; i < 2 * T::STAGES; ++i)
      mbar_wait(smem_u32(&ctl->full[i & 1][i >> 1]), ctl->last[i & 1][i >> 1], nullptr, DRAIN_LIMIT_CYCLES / 64);
  }
  if (warp == S_WARP) tmem_dealloc(tmem, T::TM_COLS);
}

// False when the pool has no tensor map (the caller then takes the warp-level kernel).
inline bool make_maps(const actkv_pool_t* pool, CUtensorMap* kmap, CUtensorMap* vmap) {
  return make_kvmap(pool, 0, kmap) && make_kvmap(pool, 1, vmap);
}
template <int D, int NR>
int launch_tc(const Args& a, const actkv_pool_t* pool, const CUtensorMap& kmap, const CUtensorMap& vmap, int64_t pieces, cudaStream_t s) {
  if (ensure_dyn_smem(attend_tc_kernel<D, NR>, smem_bytes<D, NR>()) != cudaSuccess) return ACTKV_E_CUDA;
  launch_pdl(attend_tc_kernel<D, NR>, (unsigned)(pieces * a.pool.n_kv_heads), THREADS, smem_bytes<D, NR>(), s, a, kmap, vmap,
             pool_needs_5d(pool) ? 1 : 0, stall_hook().wait_cycles.load(), (int)stall_hook().stall_tile.load());
  ACTKV_CHECK_LAUNCH();
  return ACTKV_OK;
}

}  // namespace tcx
}  // namespace at
}  // namespace actkv
