// Shared structures and the K-tile producers of the tcgen05 / TMEM / TMA score kernels (sm_100a).
#pragma once

#include "compact_job.cuh"
#include "ring.cuh"
#include "score_mma.cuh"
#include "tc_ptx.cuh"

namespace actkv {
namespace tc {

constexpr int TK = 128;                      // keys per tile
constexpr int HD = 128;                      // head dim
constexpr uint32_t HALF_BYTES = TK * 64 * 2;         // 16 KB
constexpr uint32_t QBLK_BYTES = 128 * HD * 2;        // 32 KB per 128 rows
constexpr size_t SMEM_LIMIT = 232448;        // 227 KB of dynamic shared memory per CTA
constexpr int MAX_ROWS = 512;                // window x group rows (padded to 128) a CTA of the pooled-score pass handles
constexpr int MAX_ROWS_TOTAL = 4096;         // ... per unit: that pass takes more than MAX_ROWS in groups of MAX_ROWS

constexpr int32_t STALL_ANSWER = ACTKV_STALL_ANSWER;       // TcArgs::stall_tile: see actkv_debug_inject_stall

struct Exp2Cubic { float c0, c1, c2, c3; };   // 2^f on [-0.5, 0.5] = c0 + f (c1 + f (c2 + f c3))

struct TcArgs {
  ScoreArgs a;
  int32_t tiles_per_cta;     // pooled-score pass: key tiles per CTA
  int32_t n_kchunks;         // pooled-score pass: CTAs per unit
  int32_t n_rg;              // LSE pass: groups of rows per unit (a grid dimension)
  int32_t row_begin;         // pooled-score pass: first row of this launch's row group (multiple of MAX_ROWS)
  int32_t n_stages;          // K stages in shared memory (at most 8)
  int32_t k5;                // K tensor map has five dimensions (pages that are not slot-major), else four
  CompactWs* copy_ws;        // pending compaction of another layer group whose copies this launch's spare warps
                             // take on (nullptr: none)
  int32_t stall_tile;        // fault-injection hook: the K-tile producers issue no tile from this one on (< 0: off)
  long long wait_cycles;     // limit of every bounded wait, in SM cycles
};

__device__ __forceinline__ int32_t page_for_tile(const TablesView& tab, int32_t n_pages, int r, int lp, int n_lp,
                                                 int32_t* status) {
  // logical pages past the end of the request re-read its last page (their keys are masked later)
  lp = min(lp, n_lp - 1);
  return checked_page(tab, n_pages, r, lp, status);
}

// The K-tile producers of both score kernels: producer p of P takes tiles p, p + P, ... of
// [t_begin, t_begin + n_tiles) of request r, head h, layer `layer` through the block table into the ring of S
// stages (tile i is entry e0 + i of the ring), one TMA box per (page, 64-dim half), one box per lane.  False when a wait gave up or the
// injected fault stopped it.  Pages of 16, 32, 64 or 128 tokens: a
// tile of 128 keys is ppt = 128 / page_size pages, a box page_size rows of 128 B.
// Measured on B200 (boxes of 16 rows x 128 B from random pages): one warp issuing a tile's 16 boxes from
// 8 lanes delivers a tile per 1950 cycles, from 16 lanes per 1570, two warps per 1235, four per 1180 (the
// memory system's rate).  Only the streaming update is bound by this.
// Page ids of four of the producer's tiles at a time, one per lane (lane / ppt = tile within the group,
// lane % ppt = page); the next group's ids are loaded while the current four tiles are being issued.
// K5: five-dimensional tensor map (pages that are not slot-major).
template <bool K5, int NH, class Bars>
__device__ __forceinline__ bool k_tile_producer(const CUtensorMap* kmap, const ScoreArgs& a, Bars* bars, uint32_t k_smem,
                                                int S, int r, int h, int layer, int L, int t_begin, int n_tiles,
                                                int lane, volatile int* abort_flag, int p, int P, long long wait_cycles,
                                                int stall_tile, int e0 = 0) {
  const int ps = a.pool.page_size;
  const int ppt = TK / ps;                                      // pages per tile: 8, 4, 2 or 1
  const int lp_shift = 31 - __clz(ppt);                         // log2(ppt)
  const uint32_t box_bytes = (uint32_t)ps * 128u;
  const int n_lp = (L + ps - 1) / ps;
  const int n_mine = (n_tiles - p + P - 1) / P;                  // tiles p, p + P, ... below n_tiles
  if (n_mine <= 0) return true;
  const int g_tile = lane >> lp_shift, g_page = lane & (ppt - 1);            // this lane's slot in a group of four tiles
  int32_t pid = page_for_tile(a.tab, a.pool.n_pages, r, (t_begin + p + min(g_tile, 3) * P) * ppt + g_page, n_lp, a.status);
  int32_t pid_next = 0;
  for (int i = 0; i < n_mine; ++i) {
    const int it = p + i * P;
    if (stall_tile >= 0 && it >= stall_tile) return false;       // injected fault: this and all later tiles never arrive
    const int s = ring_stage(e0 + it, S);
    const uint32_t ph = ring_parity(e0 + it, S);
    if ((i & 3) == 0 && i + 4 < n_mine)
      pid_next = page_for_tile(a.tab, a.pool.n_pages, r, (t_begin + p + (i + 4 + min(g_tile, 3)) * P) * ppt + g_page, n_lp,
                               a.status);
    int ok = 1;
    if (lane == 0) {
      ok = mbar_wait(smem_u32(&bars->k_empty[s]), ph ^ 1u, abort_flag, wait_cycles) ? 1 : 0;
      if (ok) { bars->k_last[s] = ph; mbar_expect_tx(smem_u32(&bars->k_full[s]), NH * HALF_BYTES); }
    }
    ok = __shfl_sync(0xffffffffu, ok, 0);
    if (!ok) return false;
    // lane j < ppt NH: page j % ppt, half j / ppt of this tile
    const int32_t my_pid = __shfl_sync(0xffffffffu, pid, ((i & 3) << lp_shift) | (lane & (ppt - 1)));
    if (lane < ppt * NH) {
      const int half = lane >> lp_shift;
      const uint32_t dst = k_smem + s * (NH * HALF_BYTES) + half * HALF_BYTES + (lane & (ppt - 1)) * box_bytes;
      const uint32_t bar = smem_u32(&bars->k_full[s]);
      if constexpr (K5) tma_load_5d(dst, kmap, bar, half * 64, 0, h, my_pid, layer);
      else tma_load_4d(dst, kmap, bar, half * 64, h, my_pid * ps, layer);
    }
    if ((i & 3) == 3) pid = pid_next;
  }
  return true;
}

// Tear-down after a give-up: the key tiles (and Q blocks) still in flight land in this CTA's shared memory; one thread waits for them, with
// a limit.  (In this form, with the parities recorded as the loads are issued: with the last load of each stage worked out here the
// pooled-score kernel was 2 % slower, 24 layers of 4 requests, head_dim 64: 471 -> 482 us, though nothing ever runs it.)
template <class Bars>
__device__ __forceinline__ void drain_loads(Bars* bars, int S) {
  for (int s = 0; s < S; ++s) mbar_wait(smem_u32(&bars->k_full[s]), bars->k_last[s], nullptr, DRAIN_LIMIT_CYCLES / 64);
}

}  // namespace tc
}  // namespace actkv
