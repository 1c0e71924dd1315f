// What the attention kernels share: arguments, requests, a CTA's way along the work, partials.
#pragma once

#include "common.cuh"

namespace actkv {
namespace at {

constexpr int SMS = 148, MAX_CTAS = 4 * SMS;
constexpr float NO_REF = -3.0e38f;        // the reference before the first logit (finite: no infinity meets another)
constexpr float REF_SLACK = 8.f;
constexpr int MAX_GROUP = 32;             // query heads per KV head, as the score kernels

struct Args {
  PoolView pool;
  TablesView tab;
  const __nv_bfloat16* q;
  const int32_t* win_indptr;
  __nv_bfloat16* out;
  float* lse;
  int2* desc;                    // [units] first and last piece of a unit
  float2* part_ml;               // [2 * MAX_CTAS][rows of a block] (m, l)
  float* part;                   // [2 * MAX_CTAS][rows of a block][DP]
  int32_t* status;
  int32_t layer_begin, nls, n_q_heads, group;
  int32_t sum_win, max_win, max_tok;
  int32_t rb_max;                // blocks of rows per request, at most
  int32_t page_shift;
  float scale_log2;
  int32_t causal, win_left;
};

struct Req {
  int L, W, win0;                // W = 0: nothing to do
  int lo_tile, tiles;            // key tiles that some row sees (one at least, so that every row is written)
};
template <int KT>                  // keys per tile
__device__ __forceinline__ Req load_req(const Args& a, int r, bool tell) {
  const int w0 = a.win_indptr[r], w1 = a.win_indptr[r + 1], L = a.tab.seq_len[r];
  Req q{L, w1 - w0, w0, 0, 0};
  const bool ok = L >= 0 && L <= a.max_tok && (int64_t)L <= (int64_t)a.tab.max_pages * a.pool.page_size && w0 >= 0 &&
                  w1 >= w0 && w1 <= a.sum_win && q.W <= a.max_win;
  if (!ok) {
    if (tell) report(a.status, ACTKV_E_INVALID, r, L);
    q.W = 0;
  }
  if (q.W > 0) {
    const int first = a.causal ? L - q.W : L - 1;                          // the position of the first row
    q.lo_tile = a.win_left > 0 ? max(0, first - a.win_left + 1) / KT : 0;
    q.tiles = max(1, (L + KT - 1) / KT - q.lo_tile);
  }
  return q;
}

// A CTA's way along its head's line.  Every warp walks it by itself (all lanes of a converged warp call these together).
struct Seg {
  Req q;
  int layer, r, rb, t_in, n_tiles;       // tiles t_in .. t_in + n_tiles - 1 of block rb of request r
  int b0, b1;                            // pieces in which the unit lies
};
template <int KT, int RB, int MIN_TILES>
struct Line {
  const Args& a;
  int h, piece, per_t, layer, r;
  uint32_t off, step;
  uint64_t per, x, x1;
  Req own;                               // up to 32 requests: kept, one per lane, and handed round
  __device__ __forceinline__ uint32_t length_of(const Req& q) const { return (uint32_t)(q.tiles * ((q.W * a.group + RB - 1) / RB)); }
  static __device__ __forceinline__ uint64_t div(uint64_t n, uint64_t d) { return (n | d) >> 32 ? n / d : (uint64_t)((uint32_t)n / (uint32_t)d); }
  __device__ __forceinline__ Req req_of(int r) const {
    if (per_t > 1) return load_req<KT>(a, r, false);
    Req q;
    q.L = __shfl_sync(0xffffffffu, own.L, r);
    q.W = __shfl_sync(0xffffffffu, own.W, r);
    q.win0 = __shfl_sync(0xffffffffu, own.win0, r);
    q.lo_tile = __shfl_sync(0xffffffffu, own.lo_tile, r);
    q.tiles = __shfl_sync(0xffffffffu, own.tiles, r);
    return q;
  }
  // lane t sums requests [t * per_t, (t + 1) * per_t); `tell`: report what is wrong with them
  __device__ __forceinline__ Line(const Args& a_, bool tell) : a(a_) {
    const int lane = threadIdx.x & 31, R = a.tab.n_req, Hkv = a.pool.n_kv_heads, pieces = gridDim.x / Hkv;
    h = blockIdx.x % Hkv;
    piece = blockIdx.x / Hkv;
    per_t = (R + 31) / 32;
    own = Req{};
    uint32_t mine = 0;
#pragma unroll 4
    for (int k = 0; k < per_t; ++k) {
      const int q = lane * per_t + k;
      if (q < R) {
        own = load_req<KT>(a, q, tell);
        mine += length_of(own);
      }
    }
    uint32_t incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t t = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += t;
    }
    const uint32_t T = __shfl_sync(0xffffffffu, incl, 31);                 // (the host has seen to it that it fits)
    const uint64_t total = (uint64_t)T * (uint32_t)a.nls;
    per = max((uint64_t)MIN_TILES, div(total + pieces - 1, pieces));
    x = (uint64_t)piece * per;
    x1 = min(total, x + per);
    step = 0;
    if (x >= x1) return;
    layer = (int)div(x, T);
    off = (uint32_t)(x - (uint64_t)layer * T);
    const int owner = __ffs(__ballot_sync(0xffffffffu, off < incl)) - 1;   // the lane whose requests hold the start
    off -= __shfl_sync(0xffffffffu, incl - mine, owner);
    r = owner * per_t;
    for (; per_t > 1; ++r) {
      const uint32_t n = length_of(load_req<KT>(a, r, false));
      if (off < n) break;
      off -= n;
    }
  }
  // The next stretch of tiles of one unit; false at the end of the piece.
  __device__ __forceinline__ bool next(Seg& s) {
    x += step;
    off += step;
    step = 0;
    while (x < x1) {
      s.q = req_of(r);
      if (off < length_of(s.q)) {
        s.layer = layer;
        s.r = r;
        s.rb = (int)(off / (uint32_t)s.q.tiles);
        s.t_in = (int)(off - (uint32_t)s.rb * s.q.tiles);
        s.n_tiles = (int)min((uint64_t)(s.q.tiles - s.t_in), x1 - x);
        const uint64_t u0 = x - s.t_in;                                    // the unit's place on the line
        s.b0 = (int)div(u0, per);
        s.b1 = (int)div(u0 + s.q.tiles - 1, per);
        step = (uint32_t)s.n_tiles;
        return true;
      }
      off = 0;
      if (++r == a.tab.n_req) { r = 0; ++layer; }
    }
    return false;
  }
  __device__ __forceinline__ int64_t slot(const Seg& s) const { return 2 * (int64_t)blockIdx.x + (piece == s.b0 ? 1 : 0); }
  __device__ __forceinline__ int64_t unit(const Seg& s) const {
    return ((int64_t)(s.layer * a.pool.n_kv_heads + h) * a.tab.n_req + s.r) * a.rb_max + s.rb;
  }
};

// Slots of the partials of a unit in pieces b0 .. b1 of head h's line: the unit begins at the end of piece b0 and goes on at
// the start of the others.
__device__ __forceinline__ int64_t slot_of(int i, int b0, int h, int Hkv) { return 2 * ((int64_t)(b0 + i) * Hkv + h) + (i == 0 ? 1 : 0); }

__device__ __forceinline__ void store_row(const Args& a, int64_t at, int d, float4 o, float sum, float M, int D) {
  if (d < D) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    __nv_bfloat162 v[2] = {__floats2bfloat162_rn(o.x * inv, o.y * inv), __floats2bfloat162_rn(o.z * inv, o.w * inv)};
    *reinterpret_cast<uint2*>(a.out + at * D + d) = *reinterpret_cast<uint2*>(v);
  }
  if (d == 0 && a.lse != nullptr) a.lse[at] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
}

}  // namespace at
}  // namespace actkv
