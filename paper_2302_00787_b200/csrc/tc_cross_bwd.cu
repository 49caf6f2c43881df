// Gradients of the exact cross attention of bf16 tensors on the tensor cores, from P = 2^(x - lse) made again:
//   dkv   per 128 keys, over the rows in tiles:  S^T = K Q^T, dP^T = V dY^T;  dV += P^T dY, dK += dS^T Q
//   dq    per 256 rows, over the keys in tiles:  S = Q K^T, dP = dY V^T;  dQ += dS K
// with dS = P (dP - D); the scores' factor is applied to the sums at the end.  P and dS, rounded to bf16, are operands in tensor
// memory; thread = key (dkv) or row (dq).  Two kernels that both make P instead of one that adds dQ up in memory with atomics: sums
// keep a fixed order.
// Bound: the tensor pipe and, beside it, shared memory: a product with both operands there moves 128 bytes per clock where N = 128 and 192
// where N = 64, its tiles' copies come on top; then the exponentials and the way from a product's end to the warps that wait for it
// (without the warpgroups' arithmetic the two kernels of 2 x 16 heads on 8, 2048 x 4096, d = 128, take 221 us of 267 and 219 of 224; of 16 x 12 x 512 x
// 1500 ragged, d = 64, 93 of 112 and 73 of 84).
#include "cross.cuh"
#include "tc_common.cuh"
#include "tc_cross.cuh"
#include "tc_layout.cuh"

using namespace tc;
using namespace tcl;
using namespace tcx;

int fs_tc_cross_map(CUtensorMap* map, const void* base, TensorAddr t, int B, int H, int L, int inner, int rows);

namespace {

constexpr int CG_WARPS = 8, CGW_TMA = 8, CGW_MMA = 9, CG_T = 384;      // (warps 10, 11 only hand their registers over)
constexpr int CG_REGS_REST = 56, CG_REGS_ROWS = 224;                   // 384 threads x 168 at launch = 128 x 56 + 256 x 224
constexpr int CG_REGS_REST2 = 32, CG_REGS_ROWS2 = 104;                 // two blocks on an SM: 384 x 80 at launch = 128 x 32 + 256 x 104
constexpr int HALF = 64;                                                // keys of a tile in dq
constexpr uint32_t HALF_BYTES = 8192;                                   // 64 rows x 128 bytes
constexpr uint32_t CG_DQ_TMEM = 512, CG_DQ_SUM = 256;                   // dq: two pairs (S, dP) of 64 columns each, then the two dQ

// Two exponentials, by the special-function unit or by the quartic.  NANS: a NaN stays one.
template <bool NANS>
__device__ __forceinline__ void exps2(uint32_t& x, uint32_t& y, bool quartic) {
  if (quartic) exp2_quartic2<NANS>(x, y);
  else { x = __float_as_uint(ex2(__uint_as_float(x))); y = __float_as_uint(ex2(__uint_as_float(y))); }
}

// ------------------------------------------------------------------------------------------ dK, dV
// The products of a tile are issued so that what the warpgroups make is wanted two products later: dV, next S^T, dK, next dP^T; each
// warpgroup has half of a tile's rows.  At d = 64 two blocks on an SM, tiles of 64 rows, hide each other's starts and ends (16 x 12 x 512 x
// 1500: 152 us with one block, 118).
// Columns of tensor memory: S^T and dP^T of the tile (T rows: T columns each; P^T and dS^T, two to a column, lie over them: the first
// warpgroup's T / 2 rows at the front, the second's from column T / 2 on, so that neither writes what the other has yet to read), dV, dK.
template <int D>
struct KvSm {
  static constexpr int T = D == 64 ? 64 : 128, BLOCKS = D == 64 ? 2 : 1, PANELS = D / 64, NS = D == 64 ? 4 : 2;      // NS: tiles of Q and of dY in flight
  static constexpr uint32_t PANEL = T * 128, BIG = PANELS * TILE_BYTES, TILE_D = PANELS * PANEL, K = 0, V = BIG, Q = 2 * BIG, G = Q + NS * TILE_D, STAT = G + NS * TILE_D;
  static constexpr uint32_t MISC = STAT + NS * 8 * T, TOTAL = MISC + 1536;
  static constexpr uint32_t S = 0, P = T, DV = 2 * T, DK = 2 * T + D, COLUMNS = BLOCKS == 2 ? 256 : 512;
  static_assert(BLOCKS * (TOTAL + 2048) <= 233472, "shared memory budget");
  static_assert(DK + D <= COLUMNS, "tensor memory");
};
struct KvMs {
  uint64_t q_full[4], q_empty[4], g_full[4], g_empty[4], s_full, p_ready, dp_full, ds_ready, kv_full, kv_empty, done;
  uint32_t tmem_base;
  int abort_flag;
  int live[CROSS_RANKED + 1];                          // tiles of keys that the sequences before one have
};
static_assert(sizeof(KvMs) <= 1536, "misc block");

// One piece of work: 128 keys against a piece of the rows of the query heads that share them.
struct KvWork {
  int unit, piece, b, hk, j0, n, t0, items;
};

// Blocks are persistent and take every gridDim.x-th piece of the work that there is: tiles behind a sequence's end are written with zeros
// on the way.  The next piece's keys and rows are copied, and its first S^T and dP^T made, while this one's sums go out.  (A block per
// piece: 17.5 us each for 16 x 12 x 512 x 1500, 11.2 of them at its tiles, and 5 us from one to the next: 117 us.)
template <int D>
__global__ void __launch_bounds__(CG_T, KvSm<D>::BLOCKS)
tc_cross_dkv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CrossArgs a, const __grid_constant__ CrossGrad gr,
                    int key_tiles, int* __restrict__ status) {
  using Sm = KvSm<D>;
  constexpr int T = Sm::T;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  KvMs* misc = reinterpret_cast<KvMs*>(sm + Sm::MISC);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abortp = &misc->abort_flag;
  const int per = (a.Lq + T - 1) / T;                  // row tiles: those of the first query head of the group, of the second, ...
  const int row_tiles = a.g * per;
  // Without lengths, or with more of them than are listed, every tile counts as live (the rows of a tile that is not come to nothing).
  const bool listed = a.key_len != nullptr && a.B <= CROSS_RANKED;

  if (threadIdx.x == 0) {
    for (int i = 0; i < Sm::NS; i++) { mbar_init(&misc->q_full[i], 1); mbar_init(&misc->q_empty[i], 1); mbar_init(&misc->g_full[i], 1); mbar_init(&misc->g_empty[i], 1); }
    mbar_init(&misc->s_full, 1);
    mbar_init(&misc->dp_full, 1);
    mbar_init(&misc->p_ready, CG_WARPS);
    mbar_init(&misc->ds_ready, CG_WARPS);
    mbar_init(&misc->kv_full, 1);
    mbar_init(&misc->kv_empty, 1);
    mbar_init(&misc->done, 1);
    misc->abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == CGW_MMA) {
    tmem_alloc(&misc->tmem_base, Sm::COLUMNS);
    tmem_relinquish();
  }
  if (listed && warp == 0) {
    // live tiles of the sequences before each
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      const int b = b0 + lane, own = b < a.B ? (cross_keys(a, b) + TILE - 1) / TILE : 0;
      int sum = own;
#pragma unroll
      for (int k = 1; k < 32; k <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, sum, k);
        if (lane >= k) sum += x;
      }
      if (b < a.B) misc->live[b + 1] = before + sum;
      before += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) misc->live[0] = 0;
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem = misc->tmem_base;
  const int kp = (a.d + 63) / 64, vp = (a.dv + 63) / 64;      // panels of 64 columns
  const int total = (listed ? misc->live[a.B] : a.B * key_tiles) * a.Hk * gr.kv_pieces;
  auto work_at = [&](int i) {
    KvWork k;
    int x = i;
    k.piece = 0;
    if (gr.kv_pieces > 1) { x = i / gr.kv_pieces; k.piece = i - x * gr.kv_pieces; }
    int tile;
    if (listed) {
      k.b = 0;
      for (int step = CROSS_RANKED / 2; step; step >>= 1)      // the last sequence that begins at x or before
        if (k.b + step < a.B && misc->live[k.b + step] * a.Hk <= x) k.b += step;
      const int own = misc->live[k.b + 1] - misc->live[k.b];
      x -= misc->live[k.b] * a.Hk;
      k.hk = x / own;
      tile = x - k.hk * own;
    } else {
      k.unit = x / key_tiles;
      tile = x - k.unit * key_tiles;
      k.b = k.unit / a.Hk;
      k.hk = k.unit - k.b * a.Hk;
    }
    k.unit = k.b * a.Hk + k.hk;
    k.j0 = tile * TILE;
    k.n = cross_keys(a, k.b);
    k.t0 = 0;
    k.items = row_tiles;
    if (gr.kv_pieces > 1) {
      k.t0 = (int)((int64_t)row_tiles * k.piece / gr.kv_pieces);
      k.items = (int)((int64_t)row_tiles * (k.piece + 1) / gr.kv_pieces) - k.t0;
    }
    return k;
  };

  if (warp >= CG_WARPS) regs_release<(Sm::BLOCKS == 2 ? CG_REGS_REST2 : CG_REGS_REST)>();
  if (warp == CGW_TMA) {
    if (lane == 0) {
      prefetch_tmap(&tmQ); prefetch_tmap(&tmG); prefetch_tmap(&tmK); prefetch_tmap(&tmV);
      int at = 0, worked = 0;                          // tiles of rows and pieces of work so far
      bool ok = true;
      for (int wi = blockIdx.x; wi < total && ok; wi += gridDim.x, worked++) {
        const KvWork k = work_at(wi);
        if (!mbar_wait(&misc->kv_empty, (worked & 1) ^ 1, abortp, status)) break;
        mbar_expect_tx(&misc->kv_full, (kp + vp) * TILE_BYTES);
        for (int p = 0; p < kp; p++) tma_load_4d(sm + Sm::K + p * TILE_BYTES, &tmK, &misc->kv_full, p * 64, k.j0, a.ak.sh ? k.hk : 0, a.ak.sb ? k.b : 0);
        for (int p = 0; p < vp; p++) tma_load_4d(sm + Sm::V + p * TILE_BYTES, &tmV, &misc->kv_full, p * 64, k.j0, a.av.sh ? k.hk : 0, a.av.sb ? k.b : 0);
        int h = k.hk * a.g + k.t0 / per, t = k.t0 % per;
        for (int i = 0; i < k.items; i++, at++) {
          const int s = at % Sm::NS;
          const uint32_t parity = ((at / Sm::NS) & 1) ^ 1;
          // (dY of a tile is done with before its Q is)
          if (!mbar_wait(&misc->q_empty[s], parity, abortp, status) || !mbar_wait(&misc->g_empty[s], parity, abortp, status)) { ok = false; break; }
          mbar_expect_tx(&misc->q_full[s], kp * Sm::PANEL + 8 * T);
          for (int p = 0; p < kp; p++)
            tma_load_4d(sm + Sm::Q + s * Sm::TILE_D + p * Sm::PANEL, &tmQ, &misc->q_full[s], p * 64, t * T, a.aq.sh ? h : 0, a.aq.sb ? k.b : 0);
          const float* st = gr.stat + ((int64_t)k.b * a.H + h) * cross_stat_floats(a.Lq) + (int64_t)(t * T / 128) * 256 + t * T % 128;
          bulk_load(sm + Sm::STAT + s * 8 * T, st, 4 * T, &misc->q_full[s]);
          bulk_load(sm + Sm::STAT + s * 8 * T + 4 * T, st + 128, 4 * T, &misc->q_full[s]);
          mbar_expect_tx(&misc->g_full[s], vp * Sm::PANEL);
          for (int p = 0; p < vp; p++)
            tma_load_4d(sm + Sm::G + s * Sm::TILE_D + p * Sm::PANEL, &tmG, &misc->g_full[s], p * 64, t * T, gr.ady.sh ? h : 0, gr.ady.sb ? k.b : 0);
          if (++t == per) { t = 0; h++; }
        }
        if (!ok) mbar_wait(&misc->kv_full, worked & 1, abortp, status, false);
      }
      // nothing of this block may still be in flight when it exits: no copy, and no arrival of a product's completion
      if (ok && worked > 0) {
        mbar_wait(&misc->kv_full, (worked - 1) & 1, abortp, status, false);
        mbar_wait(&misc->kv_empty, (worked - 1) & 1, abortp, status);
      }
      for (int k = max(0, at - Sm::NS); k < at; k++) {
        const uint32_t parity = (k / Sm::NS) & 1;
        mbar_wait(&misc->q_full[k % Sm::NS], parity, abortp, status, false);
        mbar_wait(&misc->g_full[k % Sm::NS], parity, abortp, status, false);
        mbar_wait(&misc->q_empty[k % Sm::NS], parity, abortp, status);
        mbar_wait(&misc->g_empty[k % Sm::NS], parity, abortp, status);
      }
    }
  } else if (warp == CGW_MMA) {
    // dV of a tile, S^T of the next, dK, dP^T of the next: each needs what the warpgroups made during the two before it.
    constexpr uint32_t ID_S = idesc_bf16(128, T, 0, 0);
    const uint32_t ID_V = idesc_bf16(128, a.dv, 0, 1), ID_K = idesc_bf16(128, a.d, 0, 1);
    const uint32_t sQ = smem_u32(sm + Sm::Q), sG = smem_u32(sm + Sm::G);
    const Desc k0 = smem_desc(smem_u32(sm + Sm::K), 16, 1024, SWZ_128B), v0 = smem_desc(smem_u32(sm + Sm::V), 16, 1024, SWZ_128B);
    const Desc q0 = smem_desc(sQ, 16, 1024, SWZ_128B), g0 = smem_desc(sG, 16, 1024, SWZ_128B);
    // the same tiles with their rows as the contraction: panels of 64 columns, 16 rows of 128 bytes per step
    const Desc qt = smem_desc(sQ, Sm::PANEL, 1024, SWZ_128B), gt = smem_desc(sG, Sm::PANEL, 1024, SWZ_128B);
    const int ks = a.d / 16, vs = a.dv / 16;
    const bool leader = elect_one();
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abortp, status); };
    auto issue_s = [&](int at) {
      const int s = at % Sm::NS;
      if (!wait(&misc->q_full[s], (at / Sm::NS) & 1)) return false;
      tcgen05_fence_after();
      if (leader) {
        Desc q = q0;
        q.lo += s * (Sm::TILE_D / 16);
        issue_rows<D / 16, TILE_BYTES, Sm::PANEL>(tmem + Sm::S, k0, q, ID_S, ks);
        mma_commit(&misc->s_full);
      }
      __syncwarp();
      return true;
    };
    auto issue_dp = [&](int at, bool last) {
      const int s = at % Sm::NS;
      if (!wait(&misc->g_full[s], (at / Sm::NS) & 1)) return false;
      tcgen05_fence_after();
      if (leader) {
        Desc g = g0;
        g.lo += s * (Sm::TILE_D / 16);
        issue_rows<D / 16, TILE_BYTES, Sm::PANEL>(tmem + Sm::P, v0, g, ID_S, vs);
        if (last) mma_commit(&misc->kv_empty);
        mma_commit(&misc->dp_full);
      }
      __syncwarp();
      return true;
    };
    int at = 0, worked = 0;
    bool ok = true;
    for (int wi = blockIdx.x; wi < total && ok; wi += gridDim.x, worked++) {
      const int items = work_at(wi).items;
      ok = wait(&misc->kv_full, worked & 1) && issue_s(at) && issue_dp(at, items == 1);
      for (int i = 0; i < items && ok; i++, at++) {
        const int s = at % Sm::NS;
        if (!(ok = wait(&misc->p_ready, at & 1))) break;
        tcgen05_fence_after();
        if (leader) {
          Desc g = gt;
          g.lo += s * (Sm::TILE_D / 16);
          issue_halves<T, T / 2>(tmem + Sm::DV, tmem + Sm::S, g, ID_V, i > 0);
          mma_commit(&misc->g_empty[s]);
        }
        __syncwarp();
        if (i + 1 < items && !(ok = issue_s(at + 1))) break;
        if (!(ok = wait(&misc->ds_ready, at & 1))) break;
        tcgen05_fence_after();
        if (leader) {
          Desc q = qt;
          q.lo += s * (Sm::TILE_D / 16);
          issue_halves<T, T / 2>(tmem + Sm::DK, tmem + Sm::P, q, ID_K, i > 0);
          mma_commit(&misc->q_empty[s]);
          if (i == items - 1) mma_commit(&misc->done);
        }
        __syncwarp();
        if (i + 1 < items) ok = issue_dp(at + 1, i + 2 == items);
      }
    }
  } else if (warp < CG_WARPS) {
    regs_acquire<(Sm::BLOCKS == 2 ? CG_REGS_ROWS2 : CG_REGS_ROWS)>();
    const int w = warp >> 2, row = (warp & 3) * 32 + lane;      // w: which half of the tile's rows; and the first writes dV, the second dK
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), tS = lanes + Sm::S + w * (T / 2), tP = lanes + Sm::P + w * (T / 2);
    const float c = a.scale * FS_LOG2E;
    // 16 values of a key's dV or dK, or of a piece's sums of them
    auto store = [&](int unit, int b, int hk, int piece, int j, int q, const float (&x)[16]) {
      const TensorAddr to = w ? gr.adk : gr.adv;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(w ? gr.dK : gr.dV) + b * to.sb + hk * to.sh + j * to.sl + q;
      float* part = gr.pkv + (((int64_t)piece * a.B * a.Hk + unit) * a.Lk + j) * (a.d + a.dv) + (w ? 0 : a.d) + q;
      store_row(j < a.Lk, x, gr.pkv ? part : nullptr, out);
    };
    const int width = w ? a.d : a.dv;
    if (listed) {
      const float none[16] = {};
      for (int i = blockIdx.x; i < a.B * a.Hk * key_tiles; i += gridDim.x) {
        const int unit = i / key_tiles, tile = i - unit * key_tiles, b = unit / a.Hk;
        if (tile >= misc->live[b + 1] - misc->live[b])
          for (int piece = 0; piece < gr.kv_pieces; piece++)
            for (int q = 0; q < width; q += 16) store(unit, b, unit - b * a.Hk, piece, tile * TILE + row, q, none);
      }
    }
    bool ok = true;
    int at = 0, worked = 0;
    for (int wi = blockIdx.x; wi < total; wi += gridDim.x, worked++) {
      const KvWork k = work_at(wi);
      for (int i = 0; i < k.items && ok; i++, at++) {
        const int s = at % Sm::NS;
        // (what a hidden key holds, NaNs too, stays in its own row of S^T, dP^T and of the sums, and is dropped at the end)
        ok = __all_sync(0xffffffffu, mbar_wait(&misc->s_full, at & 1, abortp, status, false) &&
                                         mbar_wait(&misc->q_full[s], (at / Sm::NS) & 1, abortp, status, false));
        if (!ok) break;
        tcgen05_fence_after();
        const float* st = reinterpret_cast<const float*>(sm + Sm::STAT + s * 8 * T) + w * (T / 2);
        uint32_t x[T / 2], g[T / 2];
#pragma unroll
        for (int q = 0; q < T / 32; q++) tmem_ld16(tS + 16 * q, *reinterpret_cast<uint32_t(*)[16]>(x + 16 * q));
        tmem_wait_ld();
#pragma unroll
        for (int q = 0; q < T / 2; q += 32) {
          uint32_t o[16];
#pragma unroll
          for (int p = 0; p < 32; p += 4) {
            const float4 nl = *reinterpret_cast<const float4*>(st + q + p);
            uint32_t* xp = x + q + p;
            fma2v(xp[0], xp[1], c, nl.x, nl.y);
            fma2v(xp[2], xp[3], c, nl.z, nl.w);
            // a NaN row of Q makes all of its P, and so all of dV, NaN.  (One in eight by the quartic: 936 us for 4 x 12 x 4096 x 8192, d = 64; one
            // in four 957, none 940; 271, 270 and 275 for 2 x 16 heads on 8, 2048 x 4096, d = 128)
            exps2<true>(xp[0], xp[1], false);
            exps2<true>(xp[2], xp[3], (p & 12) == 12);
            o[p / 2] = pack_bf16(__uint_as_float(xp[0]), __uint_as_float(xp[1]));
            o[p / 2 + 1] = pack_bf16(__uint_as_float(xp[2]), __uint_as_float(xp[3]));
          }
          tmem_st16(tS + q / 2, o);
        }
        tmem_wait_st();
        tcgen05_fence_before();
        mbar_arrive_warp(&misc->p_ready, lane);
        ok = __all_sync(0xffffffffu, mbar_wait(&misc->dp_full, at & 1, abortp, status, false));
        if (!ok) break;
        tcgen05_fence_after();
#pragma unroll
        for (int q = 0; q < T / 32; q++) tmem_ld16(tP + 16 * q, *reinterpret_cast<uint32_t(*)[16]>(g + 16 * q));
        tmem_wait_ld();
#pragma unroll
        for (int q = 0; q < T / 2; q += 32) {
          uint32_t u[16];
#pragma unroll
          for (int p = 0; p < 32; p += 4) {
            const float4 nd = *reinterpret_cast<const float4*>(st + T + q + p);
            uint32_t *xp = x + q + p, *gp = g + q + p;
            addmul2(gp[0], gp[1], nd.x, nd.y, xp[0], xp[1]);
            addmul2(gp[2], gp[3], nd.z, nd.w, xp[2], xp[3]);
            u[p / 2] = pack_bf16(__uint_as_float(gp[0]), __uint_as_float(gp[1]));
            u[p / 2 + 1] = pack_bf16(__uint_as_float(gp[2]), __uint_as_float(gp[3]));
          }
          tmem_st16(tP + q / 2, u);
        }
        tmem_wait_st();
        tcgen05_fence_before();
        mbar_arrive_warp(&misc->ds_ready, lane);
      }
      ok = ok && __all_sync(0xffffffffu, mbar_wait(&misc->done, worked & 1, abortp, status, false));
      if (!ok) break;
      tcgen05_fence_after();
      const int j = k.j0 + row;
      const bool on = cross_seen(a, k.b, j, k.n);
      const float f = w ? a.scale : 1.f;
      for (int q = 0; q < width; q += 16) {
        uint32_t t[16];
        tmem_ld16(lanes + (w ? Sm::DK : Sm::DV) + q, t);
        tmem_wait_ld();
        float x[16];
#pragma unroll
        for (int p = 0; p < 16; p++) x[p] = on ? __uint_as_float(t[p]) * f : 0.f;
        store(k.unit, k.b, k.hk, k.piece, j, q, x);
      }
      tcgen05_fence_before();                          // (the sums have been read before the next P and dS are handed over)
    }
  }
  tcgen05_fence_before();
  __syncthreads();
  if (warp == CGW_MMA) {
    tcgen05_fence_after();
    tmem_dealloc(tmem, Sm::COLUMNS);
  }
}

// ------------------------------------------------------------------------------------------ dQ
// Up to 256 rows of a unit per block, 128 per warpgroup, over the keys in tiles of 64; each warpgroup has S, dP (dS, two to a column, lies
// over S) and dQ of its own, and they share every K and V tile (up to 128 rows: tiles in turn, two partial dQ that meet at the end).
// (128 rows per block, both warpgroups on halves of its tiles: twice the copies, 278 us instead of 234 for 2 x 16 heads on 8,
// 2048 x 4096, d = 128, the same 92 us for 16 x 12 x 512 x 1500, d = 64.)
template <int D>
struct DqSm {
  static constexpr int PANELS = D / 64, NS = D == 64 ? 6 : 3;
  static constexpr uint32_t BIG = PANELS * TILE_BYTES, Q = 0, G = 2 * BIG, RING = 4 * BIG, SLOT = PANELS * HALF_BYTES, STAGE = 2 * SLOT;
  static constexpr uint32_t MISC = RING + NS * STAGE, TOTAL = MISC + 512;
  static_assert(TOTAL + 1024 <= 232448, "shared memory budget");
  static_assert(4 * BIG >= 128 * (D + 1) * 4, "the warpgroups' exchange");
};
struct DqMs {
  uint64_t full[8], empty[8], sp_full[2], ready[2], done[2], q_ready;
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(DqMs) <= 512, "misc block");

template <int D>
__global__ void __launch_bounds__(CG_T, 1)
tc_cross_dq_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CrossArgs a,
                   const __grid_constant__ CrossGrad gr, int* __restrict__ status) {
  using Sm = DqSm<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  DqMs* misc = reinterpret_cast<DqMs*>(sm + Sm::MISC);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abortp = &misc->abort_flag;
  const int unit = cross_unit(a, reinterpret_cast<int*>(sm + Sm::Q)), piece = blockIdx.x % gr.q_pieces, r0 = (int)(blockIdx.x / gr.q_pieces) * 256;
  const int b = unit / a.Hk, hk = unit % a.Hk, R = a.g * a.Lq;
  const int n = cross_keys(a, b), tiles = (n + HALF - 1) / HALF;
  const int t0 = (int)((int64_t)tiles * piece / gr.q_pieces), nt = (int)((int64_t)tiles * (piece + 1) / gr.q_pieces) - t0;
  const bool both = R - r0 > TILE;                     // each warpgroup has rows of its own
  const int items = both ? 2 * nt : nt;                // item i: warpgroup i & 1, tile i / 2 or i

  const int kp = (a.d + 63) / 64, vp = (a.dv + 63) / 64;      // panels of 64 columns
  auto load = [&](int i) {                             // tile i of K and of V
    const int s = i % Sm::NS, tok = (t0 + i) * HALF;
    uint8_t* base = sm + Sm::RING + s * Sm::STAGE;
    mbar_expect_tx(&misc->full[s], (kp + vp) * HALF_BYTES);
    for (int p = 0; p < kp; p++) tma_load_4d(base + p * HALF_BYTES, &tmK, &misc->full[s], p * 64, tok, a.ak.sh ? hk : 0, a.ak.sb ? b : 0);
    for (int p = 0; p < vp; p++) tma_load_4d(base + Sm::SLOT + p * HALF_BYTES, &tmV, &misc->full[s], p * 64, tok, a.av.sh ? hk : 0, a.av.sb ? b : 0);
  };
  if (threadIdx.x == CGW_TMA * 32) {                   // (the thread that issues the copies)
    for (int i = 0; i < Sm::NS; i++) { mbar_init(&misc->full[i], 1); mbar_init(&misc->empty[i], 1); }
    for (int w = 0; w < 2; w++) { mbar_init(&misc->sp_full[w], 1); mbar_init(&misc->ready[w], 4); mbar_init(&misc->done[w], 1); }
    mbar_init(&misc->q_ready, CG_WARPS);
    misc->abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
    for (int i = 0; i < Sm::NS && i < nt; i++) load(i);      // the ring's first round, while the others make ready
  }
  if (warp < CG_WARPS) {
    // the block's rows of Q and dY into shared memory, rows and columns that there are none of as zeros
    constexpr int CH = D / 8;
    const int rows = both ? 256 : 128;
    for (int i = threadIdx.x; i < 2 * rows * CH; i += 256) {
      const int which = i >= rows * CH, k = i - which * rows * CH, rr = k / CH, ch = k % CH, r = r0 + rr;
      const TensorAddr t = which ? gr.ady : a.aq;
      const __nv_bfloat16* X = static_cast<const __nv_bfloat16*>(which ? gr.dY : a.Q) + b * t.sb;
      const bool some = r < R && ch * 8 < (which ? a.dv : a.d);
      copy16(sm + (which ? Sm::G : Sm::Q) + (rr >> 7) * Sm::BIG + (ch >> 3) * TILE_BYTES + sw128_offset(rr & 127, (ch & 7) * 8),
             X + (some ? (int64_t)(hk * a.g + r / a.Lq) * t.sh + (int64_t)(r % a.Lq) * t.sl + ch * 8 : 0), some);
    }
  }
  if (warp == CGW_MMA) {
    tmem_alloc(&misc->tmem_base, CG_DQ_TMEM);
    tmem_relinquish();
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem = misc->tmem_base;

  if (warp >= CG_WARPS) regs_release<CG_REGS_REST>();
  if (warp == CGW_TMA) {
    if (lane == 0) {
      int i = min(Sm::NS, nt);
      for (; i < nt; i++) {
        if (!mbar_wait(&misc->empty[i % Sm::NS], ((i / Sm::NS) & 1) ^ 1, abortp, status)) break;
        load(i);
      }
      // nothing of this block may still be in flight when it exits: no copy, and no arrival of a product's completion
      for (int k = max(0, i - Sm::NS); k < i; k++) {
        mbar_wait(&misc->full[k % Sm::NS], (k / Sm::NS) & 1, abortp, status, false);
        mbar_wait(&misc->empty[k % Sm::NS], (k / Sm::NS) & 1, abortp, status);
      }
    }
  } else if (warp == CGW_MMA) {
    constexpr uint32_t ID_S = idesc_bf16(128, HALF, 0, 0);
    const uint32_t ID_Q = idesc_bf16(128, a.d, 0, 1);
    const uint32_t sR = smem_u32(sm + Sm::RING), sQ = smem_u32(sm + Sm::Q), sG = smem_u32(sm + Sm::G);
    const int ks = a.d / 16, vs = a.dv / 16;
    const Desc q0 = smem_desc(sQ, 16, 1024, SWZ_128B), g0 = smem_desc(sG, 16, 1024, SWZ_128B);
    const Desc k0 = smem_desc(sR, 16, 1024, SWZ_128B), kt = smem_desc(sR, HALF_BYTES, 1024, SWZ_128B);      // V: a slot behind K
    const bool leader = elect_one();
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abortp, status); };
    int slot = 0, phase = 0, done = 0;                 // the next tile's stage; the stage of the tile whose sums come next
    auto issue_sp = [&](int w) {                       // S and dP of the next item, which is warpgroup w's
      if (!wait(&misc->full[slot], phase)) return false;
      tcgen05_fence_after();
      if (leader) {
        Desc q = q0, g = g0, k = k0;
        q.lo += (both ? w : 0) * (Sm::BIG / 16);
        g.lo += (both ? w : 0) * (Sm::BIG / 16);
        k.lo += slot * (Sm::STAGE / 16);
        issue_rows<D / 16, TILE_BYTES, HALF_BYTES>(tmem + w * 128, q, k, ID_S, ks);
        k.lo += Sm::SLOT / 16;
        issue_rows<D / 16, TILE_BYTES, HALF_BYTES>(tmem + w * 128 + 64, g, k, ID_S, vs);
        mma_commit(&misc->sp_full[w]);
      }
      __syncwarp();
      if ((!both || w) && ++slot == Sm::NS) { slot = 0; phase ^= 1; }
      return true;
    };
    bool ok = nt > 0 && wait(&misc->q_ready, 0);
    if (ok) {
      tcgen05_fence_after();
      ok = issue_sp(0) && (items < 2 || issue_sp(1));
    }
    auto item = [&](int i, int w) {
      if (!wait(&misc->ready[w], (i >> 1) & 1)) return false;
      tcgen05_fence_after();
      if (leader) {
        Desc k = kt;                                   // its keys as the contraction
        k.lo += done * (Sm::STAGE / 16);
        issue_cols<4>(tmem + CG_DQ_SUM + w * 128, tmem + w * 128, k, ID_Q, i > 1);
        if (!both || w) mma_commit(&misc->empty[done]);
        if (i + 2 >= items) mma_commit(&misc->done[w]);
      }
      __syncwarp();
      if ((!both || w) && ++done == Sm::NS) done = 0;
      return i + 2 >= items || issue_sp(w);
    };
    for (int i = 0; i < items && ok; i += 2) ok = item(i, 0) && (i + 1 >= items || item(i + 1, 1));
  } else if (warp < CG_WARPS) {
    regs_acquire<CG_REGS_ROWS>();
    const int w = warp >> 2, row = (warp & 3) * 32 + lane;
    copies_done();
    fence_proxy_async_smem();
    mbar_arrive_warp(&misc->q_ready, lane);
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), tS = lanes + w * 128, tP = tS + 64, tQ = lanes + CG_DQ_SUM + w * 128;
    const int first = r0 + (both ? w * TILE : 0), r = first + row;
    const bool idle = first + (warp & 3) * 32 >= R;
    const int mine = both ? nt : (nt + 1 - w) / 2;
    const float c = a.scale * FS_LOG2E;
    const float2 st = r < R ? cross_stat(gr.stat, (int64_t)b * a.H + hk * a.g + r / a.Lq, a.Lq, r % a.Lq) : make_float2(-INFINITY, 0.f);
    bool ok = true;
    for (int i = 0; i < mine; i++) {
      const int t = both ? i : 2 * i + w, jj = (t0 + t) * HALF, s = t % Sm::NS;
      ok = __all_sync(0xffffffffu, mbar_wait(&misc->sp_full[w], i & 1, abortp, status, false) &&
                                       mbar_wait(&misc->full[s], (t / Sm::NS) & 1, abortp, status, false));
      if (!ok) break;
      tcgen05_fence_after();
      uint32_t seen[2] = {~0u, ~0u};
      if (a.key_mask != nullptr || jj + HALF > n) {
#pragma unroll
        for (int q = 0; q < 2; q++) seen[q] = __ballot_sync(0xffffffffu, cross_seen(a, b, jj + q * 32 + lane, n));
        // a hidden key's K becomes zeros (it may hold anything) before dS multiplies it; a warp does 16 of the 64 keys.  The other
        // warpgroup's scores of the same key, made before or after, are dropped like this one's
        if ((!both || w == 0) && lane < 16) {
          const int key = (warp & 3) * 16 + lane;
          if (!(seen[key >> 5] >> (key & 31) & 1u))
            for (int p = 0; p < kp; p++)
              for (int k = 0; k < 8; k++)
                *reinterpret_cast<uint4*>(sm + Sm::RING + s * Sm::STAGE + p * HALF_BYTES + key * 128 + k * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
      }
      if (!idle) {
        uint32_t x[64], g[64];
#pragma unroll
        for (int q = 0; q < 4; q++) tmem_ld16(tS + 16 * q, *reinterpret_cast<uint32_t(*)[16]>(x + 16 * q));
#pragma unroll
        for (int q = 0; q < 4; q++) tmem_ld16(tP + 16 * q, *reinterpret_cast<uint32_t(*)[16]>(g + 16 * q));
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < 64; k += 4) {
          fma2(x[k], x[k + 1], c, st.x);
          fma2(x[k + 2], x[k + 3], c, st.x);
          // (a NaN of P needs no handing on here: D of its row is NaN.  One in four by the quartic: 884 us for 4 x 12 x 4096 x 8192, one in
          // eight 902, none 917)
          exps2<false>(x[k], x[k + 1], false);
          exps2<false>(x[k + 2], x[k + 3], (k & 4) != 0);
          addmul2(g[k], g[k + 1], st.y, st.y, x[k], x[k + 1]);
          addmul2(g[k + 2], g[k + 3], st.y, st.y, x[k + 2], x[k + 3]);
        }
        if ((seen[0] & seen[1]) != ~0u) {
#pragma unroll
          for (int k = 0; k < 64; k++) g[k] = (seen[k >> 5] >> (k & 31)) & 1u ? g[k] : 0u;
        }
#pragma unroll
        for (int q = 0; q < 64; q += 32) {
          uint32_t u[16];
#pragma unroll
          for (int k = 0; k < 16; k++) u[k] = pack_bf16(__uint_as_float(g[q + 2 * k]), __uint_as_float(g[q + 2 * k + 1]));
          tmem_st16(tS + q / 2, u);
        }
        tmem_wait_st();
      }
      tcgen05_fence_before();
      mbar_arrive_warp(&misc->ready[w], lane);
    }
    if (ok && mine > 0) ok = mbar_wait(&misc->done[w], 0, abortp, status, false);
    if (ok && !both && (nt + w) / 2 > 0) ok = mbar_wait(&misc->done[w ^ 1], 0, abortp, status, false);
    ok = __all_sync(0xffffffffu, ok);
    tcgen05_fence_after();
    // (every warp comes to the barrier below, also after a wait that ran out; the exchange lies where Q and dY were)
    float* xo = reinterpret_cast<float*>(sm + Sm::Q);
    if (!both) {
      if (w == 1 && ok)
        for (int q = 0; q < a.d; q += 16) {
          uint32_t o[16] = {};
          if (mine > 0) {
            tmem_ld16(tQ + q, o);
            tmem_wait_ld();
          }
#pragma unroll
          for (int k = 0; k < 16; k++) xo[row * (D + 1) + q + k] = __uint_as_float(o[k]);
        }
      named_bar_sync(3, 256);
    }
    if ((both || w == 0) && ok) {
      const int h = hk * a.g + r / a.Lq, tok = r % a.Lq;
      float* part = gr.pq + (((int64_t)piece * a.B * a.Hk + unit) * R + r) * a.d;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(gr.dQ) + b * gr.adq.sb + h * gr.adq.sh + tok * gr.adq.sl;
      for (int q = 0; q < a.d; q += 16) {
        uint32_t o[16] = {};
        if (mine > 0) {
          tmem_ld16(tQ + q, o);
          tmem_wait_ld();
        }
        float x[16];
#pragma unroll
        for (int k = 0; k < 16; k++) x[k] = a.scale * (__uint_as_float(o[k]) + (both ? 0.f : xo[row * (D + 1) + q + k]));
        store_row(r < R, x, gr.pq ? part + q : nullptr, out + q);
      }
    }
  }
  tcgen05_fence_before();
  __syncthreads();
  if (warp == CGW_MMA) {
    tcgen05_fence_after();
    tmem_dealloc(tmem, CG_DQ_TMEM);
  }
}

template <int D>
int launch(fsharp_ctx* ctx, const CrossArgs& a, const CrossGrad& gr) {
  const int64_t keys = ((int64_t)a.Lk + TILE - 1) / TILE, works = keys * gr.kv_pieces * a.B * a.Hk, gq = ((int64_t)a.g * a.Lq + 255) / 256 * gr.q_pieces;
  if (works > 0x7fff0000 || gq > 0x7fffffff) return FSHARP_E_SHAPE;
  const int64_t resident = (int64_t)ctx->sm_count * KvSm<D>::BLOCKS;
  CUtensorMap tmQ, tmG, tmK, tmV, tmKt, tmVt;
  FS_TRY(fs_tc_cross_map(&tmQ, a.Q, a.aq, a.B, a.H, a.Lq, a.d, KvSm<D>::T));
  FS_TRY(fs_tc_cross_map(&tmG, gr.dY, gr.ady, a.B, a.H, a.Lq, a.dv, KvSm<D>::T));
  FS_TRY(fs_tc_cross_map(&tmK, a.K, a.ak, a.B, a.Hk, a.Lk, a.d, TILE));
  FS_TRY(fs_tc_cross_map(&tmV, a.V, a.av, a.B, a.Hk, a.Lk, a.dv, TILE));
  FS_TRY(fs_tc_cross_map(&tmKt, a.K, a.ak, a.B, a.Hk, a.Lk, a.d, HALF));
  FS_TRY(fs_tc_cross_map(&tmVt, a.V, a.av, a.B, a.Hk, a.Lk, a.dv, HALF));
  FS_CUDA_OK(fs_allow_smem(tc_cross_dkv_kernel<D>));
  FS_CUDA_OK(fs_allow_smem(tc_cross_dq_kernel<D>));
  FS_TIME_BEGIN(ctx, FS_K_TC_CROSS_DKV);
  tc_cross_dkv_kernel<D><<<dim3((unsigned)(works < resident ? works : resident)), CG_T, KvSm<D>::TOTAL + 1024, ctx->stream>>>(
      tmQ, tmG, tmK, tmV, a, gr, (int)keys, ctx->d_status);
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  CrossArgs aq = a;
  aq.ranked = cross_ranked(ctx, a, gq * a.B * a.Hk);
  FS_TIME_BEGIN(ctx, FS_K_TC_CROSS_DQ);
  tc_cross_dq_kernel<D><<<dim3((unsigned)gq, (unsigned)(a.B * a.Hk)), CG_T, DqSm<D>::TOTAL + 1024, ctx->stream>>>(tmKt, tmVt, aq, gr, ctx->d_status);
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  return FSHARP_OK;
}

// Pieces that bring `blocks` blocks up to one per SM, each with two tiles at least.
int pieces_for(const fsharp_ctx* ctx, int64_t blocks, int64_t tiles) {
  int64_t p = ctx->sm_count / blocks;
  if (p > tiles / 2) p = tiles / 2;
  if (p > 64) p = 64;
  return p < 1 ? 1 : (int)p;
}

}  // namespace

void fs_tc_cross_grad_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int* kv_pieces, int* q_pieces) {
  const int64_t g = dm->H / dm->Hk, units = (int64_t)dm->B * dm->Hk, keys = ((int64_t)dm->Lk + TILE - 1) / TILE;
  *kv_pieces = pieces_for(ctx, units * keys, g * (((int64_t)dm->Lq + TILE - 1) / TILE));
  *q_pieces = pieces_for(ctx, units * ((g * dm->Lq + 255) / 256), keys);
}

int fs_tc_cross_grad(fsharp_ctx* ctx, const CrossArgs& a, const CrossGrad& gr) {
  return a.d > 64 || a.dv > 64 ? launch<128>(ctx, a, gr) : launch<64>(ctx, a, gr);
}
