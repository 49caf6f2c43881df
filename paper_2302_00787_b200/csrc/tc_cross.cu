// Exact cross attention of bf16 tensors on the tensor cores:  Y = softmax(scale Q K^T) V  with a running maximum.
//
// A block has up to 256 rows of a unit (rows are packed over the query heads that share a key head) and walks the unit's keys
// in tiles of 128.  Two warpgroups, thread = row: each has scores S (lanes: rows, columns: keys of tensor memory), from which its
// threads read a row, take the maximum and the exponentials and put them back as bf16 P (beside S or over it), and an output O that the
// tensor core adds P V to from there.  Warps of their own copy K and V tiles (TMA, one ring, K before V) and issue the
// products: S of the next tile and P V of one warpgroup run while the other one is at its exponentials.
// With more than 128 rows the warpgroups take 128 rows each and share every K and V tile; with fewer they take the tiles in
// turn, as if one were another piece of the keys, and meet in shared memory at the end.
// O is only rescaled when a row's maximum has grown by more than 2^8 (l and O always have the same factor); P is then at most 2^8,
// which bf16 holds as well as 1.
// P is rounded to bf16 (2^-8 relative) as the tensor core's operand; l sums the exponentials before that rounding, in fp32.
// Bound: exponentials (128 x 128 per tile and warpgroup at 16 per clock, one in eight by a quartic on the multiply-add pipe) and the
// instructions around them.  4 x 12 x 4096 queries, 8192 keys, d = 64: 617 us, 669 TFLOP/s; without the warpgroups' arithmetic 459.
// 16 heads on 4, 2049 x 10007, masked, d = 128: 181 us, without it 132.  (Two threads per row, half of the keys each, 16 warps: 679 us; two blocks per SM with tiles of 64
// keys: 726 us.)
#include "cross.cuh"
#include "tc_common.cuh"
#include "tc_cross.cuh"
#include "tc_layout.cuh"

using namespace tc;
using namespace tcl;
using namespace tcx;

namespace {

constexpr int CX_WARPS = 8, CXW_TMA = 8, CXW_MMA = 9, CX_T = 384;      // (warps 10, 11 only hand their registers over)
constexpr int CX_REGS_REST = 56, CX_REGS_ROWS = 224;                   // 384 threads x 168 at launch = 128 x 56 + 256 x 224
constexpr uint32_t CX_TMEM = 512;
constexpr float CX_SLACK = 8.f;

template <int D>
struct CxSm {
  static constexpr int PANELS = D / 64, KT = 128, NS = D == 64 ? 8 : 5;      // keys per tile; slots of the ring: a K or V tile each
  static constexpr uint32_t PANEL = KT * 128, SLOT = PANELS * PANEL, QT = PANELS * TILE_BYTES, Q = 0, RING = 2 * QT;
  static constexpr uint32_t MISC = RING + NS * SLOT, TOTAL = MISC + 768;
  // Columns of a warpgroup: S, P (two to a column), O.  At d = 64 P has a place of its own and S is free for the next tile as soon as
  // it has been read; d = 128 has no room for that, there P lies over S.  (Tiles of 64 keys would make room; their S, N = 64, is
  // bound by shared memory: 16 heads on 4, 2049 x 10007, 285 us instead of 228.)
  static constexpr bool OVER = D == 128;
  static constexpr uint32_t S = 0, P = OVER ? 0 : KT, O = OVER ? KT : KT + KT / 2, GROUP = 256;
  static_assert(TOTAL + 1024 <= 232448, "shared memory budget");
  static_assert(QT >= 128 * (8 + 17 * 4), "the warpgroups' exchange");
  static_assert(O + D <= GROUP, "tensor memory");
};
struct CxMs {
  uint64_t full[8], empty[8], s_full[2], s_free[2], p_ready[2], o_full[2], q_ready;
  uint32_t tmem_base;
  int abort_flag;
  uint8_t order[CROSS_RANKED];
};
static_assert(sizeof(CxMs) <= 768, "misc block");

// One piece of work: up to 256 rows of a unit against a piece of its keys.
struct CxWork {
  int unit, piece, b, hk, r0, n, t0, nt;
  bool both;                                           // each warpgroup has rows of its own
};

// MASK: some keys may be hidden anywhere, not only behind a sequence's end.
// Blocks are persistent, one per SM, and take every gridDim.x-th piece of work: the next one's K and V are copied, and its rows of Q,
// while this one's last products and its output are made.  (A block per piece of work: 2.3 us before its first tile and 3.5 behind its last.)
template <int D, bool MASK>
__global__ void __launch_bounds__(CX_T, 1)
tc_cross_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CrossArgs a,
                __nv_bfloat16* __restrict__ Y, TensorAddr ay, float* __restrict__ lse, CrossPart part, int per_unit, int total,
                int* __restrict__ status) {
  using Sm = CxSm<D>;
  constexpr int KT = Sm::KT;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  CxMs* misc = reinterpret_cast<CxMs*>(sm + Sm::MISC);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abortp = &misc->abort_flag;
  const int R = a.g * a.Lq;

  if (threadIdx.x == 0) {
    for (int i = 0; i < Sm::NS; i++) { mbar_init(&misc->full[i], 1); mbar_init(&misc->empty[i], 1); }
    for (int w = 0; w < 2; w++) { mbar_init(&misc->s_full[w], 1); mbar_init(&misc->s_free[w], 4); mbar_init(&misc->p_ready[w], 4); mbar_init(&misc->o_full[w], 1); }
    mbar_init(&misc->q_ready, CX_WARPS);
    misc->abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == CXW_MMA) {
    tmem_alloc(&misc->tmem_base, CX_TMEM);
    tmem_relinquish();
  }
  if (a.ranked) cross_rank(a, reinterpret_cast<int*>(sm + Sm::Q), misc->order);
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem = misc->tmem_base;
  const int kp = (a.d + 63) / 64, vp = (a.dv + 63) / 64;      // panels of 64 columns
  // The block's round-th piece of work: there and back, so that who has the longest of one round has the shortest of the next.
  auto place = [&](int round) { return round * (int)gridDim.x + (round & 1 ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x); };
  auto work_at = [&](int round) {
    CxWork k;
    const int i = place(round), u = i / per_unit, x = i - u * per_unit;
    k.hk = u % a.Hk;
    k.b = a.ranked ? misc->order[u / a.Hk] : u / a.Hk;
    k.unit = k.b * a.Hk + k.hk;
    k.piece = x % part.pieces;
    k.r0 = x / part.pieces * 256;
    k.n = cross_keys(a, k.b);
    const int tiles = (k.n + KT - 1) / KT;
    k.t0 = 0;
    k.nt = tiles;
    if (part.pieces > 1) {
      k.t0 = (int)((int64_t)tiles * k.piece / part.pieces);
      k.nt = (int)((int64_t)tiles * (k.piece + 1) / part.pieces) - k.t0;
    }
    k.both = R - k.r0 > TILE;
    return k;
  };

  if (warp >= CX_WARPS) regs_release<CX_REGS_REST>();
  if (warp == CXW_TMA) {
    if (lane == 0) {
      prefetch_tmap(&tmK); prefetch_tmap(&tmV);
      int issued = 0;
      bool ok = true;
      for (int round = 0; place(round) < total && ok; round++) {
        const CxWork k = work_at(round);
        // (a stride of zero, one entry for all, is a dimension of size one in the tensor map)
        const int ch[2] = {a.ak.sh ? k.hk : 0, a.av.sh ? k.hk : 0}, cb[2] = {a.ak.sb ? k.b : 0, a.av.sb ? k.b : 0};
        for (int i = 0; i < 2 * k.nt; i++, issued++) {
          const int s = issued % Sm::NS, panels = i & 1 ? vp : kp;
          if (!mbar_wait(&misc->empty[s], ((issued / Sm::NS) & 1) ^ 1, abortp, status)) { ok = false; break; }
          uint8_t* base = sm + Sm::RING + s * Sm::SLOT;
          mbar_expect_tx(&misc->full[s], panels * Sm::PANEL);
          for (int p = 0; p < panels; p++)
            tma_load_4d(base + p * Sm::PANEL, i & 1 ? &tmV : &tmK, &misc->full[s], p * 64, (k.t0 + i / 2) * KT, ch[i & 1], cb[i & 1]);
        }
      }
      // nothing of this block may still be in flight when it exits: no copy, and no arrival of a product's completion
      for (int i = max(0, issued - Sm::NS); i < issued; i++) {
        mbar_wait(&misc->full[i % Sm::NS], (i / Sm::NS) & 1, abortp, status, false);
        mbar_wait(&misc->empty[i % Sm::NS], (i / Sm::NS) & 1, abortp, status);
      }
    }
  } else if (warp == CXW_MMA) {
    // The whole warp walks the schedule (waits and descriptor arithmetic stay warp-uniform); an elected lane issues.  (One warp for
    // both warpgroups: with one each, whose short products then alternate on the tensor pipe, 677 us became 714 and 228 us 290.)
    const uint32_t ID_S = idesc_bf16(128, KT, 0, 0), ID_O = idesc_bf16(128, a.dv, 0, 1);
    const uint32_t sR = smem_u32(sm + Sm::RING);
    const int ksteps = a.d / 16;
    const Desc q0 = smem_desc(smem_u32(sm + Sm::Q), 16, 1024, SWZ_128B), k0 = smem_desc(sR, 16, 1024, SWZ_128B), v0 = smem_desc(sR, Sm::PANEL, 1024, SWZ_128B);
    const bool leader = elect_one();
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abortp, status); };
    int kslot = 0, kphase = 0, vslot = 1, vphase = 0;      // where the next K and V tiles are
    int sn[2] = {0, 0}, pn[2] = {0, 0};                // S and P V issued for either warpgroup so far
    bool ok = true, both = false;
    int worked = 0;
    auto issue_s = [&](int w) {                        // S of the next item, which is warpgroup w's
      // as soon as the scores that lie there have been read (OVER: P V of the item before was issued before)
      if (!Sm::OVER && sn[w] > 0 && !wait(&misc->s_free[w], (sn[w] - 1) & 1)) return false;
      if (!wait(&misc->full[kslot], kphase)) return false;
      tcgen05_fence_after();
      if (leader) {
        Desc q = q0, k = k0;
        q.lo += (both ? w : 0) * (Sm::QT / 16);
        k.lo += kslot * (Sm::SLOT / 16);
        issue_rows<D / 16, TILE_BYTES, Sm::PANEL>(tmem + w * Sm::GROUP + Sm::S, q, k, ID_S, ksteps);
        if (!both || w) mma_commit(&misc->empty[kslot]);
        mma_commit(&misc->s_full[w]);
      }
      __syncwarp();
      sn[w]++;
      if (!both || w) {
        kslot += 2;
        if (kslot >= Sm::NS) { kslot -= Sm::NS; kphase ^= 1; }
      }
      return true;
    };
    for (int round = 0; place(round) < total && ok; round++) {
      const CxWork k = work_at(round);
      if (k.nt == 0) continue;
      both = k.both;
      const int items = both ? 2 * k.nt : k.nt;        // item i: warpgroup i & 1, tile i / 2 or i
      ok = wait(&misc->q_ready, worked++ & 1);
      if (ok) ok = issue_s(0) && (items < 2 || issue_s(1));
      auto item = [&](int i, int w) {
        if (!Sm::OVER && i + 2 < items && !issue_s(w)) return false;
        if (!wait(&misc->full[vslot], vphase) || !wait(&misc->p_ready[w], pn[w] & 1)) return false;
        tcgen05_fence_after();
        if (leader) {
          // V: panels of 64 columns (leading offset = their distance), 16 keys per step = 16 rows of 128 bytes
          Desc v = v0;
          v.lo += vslot * (Sm::SLOT / 16);
          issue_cols<KT / 16>(tmem + w * Sm::GROUP + Sm::O, tmem + w * Sm::GROUP + Sm::P, v, ID_O, i > 1);
          if (!both || w) mma_commit(&misc->empty[vslot]);
          // (OVER: the next S tells as much of the products before the last; a phase that nobody waits for is not completed)
          if (!Sm::OVER || i + 2 >= items) mma_commit(&misc->o_full[w]);
        }
        __syncwarp();
        pn[w]++;
        if (!both || w) {
          vslot += 2;
          if (vslot >= Sm::NS) { vslot -= Sm::NS; vphase ^= 1; }
        }
        return !Sm::OVER || i + 2 >= items || issue_s(w);
      };
      for (int i = 0; i < items && ok; i += 2) ok = item(i, 0) && (i + 1 >= items || item(i + 1, 1));
    }
  } else if (warp < CX_WARPS) {
    regs_acquire<CX_REGS_ROWS>();
    const int w = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), tS = lanes + w * Sm::GROUP + Sm::S, tP = lanes + w * Sm::GROUP + Sm::P, tO = lanes + w * Sm::GROUP + Sm::O;
    const float c = fmaxf(a.scale * FS_LOG2E, 1.2e-38f);                // (hidden scores are -inf: 0 would make them NaN)
    // This warpgroup's rows of Q of a piece of work into its place in shared memory, rows and columns that there are none of as zeros.
    // (Every product of S with what lay there is done: this warpgroup's own, or, where both had the first's rows, both.)
    auto fetch = [&](const CxWork& k) {
      if (k.both || w == 0) {
        // a thread has one 16-byte piece of every (128 / CH)-th row
        constexpr int CH = D / 8, STEP = 128 / CH;
        const int ch = threadIdx.x % CH, base = k.r0 + (k.both ? w * TILE : 0);
        int rr = (threadIdx.x & 127) / CH, h = (base + rr) / a.Lq, tok = (base + rr) - h * a.Lq;
        const __nv_bfloat16* Q = static_cast<const __nv_bfloat16*>(a.Q) + k.b * a.aq.sb + (int64_t)k.hk * a.g * a.aq.sh + ch * 8;
        uint8_t* to = sm + Sm::Q + w * Sm::QT + (ch >> 3) * TILE_BYTES;
#pragma unroll 4
        for (; rr < TILE; rr += STEP) {
          const bool some = base + rr < R && ch * 8 < a.d;
          copy16(to + sw128_offset(rr, (ch & 7) * 8), Q + (some ? h * a.aq.sh + tok * a.aq.sl : 0), some);
          tok += STEP;
          if (tok >= a.Lq) { h += tok / a.Lq; tok %= a.Lq; }
        }
      }
    };
    auto fetched = [&]() {
      copies_done();
      fence_proxy_async_smem();
      mbar_arrive_warp(&misc->q_ready, lane);
    };
    int done = 0;                                      // tiles of this warpgroup so far
    int ring = 0;                                      // copies of K and V so far
    int outs = 0;                                      // OVER: pieces of work with tiles of this warpgroup so far
    bool ok = true;
    CxWork next = work_at(0);
    if (next.nt) fetch(next);
    for (int round = 0; place(round) < total; round++) {
      const CxWork k = next;
      const int b = k.b, n = k.n, nt = k.nt;
      const bool both = k.both;
      if (nt) fetched();
      const int first = k.r0 + (both ? w * TILE : 0), r = first + row;  // this thread's row
      const bool idle = first + (warp & 3) * 32 >= R;                   // no row of this warp exists
      const int mine = both ? nt : (nt + 1 - w) / 2;                    // its tiles
      float m = -INFINITY;
      uint32_t l[2] = {0u, 0u};
      // The mask's bytes of a tile are asked for one tile ahead.
      uint8_t look[KT / 32];
      auto peek = [&](int t) {
#pragma unroll
        for (int q = 0; q < KT / 32; q++) {
          const int j = (k.t0 + t) * KT + q * 32 + lane;
          look[q] = j < n ? a.key_mask[b * a.mask_stride + j] : 1;
        }
      };
      if (MASK && mine > 0) peek(both ? 0 : w);
      for (int i = 0; i < mine && ok; i++, done++) {
        const int t = both ? i : 2 * i + w, j0 = (k.t0 + t) * KT;
        uint32_t seen[KT / 32];
        const bool some = MASK || j0 + KT > n;         // some key of the tile may be hidden
        if (some) {
#pragma unroll
          for (int q = 0; q < KT / 32; q++) seen[q] = __ballot_sync(0xffffffffu, j0 + q * 32 + lane < n && (!MASK || look[q] != 0));
          if (!both || w == 0) {
            // what a hidden key's V holds may be anything: zeros in its place, thread = key (one warpgroup does it for both: the
            // other's product is issued behind its own)
            const int at = ring + 2 * t + 1, slot = at % Sm::NS;
            ok = __all_sync(0xffffffffu, mbar_wait(&misc->full[slot], (at / Sm::NS) & 1, abortp, status, false));
            if (ok && row < KT && !(seen[(warp & 3) % (KT / 32)] >> lane & 1u))
              for (int p = 0; p < vp; p++)
                for (int q = 0; q < 8; q++)
                  *reinterpret_cast<uint4*>(sm + Sm::RING + slot * Sm::SLOT + p * Sm::PANEL + row * 128 + q * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
          }
        }
        ok = ok && __all_sync(0xffffffffu, mbar_wait(&misc->s_full[w], done & 1, abortp, status, false));
        if (!ok) break;
        tcgen05_fence_after();
        if (MASK && i + 1 < mine) peek(both ? i + 1 : 2 * i + 2 + w);
        if (!idle) {
          uint32_t s[KT];
#pragma unroll
          for (int q = 0; q < KT; q += 16) tmem_ld16(tS + q, *reinterpret_cast<uint32_t(*)[16]>(s + q));
          tmem_wait_ld();
          if (!Sm::OVER) {
            tcgen05_fence_before();
            mbar_arrive_warp(&misc->s_free[w], lane);
          }
          if (some) {
#pragma unroll
            for (int q = 0; q < KT; q++) s[q] = (seen[q >> 5] >> (q & 31)) & 1u ? s[q] : 0xff800000u;
          }
          float top = __uint_as_float(s[0]);
          {
            float t1 = __uint_as_float(s[1]), t2 = __uint_as_float(s[2]), t3 = __uint_as_float(s[3]);
#pragma unroll
            for (int q = 4; q < KT - 4; q += 8) {
              top = max3n(top, __uint_as_float(s[q]), __uint_as_float(s[q + 1]));
              t1 = max3n(t1, __uint_as_float(s[q + 2]), __uint_as_float(s[q + 3]));
              t2 = max3n(t2, __uint_as_float(s[q + 4]), __uint_as_float(s[q + 5]));
              t3 = max3n(t3, __uint_as_float(s[q + 6]), __uint_as_float(s[q + 7]));
            }
            top = max3n(top, __uint_as_float(s[KT - 4]), __uint_as_float(s[KT - 3]));
            t1 = max3n(t1, __uint_as_float(s[KT - 2]), __uint_as_float(s[KT - 1]));
            top = max3n(max3n(top, t1, t2), t3, t3);
          }
          top *= c;
          // (an infinite score makes the row NaN as its definition does: the quartic below would drop inf - inf)
          if (top == INFINITY) top = __uint_as_float(0x7fc00000u);
          const bool grown = !(top <= m + CX_SLACK) && top != -INFINITY;
          // the product that reads P and adds to O is done (OVER: S came behind it)
          if (!Sm::OVER && i > 0) {
            ok = __all_sync(0xffffffffu, mbar_wait(&misc->o_full[w], (done - 1) & 1, abortp, status, false));
            if (!ok) break;
            tcgen05_fence_after();
          }
          if (__any_sync(0xffffffffu, grown)) {
            const float f = grown ? ex2(m - top) : 1.f;
            if (grown) m = top;
            l[0] = __float_as_uint(__uint_as_float(l[0]) * f);
            l[1] = __float_as_uint(__uint_as_float(l[1]) * f);
            if (i > 0) {
              for (int q = 0; q < a.dv; q += 16) {
                uint32_t o[16];
                tmem_ld16(tO + q, o);
                tmem_wait_ld();
#pragma unroll
                for (int p = 0; p < 16; p++) o[p] = __float_as_uint(__uint_as_float(o[p]) * f);
                tmem_st16(tO + q, o);
              }
            }
          }
          const float base = m == -INFINITY ? 0.f : -m;
#pragma unroll
          for (int q = 0; q < KT; q += 32) {
            uint32_t o[16];
#pragma unroll
            for (int p = 0; p < 32; p += 2) {
              fma2(s[q + p], s[q + p + 1], c, base);
              if ((p & 15) < 14) {                       // (one pair of eight by the quartic: 624 us, as by a cubic; by a quintic 645, none 647, two cubics 632, three 686)
                s[q + p] = __float_as_uint(ex2(__uint_as_float(s[q + p])));
                s[q + p + 1] = __float_as_uint(ex2(__uint_as_float(s[q + p + 1])));
              } else {
                exp2_quartic2<false>(s[q + p], s[q + p + 1]);
              }
              add2(l[0], l[1], __uint_as_float(s[q + p]), __uint_as_float(s[q + p + 1]));
              o[p / 2] = pack_bf16(__uint_as_float(s[q + p]), __uint_as_float(s[q + p + 1]));
            }
            tmem_st16(tP + q / 2, o);
          }
          tmem_wait_st();
        } else {
          if (!Sm::OVER) mbar_arrive_warp(&misc->s_free[w], lane);
          // (in step with the warps that have rows: an arrival below belongs to this tile's product)
          ok = Sm::OVER || i == 0 || __all_sync(0xffffffffu, mbar_wait(&misc->o_full[w], (done - 1) & 1, abortp, status, false));
          if (!ok) break;
        }
        tcgen05_fence_before();
        mbar_arrive_warp(&misc->p_ready[w], lane);
      }
      ring += 2 * nt;
      next.nt = 0;
      if (place(round + 1) < total) next = work_at(round + 1);
      // (a warpgroup's own rows have been read when its last S is there; rows that both have read, only behind the barrier below)
      if (both && next.nt) fetch(next);
      if (ok && mine > 0) ok = __all_sync(0xffffffffu, mbar_wait(&misc->o_full[w], (Sm::OVER ? outs++ : done - 1) & 1, abortp, status, false));
      tcgen05_fence_after();
      float sum = m == -INFINITY ? 0.f : __uint_as_float(l[0]) + __uint_as_float(l[1]);      // (2^-125 per hidden key from the quartic)
      const int h = k.hk * a.g + r / a.Lq, tok = r % a.Lq;
      const int64_t at = ((int64_t)k.unit * part.pieces + k.piece) * R + r;
      __nv_bfloat16* y = Y + b * ay.sb + h * ay.sh + tok * ay.sl;
      // The second warpgroup's sums, where it has worked on the first one's rows: its maximum and sum, then its O 16 columns at a time,
      // where the second one's rows of Q would be.  (Every warp comes to the barriers, also after a wait that ran out.)
      float f0 = 1.f, f1 = 0.f;
      float2* xs = reinterpret_cast<float2*>(sm + Sm::Q + Sm::QT);      // [128]
      float* xo = reinterpret_cast<float*>(xs + 128);                   // [128][17]
      if (!both) {
        if (w == 1) xs[row] = make_float2(m, sum);
        named_bar_sync(3, 256);
        if (w == 0) {
          const float2 other = xs[row];
          const float top = fmaxf(m, other.x), base = top == -INFINITY ? 0.f : top;
          f0 = ex2(m - base); f1 = ex2(other.x - base);
          sum = sum * f0 + other.y * f1;
          m = top;
        }
      }
      const float inv = part.pieces > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
      for (int q = 0; q < a.dv; q += 16) {
        uint32_t o[16] = {};
        if (mine > 0 && ok) {
          tmem_ld16(tO + q, o);
          tmem_wait_ld();
        }
        float x[16];
#pragma unroll
        for (int p = 0; p < 16; p++) x[p] = __uint_as_float(o[p]) * f0;
        if (!both) {
          if (w == 1)
#pragma unroll
            for (int p = 0; p < 16; p++) xo[row * 17 + p] = x[p];
          named_bar_sync(3, 256);
          // (a warpgroup that saw nothing has a factor of zero; its sums are zeros)
          if (w == 0)
#pragma unroll
            for (int p = 0; p < 16; p++) x[p] += xo[row * 17 + p] * f1;
          named_bar_sync(3, 256);
        }
#pragma unroll
        for (int p = 0; p < 16; p++) x[p] *= inv;
        store_row((both || w == 0) && ok && r < R, x, part.pieces > 1 ? part.o + at * a.dv + q : nullptr, y + q);
      }
      tcgen05_fence_before();                          // (O has been read before the next P is handed over)
      if ((both || w == 0) && ok && r < R) {
        if (part.pieces > 1) part.ml[at] = make_float2(m, sum);
        else if (lse) lse[((int64_t)b * a.H + h) * a.Lq + tok] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * FS_LN2;
      }
      __syncwarp();
      if (!both && next.nt) fetch(next);
    }
  }
  tcgen05_fence_before();
  __syncthreads();
  if (warp == CXW_MMA) {
    tcgen05_fence_after();
    tmem_dealloc(tmem, CX_TMEM);
  }
}

template <int D>
int launch(fsharp_ctx* ctx, const CUtensorMap& tmK, const CUtensorMap& tmV, CrossArgs a, void* Y, TensorAddr ay, float* lse, CrossPart part) {
  const int64_t gx = ((int64_t)a.g * a.Lq + 255) / 256 * part.pieces, total = gx * a.B * a.Hk;
  if (total > 0x7fff0000) return FSHARP_E_SHAPE;
  a.ranked = cross_ranked(ctx, a, total);
  const auto kernel = a.key_mask ? tc_cross_kernel<D, true> : tc_cross_kernel<D, false>;
  FS_CUDA_OK(fs_allow_smem(kernel));
  FS_TIME_BEGIN(ctx, FS_K_TC_CROSS);
  kernel<<<dim3((unsigned)(total < ctx->sm_count ? total : ctx->sm_count)), CX_T, CxSm<D>::TOTAL + 1024, ctx->stream>>>(
      tmK, tmV, a, static_cast<__nv_bfloat16*>(Y), ay, lse, part, (int)gx, (int)total, ctx->d_status);
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  return FSHARP_OK;
}

}  // namespace

namespace tchost {
int make_map_rows(CUtensorMap* map, const void* base, TensorAddr a, int B, int H, int L, int inner, int box_rows);
}

// A tensor as a map of boxes of `rows` tokens.  A dimension of size one may carry any stride, which nothing reads; one whose entries are all the
// same (stride zero) becomes a dimension of size one.
int fs_tc_cross_map(CUtensorMap* map, const void* base, TensorAddr t, int B, int H, int L, int inner, int rows) {
  if (t.sh == 0) H = 1;
  if (t.sb == 0) B = 1;
  if (L == 1) t.sl = inner;
  if (H == 1) t.sh = t.sl * L;
  if (B == 1) t.sb = t.sh * H;
  return tchost::make_map_rows(map, base, t, B, H, L, inner, rows);
}

// Pieces that bring the blocks up to what is resident at once, each with 256 keys at least.
int fs_tc_cross_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm) {
  const int64_t R = (int64_t)dm->H / dm->Hk * dm->Lq, blocks = (int64_t)dm->B * dm->Hk * ((R + 255) / 256), some = ((int64_t)dm->Lk + 255) / 256;
  int64_t p = ctx->sm_count / blocks;
  if (p > some) p = some;
  if (p > 64) p = 64;
  return p < 1 ? 1 : (int)p;
}

int fs_tc_cross(fsharp_ctx* ctx, const CrossArgs& a, void* Y, TensorAddr ay, float* lse, CrossPart part) {
  CUtensorMap tmK, tmV;
  const int rows = a.d > 64 || a.dv > 64 ? CxSm<128>::KT : CxSm<64>::KT;
  FS_TRY(fs_tc_cross_map(&tmK, a.K, a.ak, a.B, a.Hk, a.Lk, a.d, rows));
  FS_TRY(fs_tc_cross_map(&tmV, a.V, a.av, a.B, a.Hk, a.Lk, a.dv, rows));
  return a.d > 64 || a.dv > 64 ? launch<128>(ctx, tmK, tmV, a, Y, ay, lse, part) : launch<64>(ctx, tmK, tmV, a, Y, ay, lse, part);
}
