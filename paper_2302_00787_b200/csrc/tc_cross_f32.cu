// Exact cross attention of fp32 tensors, d and dv up to 64, on the tensor cores: every operand is the sum of three bf16 parts
// (split3.cuh), every product the sum of six part products, the small ones first because the accumulator truncates at every
// step.  Sums over many keys or rows leave the accumulator after every tile of 64 and are carried in fp32 registers: kept in it
// they would lose some 2^-25 of their size per step of 16 (8192 keys: 1e-4).  The schedules are those of tc_cross.cu and
// tc_cross_bwd.cu with tiles of 64; K, V (and, backward, Q and dY) are split once by cross_split_kernel, P and dS by the threads
// that make them.  An infinity that is seen gives NaN (its parts do), values below 2^-109 in magnitude carry fewer than 24 bits.
// Bound: the tensor pipe and shared memory (six products of 128 x 64 x 64 each; 4 x 8 x 701 x 1501, d = 32, forward: multiply-add
// tiles 202 us).
#include "cross.cuh"
#include "split3.cuh"
#include "tc_common.cuh"
#include "tc_cross.cuh"
#include "tc_layout.cuh"

using namespace tc;
using namespace tcl;
using namespace tcx;

int fs_tc_cross_map(CUtensorMap* map, const void* base, TensorAddr t, int B, int H, int L, int inner, int rows);

namespace {

constexpr int CF_WARPS = 8, CFW_TMA = 8, CFW_MMA = 9, CF_T = 384;      // (warps 10, 11 only hand their registers over)
constexpr int CF_REGS_REST = 56, CF_REGS_ROWS = 224;                   // 384 threads x 168 at launch = 128 x 56 + 256 x 224
constexpr int KT = 64;                                                  // keys or rows of a walked tile
constexpr uint32_t SMALL = 8192, SMALL3 = 3 * SMALL;                    // 64 rows x 128 bytes, and its three parts
constexpr uint32_t BIG = TILE_BYTES, BIG3 = 3 * BIG;                    // 128 rows
constexpr uint32_t CF_TMEM = 512;

// The part products of two operands, smallest first: A's part, B's part.
__device__ constexpr int PA[6] = {2, 0, 1, 1, 0, 0}, PB[6] = {0, 2, 1, 0, 1, 0};

// ------------------------------------------------------------------------------------------ parts
// Up to four tensors x [B,H,L,d] fp32 -> their parts [3][B H][L][d] bf16, one after the other; eight values per thread.
struct SplitJob {
  const float* x;
  TensorAddr ax;
  int64_t rows, end;           // rows of all heads; threads of this tensor and of those before it
  __nv_bfloat16* parts;
  int H, L, d;
};
struct SplitJobs {
  SplitJob job[4];
};
__global__ void __launch_bounds__(256)
cross_split_kernel(const __grid_constant__ SplitJobs jobs, int n) {
  int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  int t = 0;
  while (t < n && i >= jobs.job[t].end) t++;
  if (t == n) return;
  const SplitJob& j = jobs.job[t];
  if (t) i -= jobs.job[t - 1].end;
  const int q = j.d / 8, e = (int)(i % q) * 8;
  const int64_t row = i / q;
  const float* p = j.x + row / ((int64_t)j.H * j.L) * j.ax.sb + row / j.L % j.H * j.ax.sh + row % j.L * j.ax.sl + e;
  float v[8];
  *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(p);
  *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(p + 4);
  uint4 h, m, l;
  split3::split8(v, h, m, l);
  const int64_t all = j.rows * j.d, at = row * j.d + e;
  *reinterpret_cast<uint4*>(j.parts + at) = h;
  *reinterpret_cast<uint4*>(j.parts + all + at) = m;
  *reinterpret_cast<uint4*>(j.parts + 2 * all + at) = l;
}

// Rows r0 .. r0 + 127 of a unit's packed rows of X, split, into a [3][128 x 64] tile by 256 threads (thread `t`).
__device__ __forceinline__ void split_rows(uint8_t* to, const void* X, const TensorAddr& ax, const CrossArgs& a, int b, int hk, int r0, int width, int t) {
  const int R = a.g * a.Lq;
  for (int i = t; i < TILE * 8; i += 256) {
    const int rr = i >> 3, ch = i & 7, r = r0 + rr;
    float v[8] = {};
    if (r < R && ch * 8 < width) {
      const float* p = static_cast<const float*>(X) + b * ax.sb + (int64_t)(hk * a.g + r / a.Lq) * ax.sh + (int64_t)(r % a.Lq) * ax.sl + ch * 8;
      *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(p);
      *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(p + 4);
    }
    uint4 h, m, l;
    split3::split8(v, h, m, l);
    uint8_t* at = to + sw128_offset(rr, ch * 8);
    *reinterpret_cast<uint4*>(at) = h;
    *reinterpret_cast<uint4*>(at + BIG) = m;
    *reinterpret_cast<uint4*>(at + 2 * BIG) = l;
  }
}

// D [128 x N] = A B^T, both [3][rows x 64] in shared memory, K-major, their parts A_PART and B_PART bytes apart
template <uint32_t A_PART, uint32_t B_PART>
__device__ __forceinline__ void issue_rows6(uint32_t d_tmem, Desc a, Desc b, uint32_t idesc, int steps) {
#pragma unroll
  for (int p = 0; p < 6; p++)
#pragma unroll
    for (int k = 0; k < 4; k++)
      if (k < steps) mma_bf16_lh(d_tmem, a.lo + (PA[p] * A_PART + k * 32) / 16, a.hi, b.lo + (PB[p] * B_PART + k * 32) / 16, b.hi, idesc, p + k > 0);
}
// D [128 x N] = A B, A [3][128 x 64] in tensor memory (32 columns per part), B [3][64 rows x 128 bytes] with its rows as the contraction
__device__ __forceinline__ void issue_cols6(uint32_t d_tmem, uint32_t a_tmem, Desc b, uint32_t idesc) {
#pragma unroll
  for (int p = 0; p < 6; p++)
#pragma unroll
    for (int k = 0; k < 4; k++)
      mma_bf16_ta_lh(d_tmem, a_tmem + PA[p] * 32 + k * 8, b.lo + (PB[p] * SMALL + k * 2048) / 16, b.hi, idesc, p + k > 0);
}
// N values (a multiple of 32) of this thread's row as parts into tensor memory: N / 2 columns of each part from `to` on
template <int N>
__device__ __forceinline__ void store_parts(uint32_t to, const uint32_t* x) {
#pragma unroll
  for (int q = 0; q < N; q += 32) {
    uint32_t h[16], m[16], l[16];
#pragma unroll
    for (int k = 0; k < 16; k++) split3::split_pair(__uint_as_float(x[q + 2 * k]), __uint_as_float(x[q + 2 * k + 1]), h[k], m[k], l[k]);
    tmem_st16(to + q / 2, h);
    tmem_st16(to + 32 + q / 2, m);
    tmem_st16(to + 64 + q / 2, l);
  }
}
// acc += the tile's sums, columns 0 .. width - 1 of N
template <int N>
__device__ __forceinline__ void fold(float (&acc)[N], uint32_t from, int width) {
#pragma unroll
  for (int q = 0; q < N; q += 16)
    if (q < width) {
      uint32_t o[16];
      tmem_ld16(from + q, o);
      tmem_wait_ld();
#pragma unroll
      for (int k = 0; k < 16; k++) acc[q + k] += __uint_as_float(o[k]);
    }
}

// ------------------------------------------------------------------------------------------ forward
struct FwSm {
  static constexpr int NS = 4;
  static constexpr uint32_t Q = 0, RING = 2 * BIG3, MISC = RING + NS * SMALL3, TOTAL = MISC + 512;
  static constexpr uint32_t S = 0, P = 64, O = 160, GROUP = 256;        // columns of a warpgroup
  static_assert(TOTAL + 1024 <= 232448, "shared memory budget");
  static_assert(NS * SMALL3 >= 128 * 65 * 4 + 1024, "the warpgroups' exchange");
};
struct FwMs {
  uint64_t full[4], empty[4], s_full[2], s_free[2], p_ready[2], o_full[2], q_ready;
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(FwMs) <= 512, "misc block");

__global__ void __launch_bounds__(CF_T, 1)
tc_cross_f32_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CrossArgs a,
                    float* __restrict__ Y, TensorAddr ay, float* __restrict__ lse, CrossPart part, int* __restrict__ status) {
  using Sm = FwSm;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  FwMs* misc = reinterpret_cast<FwMs*>(sm + Sm::MISC);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abortp = &misc->abort_flag;
  const int unit = cross_unit(a, reinterpret_cast<int*>(sm + Sm::Q)), piece = blockIdx.x % part.pieces, r0 = (int)(blockIdx.x / part.pieces) * 256;
  const int b = unit / a.Hk, hk = unit % a.Hk, R = a.g * a.Lq;
  const int n = cross_keys(a, b), tiles = (n + KT - 1) / KT;
  const int t0 = (int)((int64_t)tiles * piece / part.pieces), nt = (int)((int64_t)tiles * (piece + 1) / part.pieces) - t0;
  const bool both = R - r0 > TILE;                     // each warpgroup has rows of its own
  const int items = both ? 2 * nt : nt;                // item i: warpgroup i & 1, tile i / 2 or i

  if (threadIdx.x == 0) {
    for (int i = 0; i < Sm::NS; i++) { mbar_init(&misc->full[i], 1); mbar_init(&misc->empty[i], 1); }
    for (int w = 0; w < 2; w++) { mbar_init(&misc->s_full[w], 1); mbar_init(&misc->s_free[w], 4); mbar_init(&misc->p_ready[w], 4); mbar_init(&misc->o_full[w], 1); }
    mbar_init(&misc->q_ready, CF_WARPS);
    misc->abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == CFW_MMA) {
    tmem_alloc(&misc->tmem_base, CF_TMEM);
    tmem_relinquish();
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem = misc->tmem_base;

  if (warp >= CF_WARPS) regs_release<CF_REGS_REST>();
  if (warp == CFW_TMA) {
    if (lane == 0) {
      prefetch_tmap(&tmK); prefetch_tmap(&tmV);
      int i = 0;
      for (; i < 2 * nt; i++) {
        const int s = i % Sm::NS, tok = (t0 + i / 2) * KT;
        if (!mbar_wait(&misc->empty[s], ((i / Sm::NS) & 1) ^ 1, abortp, status)) break;
        mbar_expect_tx(&misc->full[s], SMALL3);
        for (int p = 0; p < 3; p++) tma_load_4d(sm + Sm::RING + s * SMALL3 + p * SMALL, i & 1 ? &tmV : &tmK, &misc->full[s], 0, tok, unit, p);
      }
      // nothing of this block may still be in flight when it exits: no copy, and no arrival of a product's completion
      for (int k = max(0, i - Sm::NS); k < i; k++) {
        mbar_wait(&misc->full[k % Sm::NS], (k / Sm::NS) & 1, abortp, status, false);
        mbar_wait(&misc->empty[k % Sm::NS], (k / Sm::NS) & 1, abortp, status);
      }
    }
  } else if (warp == CFW_MMA) {
    constexpr uint32_t ID_S = idesc_bf16(128, KT, 0, 0);
    const uint32_t ID_O = idesc_bf16(128, a.dv, 0, 1);
    const uint32_t sR = smem_u32(sm + Sm::RING);
    const Desc q0 = smem_desc(smem_u32(sm + Sm::Q), 16, 1024, SWZ_128B), k0 = smem_desc(sR, 16, 1024, SWZ_128B), v0 = smem_desc(sR, SMALL, 1024, SWZ_128B);
    const int ks = a.d / 16;
    const bool leader = elect_one();
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abortp, status); };
    int kslot = 0, kphase = 0, vslot = 1, vphase = 0;      // where the next K and V tiles are
    auto issue_s = [&](int w) {                        // S of the next item, which is warpgroup w's
      if (!wait(&misc->full[kslot], kphase)) return false;
      tcgen05_fence_after();
      if (leader) {
        Desc q = q0, k = k0;
        q.lo += (both ? w : 0) * (BIG3 / 16);
        k.lo += kslot * (SMALL3 / 16);
        issue_rows6<BIG, SMALL>(tmem + w * Sm::GROUP + Sm::S, q, k, ID_S, ks);
        if (!both || w) mma_commit(&misc->empty[kslot]);
        mma_commit(&misc->s_full[w]);
      }
      __syncwarp();
      if (!both || w) {
        kslot += 2;
        if (kslot >= Sm::NS) { kslot -= Sm::NS; kphase ^= 1; }
      }
      return true;
    };
    bool ok = nt > 0 && wait(&misc->q_ready, 0);
    if (ok) ok = issue_s(0) && (items < 2 || issue_s(1));
    auto item = [&](int i, int w) {
      // S of the item after the next, as soon as the scores that lie there have been read
      if (i + 2 < items && (!wait(&misc->s_free[w], (i >> 1) & 1) || !issue_s(w))) return false;
      if (!wait(&misc->full[vslot], vphase) || !wait(&misc->p_ready[w], (i >> 1) & 1)) return false;
      tcgen05_fence_after();
      if (leader) {
        Desc v = v0;
        v.lo += vslot * (SMALL3 / 16);
        issue_cols6(tmem + w * Sm::GROUP + Sm::O, tmem + w * Sm::GROUP + Sm::P, v, ID_O);
        if (!both || w) mma_commit(&misc->empty[vslot]);
        mma_commit(&misc->o_full[w]);
      }
      __syncwarp();
      if (!both || w) {
        vslot += 2;
        if (vslot >= Sm::NS) { vslot -= Sm::NS; vphase ^= 1; }
      }
      return true;
    };
    for (int i = 0; i < items && ok; i += 2) ok = item(i, 0) && (i + 1 >= items || item(i + 1, 1));
  } else if (warp < CF_WARPS) {
    regs_acquire<CF_REGS_ROWS>();
    const int w = warp >> 2, row = (warp & 3) * 32 + lane;
    split_rows(sm + Sm::Q, a.Q, a.aq, a, b, hk, r0, a.d, threadIdx.x);
    if (both) split_rows(sm + Sm::Q + BIG3, a.Q, a.aq, a, b, hk, r0 + TILE, a.d, threadIdx.x);
    fence_proxy_async_smem();
    mbar_arrive_warp(&misc->q_ready, lane);
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + w * Sm::GROUP;
    const int first = r0 + (both ? w * TILE : 0), r = first + row;      // this thread's row
    const bool idle = first + (warp & 3) * 32 >= R;                     // no row of this warp exists
    const int mine = both ? nt : (nt + 1 - w) / 2;                      // its tiles
    const float c = fmaxf(a.scale * FS_LOG2E, 1.2e-38f);                // (hidden scores are -inf: 0 would make them NaN)
    float m = -INFINITY, o[64];
#pragma unroll
    for (int k = 0; k < 64; k++) o[k] = 0.f;
    uint32_t l[2] = {0u, 0u};
    bool ok = true;
    uint8_t look[2];                                                    // the mask's bytes of a tile, asked for one tile ahead
    auto peek = [&](int t) {
#pragma unroll
      for (int q = 0; q < 2; q++) {
        const int j = (t0 + t) * KT + q * 32 + lane;
        look[q] = a.key_mask && j < n ? a.key_mask[b * a.mask_stride + j] : 1;
      }
    };
    if (mine > 0) peek(both ? 0 : w);
    for (int i = 0; i < mine; i++) {
      const int t = both ? i : 2 * i + w, j0 = (t0 + t) * KT;
      uint32_t seen[2];
      const bool some = a.key_mask != nullptr || j0 + KT > n;
      if (some) {
#pragma unroll
        for (int q = 0; q < 2; q++) seen[q] = __ballot_sync(0xffffffffu, j0 + q * 32 + lane < n && look[q] != 0);
      }
      if (i + 1 < mine) peek(both ? i + 1 : 2 * i + 2 + w);
      ok = __all_sync(0xffffffffu, mbar_wait(&misc->s_full[w], i & 1, abortp, status, false));
      if (!ok) break;
      tcgen05_fence_after();
      uint32_t s[KT];
      if (!idle) {
#pragma unroll
        for (int q = 0; q < KT; q += 16) tmem_ld16(lanes + Sm::S + q, *reinterpret_cast<uint32_t(*)[16]>(s + q));
        tmem_wait_ld();
      }
      tcgen05_fence_before();
      mbar_arrive_warp(&misc->s_free[w], lane);
      // the product that reads P is done; its sums join the others
      if (i > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(&misc->o_full[w], (i - 1) & 1, abortp, status, false));
        if (!ok) break;
        tcgen05_fence_after();
        if (!idle) fold<64>(o, lanes + Sm::O, a.dv);
      }
      if (some && (!both || w == 0)) {
        // What a hidden key's V holds may be anything: zeros in its place, a thread per key (one warpgroup does it for both: the
        // other's product is issued behind its own).  Here, behind the product before, and not earlier: with tiles in turn the slot held
        // this warpgroup's tile before, and until that one is known to have come, the wait below could be for its phase.
        const int slot = (2 * t + 1) % Sm::NS;
        ok = __all_sync(0xffffffffu, mbar_wait(&misc->full[slot], ((2 * t + 1) / Sm::NS) & 1, abortp, status, false));
        if (!ok) break;
        if (row < KT && !(seen[warp & 1] >> lane & 1u))
          for (int p = 0; p < 3; p++)
            for (int k = 0; k < 8; k++) *reinterpret_cast<uint4*>(sm + Sm::RING + slot * SMALL3 + p * SMALL + row * 128 + k * 16) = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
      }
      if (!idle) {
        if (some) {
#pragma unroll
          for (int q = 0; q < KT; q++) s[q] = (seen[q >> 5] >> (q & 31)) & 1u ? s[q] : 0xff800000u;
        }
        float top = max3n(__uint_as_float(s[0]), __uint_as_float(s[1]), __uint_as_float(s[2])), t1 = __uint_as_float(s[3]);
#pragma unroll
        for (int q = 4; q < KT; q += 4) {
          top = max3n(top, __uint_as_float(s[q]), __uint_as_float(s[q + 1]));
          t1 = max3n(t1, __uint_as_float(s[q + 2]), __uint_as_float(s[q + 3]));
        }
        top = max3n(top, t1, t1) * c;
        if (top == INFINITY) top = __uint_as_float(0x7fc00000u);        // (the row is NaN, as inf - inf)
        if (!(top <= m) && top != -INFINITY) {
          const float f = ex2(m - top);
          m = top;
          l[0] = __float_as_uint(__uint_as_float(l[0]) * f);
          l[1] = __float_as_uint(__uint_as_float(l[1]) * f);
#pragma unroll
          for (int k = 0; k < 64; k++) o[k] *= f;
        }
        __syncwarp();
        const float base = m == -INFINITY ? 0.f : -m;
#pragma unroll
        for (int k = 0; k < KT; k += 2) {
          fma2(s[k], s[k + 1], c, base);
          s[k] = __float_as_uint(ex2(__uint_as_float(s[k])));
          s[k + 1] = __float_as_uint(ex2(__uint_as_float(s[k + 1])));
          add2(l[0], l[1], __uint_as_float(s[k]), __uint_as_float(s[k + 1]));
        }
        store_parts<KT>(lanes + Sm::P, s);
        tmem_wait_st();
      }
      tcgen05_fence_before();
      mbar_arrive_warp(&misc->p_ready[w], lane);
    }
    if (ok && mine > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait(&misc->o_full[w], (mine - 1) & 1, abortp, status, false));
      tcgen05_fence_after();
      if (ok && !idle) fold<64>(o, lanes + Sm::O, a.dv);
    }
    float sum = __uint_as_float(l[0]) + __uint_as_float(l[1]);
    if (!both) {
      // (every warp comes to the barriers, also after a wait that ran out; behind the first one no product reads the ring)
      float* xo = reinterpret_cast<float*>(sm + Sm::RING);              // [128][65]
      float2* xm = reinterpret_cast<float2*>(sm + Sm::RING + 128 * 65 * 4);
      named_bar_sync(3, 256);
      if (w == 1) {
#pragma unroll
        for (int k = 0; k < 64; k++) xo[row * 65 + k] = o[k];
        xm[row] = make_float2(m, sum);
      }
      named_bar_sync(3, 256);
      if (w == 0) {
        const float2 other = xm[row];
        const float top = fmaxf(m, other.x), base = top == -INFINITY ? 0.f : top, f0 = ex2(m - base), f1 = ex2(other.x - base);
        sum = sum * f0 + other.y * f1;
        m = top;
#pragma unroll
        for (int k = 0; k < 64; k++) o[k] = o[k] * f0 + xo[row * 65 + k] * f1;
      }
    }
    if ((both || w == 0) && ok && r < R) {
      const int h = hk * a.g + r / a.Lq, tok = r % a.Lq;
      const float inv = part.pieces > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
      const int64_t at = ((int64_t)unit * part.pieces + piece) * R + r;
      float* y = part.pieces > 1 ? part.o + at * a.dv : Y + b * ay.sb + h * ay.sh + tok * ay.sl;
#pragma unroll
      for (int k = 0; k < 64; k += 4)
        if (k < a.dv) *reinterpret_cast<float4*>(y + k) = make_float4(o[k] * inv, o[k + 1] * inv, o[k + 2] * inv, o[k + 3] * inv);
      if (part.pieces > 1) part.ml[at] = make_float2(m, sum);
      else if (lse) lse[((int64_t)b * a.H + h) * a.Lq + tok] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * FS_LN2;
    }
    __syncwarp();
  }
  tcgen05_fence_before();
  __syncthreads();
  if (warp == CFW_MMA) {
    tcgen05_fence_after();
    tmem_dealloc(tmem, CF_TMEM);
  }
}

// ------------------------------------------------------------------------------------------ dK, dV
// Per 128 keys, over the rows in tiles of 64: the products in the order dV, next S^T, dK, next dP^T, each warpgroup half of a tile's rows.
struct FkSm {
  static constexpr int NS = 2;
  static constexpr uint32_t K = 0, V = BIG3, Q = 2 * BIG3, G = Q + NS * SMALL3, STAT = G + NS * SMALL3, MISC = STAT + NS * 512, TOTAL = MISC + 512;
  static constexpr uint32_t S = 0, DP = 64, P = 128, DS = 224, DV = 320, DK = 384;      // columns
  static_assert(TOTAL + 1024 <= 232448, "shared memory budget");
};
struct FkMs {
  uint64_t q_full[2], q_empty[2], g_full[2], g_empty[2], s_full, p_ready, dp_full, ds_ready, kv_full, done;
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(FkMs) <= 512, "misc block");

__global__ void __launch_bounds__(CF_T, 1)
tc_cross_f32_dkv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmK,
                        const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CrossArgs a, const __grid_constant__ CrossGrad gr,
                        int* __restrict__ status) {
  using Sm = FkSm;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  FkMs* misc = reinterpret_cast<FkMs*>(sm + Sm::MISC);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abortp = &misc->abort_flag;
  const int unit = blockIdx.y, piece = blockIdx.x % gr.kv_pieces, j0 = (int)(blockIdx.x / gr.kv_pieces) * TILE;
  const int b = unit / a.Hk, hk = unit % a.Hk, n = cross_keys(a, b);
  const int per = (a.Lq + KT - 1) / KT;                // row tiles: those of the first query head of the group, of the second, ...
  const int64_t tiles = j0 < n ? (int64_t)a.g * per : 0;
  const int t0 = (int)(tiles * piece / gr.kv_pieces), items = (int)(tiles * (piece + 1) / gr.kv_pieces) - t0;

  if (threadIdx.x == 0) {
    for (int i = 0; i < Sm::NS; i++) { mbar_init(&misc->q_full[i], 1); mbar_init(&misc->q_empty[i], 1); mbar_init(&misc->g_full[i], 1); mbar_init(&misc->g_empty[i], 1); }
    mbar_init(&misc->s_full, 1);
    mbar_init(&misc->dp_full, 1);
    mbar_init(&misc->p_ready, CF_WARPS);
    mbar_init(&misc->ds_ready, CF_WARPS);
    mbar_init(&misc->kv_full, 1);
    mbar_init(&misc->done, 1);
    misc->abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == CFW_MMA) {
    tmem_alloc(&misc->tmem_base, CF_TMEM);
    tmem_relinquish();
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem = misc->tmem_base;

  if (warp >= CF_WARPS) regs_release<CF_REGS_REST>();
  if (warp == CFW_TMA) {
    if (lane == 0 && items > 0) {
      prefetch_tmap(&tmQ); prefetch_tmap(&tmG); prefetch_tmap(&tmK); prefetch_tmap(&tmV);
      mbar_expect_tx(&misc->kv_full, 2 * BIG3);
      for (int p = 0; p < 3; p++) {
        tma_load_4d(sm + Sm::K + p * BIG, &tmK, &misc->kv_full, 0, j0, unit, p);
        tma_load_4d(sm + Sm::V + p * BIG, &tmV, &misc->kv_full, 0, j0, unit, p);
      }
      int i = 0;
      for (; i < items; i++) {
        const int s = i % Sm::NS, h = hk * a.g + (t0 + i) / per, t = (t0 + i) % per, bh = b * a.H + h;
        const uint32_t parity = ((i / Sm::NS) & 1) ^ 1;
        // (dY of a tile is done with before its Q is)
        if (!mbar_wait(&misc->q_empty[s], parity, abortp, status) || !mbar_wait(&misc->g_empty[s], parity, abortp, status)) break;
        mbar_expect_tx(&misc->q_full[s], SMALL3 + 512);
        for (int p = 0; p < 3; p++) tma_load_4d(sm + Sm::Q + s * SMALL3 + p * SMALL, &tmQ, &misc->q_full[s], 0, t * KT, bh, p);
        const float* st = gr.stat + (int64_t)bh * cross_stat_floats(a.Lq) + (int64_t)(t >> 1) * 256 + (t & 1) * 64;
        bulk_load(sm + Sm::STAT + s * 512, st, 256, &misc->q_full[s]);
        bulk_load(sm + Sm::STAT + s * 512 + 256, st + 128, 256, &misc->q_full[s]);
        mbar_expect_tx(&misc->g_full[s], SMALL3);
        for (int p = 0; p < 3; p++) tma_load_4d(sm + Sm::G + s * SMALL3 + p * SMALL, &tmG, &misc->g_full[s], 0, t * KT, bh, p);
      }
      // nothing of this block may still be in flight when it exits: no copy, and no arrival of a product's completion
      mbar_wait(&misc->kv_full, 0, abortp, status, false);
      for (int k = max(0, i - Sm::NS); k < i; k++) {
        const uint32_t parity = (k / Sm::NS) & 1;
        mbar_wait(&misc->q_full[k % Sm::NS], parity, abortp, status, false);
        mbar_wait(&misc->g_full[k % Sm::NS], parity, abortp, status, false);
        mbar_wait(&misc->q_empty[k % Sm::NS], parity, abortp, status);
        mbar_wait(&misc->g_empty[k % Sm::NS], parity, abortp, status);
      }
    }
  } else if (warp == CFW_MMA) {
    constexpr uint32_t ID_S = idesc_bf16(128, KT, 0, 0);
    const uint32_t ID_V = idesc_bf16(128, a.dv, 0, 1), ID_K = idesc_bf16(128, a.d, 0, 1);
    const uint32_t sQ = smem_u32(sm + Sm::Q), sG = smem_u32(sm + Sm::G);
    const Desc k0 = smem_desc(smem_u32(sm + Sm::K), 16, 1024, SWZ_128B), v0 = smem_desc(smem_u32(sm + Sm::V), 16, 1024, SWZ_128B);
    const Desc q0 = smem_desc(sQ, 16, 1024, SWZ_128B), g0 = smem_desc(sG, 16, 1024, SWZ_128B);
    const Desc qt = smem_desc(sQ, SMALL, 1024, SWZ_128B), gt = smem_desc(sG, SMALL, 1024, SWZ_128B);      // their rows as the contraction
    const int ks = a.d / 16, vs = a.dv / 16;
    const bool leader = elect_one();
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abortp, status); };
    auto issue = [&](uint64_t* full, int i, Desc left, Desc right, uint32_t to, int steps, uint64_t* then) {
      const int s = i % Sm::NS;
      if (!wait(full + s, (i / Sm::NS) & 1)) return false;
      tcgen05_fence_after();
      if (leader) {
        right.lo += s * (SMALL3 / 16);
        issue_rows6<BIG, SMALL>(tmem + to, left, right, ID_S, steps);
        mma_commit(then);
      }
      __syncwarp();
      return true;
    };
    auto issue_s = [&](int i) { return issue(misc->q_full, i, k0, q0, Sm::S, ks, &misc->s_full); };
    auto issue_dp = [&](int i) { return issue(misc->g_full, i, v0, g0, Sm::DP, vs, &misc->dp_full); };
    bool ok = items > 0 && wait(&misc->kv_full, 0) && issue_s(0) && issue_dp(0);
    for (int i = 0; i < items && ok; i++) {
      const int s = i % Sm::NS;
      if (!(ok = wait(&misc->p_ready, i & 1))) break;
      tcgen05_fence_after();
      if (leader) {
        Desc g = gt;
        g.lo += s * (SMALL3 / 16);
        issue_cols6(tmem + Sm::DV, tmem + Sm::P, g, ID_V);
        mma_commit(&misc->g_empty[s]);
      }
      __syncwarp();
      if (i + 1 < items && !(ok = issue_s(i + 1))) break;
      if (!(ok = wait(&misc->ds_ready, i & 1))) break;
      tcgen05_fence_after();
      if (leader) {
        Desc q = qt;
        q.lo += s * (SMALL3 / 16);
        issue_cols6(tmem + Sm::DK, tmem + Sm::DS, q, ID_K);
        mma_commit(&misc->q_empty[s]);
        if (i == items - 1) mma_commit(&misc->done);
      }
      __syncwarp();
      if (i + 1 < items) ok = issue_dp(i + 1);
    }
  } else if (warp < CF_WARPS) {
    regs_acquire<CF_REGS_ROWS>();
    const int w = warp >> 2, row = (warp & 3) * 32 + lane;      // w: which half of the tile's rows; and the first carries dV, the second dK
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const float c = a.scale * FS_LOG2E;
    float acc[64];
#pragma unroll
    for (int k = 0; k < 64; k++) acc[k] = 0.f;
    bool ok = true;
    for (int i = 0; i < items; i++) {
      const int s = i % Sm::NS;
      // (what a hidden key holds, NaNs too, stays in its own row of S^T, dP^T and of the sums, and is dropped at the end)
      ok = __all_sync(0xffffffffu, mbar_wait(&misc->s_full, i & 1, abortp, status, false) &&
                                       mbar_wait(&misc->q_full[s], (i / Sm::NS) & 1, abortp, status, false));
      if (!ok) break;
      tcgen05_fence_after();
      const float* st = reinterpret_cast<const float*>(sm + Sm::STAT + s * 512) + w * 32;
      uint32_t x[32], g[32];
      tmem_ld16(lanes + Sm::S + w * 32, *reinterpret_cast<uint32_t(*)[16]>(x));
      tmem_ld16(lanes + Sm::S + w * 32 + 16, *reinterpret_cast<uint32_t(*)[16]>(x + 16));
      tmem_wait_ld();
#pragma unroll
      for (int k = 0; k < 32; k += 4) {
        const float4 nl = *reinterpret_cast<const float4*>(st + k);
        fma2v(x[k], x[k + 1], c, nl.x, nl.y);
        fma2v(x[k + 2], x[k + 3], c, nl.z, nl.w);
#pragma unroll
        for (int q = 0; q < 4; q++) x[k + q] = __float_as_uint(ex2(__uint_as_float(x[k + q])));
      }
      store_parts<32>(lanes + Sm::P + w * 16, x);
      // S^T of this tile came behind dV of the last one, dP^T behind its dK: they are there, and free when P and dS are handed over
      if (i > 0 && w == 0) fold<64>(acc, lanes + Sm::DV, a.dv);
      tmem_wait_st();
      tcgen05_fence_before();
      mbar_arrive_warp(&misc->p_ready, lane);
      ok = __all_sync(0xffffffffu, mbar_wait(&misc->dp_full, i & 1, abortp, status, false));
      if (!ok) break;
      tcgen05_fence_after();
      tmem_ld16(lanes + Sm::DP + w * 32, *reinterpret_cast<uint32_t(*)[16]>(g));
      tmem_ld16(lanes + Sm::DP + w * 32 + 16, *reinterpret_cast<uint32_t(*)[16]>(g + 16));
      tmem_wait_ld();
#pragma unroll
      for (int k = 0; k < 32; k += 4) {
        const float4 nd = *reinterpret_cast<const float4*>(st + 64 + k);
        addmul2(g[k], g[k + 1], nd.x, nd.y, x[k], x[k + 1]);
        addmul2(g[k + 2], g[k + 3], nd.z, nd.w, x[k + 2], x[k + 3]);
      }
      store_parts<32>(lanes + Sm::DS + w * 16, g);
      if (i > 0 && w == 1) fold<64>(acc, lanes + Sm::DK, a.d);
      tmem_wait_st();
      tcgen05_fence_before();
      mbar_arrive_warp(&misc->ds_ready, lane);
    }
    if (ok && items > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait(&misc->done, 0, abortp, status, false));
      tcgen05_fence_after();
      if (ok) fold<64>(acc, lanes + (w ? Sm::DK : Sm::DV), w ? a.d : a.dv);
    }
    const int j = j0 + row, width = w ? a.d : a.dv;
    if (ok && j < a.Lk) {
      const float f = w ? a.scale : 1.f;
      const bool on = cross_seen(a, b, j, n);
      const TensorAddr to = w ? gr.adk : gr.adv;
      float* out = gr.pkv ? gr.pkv + (((int64_t)piece * a.B * a.Hk + unit) * a.Lk + j) * (a.d + a.dv) + (w ? 0 : a.d)
                          : static_cast<float*>(w ? gr.dK : gr.dV) + b * to.sb + hk * to.sh + j * to.sl;
#pragma unroll
      for (int k = 0; k < 64; k += 4)
        if (k < width)
          *reinterpret_cast<float4*>(out + k) = on ? make_float4(acc[k] * f, acc[k + 1] * f, acc[k + 2] * f, acc[k + 3] * f) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncwarp();
  }
  tcgen05_fence_before();
  __syncthreads();
  if (warp == CFW_MMA) {
    tcgen05_fence_after();
    tmem_dealloc(tmem, CF_TMEM);
  }
}

// ------------------------------------------------------------------------------------------ dQ
// Per 128 rows, over the keys in tiles of 64, each warpgroup half of a tile's keys: next S and next dP are made while dS is.
struct FqSm {
  static constexpr int NS = 2;
  static constexpr uint32_t Q = 0, G = BIG3, K = 2 * BIG3, V = K + NS * SMALL3, MISC = V + NS * SMALL3, TOTAL = MISC + 512;
  static constexpr uint32_t S = 0, DP = 64, DS = 128, DQ = 224;         // columns
  static_assert(TOTAL + 1024 <= 232448, "shared memory budget");
};
struct FqMs {
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full, s_free, dp_full, dp_free, ds_ready, dq_done, q_ready;
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(FqMs) <= 512, "misc block");

__global__ void __launch_bounds__(CF_T, 1)
tc_cross_f32_dq_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CrossArgs a,
                       const __grid_constant__ CrossGrad gr, int* __restrict__ status) {
  using Sm = FqSm;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  FqMs* misc = reinterpret_cast<FqMs*>(sm + Sm::MISC);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abortp = &misc->abort_flag;
  const int unit = cross_unit(a, reinterpret_cast<int*>(sm + Sm::Q)), piece = blockIdx.x % gr.q_pieces, r0 = (int)(blockIdx.x / gr.q_pieces) * TILE;
  const int b = unit / a.Hk, hk = unit % a.Hk, R = a.g * a.Lq;
  const int n = cross_keys(a, b), tiles = (n + KT - 1) / KT;
  const int t0 = (int)((int64_t)tiles * piece / gr.q_pieces), nt = (int)((int64_t)tiles * (piece + 1) / gr.q_pieces) - t0;

  if (threadIdx.x == 0) {
    for (int i = 0; i < Sm::NS; i++) { mbar_init(&misc->k_full[i], 1); mbar_init(&misc->k_empty[i], 1); mbar_init(&misc->v_full[i], 1); mbar_init(&misc->v_empty[i], 1); }
    mbar_init(&misc->s_full, 1);
    mbar_init(&misc->dp_full, 1);
    mbar_init(&misc->dq_done, 1);
    mbar_init(&misc->s_free, CF_WARPS);
    mbar_init(&misc->dp_free, CF_WARPS);
    mbar_init(&misc->ds_ready, CF_WARPS);
    mbar_init(&misc->q_ready, CF_WARPS);
    misc->abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == CFW_MMA) {
    tmem_alloc(&misc->tmem_base, CF_TMEM);
    tmem_relinquish();
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem = misc->tmem_base;

  if (warp >= CF_WARPS) regs_release<CF_REGS_REST>();
  if (warp == CFW_TMA) {
    if (lane == 0) {
      prefetch_tmap(&tmK); prefetch_tmap(&tmV);
      int i = 0;
      for (; i < nt; i++) {
        const int s = i % Sm::NS, tok = (t0 + i) * KT;
        const uint32_t parity = ((i / Sm::NS) & 1) ^ 1;
        // (V of a tile is done with before its K is)
        if (!mbar_wait(&misc->k_empty[s], parity, abortp, status) || !mbar_wait(&misc->v_empty[s], parity, abortp, status)) break;
        mbar_expect_tx(&misc->k_full[s], SMALL3);
        mbar_expect_tx(&misc->v_full[s], SMALL3);
        for (int p = 0; p < 3; p++) tma_load_4d(sm + Sm::K + s * SMALL3 + p * SMALL, &tmK, &misc->k_full[s], 0, tok, unit, p);
        for (int p = 0; p < 3; p++) tma_load_4d(sm + Sm::V + s * SMALL3 + p * SMALL, &tmV, &misc->v_full[s], 0, tok, unit, p);
      }
      // nothing of this block may still be in flight when it exits: no copy, and no arrival of a product's completion
      for (int k = max(0, i - Sm::NS); k < i; k++) {
        const uint32_t parity = (k / Sm::NS) & 1;
        mbar_wait(&misc->k_full[k % Sm::NS], parity, abortp, status, false);
        mbar_wait(&misc->v_full[k % Sm::NS], parity, abortp, status, false);
        mbar_wait(&misc->k_empty[k % Sm::NS], parity, abortp, status);
        mbar_wait(&misc->v_empty[k % Sm::NS], parity, abortp, status);
      }
    }
  } else if (warp == CFW_MMA) {
    constexpr uint32_t ID_S = idesc_bf16(128, KT, 0, 0);
    const uint32_t ID_Q = idesc_bf16(128, a.d, 0, 1);
    const uint32_t sK = smem_u32(sm + Sm::K);
    const Desc q0 = smem_desc(smem_u32(sm + Sm::Q), 16, 1024, SWZ_128B), g0 = smem_desc(smem_u32(sm + Sm::G), 16, 1024, SWZ_128B);
    const Desc k0 = smem_desc(sK, 16, 1024, SWZ_128B), v0 = smem_desc(smem_u32(sm + Sm::V), 16, 1024, SWZ_128B);
    const Desc kt = smem_desc(sK, SMALL, 1024, SWZ_128B);                // its keys as the contraction
    const int ks = a.d / 16, vs = a.dv / 16;
    const bool leader = elect_one();
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abortp, status); };
    auto issue_s = [&](int i) {
      const int s = i % Sm::NS;
      if (!wait(&misc->k_full[s], (i / Sm::NS) & 1)) return false;
      tcgen05_fence_after();
      if (leader) {
        Desc k = k0;
        k.lo += s * (SMALL3 / 16);
        issue_rows6<BIG, SMALL>(tmem + Sm::S, q0, k, ID_S, ks);
        mma_commit(&misc->s_full);
      }
      __syncwarp();
      return true;
    };
    auto issue_dp = [&](int i) {
      const int s = i % Sm::NS;
      if (!wait(&misc->v_full[s], (i / Sm::NS) & 1)) return false;
      tcgen05_fence_after();
      if (leader) {
        Desc v = v0;
        v.lo += s * (SMALL3 / 16);
        issue_rows6<BIG, SMALL>(tmem + Sm::DP, g0, v, ID_S, vs);
        mma_commit(&misc->v_empty[s]);
        mma_commit(&misc->dp_full);
      }
      __syncwarp();
      return true;
    };
    bool ok = nt > 0 && wait(&misc->q_ready, 0) && issue_s(0) && issue_dp(0);
    for (int i = 0; i < nt && ok; i++) {
      const int s = i % Sm::NS;
      if (i + 1 < nt && !(ok = wait(&misc->s_free, i & 1) && issue_s(i + 1) && wait(&misc->dp_free, i & 1) && issue_dp(i + 1))) break;
      if (!(ok = wait(&misc->ds_ready, i & 1))) break;
      tcgen05_fence_after();
      if (leader) {
        Desc k = kt;
        k.lo += s * (SMALL3 / 16);
        issue_cols6(tmem + Sm::DQ, tmem + Sm::DS, k, ID_Q);
        mma_commit(&misc->k_empty[s]);
        mma_commit(&misc->dq_done);
      }
      __syncwarp();
    }
  } else if (warp < CF_WARPS) {
    regs_acquire<CF_REGS_ROWS>();
    const int w = warp >> 2, row = (warp & 3) * 32 + lane;      // w: which half of the tile's keys, and of dQ's columns
    split_rows(sm + Sm::Q, a.Q, a.aq, a, b, hk, r0, a.d, threadIdx.x);
    split_rows(sm + Sm::G, gr.dY, gr.ady, a, b, hk, r0, a.dv, threadIdx.x);
    fence_proxy_async_smem();
    mbar_arrive_warp(&misc->q_ready, lane);
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const int r = r0 + row, width = a.d - w * 32;               // of its 32 columns of dQ, those that there are
    const bool idle = r0 + (warp & 3) * 32 >= R;                // no row of this warp exists
    const float c = a.scale * FS_LOG2E;
    const float2 st = r < R ? cross_stat(gr.stat, (int64_t)b * a.H + hk * a.g + r / a.Lq, a.Lq, r % a.Lq) : make_float2(-INFINITY, 0.f);
    float acc[32];
#pragma unroll
    for (int k = 0; k < 32; k++) acc[k] = 0.f;
    bool ok = true;
    uint8_t look = 1;                                           // the mask's byte of a tile, asked for one tile ahead
    auto peek = [&](int t) {
      const int j = (t0 + t) * KT + w * 32 + lane;
      look = a.key_mask && j < n ? a.key_mask[b * a.mask_stride + j] : 1;
    };
    if (nt > 0) peek(0);
    for (int i = 0; i < nt; i++) {
      const int s = i % Sm::NS, j0 = (t0 + i) * KT + w * 32;
      ok = __all_sync(0xffffffffu, mbar_wait(&misc->s_full, i & 1, abortp, status, false));
      if (!ok) break;
      tcgen05_fence_after();
      const uint32_t seen = __ballot_sync(0xffffffffu, j0 + lane < n && look != 0);
      if (i + 1 < nt) peek(i + 1);
      uint32_t x[32], g[32];
      if (!idle) {
        tmem_ld16(lanes + Sm::S + w * 32, *reinterpret_cast<uint32_t(*)[16]>(x));
        tmem_ld16(lanes + Sm::S + w * 32 + 16, *reinterpret_cast<uint32_t(*)[16]>(x + 16));
        tmem_wait_ld();
      }
      tcgen05_fence_before();
      mbar_arrive_warp(&misc->s_free, lane);
      if (!idle) {
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
          fma2(x[k], x[k + 1], c, st.x);
          x[k] = __float_as_uint(ex2(__uint_as_float(x[k])));
          x[k + 1] = __float_as_uint(ex2(__uint_as_float(x[k + 1])));
        }
      }
      ok = __all_sync(0xffffffffu, mbar_wait(&misc->dp_full, i & 1, abortp, status, false) &&
                                       (i == 0 || mbar_wait(&misc->dq_done, (i - 1) & 1, abortp, status, false)));
      if (!ok) break;
      tcgen05_fence_after();
      if (!idle) {
        tmem_ld16(lanes + Sm::DP + w * 32, *reinterpret_cast<uint32_t(*)[16]>(g));
        tmem_ld16(lanes + Sm::DP + w * 32 + 16, *reinterpret_cast<uint32_t(*)[16]>(g + 16));
        tmem_wait_ld();
      }
      tcgen05_fence_before();
      mbar_arrive_warp(&misc->dp_free, lane);
      if (seen != ~0u) {
        // a hidden key's K becomes zeros (it may hold anything) before dS, zero there, multiplies it: S, its other reader, has been made
        if ((warp & 3) == 0 && !(seen >> lane & 1u))
          for (int p = 0; p < 3; p++)
            for (int k = 0; k < 8; k++) *reinterpret_cast<uint4*>(sm + Sm::K + s * SMALL3 + p * SMALL + (w * 32 + lane) * 128 + k * 16) = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
      }
      if (!idle) {
        if (i > 0) fold<32>(acc, lanes + Sm::DQ + w * 32, width);
#pragma unroll
        for (int k = 0; k < 32; k += 2) addmul2(g[k], g[k + 1], st.y, st.y, x[k], x[k + 1]);
        if (seen != ~0u) {
#pragma unroll
          for (int k = 0; k < 32; k++) g[k] = (seen >> k) & 1u ? g[k] : 0u;
        }
        store_parts<32>(lanes + Sm::DS + w * 16, g);
        tmem_wait_st();
      }
      tcgen05_fence_before();
      mbar_arrive_warp(&misc->ds_ready, lane);
    }
    if (ok && nt > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait(&misc->dq_done, (nt - 1) & 1, abortp, status, false));
      tcgen05_fence_after();
      if (ok && !idle) fold<32>(acc, lanes + Sm::DQ + w * 32, width);
    }
    if (ok && r < R) {
      const int h = hk * a.g + r / a.Lq, tok = r % a.Lq;
      float* out = gr.pq ? gr.pq + (((int64_t)piece * a.B * a.Hk + unit) * R + r) * a.d
                         : static_cast<float*>(gr.dQ) + b * gr.adq.sb + h * gr.adq.sh + tok * gr.adq.sl;
      out += w * 32;
#pragma unroll
      for (int k = 0; k < 32; k += 4)
        if (k < width) *reinterpret_cast<float4*>(out + k) = make_float4(acc[k] * a.scale, acc[k + 1] * a.scale, acc[k + 2] * a.scale, acc[k + 3] * a.scale);
    }
    __syncwarp();
  }
  tcgen05_fence_before();
  __syncthreads();
  if (warp == CFW_MMA) {
    tcgen05_fence_after();
    tmem_dealloc(tmem, CF_TMEM);
  }
}

int64_t parts_of(int64_t rows, int d) { return 3 * rows * d; }
// Collects tensors to split; `next` is where the next one's parts go.
struct Split {
  SplitJobs jobs;
  int n = 0;
  int64_t threads = 0;
  __nv_bfloat16* next;
  __nv_bfloat16* add(const void* x, TensorAddr ax, int B, int H, int L, int d) {
    __nv_bfloat16* parts = next;
    const int64_t rows = (int64_t)B * H * L;
    threads += rows * (d / 8);
    next += parts_of(rows, d);
    jobs.job[n++] = SplitJob{static_cast<const float*>(x), ax, rows, threads, parts, H, L, d};
    return parts;
  }
  int run(fsharp_ctx* ctx) {
    const int64_t blocks = (threads + 255) / 256;
    if (blocks > 0x7fffffff) return FSHARP_E_SHAPE;
    FS_TIME_BEGIN(ctx, FS_K_CROSS_SPLIT);
    cross_split_kernel<<<(unsigned)blocks, 256, 0, ctx->stream>>>(jobs, n);
    FS_TIME_END(ctx);
    FS_LAUNCH_CHECK(ctx);
    return FSHARP_OK;
  }
};
// parts [3][B H][L][d]
int parts_map(CUtensorMap* map, const __nv_bfloat16* parts, int BH, int L, int d, int rows) {
  return fs_tc_cross_map(map, parts, TensorAddr{(int64_t)BH * L * d, (int64_t)L * d, d}, 3, BH, L, d, rows);
}
// Pieces that bring `blocks` blocks up to one per SM (one is resident there), `most` at most: each has two tiles of keys forward, one of 128 rows or
// keys backward.
int pieces_for(const fsharp_ctx* ctx, int64_t blocks, int64_t most) {
  int64_t p = ctx->sm_count / blocks;
  if (p > most) p = most;
  if (p > 64) p = 64;
  return p < 1 ? 1 : (int)p;
}

}  // namespace

int fs_tc_cross_f32_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm) {
  const int64_t R = (int64_t)dm->H / dm->Hk * dm->Lq;
  return pieces_for(ctx, (int64_t)dm->B * dm->Hk * ((R + 255) / 256), ((int64_t)dm->Lk + 127) / 128);
}
// bf16 values of scratch for the parts of K and V (and Q and dY)
int64_t fs_tc_cross_f32_parts(const fsharp_cross_dims* dm, int backward) {
  const int64_t keys = (int64_t)dm->B * dm->Hk * dm->Lk, rows = (int64_t)dm->B * dm->H * dm->Lq;
  return parts_of(keys, dm->d) + parts_of(keys, dm->dv) + (backward ? parts_of(rows, dm->d) + parts_of(rows, dm->dv) : 0);
}
int fs_tc_cross_f32(fsharp_ctx* ctx, const CrossArgs& a, void* Y, TensorAddr ay, float* lse, CrossPart part, void* scratch) {
  Split split;
  split.next = static_cast<__nv_bfloat16*>(scratch);
  const __nv_bfloat16 *pk = split.add(a.K, a.ak, a.B, a.Hk, a.Lk, a.d), *pv = split.add(a.V, a.av, a.B, a.Hk, a.Lk, a.dv);
  FS_TRY(split.run(ctx));
  CUtensorMap tmK, tmV;
  FS_TRY(parts_map(&tmK, pk, a.B * a.Hk, a.Lk, a.d, KT));
  FS_TRY(parts_map(&tmV, pv, a.B * a.Hk, a.Lk, a.dv, KT));
  const int64_t gx = ((int64_t)a.g * a.Lq + 255) / 256 * part.pieces;
  if (gx > 0x7fffffff) return FSHARP_E_SHAPE;
  FS_CUDA_OK(fs_allow_smem(tc_cross_f32_kernel));
  CrossArgs af = a;
  af.ranked = cross_ranked(ctx, a, gx * a.B * a.Hk);
  FS_TIME_BEGIN(ctx, FS_K_TC_CROSS);
  tc_cross_f32_kernel<<<dim3((unsigned)gx, (unsigned)(a.B * a.Hk)), CF_T, FwSm::TOTAL + 1024, ctx->stream>>>(tmK, tmV, af, static_cast<float*>(Y), ay, lse, part, ctx->d_status);
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  return FSHARP_OK;
}
void fs_tc_cross_f32_grad_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int* kv_pieces, int* q_pieces) {
  const int64_t g = dm->H / dm->Hk, units = (int64_t)dm->B * dm->Hk, kt = ((int64_t)dm->Lk + TILE - 1) / TILE;
  *kv_pieces = pieces_for(ctx, units * kt, g * (((int64_t)dm->Lq + TILE - 1) / TILE));
  *q_pieces = pieces_for(ctx, units * ((g * dm->Lq + TILE - 1) / TILE), kt);
}
int fs_tc_cross_f32_grad(fsharp_ctx* ctx, const CrossArgs& a, const CrossGrad& gr, void* scratch) {
  Split split;
  split.next = static_cast<__nv_bfloat16*>(scratch);
  const __nv_bfloat16 *pk = split.add(a.K, a.ak, a.B, a.Hk, a.Lk, a.d), *pv = split.add(a.V, a.av, a.B, a.Hk, a.Lk, a.dv),
                      *pq = split.add(a.Q, a.aq, a.B, a.H, a.Lq, a.d), *pg = split.add(gr.dY, gr.ady, a.B, a.H, a.Lq, a.dv);
  FS_TRY(split.run(ctx));
  CUtensorMap tmQ, tmG, tmK, tmV, tmKt, tmVt;
  FS_TRY(parts_map(&tmQ, pq, a.B * a.H, a.Lq, a.d, KT));
  FS_TRY(parts_map(&tmG, pg, a.B * a.H, a.Lq, a.dv, KT));
  FS_TRY(parts_map(&tmK, pk, a.B * a.Hk, a.Lk, a.d, TILE));
  FS_TRY(parts_map(&tmV, pv, a.B * a.Hk, a.Lk, a.dv, TILE));
  FS_TRY(parts_map(&tmKt, pk, a.B * a.Hk, a.Lk, a.d, KT));
  FS_TRY(parts_map(&tmVt, pv, a.B * a.Hk, a.Lk, a.dv, KT));
  const int64_t gk = ((int64_t)a.Lk + TILE - 1) / TILE * gr.kv_pieces, gq = ((int64_t)a.g * a.Lq + TILE - 1) / TILE * gr.q_pieces;
  if (gk > 0x7fffffff || gq > 0x7fffffff) return FSHARP_E_SHAPE;
  FS_CUDA_OK(fs_allow_smem(tc_cross_f32_dkv_kernel));
  FS_CUDA_OK(fs_allow_smem(tc_cross_f32_dq_kernel));
  FS_TIME_BEGIN(ctx, FS_K_TC_CROSS_DKV);
  tc_cross_f32_dkv_kernel<<<dim3((unsigned)gk, (unsigned)(a.B * a.Hk)), CF_T, FkSm::TOTAL + 1024, ctx->stream>>>(tmQ, tmG, tmK, tmV, a, gr, ctx->d_status);
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  CrossArgs aq = a;
  aq.ranked = cross_ranked(ctx, a, gq * a.B * a.Hk);
  FS_TIME_BEGIN(ctx, FS_K_TC_CROSS_DQ);
  tc_cross_f32_dq_kernel<<<dim3((unsigned)gq, (unsigned)(a.B * a.Hk)), CF_T, FqSm::TOTAL + 1024, ctx->stream>>>(tmKt, tmVt, aq, gr, ctx->d_status);
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  return FSHARP_OK;
}
