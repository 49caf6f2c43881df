// Cross attention and its gradients on the multiply-add pipe, fp32 throughout: fp32 tensors of wide heads (and any where the tensor-core
// kernels are not wanted).  Blocks of 256 threads; tiles of 64 keys and 16 or 64 rows lie row by row in shared memory as fp32,
// every product is 4 x 4 (or 4 x D / 16) sums per thread with 16-byte loads of both operands: four loads of an operand row
// serve 16 multiply-adds, which keeps the multiply-add pipe, not shared memory, the bound.
//   forward   S = Q K^T (row by row dots), softmax over the tile with a running maximum and sum, O += P V
//   dkv       per 64 keys, over the rows: P^T from lse, dS^T = P^T (V dY^T - D), dV += P^T dY, dK += dS^T Q
//   dq        per 64 rows, over the keys: dQ += dS K
// The gradients' kernels recompute P; two kernels instead of one with atomics, so that sums have a fixed order.
#include "cross.cuh"
#include "tc_common.cuh"

namespace {

// Blocks on an SM that registers are kept for (4 x 8 x 701 x 1501, d = 32, forward: 247 us with two, 202 with three).
__host__ __device__ constexpr int fm_blocks(int D) { return D == 32 ? 3 : D == 64 ? 2 : 1; }
constexpr int FM_T = 256, FM_KEYS = 64, FM_LP = FM_KEYS + 4;

__device__ __forceinline__ float4 widen4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 widen4(const __nv_bfloat16* p) {
  const uint2 x = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u));
}
template <typename T> __device__ __forceinline__ const T* row_of(const void* base, const TensorAddr& t, int b, int h, int i) {
  return static_cast<const T*>(base) + b * t.sb + h * t.sh + i * t.sl;
}

// N rows of D values, zero from column `width` on and in rows that `at` has no place for.
template <typename T, int D, int N, class At>
__device__ __forceinline__ void load_tile(float* to, int width, At at) {
  constexpr int Q = D / 4;
  for (int i = threadIdx.x; i < N * Q; i += FM_T) {
    const int r = i / Q, e = i % Q * 4;
    const T* p = e < width ? at(r) : nullptr;
    *reinterpret_cast<float4*>(to + r * (D + 4) + e) = p ? widen4(p + e) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
}
// acc[i][j] += sum_k A[ty + 16 i][k] B[tx + 16 j][k], k < K (a multiple of 16; not the tiles' D, which is the larger of d and dv)
template <int MT, int NT>
__device__ __forceinline__ void dots(float (&acc)[MT][NT], const float* A, const float* B, int ld, int K) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll 4
  for (int k = 0; k < K; k += 4) {
    float4 x[MT], y[NT];
#pragma unroll
    for (int i = 0; i < MT; i++) x[i] = *reinterpret_cast<const float4*>(A + (ty + 16 * i) * ld + k);
#pragma unroll
    for (int j = 0; j < NT; j++) y[j] = *reinterpret_cast<const float4*>(B + (tx + 16 * j) * ld + k);
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
      for (int j = 0; j < NT; j++) {
        acc[i][j] = fmaf(x[i].x, y[j].x, acc[i][j]);
        acc[i][j] = fmaf(x[i].y, y[j].y, acc[i][j]);
        acc[i][j] = fmaf(x[i].z, y[j].z, acc[i][j]);
        acc[i][j] = fmaf(x[i].w, y[j].w, acc[i][j]);
      }
  }
}
// The columns of a thread's sums over D values: 4 tx .. + 3 (and 64 + those for D = 128), 2 tx, 2 tx + 1 for D = 32.
template <int D> __device__ __forceinline__ int col_of(int c) {
  const int tx = threadIdx.x & 15;
  return D == 32 ? 2 * tx + c : 4 * tx + (c & 3) + (c >> 2) * 64;
}
// acc[i][c] += sum_k A[ty + 16 i][k] B[k][col(c)], k < 64 (A with rows of FM_LP, B of D + 4).  D = 128: the upper columns only where
// `width` has them.
template <int MT, int D>
__device__ __forceinline__ void add_rows(float (&acc)[MT][D / 16], const float* A, const float* B, int width) {
  const int ty = threadIdx.x >> 4;
  if constexpr (D == 128) {
    if (width <= 64) {
#pragma unroll 2
      for (int k = 0; k < 64; k += 4) {
        float x[MT][4];
#pragma unroll
        for (int i = 0; i < MT; i++) *reinterpret_cast<float4*>(x[i]) = *reinterpret_cast<const float4*>(A + (ty + 16 * i) * FM_LP + k);
#pragma unroll
        for (int q = 0; q < 4; q++) {
          float y[4];
          *reinterpret_cast<float4*>(y) = *reinterpret_cast<const float4*>(B + (k + q) * (D + 4) + col_of<D>(0));
#pragma unroll
          for (int i = 0; i < MT; i++)
#pragma unroll
            for (int c = 0; c < 4; c++) acc[i][c] = fmaf(x[i][q], y[c], acc[i][c]);
        }
      }
      return;
    }
  }
#pragma unroll 2
  for (int k = 0; k < 64; k += 4) {
    float x[MT][4];
#pragma unroll
    for (int i = 0; i < MT; i++) *reinterpret_cast<float4*>(x[i]) = *reinterpret_cast<const float4*>(A + (ty + 16 * i) * FM_LP + k);
#pragma unroll
    for (int q = 0; q < 4; q++) {
      float y[D / 16];
      const float* row = B + (k + q) * (D + 4);
      if constexpr (D == 32) *reinterpret_cast<float2*>(y) = *reinterpret_cast<const float2*>(row + col_of<D>(0));
      else
#pragma unroll
        for (int c = 0; c < D / 16; c += 4) *reinterpret_cast<float4*>(y + c) = *reinterpret_cast<const float4*>(row + col_of<D>(c));
#pragma unroll
      for (int i = 0; i < MT; i++)
#pragma unroll
        for (int c = 0; c < D / 16; c++) acc[i][c] = fmaf(x[i][q], y[c], acc[i][c]);
    }
  }
}

template <int D, int MT> constexpr size_t fwd_smem() { return sizeof(float) * ((16 * MT + 2 * FM_KEYS) * (D + 4) + 16 * MT * FM_LP + FM_KEYS); }

template <typename T, int D, int MT>
__global__ void __launch_bounds__(FM_T, fm_blocks(D))
cross_fma_kernel(const __grid_constant__ CrossArgs a, T* __restrict__ Y, TensorAddr ay, float* __restrict__ lse, CrossPart part) {
  constexpr int RT = 16 * MT, LD = D + 4;
  extern __shared__ __align__(16) float fm_smem[];
  float *sq = fm_smem, *sk = sq + RT * LD, *sv = sk + FM_KEYS * LD, *sp = sv + FM_KEYS * LD;
  int* seen = reinterpret_cast<int*>(sp + RT * FM_LP);
  const int unit = blockIdx.y, piece = blockIdx.x % part.pieces, r0 = (int)(blockIdx.x / part.pieces) * RT;
  const int b = unit / a.Hk, hk = unit % a.Hk, R = a.g * a.Lq, ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const int n = cross_keys(a, b), tiles = (n + FM_KEYS - 1) / FM_KEYS;
  const int t0 = (int)((int64_t)tiles * piece / part.pieces), t1 = (int)((int64_t)tiles * (piece + 1) / part.pieces);
  const float c = a.scale * FS_LOG2E;
  load_tile<T, D, RT>(sq, a.d, [&](int r) { return r0 + r < R ? row_of<T>(a.Q, a.aq, b, hk * a.g + (r0 + r) / a.Lq, (r0 + r) % a.Lq) : nullptr; });
  float m[MT], l[MT], o[MT][D / 16];
#pragma unroll
  for (int i = 0; i < MT; i++) {
    m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; k++) o[i][k] = 0.f;
  }
  for (int t = t0; t < t1; t++) {
    const int j0 = t * FM_KEYS;
    __syncthreads();
    load_tile<T, D, FM_KEYS>(sk, a.d, [&](int j) { return j0 + j < n ? row_of<T>(a.K, a.ak, b, hk, j0 + j) : nullptr; });
    load_tile<T, D, FM_KEYS>(sv, a.dv, [&](int j) { return cross_seen(a, b, j0 + j, n) ? row_of<T>(a.V, a.av, b, hk, j0 + j) : nullptr; });
    if (threadIdx.x < FM_KEYS) seen[threadIdx.x] = cross_seen(a, b, j0 + threadIdx.x, n);
    __syncthreads();
    float s[MT][4] = {};
    dots<MT, 4>(s, sq, sk, LD, a.d);
#pragma unroll
    for (int i = 0; i < MT; i++) {
      float top = m[i];
#pragma unroll
      for (int j = 0; j < 4; j++) {
        s[i][j] = seen[tx + 16 * j] ? s[i][j] * c : -INFINITY;
        top = fmaxf(top, s[i][j]);
      }
#pragma unroll
      for (int w = 1; w < 16; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
      const float base = top == -INFINITY ? 0.f : top, corr = tc::ex2(m[i] - base);
      m[i] = top;
      l[i] *= corr;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const float p = tc::ex2(s[i][j] - base);
        l[i] += p;                                   // this thread's four columns: added up over the row at the end
        sp[(ty + 16 * i) * FM_LP + tx + 16 * j] = p;
      }
#pragma unroll
      for (int k = 0; k < D / 16; k++) o[i][k] *= corr;
    }
    __syncthreads();
    // (a tile's sums on their own first: one sum over all keys is off by more, 1.1e-6 of the result instead of 3e-7 for 6127 keys)
    float sum[MT][D / 16] = {};
    add_rows<MT, D>(sum, sp, sv, a.dv);
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
      for (int k = 0; k < D / 16; k++) o[i][k] += sum[i][k];
  }
#pragma unroll
  for (int i = 0; i < MT; i++) {
    float sum = l[i];
#pragma unroll
    for (int w = 1; w < 16; w <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    const int r = r0 + ty + 16 * i;
    if (r >= R) continue;
    if (part.pieces > 1) {
      const int64_t at = ((int64_t)unit * part.pieces + piece) * R + r;
#pragma unroll
      for (int k = 0; k < D / 16; k++)
        if (col_of<D>(k) < a.dv) part.o[at * a.dv + col_of<D>(k)] = o[i][k];
      if (tx == 0) part.ml[at] = make_float2(m[i], sum);
    } else {
      const int h = hk * a.g + r / a.Lq, tok = r % a.Lq;
      T* y = Y + b * ay.sb + h * ay.sh + tok * ay.sl;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int k = 0; k < D / 16; k++)
        if (col_of<D>(k) < a.dv) fs_store(y + col_of<D>(k), o[i][k] * inv);
      if (lse && tx == 0) lse[((int64_t)b * a.H + h) * a.Lq + tok] = sum == 0.f ? -INFINITY : (m[i] + log2f(sum)) * FS_LN2;
    }
  }
}

// ---------------------------------------------------------------- gradients
// What both kernels make of a pair of tiles: P and dS of rows ty + 16 i and keys tx + 16 j.
template <int D>
__device__ __forceinline__ void p_ds(float (&p)[4][4], float (&ds)[4][4], const float* sq, const float* sg, const float* sk, const float* sv,
                                     const float2* stat, const int* seen, float c, float scale, int d, int dv) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int j = 0; j < 4; j++) p[i][j] = ds[i][j] = 0.f;
  dots<4, 4>(p, sq, sk, D + 4, d);
  dots<4, 4>(ds, sg, sv, D + 4, dv);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float2 st = stat[ty + 16 * i];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const bool on = seen[tx + 16 * j];
      p[i][j] = on ? tc::ex2(fmaf(p[i][j], c, st.x)) : 0.f;
      ds[i][j] = on ? p[i][j] * (ds[i][j] + st.y) * scale : 0.f;
    }
  }
}

__device__ __forceinline__ float2 stat_of(const CrossArgs& a, const CrossGrad& gr, int b, int hk, int r) {
  return r < a.g * a.Lq ? cross_stat(gr.stat, (int64_t)b * a.H + hk * a.g + r / a.Lq, a.Lq, r % a.Lq) : make_float2(-INFINITY, 0.f);
}

template <int D> constexpr size_t dkv_smem() { return sizeof(float) * (4 * 64 * (D + 4) + 2 * 64 * FM_LP + 3 * 64); }
template <int D> constexpr size_t dq_smem() { return sizeof(float) * (4 * 64 * (D + 4) + 64 * FM_LP + 3 * 64); }

template <typename T, int D>
__global__ void __launch_bounds__(FM_T, fm_blocks(D))
cross_dkv_kernel(const __grid_constant__ CrossArgs a, const __grid_constant__ CrossGrad gr) {
  constexpr int LD = D + 4;
  extern __shared__ __align__(16) float fm_smem[];
  float *sk = fm_smem, *sv = sk + 64 * LD, *sq = sv + 64 * LD, *sg = sq + 64 * LD, *spt = sg + 64 * LD, *sdt = spt + 64 * FM_LP;
  float2* stat = reinterpret_cast<float2*>(sdt + 64 * FM_LP);
  int* seen = reinterpret_cast<int*>(stat + 64);
  const int unit = blockIdx.y, piece = blockIdx.x % gr.kv_pieces, j0 = (int)(blockIdx.x / gr.kv_pieces) * 64;
  const int b = unit / a.Hk, hk = unit % a.Hk, R = a.g * a.Lq, ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const int n = cross_keys(a, b), tiles = j0 < n ? (R + 63) / 64 : 0;
  const int t0 = (int)((int64_t)tiles * piece / gr.kv_pieces), t1 = (int)((int64_t)tiles * (piece + 1) / gr.kv_pieces);
  const float c = a.scale * FS_LOG2E;
  if (threadIdx.x < 64) seen[threadIdx.x] = cross_seen(a, b, j0 + threadIdx.x, n);
  load_tile<T, D, 64>(sk, a.d, [&](int j) { return cross_seen(a, b, j0 + j, n) ? row_of<T>(a.K, a.ak, b, hk, j0 + j) : nullptr; });
  load_tile<T, D, 64>(sv, a.dv, [&](int j) { return cross_seen(a, b, j0 + j, n) ? row_of<T>(a.V, a.av, b, hk, j0 + j) : nullptr; });
  float dk[4][D / 16] = {}, dv[4][D / 16] = {};
  for (int t = t0; t < t1; t++) {
    const int r0 = t * 64;
    __syncthreads();
    load_tile<T, D, 64>(sq, a.d, [&](int r) { return r0 + r < R ? row_of<T>(a.Q, a.aq, b, hk * a.g + (r0 + r) / a.Lq, (r0 + r) % a.Lq) : nullptr; });
    load_tile<T, D, 64>(sg, a.dv, [&](int r) { return r0 + r < R ? row_of<T>(gr.dY, gr.ady, b, hk * a.g + (r0 + r) / a.Lq, (r0 + r) % a.Lq) : nullptr; });
    if (threadIdx.x < 64) stat[threadIdx.x] = stat_of(a, gr, b, hk, r0 + threadIdx.x);
    __syncthreads();
    float p[4][4], ds[4][4];
    p_ds<D>(p, ds, sq, sg, sk, sv, stat, seen, c, a.scale, a.d, a.dv);
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        spt[(tx + 16 * j) * FM_LP + ty + 16 * i] = p[i][j];
        sdt[(tx + 16 * j) * FM_LP + ty + 16 * i] = ds[i][j];
      }
    __syncthreads();
    add_rows<4, D>(dv, spt, sg, a.dv);
    add_rows<4, D>(dk, sdt, sq, a.d);
  }
  __syncthreads();      // (seen, where no tile was walked)
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int jj = ty + 16 * i, j = j0 + jj;
    if (j >= a.Lk) continue;
    const bool on = seen[jj];                        // (infinite queries or cotangents reach no key that is not seen)
    float* part = gr.pkv + (((int64_t)piece * a.B * a.Hk + unit) * a.Lk + j) * (a.d + a.dv);
    T* gk = static_cast<T*>(gr.dK) + b * gr.adk.sb + hk * gr.adk.sh + j * gr.adk.sl;
    T* gv = static_cast<T*>(gr.dV) + b * gr.adv.sb + hk * gr.adv.sh + j * gr.adv.sl;
#pragma unroll
    for (int k = 0; k < D / 16; k++) {
      const int e = col_of<D>(k);
      const float x = on ? dk[i][k] : 0.f, y = on ? dv[i][k] : 0.f;
      if (gr.pkv) {
        if (e < a.d) part[e] = x;
        if (e < a.dv) part[a.d + e] = y;
      } else {
        if (e < a.d) fs_store(gk + e, x);
        if (e < a.dv) fs_store(gv + e, y);
      }
    }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(FM_T, fm_blocks(D))
cross_dq_kernel(const __grid_constant__ CrossArgs a, const __grid_constant__ CrossGrad gr) {
  constexpr int LD = D + 4;
  extern __shared__ __align__(16) float fm_smem[];
  float *sk = fm_smem, *sv = sk + 64 * LD, *sq = sv + 64 * LD, *sg = sq + 64 * LD, *sd = sg + 64 * LD;
  float2* stat = reinterpret_cast<float2*>(sd + 64 * FM_LP);
  int* seen = reinterpret_cast<int*>(stat + 64);
  const int unit = blockIdx.y, piece = blockIdx.x % gr.q_pieces, r0 = (int)(blockIdx.x / gr.q_pieces) * 64;
  const int b = unit / a.Hk, hk = unit % a.Hk, R = a.g * a.Lq, ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const int n = cross_keys(a, b), tiles = (n + 63) / 64;
  const int t0 = (int)((int64_t)tiles * piece / gr.q_pieces), t1 = (int)((int64_t)tiles * (piece + 1) / gr.q_pieces);
  const float c = a.scale * FS_LOG2E;
  load_tile<T, D, 64>(sq, a.d, [&](int r) { return r0 + r < R ? row_of<T>(a.Q, a.aq, b, hk * a.g + (r0 + r) / a.Lq, (r0 + r) % a.Lq) : nullptr; });
  load_tile<T, D, 64>(sg, a.dv, [&](int r) { return r0 + r < R ? row_of<T>(gr.dY, gr.ady, b, hk * a.g + (r0 + r) / a.Lq, (r0 + r) % a.Lq) : nullptr; });
  if (threadIdx.x < 64) stat[threadIdx.x] = stat_of(a, gr, b, hk, r0 + threadIdx.x);
  float dq[4][D / 16] = {};
  for (int t = t0; t < t1; t++) {
    const int j0 = t * 64;
    __syncthreads();
    if (threadIdx.x < 64) seen[threadIdx.x] = cross_seen(a, b, j0 + threadIdx.x, n);
    load_tile<T, D, 64>(sk, a.d, [&](int j) { return cross_seen(a, b, j0 + j, n) ? row_of<T>(a.K, a.ak, b, hk, j0 + j) : nullptr; });
    load_tile<T, D, 64>(sv, a.dv, [&](int j) { return cross_seen(a, b, j0 + j, n) ? row_of<T>(a.V, a.av, b, hk, j0 + j) : nullptr; });
    __syncthreads();
    float p[4][4], ds[4][4];
    p_ds<D>(p, ds, sq, sg, sk, sv, stat, seen, c, a.scale, a.d, a.dv);
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int j = 0; j < 4; j++) sd[(ty + 16 * i) * FM_LP + tx + 16 * j] = ds[i][j];
    __syncthreads();
    add_rows<4, D>(dq, sd, sk, a.d);
  }
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int r = r0 + ty + 16 * i;
    if (r >= R) continue;
    float* part = gr.pq + (((int64_t)piece * a.B * a.Hk + unit) * R + r) * a.d;
    T* out = static_cast<T*>(gr.dQ) + b * gr.adq.sb + (hk * a.g + r / a.Lq) * gr.adq.sh + r % a.Lq * gr.adq.sl;
#pragma unroll
    for (int k = 0; k < D / 16; k++) {
      const int e = col_of<D>(k);
      if (e >= a.d) continue;
      if (gr.pq) part[e] = dq[i][k];
      else fs_store(out + e, dq[i][k]);
    }
  }
}

template <typename T, int D, int MT>
int launch_fwd(fsharp_ctx* ctx, const CrossArgs& a, T* Y, TensorAddr ay, float* lse, CrossPart part) {
  const int64_t gx = ((int64_t)a.g * a.Lq + 16 * MT - 1) / (16 * MT) * part.pieces;
  if (gx > 0x7fffffff) return FSHARP_E_SHAPE;
  FS_CUDA_OK(fs_allow_smem(cross_fma_kernel<T, D, MT>));
  FS_TIME_BEGIN(ctx, FS_K_CROSS_FMA);
  cross_fma_kernel<T, D, MT><<<dim3((unsigned)gx, (unsigned)(a.B * a.Hk)), FM_T, fwd_smem<D, MT>(), ctx->stream>>>(a, Y, ay, lse, part);
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  return FSHARP_OK;
}
template <typename T, int D>
int launch_rows_of(fsharp_ctx* ctx, const CrossArgs& a, T* Y, TensorAddr ay, float* lse, CrossPart part) {
  return a.g * a.Lq <= 16 ? launch_fwd<T, D, 1>(ctx, a, Y, ay, lse, part) : launch_fwd<T, D, 4>(ctx, a, Y, ay, lse, part);
}
template <typename T>
int run_fwd(fsharp_ctx* ctx, const CrossArgs& a, T* Y, TensorAddr ay, float* lse, CrossPart part) {
  const int D = a.d > a.dv ? a.d : a.dv;
  if (D <= 32) return launch_rows_of<T, 32>(ctx, a, Y, ay, lse, part);
  if (D == 64) return launch_rows_of<T, 64>(ctx, a, Y, ay, lse, part);
  return launch_rows_of<T, 128>(ctx, a, Y, ay, lse, part);
}

template <typename T, int D>
int launch_grad(fsharp_ctx* ctx, const CrossArgs& a, const CrossGrad& gr) {
  const int64_t gk = ((int64_t)a.Lk + 63) / 64 * gr.kv_pieces, gq = ((int64_t)a.g * a.Lq + 63) / 64 * gr.q_pieces;
  if (gk > 0x7fffffff || gq > 0x7fffffff) return FSHARP_E_SHAPE;
  FS_CUDA_OK(fs_allow_smem(cross_dkv_kernel<T, D>));
  FS_CUDA_OK(fs_allow_smem(cross_dq_kernel<T, D>));
  if (gk) {
    FS_TIME_BEGIN(ctx, FS_K_CROSS_DKV);
    cross_dkv_kernel<T, D><<<dim3((unsigned)gk, (unsigned)(a.B * a.Hk)), FM_T, dkv_smem<D>(), ctx->stream>>>(a, gr);
    FS_TIME_END(ctx);
    FS_LAUNCH_CHECK(ctx);
  }
  if (gq) {
    FS_TIME_BEGIN(ctx, FS_K_CROSS_DQ);
    cross_dq_kernel<T, D><<<dim3((unsigned)gq, (unsigned)(a.B * a.Hk)), FM_T, dq_smem<D>(), ctx->stream>>>(a, gr);
    FS_TIME_END(ctx);
    FS_LAUNCH_CHECK(ctx);
  }
  return FSHARP_OK;
}
template <typename T>
int run_grad(fsharp_ctx* ctx, const CrossArgs& a, const CrossGrad& gr) {
  const int D = a.d > a.dv ? a.d : a.dv;
  if (D <= 32) return launch_grad<T, 32>(ctx, a, gr);
  if (D == 64) return launch_grad<T, 64>(ctx, a, gr);
  return launch_grad<T, 128>(ctx, a, gr);
}

// Pieces that bring `blocks` blocks up to two per SM, none of less than one tile.
int pieces_for(const fsharp_ctx* ctx, int64_t blocks, int64_t tiles) {
  if (blocks < 1) return 1;
  int64_t p = 2 * (int64_t)ctx->sm_count / blocks;
  if (p > tiles) p = tiles;
  if (p > 64) p = 64;
  return p < 1 ? 1 : (int)p;
}

}  // namespace

int fs_cross_fma_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm) {
  const int64_t R = (int64_t)dm->H / dm->Hk * dm->Lq, rt = R <= 16 ? 16 : 64;
  return pieces_for(ctx, (int64_t)dm->B * dm->Hk * ((R + rt - 1) / rt), ((int64_t)dm->Lk + 63) / 64);
}
int fs_cross_fma(fsharp_ctx* ctx, const CrossArgs& a, int dtype, void* Y, TensorAddr ay, float* lse, CrossPart part) {
  return dtype == FSHARP_F32 ? run_fwd<float>(ctx, a, static_cast<float*>(Y), ay, lse, part)
                             : run_fwd<__nv_bfloat16>(ctx, a, static_cast<__nv_bfloat16*>(Y), ay, lse, part);
}
void fs_cross_fma_grad_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int* kv_pieces, int* q_pieces) {
  const int64_t rt = ((int64_t)dm->H / dm->Hk * dm->Lq + 63) / 64, kt = ((int64_t)dm->Lk + 63) / 64, units = (int64_t)dm->B * dm->Hk;
  *kv_pieces = pieces_for(ctx, units * kt, rt);
  *q_pieces = pieces_for(ctx, units * rt, kt);
}
int fs_cross_fma_grad(fsharp_ctx* ctx, const CrossArgs& a, int dtype, const CrossGrad& gr) {
  return dtype == FSHARP_F32 ? run_grad<float>(ctx, a, gr) : run_grad<__nv_bfloat16>(ctx, a, gr);
}
