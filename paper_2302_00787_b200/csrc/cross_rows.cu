// Cross attention of few query rows per key head (decoding steps): K and V are streamed once.  A key's d values lie across
// D / VE lanes (16 bytes each), a warp's copy covers 512 bytes of K or V, and asynchronous copies of a few turns of keys and values per lane
// are in flight (up to 190 KB per SM); scores are sums over a key's lanes by shuffles.
// Each lane group keeps a maximum, a sum and an output of its own; they meet once at the end: warp, block, then the pieces of
// the keys, which are the blocks of a cluster (up to eight; one launch) or meet in scratch (cross_join_kernel).
// Bound: HBM (2 n d values per unit).
#include "cross.cuh"
#include "tc_common.cuh"

namespace {

constexpr int RW_T = 128, RW_WARPS = RW_T / 32;
// Keys per lane and turn, and turns in flight: 32 KB of copies per block, six blocks on an SM; heads of 128, whose turns are half as many
// keys, 48 KB.  (64 x 12 sequences of 1500 keys, d = 64: 53 us so, 62 with 4 and 3; 16 x 8 of 16384, d = 128: 176 with 4 and 3, 208 with 2 and 4.)
__host__ __device__ constexpr int rows_u(int D) { return D == 128 ? 4 : 2; }
__host__ __device__ constexpr int rows_stages(int D) { return D == 128 ? 3 : 4; }
constexpr int RW_CLUSTER = 8;      // most pieces that meet in a cluster

template <typename T> __device__ __forceinline__ void widen(const uint4& x, float* v);
template <> __device__ __forceinline__ void widen<float>(const uint4& x, float* v) {
  v[0] = __uint_as_float(x.x); v[1] = __uint_as_float(x.y); v[2] = __uint_as_float(x.z); v[3] = __uint_as_float(x.w);
}
template <> __device__ __forceinline__ void widen<__nv_bfloat16>(const uint4& x, float* v) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; i++) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}

__host__ __device__ constexpr int rows_step(int D, int es) { return RW_WARPS * (32 / (D * es / 16)) * rows_u(D); }    // keys per turn of a block

template <typename T, int D, int R>
__global__ void __launch_bounds__(RW_T)
cross_rows_kernel(const __grid_constant__ CrossArgs a, T* __restrict__ Y, TensorAddr ay, float* __restrict__ lse, CrossPart part) {
  constexpr int RW_U = rows_u(D), RW_STAGES = rows_stages(D), VE = 16 / (int)sizeof(T), LPK = D / VE, KPW = 32 / LPK, STEP = RW_WARPS * KPW * RW_U;
  static_assert(STEP == rows_step(D, sizeof(T)), "");
  __shared__ float so[RW_WARPS][R][D];
  __shared__ float sm[RW_WARPS][R], sl[RW_WARPS][R];
  const int unit = blockIdx.y, piece = blockIdx.x, b = unit / a.Hk, hk = unit % a.Hk, rows = a.g * a.Lq;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = lane / LPK, e0 = lane % LPK * VE;
  const float c = a.scale * FS_LOG2E;
  const bool inq = e0 < a.d, inv = e0 < a.dv;
  float q[R][VE];
#pragma unroll
  for (int r = 0; r < R; r++) {
    uint4 x = make_uint4(0, 0, 0, 0);
    if (r < rows && inq)
      x = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.Q) + b * a.aq.sb + (int64_t)(hk * a.g + r / a.Lq) * a.aq.sh +
                                          (int64_t)(r % a.Lq) * a.aq.sl + e0);
    widen<T>(x, q[r]);
#pragma unroll
    for (int k = 0; k < VE; k++) q[r][k] *= c;
  }
  const T* Kb = static_cast<const T*>(a.K) + b * a.ak.sb + hk * a.ak.sh + e0;
  const T* Vb = static_cast<const T*>(a.V) + b * a.av.sb + hk * a.av.sh + e0;
  const int n = cross_keys(a, b), turns = (n + STEP - 1) / STEP;
  const int t0 = (int)((int64_t)turns * piece / part.pieces), t1 = (int)((int64_t)turns * (piece + 1) / part.pieces);
  float m[R], l[R], o[R][VE];
#pragma unroll
  for (int r = 0; r < R; r++) {
    m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
    for (int k = 0; k < VE; k++) o[r][k] = 0.f;
  }
  // A thread's ring in shared memory, RW_STAGES turns of its own 16-byte pieces: nobody else touches them, so waiting for the thread's
  // own copies is all the order they need.
  extern __shared__ uint4 ring[];
  uint4* mine = ring + threadIdx.x;
  auto fetch = [&](int t) {
    if (t < t1) {
      uint4* to = mine + (t % RW_STAGES) * 2 * RW_U * RW_T;
#pragma unroll
      for (int u = 0; u < RW_U; u++) {
        const int64_t j = t * STEP + (u * RW_WARPS + warp) * KPW + grp;
        tc::copy16(to + 2 * u * RW_T, Kb + (j < n ? j * a.ak.sl : 0), j < n && inq);
        tc::copy16(to + (2 * u + 1) * RW_T, Vb + (j < n ? j * a.av.sl : 0), j < n && inv);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  bool next[RW_U];                                       // which keys of the coming turn are seen
  auto look = [&](int t) {
#pragma unroll
    for (int u = 0; u < RW_U; u++) next[u] = cross_seen(a, b, t * STEP + (u * RW_WARPS + warp) * KPW + grp, n);
  };
#pragma unroll
  for (int t = 0; t < RW_STAGES - 1; t++) fetch(t0 + t);
  if (t0 < t1) look(t0);
  for (int t = t0; t < t1; t++) {
    fetch(t + RW_STAGES - 1);
    bool on[RW_U];
#pragma unroll
    for (int u = 0; u < RW_U; u++) on[u] = next[u];
    if (t + 1 < t1) look(t + 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(RW_STAGES - 1) : "memory");
    const uint4* from = mine + (t % RW_STAGES) * 2 * RW_U * RW_T;
    float s[RW_U][R];
#pragma unroll
    for (int u = 0; u < RW_U; u++) {
      float k[VE];
      widen<T>(from[2 * u * RW_T], k);
#pragma unroll
      for (int r = 0; r < R; r++) {
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < VE; e++) x = fmaf(q[r][e], k[e], x);
        s[u][r] = x;
      }
    }
#pragma unroll
    for (int w = 1; w < LPK; w <<= 1)
#pragma unroll
      for (int u = 0; u < RW_U; u++)
#pragma unroll
        for (int r = 0; r < R; r++) s[u][r] += __shfl_xor_sync(0xffffffffu, s[u][r], w);
#pragma unroll
    for (int r = 0; r < R; r++) {
      float top = m[r];
#pragma unroll
      for (int u = 0; u < RW_U; u++) {
        if (!on[u]) s[u][r] = -INFINITY;
        top = fmaxf(top, s[u][r]);
      }
      const float base = top == -INFINITY ? 0.f : top, corr = tc::ex2(m[r] - base);
      m[r] = top;
      l[r] *= corr;
#pragma unroll
      for (int u = 0; u < RW_U; u++) {
        s[u][r] = tc::ex2(s[u][r] - base);
        l[r] += s[u][r];
      }
#pragma unroll
      for (int e = 0; e < VE; e++) o[r][e] *= corr;
    }
#pragma unroll
    for (int u = 0; u < RW_U; u++) {
      uint4 y = from[(2 * u + 1) * RW_T];
      if (!on[u]) y = make_uint4(0, 0, 0, 0);            // what a hidden key holds may be anything
      float v[VE];
      widen<T>(y, v);
#pragma unroll
      for (int r = 0; r < R; r++)
#pragma unroll
        for (int e = 0; e < VE; e++) o[r][e] = fmaf(s[u][r], v[e], o[r][e]);
    }
  }
  // the warp's lane groups, then the block's warps
#pragma unroll
  for (int r = 0; r < R; r++) {
    float top = m[r];
#pragma unroll
    for (int w = LPK; w < 32; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
    const float f = tc::ex2(m[r] - (top == -INFINITY ? 0.f : top));
    l[r] *= f;
#pragma unroll
    for (int e = 0; e < VE; e++) o[r][e] *= f;
#pragma unroll
    for (int w = LPK; w < 32; w <<= 1) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], w);
#pragma unroll
      for (int e = 0; e < VE; e++) o[r][e] += __shfl_xor_sync(0xffffffffu, o[r][e], w);
    }
    if (grp == 0) {
#pragma unroll
      for (int e = 0; e < VE; e++) so[warp][r][e0 + e] = o[r][e];
      if (lane == 0) { sm[warp][r] = top; sl[warp][r] = l[r]; }
    }
  }
  __syncthreads();
  // the block's sums, in the first warp's place
  for (int i = threadIdx.x; i < R * D; i += RW_T) {
    const int r = i / D, e = i % D;
    float top = sm[0][r], x = 0.f;
#pragma unroll
    for (int w = 1; w < RW_WARPS; w++) top = fmaxf(top, sm[w][r]);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < RW_WARPS; w++) x = fmaf(tc::ex2(sm[w][r] - base), so[w][r][e], x);
    so[0][r][e] = x;
  }
  __syncthreads();
  if (threadIdx.x < R) {
    const int r = threadIdx.x;
    float top = sm[0][r], sum = 0.f;
#pragma unroll
    for (int w = 1; w < RW_WARPS; w++) top = fmaxf(top, sm[w][r]);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < RW_WARPS; w++) sum = fmaf(tc::ex2(sm[w][r] - base), sl[w][r], sum);
    sm[0][r] = top;
    sl[0][r] = sum;
  }
  const bool cluster = !part.o && part.pieces > 1;
  if (cluster) tc::cluster_sync();
  else __syncthreads();
  if (!cluster || piece == 0)
    for (int i = threadIdx.x; i < R * D; i += RW_T) {
      const int r = i / D, e = i % D;
      if (r >= rows || e >= a.dv) continue;
      float top = sm[0][r], sum = sl[0][r], x = so[0][r][e];
      if (cluster) {
        const uint32_t am = tc::smem_u32(&sm[0][r]), al = tc::smem_u32(&sl[0][r]), ao = tc::smem_u32(&so[0][r][e]);
        for (int p = 1; p < part.pieces; p++) top = fmaxf(top, tc::load_cluster(tc::map_cluster(am, p)));
        const float base = top == -INFINITY ? 0.f : top;
        sum = x = 0.f;
        for (int p = 0; p < part.pieces; p++) {
          const float f = tc::ex2(tc::load_cluster(tc::map_cluster(am, p)) - base);
          sum = fmaf(f, tc::load_cluster(tc::map_cluster(al, p)), sum);
          x = fmaf(f, tc::load_cluster(tc::map_cluster(ao, p)), x);
        }
      }
      if (part.o) {
        const int64_t at = ((int64_t)unit * part.pieces + piece) * rows + r;
        part.o[at * a.dv + e] = x;
        if (e == 0) part.ml[at] = make_float2(top, sum);
      } else {
        const int h = hk * a.g + r / a.Lq, tok = r % a.Lq;
        fs_store(Y + b * ay.sb + h * ay.sh + tok * ay.sl + e, sum == 0.f ? 0.f : x / sum);
        if (lse && e == 0) lse[((int64_t)b * a.H + h) * a.Lq + tok] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * FS_LN2;
      }
    }
  if (cluster) tc::cluster_sync();      // (a block's shared memory is read until here)
}

// Y and lse from the pieces' partial results: a thread per row and four values.
template <typename T>
__global__ void __launch_bounds__(256)
cross_join_kernel(CrossPart part, int64_t units, int Hk, int R, int g, int Lq, int dv, T* __restrict__ Y, TensorAddr ay, float* __restrict__ lse) {
  fs_grid_dependency_wait();
  const int q = dv / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / q;
  const int e = (int)(i % q) * 4;
  if (row >= units * R) return;
  const int64_t unit = row / R;
  const int r = (int)(row % R);
  float top = -INFINITY;
  for (int p = 0; p < part.pieces; p++) top = fmaxf(top, part.ml[(unit * part.pieces + p) * R + r].x);
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int p = 0; p < part.pieces; p++) {
    const int64_t at = (unit * part.pieces + p) * R + r;
    const float2 ml = part.ml[at];
    const float4 o = *reinterpret_cast<const float4*>(part.o + at * dv + e);
    const float f = tc::ex2(ml.x - base);
    sum = fmaf(f, ml.y, sum);
    x.x = fmaf(f, o.x, x.x); x.y = fmaf(f, o.y, x.y); x.z = fmaf(f, o.z, x.z); x.w = fmaf(f, o.w, x.w);
  }
  const int64_t b = unit / Hk;
  const int h = (int)(unit % Hk) * g + r / Lq, tok = r % Lq;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T* y = Y + b * ay.sb + h * ay.sh + tok * ay.sl + e;
  fs_store(y, x.x * inv); fs_store(y + 1, x.y * inv); fs_store(y + 2, x.z * inv); fs_store(y + 3, x.w * inv);
  if (lse && e == 0) lse[(b * Hk * g + h) * Lq + tok] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * FS_LN2;
}

template <typename T, int D, int R>
int launch_rows(fsharp_ctx* ctx, const CrossArgs& a, T* Y, TensorAddr ay, float* lse, CrossPart part) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)part.pieces, (unsigned)(a.B * a.Hk));
  cfg.blockDim = dim3(RW_T);
  cfg.dynamicSmemBytes = (size_t)rows_stages(D) * 2 * rows_u(D) * RW_T * 16;
  cfg.stream = ctx->stream;
  cudaLaunchAttribute at[1];
  if (!part.o && part.pieces > 1) {
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)part.pieces;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
  }
  FS_CUDA_OK(fs_allow_smem(cross_rows_kernel<T, D, R>, sizeof(float) * RW_WARPS * R * (D + 2)));
  FS_TIME_BEGIN(ctx, FS_K_CROSS_ROWS);
  FS_CUDA_OK(cudaLaunchKernelEx(&cfg, cross_rows_kernel<T, D, R>, a, Y, ay, lse, part));
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  return FSHARP_OK;
}

template <typename T, int R>
int run_rows(fsharp_ctx* ctx, const CrossArgs& a, void* Yv, TensorAddr ay, float* lse, CrossPart part) {
  const int D = a.d > a.dv ? a.d : a.dv;
  T* Y = static_cast<T*>(Yv);
  if (D == 16) return launch_rows<T, 16, R>(ctx, a, Y, ay, lse, part);
  if (D == 32) return launch_rows<T, 32, R>(ctx, a, Y, ay, lse, part);
  if (D == 64) return launch_rows<T, 64, R>(ctx, a, Y, ay, lse, part);
  return launch_rows<T, 128, R>(ctx, a, Y, ay, lse, part);
}

template <typename T>
int run_join(fsharp_ctx* ctx, const CrossArgs& a, T* Y, TensorAddr ay, float* lse, CrossPart part) {
  const int R = a.g * a.Lq;
  const int64_t units = (int64_t)a.B * a.Hk, blocks = (units * R * (a.dv / 4) + 255) / 256;
  if (blocks > 0x7fffffff) return FSHARP_E_SHAPE;
  FS_TIME_BEGIN(ctx, FS_K_CROSS_JOIN);
  FS_CUDA_OK(fs_launch_chained(cross_join_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, ctx->stream, part, units, a.Hk, R, a.g, a.Lq,
                               a.dv, Y, ay, lse));
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  return FSHARP_OK;
}

}  // namespace

// Up to how many rows of a unit this kernel is the one to take: one of bf16, four of fp32.  Each call whole, us, by this kernel (with
// its two- to eight-row forms of either type built for the measurement) for 1 | 2 | 4 | 8 rows, and by the other one, whose time hardly
// depends on the rows up to 16:
//                                     bf16, here          tensor cores    fp32, here              multiply-add tiles
//   64 x 12 x 1500 keys, d = 64       70 | 70 | 88 | 191       100        115 | 115 | 131 | 195         594
//   8 x 12 x 32768 keys, d = 64       174 | 182 | 223 | 408    207        301 | 317 | 365 | 537        1411
//   32 x 8 x 1024 keys, d = 128       39 | 43 | 59 | 109       45         66 | 68 | 103 | 121           229
//   16 x 4 x 16384 keys, d = 128      119 | 127 | 174 | 260    106        199 | 215 | 420 | 430         878
//   1 x 8 x 512 keys, d = 64          8.2 | 10 | 10 | 16       14         12 | 12 | 12 | 14              16
// So the rule is on the safe side: two bf16 rows of d = 64 and five to eight fp32 rows would still be faster here; one bf16 row against
// long sequences of d = 128 would be 12 % faster on the tensor cores.
int fs_cross_rows_most(int dtype) { return dtype == FSHARP_F32 ? 4 : 1; }

// Pieces of the keys: enough for six blocks per SM, each with two turns of keys, where eight pieces (a cluster, which joins them
// itself) do; where they leave SMs without work, as many more, through scratch, as give every SM two blocks.
int fs_cross_rows_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int dtype, bool* cluster) {
  const int es = dtype == FSHARP_F32 ? 4 : 2, D = dm->d > dm->dv ? dm->d : dm->dv, step = rows_step(D, es);
  const int64_t units = (int64_t)dm->B * dm->Hk, turns = ((int64_t)dm->Lk + step - 1) / step, sms = ctx->sm_count;
  int64_t p = (6 * sms + units - 1) / units;
  if (p > turns / 2) p = turns / 2;
  *cluster = p <= RW_CLUSTER || units * RW_CLUSTER >= 2 * sms;
  if (*cluster) p = p > RW_CLUSTER ? RW_CLUSTER : p;
  else p = p < 2 * sms / units ? p : 2 * sms / units;
  return p < 1 ? 1 : p > 256 ? 256 : (int)p;
}

int fs_cross_rows(fsharp_ctx* ctx, const CrossArgs& a, int dtype, void* Y, TensorAddr ay, float* lse, CrossPart part) {
  const int R = a.g * a.Lq;
  if (dtype == FSHARP_BF16) return run_rows<__nv_bfloat16, 1>(ctx, a, Y, ay, lse, part);
  return R == 1 ? run_rows<float, 1>(ctx, a, Y, ay, lse, part) : R == 2 ? run_rows<float, 2>(ctx, a, Y, ay, lse, part)
                                                               : run_rows<float, 4>(ctx, a, Y, ay, lse, part);
}
int fs_cross_join(fsharp_ctx* ctx, const CrossArgs& a, int dtype, void* Y, TensorAddr ay, float* lse, CrossPart part) {
  return dtype == FSHARP_F32 ? run_join<float>(ctx, a, static_cast<float*>(Y), ay, lse, part)
                             : run_join<__nv_bfloat16>(ctx, a, static_cast<__nv_bfloat16*>(Y), ay, lse, part);
}
