// Entry points of the exact cross attention: argument checks, choice of the kernels, the backward pass's row statistics and
// the sums over pieces.
#include <math.h>

#include "cross.cuh"

namespace {

// -lse log2(e) and -D, D = dY . Y, of every row and of the places up to a multiple of 128 (cross.cuh).  dv / VE lanes share a
// row's dv values, 16 bytes each.
template <typename T>
__global__ void __launch_bounds__(256)
cross_delta_kernel(const T* __restrict__ Y, TensorAddr ay, const T* __restrict__ dY, TensorAddr ady, const float* __restrict__ lse,
                   int64_t places, int H, int Lq, int dv, float* __restrict__ stat) {
  constexpr int VE = 16 / (int)sizeof(T);
  const int lpr = dv / VE, Lp = (Lq + 127) / 128 * 128;  // lpr: 2 .. 32, a power of two
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, place = i / lpr, bh = place / Lp;
  const int e = (int)(i % lpr) * VE, tok = (int)(place % Lp);
  const bool row = place < places && tok < Lq;
  float sum = 0.f;
  if (row) {
    const int64_t b = bh / H, h = bh % H;
    const uint4 y = *reinterpret_cast<const uint4*>(Y + b * ay.sb + h * ay.sh + tok * ay.sl + e);
    const uint4 g = *reinterpret_cast<const uint4*>(dY + b * ady.sb + h * ady.sh + tok * ady.sl + e);
    const T *py = reinterpret_cast<const T*>(&y), *pg = reinterpret_cast<const T*>(&g);
#pragma unroll
    for (int k = 0; k < VE; k++) sum = fmaf(fs_load(py + k), fs_load(pg + k), sum);
  }
  for (int w = 1; w < lpr; w <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
  if (place < places && e == 0) {
    const float x = row ? lse[bh * Lq + tok] : -INFINITY;
    float* to = stat + bh * cross_stat_floats(Lq) + (int64_t)(tok >> 7) * 256 + (tok & 127);
    to[0] = x == -INFINITY ? -INFINITY : -x * FS_LOG2E;
    to[128] = row ? -sum : 0.f;
  }
}

// out [B,H,L,width] = the sum over the pieces, in their order, of part [piece][B H L][ld] from column `off` on.
template <typename T>
__global__ void __launch_bounds__(256)
cross_sum_kernel(const float* __restrict__ part, int pieces, int64_t rows, int ld, int off, int width, int H, int L, T* __restrict__ out,
                 TensorAddr to) {
  fs_grid_dependency_wait();
  const int q = width / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / q;
  const int e = (int)(i % q) * 4;
  if (row >= rows) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int p = 0; p < pieces; p++) {
    const float4 x = *reinterpret_cast<const float4*>(part + (p * rows + row) * ld + off + e);
    s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
  }
  T* y = out + row / ((int64_t)H * L) * to.sb + row / L % H * to.sh + row % L * to.sl + e;
  fs_store(y, s.x); fs_store(y + 1, s.y); fs_store(y + 2, s.z); fs_store(y + 3, s.w);
}

template <typename T>
int run_delta(fsharp_ctx* ctx, const CrossArgs& a, const void* Y, TensorAddr ay, const void* dY, TensorAddr ady, const float* lse, float* stat) {
  const int64_t places = (int64_t)a.B * a.H * (((int64_t)a.Lq + 127) / 128 * 128), blocks = (places * (a.dv * (int64_t)sizeof(T) / 16) + 255) / 256;
  if (blocks > 0x7fffffff) return FSHARP_E_SHAPE;
  FS_TIME_BEGIN(ctx, FS_K_CROSS_DELTA);
  cross_delta_kernel<T><<<(unsigned)blocks, 256, 0, ctx->stream>>>(static_cast<const T*>(Y), ay, static_cast<const T*>(dY), ady, lse, places,
                                                                    a.H, a.Lq, a.dv, stat);
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  return FSHARP_OK;
}
template <typename T>
int run_sum(fsharp_ctx* ctx, const float* part, int pieces, int64_t rows, int ld, int off, int width, int H, int L, void* out, TensorAddr to) {
  const int64_t blocks = (rows * (width / 4) + 255) / 256;
  if (blocks > 0x7fffffff) return FSHARP_E_SHAPE;
  FS_TIME_BEGIN(ctx, FS_K_CROSS_SUM);
  FS_CUDA_OK(fs_launch_chained(cross_sum_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, ctx->stream, part, pieces, rows, ld, off, width,
                               H, L, static_cast<T*>(out), to));
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  return FSHARP_OK;
}

bool head_ok(int d) { return d == 16 || d == 32 || d == 64 || d == 128; }

int check(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int dtype) {
  if (!ctx || !dm) return FSHARP_E_BADARG;
  if (dm->B < 0 || dm->H < 0 || dm->Hk < 0 || dm->Lq < 0 || dm->Lk < 0) return FSHARP_E_SHAPE;
  if (!head_ok(dm->d) || !head_ok(dm->dv)) return FSHARP_E_SHAPE;
  if (dm->Hk ? dm->H % dm->Hk != 0 : dm->H != 0) return FSHARP_E_SHAPE;
  if ((int64_t)dm->B * dm->Hk > 65535) return FSHARP_E_SHAPE;
  // rows of a unit and keys are 32-bit indexes, with room for a tile behind the last
  if (dm->Hk && (int64_t)(dm->H / dm->Hk) * dm->Lq > 0x7ffffe00) return FSHARP_E_SHAPE;
  if (dm->Lk > 0x7ffffe00) return FSHARP_E_SHAPE;
  if (dtype != FSHARP_F32 && dtype != FSHARP_BF16) return FSHARP_E_DTYPE;
  if (ctx->impl == FSHARP_IMPL_TENSOR && dtype != FSHARP_BF16 && (dm->d > 64 || dm->dv > 64)) return FSHARP_E_SHAPE;
  return FSHARP_OK;
}

int check_tensor(const void* p, int dtype, const int64_t s[3]) {
  if (!p) return FSHARP_E_BADARG;
  const size_t es = dtype == FSHARP_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return FSHARP_E_ALIGN;
  for (int i = 0; i < 3; i++)
    if (s[i] < 0 || (s[i] * es) % 16 != 0) return FSHARP_E_ALIGN;
  return FSHARP_OK;
}

// The same, and a token stride that tells the tokens apart (a tensor map has no other).
int check_tokens(const void* p, int dtype, const int64_t s[3], int L) {
  FS_TRY(check_tensor(p, dtype, s));
  return L > 1 && s[2] == 0 && (s[0] != 0 || s[1] != 0) ? FSHARP_E_SHAPE : FSHARP_OK;
}

enum Kind { ROWS, FMA, TC, TC32 };
struct Plan {
  Kind kind;
  int pieces;
  bool join;                   // the pieces meet in scratch
  int64_t o_floats, ml;        // partial results
  int64_t parts;               // bf16 parts of fp32 operands
};

// Rows of a unit up to which fp32 takes the multiply-add tiles of 16 rows: 16 rows there and 17 on the tensor cores, whose time does not
// depend on them, 64 x 12 units of 1500 keys, d = 64: 596 us (17 rows: 807) and 618; 8 x 12 of 32768: 1415 (1907) and 1905; 1 x 4 of 300, d = 32:
// 12 (14) and 19.
constexpr int FMA_MOST_ROWS = 16;
// fp32 on the tensor cores: heads that leave room for three parts of every operand in shared memory.
bool parts_fit(const fsharp_cross_dims* dm) { return dm->d <= 64 && dm->dv <= 64; }

Plan plan_forward(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int dtype) {
  Plan p = {};
  const int64_t R = (int64_t)dm->H / dm->Hk * dm->Lq, units = (int64_t)dm->B * dm->Hk;
  const bool bf16 = dtype == FSHARP_BF16;
  if (ctx->impl == FSHARP_IMPL_TENSOR) p.kind = bf16 ? TC : TC32;
  else if (R <= fs_cross_rows_most(dtype)) p.kind = ROWS;
  else if (ctx->impl == FSHARP_IMPL_SIMT) p.kind = FMA;
  else p.kind = bf16 ? TC : parts_fit(dm) && R > FMA_MOST_ROWS ? TC32 : FMA;
  if (dm->Lk == 0) p.kind = FMA;       // (zeros: there is no key that a tensor map could describe)
  bool cluster = false;
  switch (p.kind) {
    case ROWS: p.pieces = fs_cross_rows_pieces(ctx, dm, dtype, &cluster); break;
    case FMA: p.pieces = fs_cross_fma_pieces(ctx, dm); break;
    case TC: p.pieces = fs_tc_cross_pieces(ctx, dm); break;
    case TC32: p.pieces = fs_tc_cross_f32_pieces(ctx, dm); p.parts = fs_tc_cross_f32_parts(dm, 0); break;
  }
  p.join = p.pieces > 1 && !cluster;
  if (p.join) {
    p.ml = units * p.pieces * R;
    p.o_floats = p.ml * dm->dv;
  }
  return p;
}

struct GradPlan {
  Kind kind;
  int64_t parts;
  int kv_pieces, q_pieces;
  int64_t stat, kv_floats, q_floats;
};
GradPlan plan_backward(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int dtype) {
  GradPlan p = {};
  const int64_t R = (int64_t)dm->H / dm->Hk * dm->Lq, units = (int64_t)dm->B * dm->Hk;
  p.kind = FMA;
  if (ctx->impl != FSHARP_IMPL_SIMT && dm->Lk > 0) p.kind = dtype == FSHARP_BF16 ? TC : parts_fit(dm) ? TC32 : FMA;
  if (p.kind == TC) fs_tc_cross_grad_pieces(ctx, dm, &p.kv_pieces, &p.q_pieces);
  else if (p.kind == TC32) fs_tc_cross_f32_grad_pieces(ctx, dm, &p.kv_pieces, &p.q_pieces);
  else fs_cross_fma_grad_pieces(ctx, dm, &p.kv_pieces, &p.q_pieces);
  if (p.kind == TC32) p.parts = fs_tc_cross_f32_parts(dm, 1);
  p.stat = (int64_t)dm->B * dm->H * cross_stat_floats(dm->Lq);
  if (p.kv_pieces > 1) p.kv_floats = p.kv_pieces * units * dm->Lk * (dm->d + dm->dv);
  if (p.q_pieces > 1) p.q_floats = p.q_pieces * units * R * dm->d;
  return p;
}

CrossArgs args_of(const fsharp_cross_dims* dm, const void* Q, const void* K, const void* V, const int32_t* key_len, const uint8_t* key_mask,
                  float scale) {
  CrossArgs a;
  a.Q = Q; a.K = K; a.V = V;
  a.aq = fs_addr(dm->q_stride, dm->H, dm->Lq, dm->d);
  a.ak = fs_addr(dm->k_stride, dm->Hk, dm->Lk, dm->d);
  a.av = fs_addr(dm->v_stride, dm->Hk, dm->Lk, dm->dv);
  a.key_len = key_len; a.key_mask = key_mask; a.mask_stride = dm->mask_stride;
  a.B = dm->B; a.H = dm->H; a.Hk = dm->Hk; a.g = dm->H / dm->Hk; a.Lq = dm->Lq; a.Lk = dm->Lk; a.d = dm->d; a.dv = dm->dv;
  a.scale = scale;
  a.ranked = 0;
  return a;
}

int64_t forward_bytes(const Plan& p) { return (int64_t)((p.join ? ws_round(p.o_floats * 4) + ws_round(p.ml * 8) : 0) + ws_round(p.parts * 2)); }
int64_t backward_bytes(const GradPlan& p) { return (int64_t)(ws_round(p.stat * 4) + ws_round(p.kv_floats * 4) + ws_round(p.q_floats * 4) + ws_round(p.parts * 2)); }

int check_scratch(const void* scratch, int64_t have, int64_t need) {
  if (need == 0) return FSHARP_OK;
  if (!scratch) return FSHARP_E_BADARG;
  if (reinterpret_cast<uintptr_t>(scratch) % 16 != 0) return FSHARP_E_ALIGN;
  return have < need ? FSHARP_E_NOMEM : FSHARP_OK;
}

}  // namespace

extern "C" {

int64_t fsharp_cross_scratch_bytes(const fsharp_ctx* ctx, const fsharp_cross_dims* dims, int dtype, int backward) {
  FS_TRY(check(ctx, dims, dtype));
  if ((int64_t)dims->B * dims->H == 0 || dims->Lq == 0) return 0;
  return backward ? backward_bytes(plan_backward(ctx, dims, dtype)) : forward_bytes(plan_forward(ctx, dims, dtype));
}

int fsharp_cross_attend(fsharp_ctx* ctx, const void* Q, const void* K, const void* V, const int32_t* key_len, const uint8_t* key_mask,
                        const fsharp_cross_dims* dims, int dtype, float scale, void* Y, float* lse, void* scratch,
                        int64_t scratch_bytes) {
  FS_RANGE("fsharp_cross_attend");
  FS_TRY(check(ctx, dims, dtype));
  if (!(scale >= 0.f) || !isfinite(scale)) return FSHARP_E_BADARG;
  if (dims->mask_stride < 0) return FSHARP_E_BADARG;
  if ((int64_t)dims->B * dims->H == 0 || dims->Lq == 0) return FSHARP_OK;
  FS_TRY(check_tensor(Q, dtype, dims->q_stride));
  if (dims->Lk) {                     // (without keys K and V are not read)
    FS_TRY(check_tokens(K, dtype, dims->k_stride, dims->Lk));
    FS_TRY(check_tokens(V, dtype, dims->v_stride, dims->Lk));
  }
  FS_TRY(check_tensor(Y, dtype, dims->y_stride));
  const Plan p = plan_forward(ctx, dims, dtype);
  FS_TRY(check_scratch(scratch, scratch_bytes, forward_bytes(p)));
  FsDevice device(ctx->device);
  if (!device.ok) return FSHARP_E_CUDA;
  const CrossArgs a = args_of(dims, Q, K, V, key_len, key_mask, scale);
  const TensorAddr ay = fs_addr(dims->y_stride, dims->H, dims->Lq, dims->dv);
  CrossPart part = {nullptr, nullptr, p.pieces};
  WsAlloc ws{static_cast<char*>(scratch), 0};
  if (p.join) {
    part.o = ws.take<float>(p.o_floats);
    part.ml = ws.take<float2>(p.ml);
  }
  if (p.kind == ROWS) FS_TRY(fs_cross_rows(ctx, a, dtype, Y, ay, lse, part));
  else if (p.kind == TC) FS_TRY(fs_tc_cross(ctx, a, Y, ay, lse, part));
  else if (p.kind == TC32) FS_TRY(fs_tc_cross_f32(ctx, a, Y, ay, lse, part, ws.take<char>(p.parts * 2)));
  else FS_TRY(fs_cross_fma(ctx, a, dtype, Y, ay, lse, part));
  return p.join ? fs_cross_join(ctx, a, dtype, Y, ay, lse, part) : FSHARP_OK;
}

int fsharp_cross_attend_backward(fsharp_ctx* ctx, const void* Q, const void* K, const void* V, const void* Y, const float* lse,
                                 const void* dY, const int32_t* key_len, const uint8_t* key_mask, const fsharp_cross_dims* dims, int dtype,
                                 float scale, void* dQ, void* dK, void* dV, void* scratch, int64_t scratch_bytes) {
  FS_RANGE("fsharp_cross_attend_backward");
  FS_TRY(check(ctx, dims, dtype));
  if (!(scale >= 0.f) || !isfinite(scale)) return FSHARP_E_BADARG;
  if (dims->mask_stride < 0) return FSHARP_E_BADARG;
  if ((int64_t)dims->B * dims->Hk == 0) return FSHARP_OK;
  if (dims->H == 0 || dims->Lq == 0) return dims->Lk == 0 ? FSHARP_OK : FSHARP_E_SHAPE;      // no query: nothing to differentiate
  FS_TRY(check_tokens(Q, dtype, dims->q_stride, dims->Lq));
  FS_TRY(check_tensor(Y, dtype, dims->y_stride));
  FS_TRY(check_tokens(dY, dtype, dims->dy_stride, dims->Lq));
  FS_TRY(check_tensor(dQ, dtype, dims->dq_stride));
  if (!lse) return FSHARP_E_BADARG;
  if (dims->Lk) {
    FS_TRY(check_tokens(K, dtype, dims->k_stride, dims->Lk));
    FS_TRY(check_tokens(V, dtype, dims->v_stride, dims->Lk));
    FS_TRY(check_tensor(dK, dtype, dims->dk_stride));
    FS_TRY(check_tensor(dV, dtype, dims->dv_stride));
  }
  const GradPlan p = plan_backward(ctx, dims, dtype);
  FS_TRY(check_scratch(scratch, scratch_bytes, backward_bytes(p)));
  FsDevice device(ctx->device);
  if (!device.ok) return FSHARP_E_CUDA;
  const CrossArgs a = args_of(dims, Q, K, V, key_len, key_mask, scale);
  WsAlloc ws{static_cast<char*>(scratch), 0};
  float* stat = ws.take<float>(p.stat);
  CrossGrad gr;
  gr.dY = dY;
  gr.ady = fs_addr(dims->dy_stride, dims->H, dims->Lq, dims->dv);
  gr.stat = stat;
  gr.dQ = dQ; gr.dK = dK; gr.dV = dV;
  gr.adq = fs_addr(dims->dq_stride, dims->H, dims->Lq, dims->d);
  gr.adk = fs_addr(dims->dk_stride, dims->Hk, dims->Lk, dims->d);
  gr.adv = fs_addr(dims->dv_stride, dims->Hk, dims->Lk, dims->dv);
  gr.kv_pieces = p.kv_pieces;
  gr.q_pieces = p.q_pieces;
  gr.pkv = p.kv_pieces > 1 ? ws.take<float>(p.kv_floats) : nullptr;
  gr.pq = p.q_pieces > 1 ? ws.take<float>(p.q_floats) : nullptr;
  const TensorAddr ay = fs_addr(dims->y_stride, dims->H, dims->Lq, dims->dv);
  const bool f32 = dtype == FSHARP_F32;
  FS_TRY(f32 ? run_delta<float>(ctx, a, Y, ay, dY, gr.ady, lse, stat) : run_delta<__nv_bfloat16>(ctx, a, Y, ay, dY, gr.ady, lse, stat));
  if (p.kind == TC) FS_TRY(fs_tc_cross_grad(ctx, a, gr));
  else if (p.kind == TC32) FS_TRY(fs_tc_cross_f32_grad(ctx, a, gr, ws.take<char>(p.parts * 2)));
  else FS_TRY(fs_cross_fma_grad(ctx, a, dtype, gr));
  const auto sum = f32 ? run_sum<float> : run_sum<__nv_bfloat16>;
  const int64_t keys = (int64_t)a.B * a.Hk * a.Lk;
  if (gr.pkv) {
    FS_TRY(sum(ctx, gr.pkv, p.kv_pieces, keys, a.d + a.dv, 0, a.d, a.Hk, a.Lk, dK, gr.adk));
    FS_TRY(sum(ctx, gr.pkv, p.kv_pieces, keys, a.d + a.dv, a.d, a.dv, a.Hk, a.Lk, dV, gr.adv));
  }
  if (gr.pq) FS_TRY(sum(ctx, gr.pq, p.q_pieces, (int64_t)a.B * a.H * a.Lq, a.d, 0, a.d, a.H, a.Lq, dQ, gr.adq));
  return FSHARP_OK;
}

}  // extern "C"
