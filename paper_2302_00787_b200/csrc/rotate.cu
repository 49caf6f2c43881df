// Rotary positions on queries and keys.  Pair j < rot / 2 of a head, (a, b) = features (j, j + rot / 2) or (2j, 2j + 1),
// of a token at position p becomes
//   (a', b') = gain (a cos t - b sin t, b cos t + a sin t),   t = 2 pi p f_j,
// f_j in turns per position; features from rot on pass through.  The transpose (the gradient) has -t.
//
// Bound: HBM, every tensor read once and written once.  A thread owns W pairs of one token (two vectors of W values per
// head) and walks the heads: the angle, a 64-bit product reduced to a fraction of a turn so that far positions lose
// nothing, and its sine and cosine are computed once per token and pair and serve `hpt` heads.
// Queries and keys share the launch: a decoding step is bound by the launch alone.
#include <math.h>

#include "common.cuh"

namespace {

constexpr int ROT_T = 256;

struct RotTensors {
  const void* x[2];      // queries, keys
  void* y[2];
  TensorAddr ax[2], ay[2];
  int H[2];
};
struct RotFreq {
  double turns[64];      // per position
};

template <typename T, int W>
struct alignas(sizeof(T) * W) Vec {
  T v[W];
};

template <typename T, int W>
__global__ void __launch_bounds__(ROT_T)
rotate_kernel(RotTensors t, const __grid_constant__ RotFreq freq, const int64_t* __restrict__ pos, int64_t pos_stride, int64_t pos0,
              int64_t tokens, int L, int d, int rot, int interleaved, int hpt, float gain, float sign) {
  const int units = d / (2 * W);                      // a power of two
  const int64_t g = (int64_t)blockIdx.x * ROT_T + threadIdx.x;
  const int64_t tok = g / units;
  const int u = (int)(g % units);
  if (tok >= tokens) return;
  const int64_t b = tok / L, i = tok % L;
  // pairs u W .. u W + W - 1; those past rot / 2 (a multiple of W) are neighbours that pass through
  const int p0 = u * W;
  const bool turn = p0 < rot / 2;
  int ja, jb;
  if (interleaved) { ja = 2 * p0; jb = ja + W; }
  else if (turn) { ja = p0; jb = p0 + rot / 2; }
  else { ja = 2 * p0; jb = ja + W; }                  // = rot + 2 (p0 - rot / 2)
  float c[W], s[W];
  if (turn) {
    const double p = (double)((pos ? pos[b * pos_stride + i] : i) + pos0);
#pragma unroll
    for (int k = 0; k < W; k++) {
      const double n = p * freq.turns[p0 + k];
      float sn, cs;
      sincospif(2.f * (float)(n - rint(n)), &sn, &cs);
      c[k] = gain * cs;
      s[k] = gain * sign * sn;
    }
  } else {
#pragma unroll
    for (int k = 0; k < W; k++) { c[k] = 1.f; s[k] = 0.f; }
  }
  const int heads = t.H[0] + t.H[1], h0 = blockIdx.y * hpt, h1 = min(heads, h0 + hpt);
  using V = Vec<T, W>;
  auto at = [&](int h, const T*& x, T*& y) {
    const int w = h >= t.H[0];
    const int64_t hh = w ? h - t.H[0] : h;
    x = static_cast<const T*>(t.x[w]) + b * t.ax[w].sb + hh * t.ax[w].sh + i * t.ax[w].sl;
    y = static_cast<T*>(t.y[w]) + b * t.ay[w].sb + hh * t.ay[w].sh + i * t.ay[w].sl;
  };
  constexpr int U = 4;                                // heads with their loads in flight together
  for (int h = h0; h < h1; h += U) {
    V a[U], e[U];
    T* out[U];
#pragma unroll
    for (int q = 0; q < U; q++)
      if (h + q < h1) {
        const T* x;
        at(h + q, x, out[q]);
        a[q] = *reinterpret_cast<const V*>(x + ja);
        e[q] = *reinterpret_cast<const V*>(x + jb);
      }
#pragma unroll
    for (int q = 0; q < U; q++)
      if (h + q < h1) {
        V ya, yb;
        if (interleaved && W > 1) {
          // the unit's 2 W values in a row: pair k is (2k, 2k + 1)
          float z[2 * W];
#pragma unroll
          for (int k = 0; k < W; k++) { z[k] = fs_load(&a[q].v[k]); z[W + k] = fs_load(&e[q].v[k]); }
#pragma unroll
          for (int k = 0; k < W; k++) {
            const float r = z[2 * k] * c[k] - z[2 * k + 1] * s[k], m = z[2 * k + 1] * c[k] + z[2 * k] * s[k];
            fs_store(2 * k < W ? &ya.v[(2 * k) % W] : &yb.v[(2 * k) % W], r);
            fs_store(2 * k + 1 < W ? &ya.v[(2 * k + 1) % W] : &yb.v[(2 * k + 1) % W], m);
          }
        } else {
#pragma unroll
          for (int k = 0; k < W; k++) {
            const float x0 = fs_load(&a[q].v[k]), x1 = fs_load(&e[q].v[k]);
            fs_store(&ya.v[k], x0 * c[k] - x1 * s[k]);
            fs_store(&yb.v[k], x1 * c[k] + x0 * s[k]);
          }
        }
        if (!turn) { ya = a[q]; yb = e[q]; }          // the bits as they are, NaNs among them
        *reinterpret_cast<V*>(out[q] + ja) = ya;
        *reinterpret_cast<V*>(out[q] + jb) = yb;
      }
  }
}

template <typename T, int W>
int launch(fsharp_ctx* ctx, const RotTensors& t, const RotFreq& f, const int64_t* pos, int64_t pos_stride, int64_t pos0, int64_t tokens,
           int L, int d, const fsharp_rope* r, int transpose) {
  const int heads = t.H[0] + t.H[1];
  const int64_t units = tokens * (d / (2 * W));
  // Heads per thread: as many as leave the GPU full (the angles are shared by them), at most 8.
  int64_t hpt = units * heads / ((int64_t)ctx->sm_count * 2048);
  hpt = hpt < 1 ? 1 : hpt > 8 ? 8 : hpt;
  const int64_t gx = (units + ROT_T - 1) / ROT_T, gy = (heads + hpt - 1) / hpt;
  if (gx > 0x7fffffff || gy > 65535) return FSHARP_E_SHAPE;
  FS_TIME_BEGIN(ctx, FS_K_ROTATE);
  rotate_kernel<T, W><<<dim3((unsigned)gx, (unsigned)gy), ROT_T, 0, ctx->stream>>>(
      t, f, pos, pos_stride, pos0, tokens, L, d, r->rot, r->layout == FSHARP_ROT_INTERLEAVED, (int)hpt, (float)r->gain,
      transpose ? -1.f : 1.f);
  FS_TIME_END(ctx);
  FS_LAUNCH_CHECK(ctx);
  return FSHARP_OK;
}

bool positive(double x) { return x > 0.0 && isfinite(x); }

int check_side(const void* x, const void* y, const int64_t sx[3], const int64_t sy[3], size_t es) {
  if (!x || !y) return FSHARP_E_BADARG;
  if (reinterpret_cast<uintptr_t>(x) % 16 || reinterpret_cast<uintptr_t>(y) % 16) return FSHARP_E_ALIGN;
  for (int k = 0; k < 3; k++)
    if (sx[k] < 0 || sy[k] < 0 || sx[k] * es % 16 || sy[k] * es % 16) return FSHARP_E_ALIGN;
  return FSHARP_OK;
}

}  // namespace

extern "C" int fsharp_rotate(fsharp_ctx* ctx, const void* Q, const void* K, const int64_t* pos, int64_t pos_stride, int64_t pos0,
                             const fsharp_rope* rope, const fsharp_rotate_dims* dims, int dtype, int transpose, void* Qout,
                             void* Kout) {
  FS_RANGE("fsharp_rotate");
  if (!ctx || !rope || !dims) return FSHARP_E_BADARG;
  const int d = dims->d, rot = rope->rot;
  if (dims->B < 0 || dims->L < 0 || dims->H < 0 || dims->Hk < 0) return FSHARP_E_SHAPE;
  if (d != 16 && d != 32 && d != 64 && d != 128) return FSHARP_E_SHAPE;
  if (rot < 2 || rot > d || rot % 2) return FSHARP_E_SHAPE;
  if (dtype != FSHARP_F32 && dtype != FSHARP_BF16) return FSHARP_E_DTYPE;
  if (rope->layout != FSHARP_ROT_HALF && rope->layout != FSHARP_ROT_INTERLEAVED) return FSHARP_E_BADARG;
  if (rope->scaling < FSHARP_ROPE_PLAIN || rope->scaling > FSHARP_ROPE_PARTS) return FSHARP_E_BADARG;
  if (!positive(rope->base) || !isfinite(rope->gain)) return FSHARP_E_BADARG;
  if (rope->scaling != FSHARP_ROPE_PLAIN && !positive(rope->factor)) return FSHARP_E_BADARG;
  if (rope->scaling == FSHARP_ROPE_NTK && rot == 2) return FSHARP_E_SHAPE;     // one pair: the exponent rot / (rot - 2) has no value
  if (rope->scaling == FSHARP_ROPE_PARTS &&
      (!positive(rope->original) || !isfinite(rope->slow) || !isfinite(rope->fast) || !(rope->fast > rope->slow)))
    return FSHARP_E_BADARG;
  if (pos_stride < 0) return FSHARP_E_BADARG;
  const int64_t tokens = (int64_t)dims->B * dims->L;
  if (tokens == 0 || dims->H + dims->Hk == 0) return FSHARP_OK;
  const size_t es = dtype == FSHARP_F32 ? 4 : 2;
  if (dims->H) FS_TRY(check_side(Q, Qout, dims->q_stride, dims->qo_stride, es));
  if (dims->Hk) FS_TRY(check_side(K, Kout, dims->k_stride, dims->ko_stride, es));
  FsDevice device(ctx->device);
  if (!device.ok) return FSHARP_E_CUDA;

  RotTensors t;
  t.x[0] = Q; t.x[1] = K; t.y[0] = Qout; t.y[1] = Kout;
  t.H[0] = dims->H; t.H[1] = dims->Hk;
  t.ax[0] = fs_addr(dims->q_stride, dims->H, dims->L, d);
  t.ax[1] = fs_addr(dims->k_stride, dims->Hk, dims->L, d);
  t.ay[0] = fs_addr(dims->qo_stride, dims->H, dims->L, d);
  t.ay[1] = fs_addr(dims->ko_stride, dims->Hk, dims->L, d);
  RotFreq f = {};
  const double turn = 6.283185307179586476925, s = rope->factor;
  const double base = rope->scaling == FSHARP_ROPE_NTK ? rope->base * pow(s, rot / (rot - 2.0)) : rope->base;
  const double step = log2(base) * 2.0 / rot;
  for (int j = 0; j < rot / 2; j++) {
    double n = exp2(-j * step) / turn;
    if (rope->scaling == FSHARP_ROPE_LINEAR) n /= s;
    if (rope->scaling == FSHARP_ROPE_PARTS) {
      double keep = (rope->original * n - rope->slow) / (rope->fast - rope->slow);     // from the turns in the trained length
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      n = n / s * (1.0 - keep) + n * keep;
    }
    f.turns[j] = n;
  }
  // The widest vectors that rot / 2 is a multiple of: a thread's pairs then all turn or all pass, and the half layout's
  // second vector is aligned.
  const int half = rot / 2;
#define FS_ROT(T, W) return launch<T, W>(ctx, t, f, pos, pos_stride, pos0, tokens, dims->L, d, rope, transpose)
  if (dtype == FSHARP_F32) {
    if (half % 4 == 0) FS_ROT(float, 4);
    if (half % 2 == 0) FS_ROT(float, 2);
    FS_ROT(float, 1);
  }
  if (half % 8 == 0) FS_ROT(__nv_bfloat16, 8);
  if (half % 4 == 0) FS_ROT(__nv_bfloat16, 4);
  if (half % 2 == 0) FS_ROT(__nv_bfloat16, 2);
  FS_ROT(__nv_bfloat16, 1);
#undef FS_ROT
}
