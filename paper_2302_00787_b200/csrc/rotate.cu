// Rotary positions on queries and keys.  Pair j < rot / 2 of a head, (a, b) = features (j, j + rot / 2) or (2j, 2j + 1),
// of a token at position p becomes
//   (a', b') = gain (a cos t - b sin t, b cos t + a sin t),   t = 2 pi p f_j,
// f_j in turns per position; features from rot on pass through.  The transpose (the gradient) has -t.
//
// Bound: HBM, every tensor read once and written once.  A thread owns W pairs of one token (two vectors of W values per
// head) and walks the heads: the angle, reduced to a fraction of a turn, and its sine and cosine are computed once per token
// and pair and serve `hpt` heads.  From 2^22 turns on f_j is the sum of two 64-bit numbers and p f_j a product with its
// remainder: with one, 2^31 f_0 would be off by 5e-8 turns (3.2e-7 radians, five half steps of an fp32 sine); nearer ones are off by 2^-31
// turns at most.  (The second number for all positions: 4 x 16 heads x 1501 tokens, fp32, 8.2 -> 9.2 us.)
// Queries and keys share the launch: a decoding step is bound by the launch alone.
#include <math.h>

#include "common.cuh"
#include "tc_common.cuh"

namespace {

constexpr int ROT_T = 256;

struct RotTensors {
  const void* x[2];      // queries, keys
  void* y[2];
  TensorAddr ax[2], ay[2];
  int H[2];
};
struct RotFreq {
  double turns[64], rest[64];      // per position, and what 64 bits leave of it
};

// W neighbouring values of a row, as one load or store; bf16 pairs are widened and rounded two at a time.
template <typename T, int W>
struct alignas(sizeof(T) * W) Vec {
  T v[W];
};
template <int W> __device__ __forceinline__ void widen(const Vec<float, W>& x, float* f) {
#pragma unroll
  for (int k = 0; k < W; k++) f[k] = x.v[k];
}
template <int W> __device__ __forceinline__ void widen(const Vec<__nv_bfloat16, W>& x, float* f) {
  if constexpr (W == 1) f[0] = __bfloat162float(x.v[0]);
  else {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(x.v);
#pragma unroll
    for (int k = 0; k < W; k += 2) { f[k] = __uint_as_float(w[k / 2] << 16); f[k + 1] = __uint_as_float(w[k / 2] & 0xffff0000u); }
  }
}
template <int W> __device__ __forceinline__ void narrow(Vec<float, W>& x, const float* f) {
#pragma unroll
  for (int k = 0; k < W; k++) x.v[k] = f[k];
}
template <int W> __device__ __forceinline__ void narrow(Vec<__nv_bfloat16, W>& x, const float* f) {
  if constexpr (W == 1) x.v[0] = __float2bfloat16_rn(f[0]);
  else {
    uint32_t* w = reinterpret_cast<uint32_t*>(x.v);
#pragma unroll
    for (int k = 0; k < W; k += 2) w[k / 2] = tc::pack_bf16(f[k], f[k + 1]);
  }
}

template <typename T, int W, bool INTERLEAVED>
__global__ void __launch_bounds__(ROT_T)
rotate_kernel(const __grid_constant__ RotTensors t, const __grid_constant__ RotFreq freq, const int64_t* __restrict__ pos, int64_t pos_stride,
              int64_t pos0, int64_t tokens, int L, int d, int rot, int hpt, float gain, float sign) {
  const int units = d / (2 * W);                      // a power of two
  const int64_t g = (int64_t)blockIdx.x * ROT_T + threadIdx.x;
  const int64_t tok = g / units;
  const int u = (int)(g % units);
  if (tok >= tokens) return;
  const int64_t b = tok / L, i = tok % L;
  // pairs u W .. u W + W - 1; those past rot / 2 (a multiple of W) are neighbours that pass through
  const int p0 = u * W;
  const bool turn = p0 < rot / 2;
  const int ja = turn && !INTERLEAVED ? p0 : 2 * p0, jb = turn && !INTERLEAVED ? p0 + rot / 2 : 2 * p0 + W;
  float c[W], s[W];
#pragma unroll
  for (int k = 0; k < W; k++) { c[k] = 1.f; s[k] = 0.f; }
  if (turn) {
    const double p = (double)((pos ? pos[b * pos_stride + i] : i) + pos0);
#pragma unroll
    for (int k = 0; k < W; k++) {
      const double f = freq.turns[p0 + k], n = p * f;
      double part = n - rint(n);
      if (fabs(n) >= 4194304.0) part += fma(p, freq.rest[p0 + k], fma(p, f, -n));
      sincospif(2.f * (float)part, &s[k], &c[k]);
      c[k] *= gain;
      s[k] *= gain * sign;
    }
  }
  using V = Vec<T, W>;
  constexpr int U = 4;                                // heads with their loads in flight together
  const int h0 = blockIdx.y * hpt, h1 = h0 + hpt;
#pragma unroll
  for (int w = 0; w < 2; w++) {
    const int first = w ? max(0, h0 - t.H[0]) : h0, last = w ? min(t.H[1], h1 - t.H[0]) : min(t.H[0], h1);
    if (first >= last) continue;
    const int64_t sx = t.ax[w].sh, sy = t.ay[w].sh;
    const T* x = static_cast<const T*>(t.x[w]) + b * t.ax[w].sb + i * t.ax[w].sl + first * sx;
    T* y = static_cast<T*>(t.y[w]) + b * t.ay[w].sb + i * t.ay[w].sl + first * sy;
    for (int h = first; h < last; h += U, x += U * sx, y += U * sy) {
      V a[U], e[U];
#pragma unroll
      for (int q = 0; q < U; q++)
        if (h + q < last) {
          a[q] = *reinterpret_cast<const V*>(x + q * sx + ja);
          e[q] = *reinterpret_cast<const V*>(x + q * sx + jb);
        }
#pragma unroll
      for (int q = 0; q < U; q++)
        if (h + q < last) {
          if (turn) {                                 // (what passes through keeps its bits, NaNs among them)
            float z[2 * W], r[2 * W];
            widen<W>(a[q], z);
            widen<W>(e[q], z + W);
#pragma unroll
            for (int k = 0; k < W; k++) {
              const int m = INTERLEAVED ? 2 * k : k, n = INTERLEAVED ? 2 * k + 1 : W + k;
              r[m] = z[m] * c[k] - z[n] * s[k];
              r[n] = z[n] * c[k] + z[m] * s[k];
            }
            narrow<W>(a[q], r);
            narrow<W>(e[q], r + W);
          }
          *reinterpret_cast<V*>(y + q * sy + ja) = a[q];
          *reinterpret_cast<V*>(y + q * sy + jb) = e[q];
        }
    }
  }
}

template <typename T, int W>
int launch(fsharp_ctx* ctx, const RotTensors& t, const RotFreq& f, const int64_t* pos, int64_t pos_stride, int64_t pos0, int64_t tokens,
           int L, int d, const fsharp_rope* r, int transpose) {
  const int heads = t.H[0] + t.H[1];
  const int64_t units = tokens * (d / (2 * W));
  // Heads per thread: as many as leave a thousand threads per SM (the angles are shared by them).
  int64_t hpt = units * heads / ((int64_t)ctx->sm_count * 1024);
  hpt = hpt < 1 ? 1 : hpt > heads ? heads : hpt;
  const int64_t gx = (units + ROT_T - 1) / ROT_T, gy = (heads + hpt - 1) / hpt;
  if (gx > 0x7fffffff || gy > 65535) return FSHARP_E_SHAPE;
  FS_TIME_BEGIN(ctx, FS_K_ROTATE);
  const auto kernel = r->layout == FSHARP_ROT_INTERLEAVED ? rotate_kernel<T, W, true> : rotate_kernel<T, W, false>;
  kernel<<<dim3((unsigned)gx, (unsigned)gy), ROT_T, 0, ctx->stream>>>(t, f, pos, pos_stride, pos0, tokens, L, d, r->rot, (int)hpt,
                                                                      (float)r->gain, transpose ? -1.f : 1.f);
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
  if (!positive(rope->base) || !isfinite((float)rope->gain)) return FSHARP_E_BADARG;
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
  // one tensor's output at the other's place: a thread would read what another has written
  if (dims->H && dims->Hk && (Qout == K || Kout == Q || Qout == Kout)) return FSHARP_E_BADARG;
  RotFreq f = {};
  const long double turn = 6.283185307179586476925286766559L, s = rope->factor;
  const long double base = rope->scaling == FSHARP_ROPE_NTK ? rope->base * powl(s, rot / (rot - 2.0L)) : (long double)rope->base;
  // one power of 64 bits' mantissa and products (off by j 2^-63 of a frequency that falls with j; a power per pair, 32 pairs: 15.1 -> 16.6 us of host time)
  const long double ratio = exp2l(-log2l(base) * 2 / rot);
  long double plain = 1 / turn;
  for (int j = 0; j < rot / 2; j++, plain *= ratio) {
    long double n = plain;
    if (rope->scaling == FSHARP_ROPE_LINEAR) n /= s;
    if (rope->scaling == FSHARP_ROPE_PARTS) {
      long double keep = (rope->original * n - rope->slow) / ((long double)rope->fast - rope->slow);     // from the turns in the trained length
      keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
      n = n / s * (1 - keep) + n * keep;
    }
    if (!isfinite((double)(n * 0x1p64L))) return FSHARP_E_BADARG;      // (a position's turns would not be finite)
    f.turns[j] = (double)n;
    f.rest[j] = (double)(n - f.turns[j]);
  }
  FsDevice device(ctx->device);
  if (!device.ok) return FSHARP_E_CUDA;
  RotTensors t;
  t.x[0] = Q; t.x[1] = K; t.y[0] = Qout; t.y[1] = Kout;
  t.H[0] = dims->H; t.H[1] = dims->Hk;
  t.ax[0] = fs_addr(dims->q_stride, dims->H, dims->L, d);
  t.ax[1] = fs_addr(dims->k_stride, dims->Hk, dims->L, d);
  t.ay[0] = fs_addr(dims->qo_stride, dims->H, dims->L, d);
  t.ay[1] = fs_addr(dims->ko_stride, dims->Hk, dims->L, d);
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
