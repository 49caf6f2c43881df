// Exact cross attention: what its kernels share.  A unit is one (batch, key head); the R = (H / Hk) Lq query rows of the heads
// that share the key head are its rows, row r = token r % Lq of the group's head r / Lq.  Scores live in the base-2 domain:
// x = S log2(e), m a running maximum of x, l the sum of 2^(x - m).
#pragma once

#include "common.cuh"

struct CrossArgs {
  const void *Q, *K, *V;
  TensorAddr aq, ak, av;
  const int32_t* key_len;
  const uint8_t* key_mask;
  int64_t mask_stride;
  int B, H, Hk, g, Lq, Lk, d, dv;
  float scale;             // of the scores; kernels multiply by log2(e) where they need it
  int ranked;              // blocks take the units in the order of their sequences' lengths (cross_rank)
};

// The keys of sequence b: no more than this many.
__device__ __forceinline__ int cross_keys(const CrossArgs& a, int b) {
  return a.key_len ? max(0, min(a.Lk, a.key_len[b])) : a.Lk;
}
__device__ __forceinline__ bool cross_seen(const CrossArgs& a, int b, int j, int n) {
  return j < n && (!a.key_mask || a.key_mask[b * a.mask_stride + j] != 0);
}

// The batch's sequences from the longest to the shortest, into order[B]: a block's time goes with its sequence's length; with the
// longest first, what runs alone at the end is short.  room: B ints of shared memory, free again when the call returns.  All
// threads of the block.
constexpr int CROSS_RANKED = 256;      // most sequences that are ranked
__device__ __forceinline__ void cross_rank(const CrossArgs& a, int* room, uint8_t* order) {
  const int t = threadIdx.x;
  if (t < a.B) room[t] = cross_keys(a, t);
  __syncthreads();
  if (t < a.B) {
    const int mine = room[t];
    int rank = 0;
    for (int b = 0; b < a.B; b++) rank += room[b] > mine || (room[b] == mine && b < t);
    order[rank] = (uint8_t)t;
  }
  __syncthreads();
}
// The unit of a block of a grid with a unit per blockIdx.y.
__device__ __forceinline__ int cross_unit(const CrossArgs& a, int* room) {
  const int u = blockIdx.y;
  if (!a.ranked) return u;
  uint8_t* order = reinterpret_cast<uint8_t*>(room + CROSS_RANKED);
  cross_rank(a, room, order);
  const int b = order[u / a.Hk];
  __syncthreads();
  return b * a.Hk + u % a.Hk;
}
// Whether it is worth it: lengths differ, and the blocks do not all run at once.
static inline int cross_ranked(const fsharp_ctx* ctx, const CrossArgs& a, int64_t blocks) {
  return a.key_len && a.B > 1 && a.B <= CROSS_RANKED && blocks > ctx->sm_count;
}

// Pieces of a unit's keys (or rows) that blocks of their own take, so that few units fill the GPU: partial results go to scratch.
// Forward: O [unit][piece][R][dv] (unnormalised) and (m, l) [unit][piece][R].
struct CrossPart {
  float* o;              // null where there is one piece, or where a unit's pieces meet in a cluster
  float2* ml;
  int pieces;
};

#define FS_LN2 0.6931471805599453f

// tensor cores (tc_cross.cu): bf16
int fs_tc_cross_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm);
int fs_tc_cross(fsharp_ctx* ctx, const CrossArgs& a, void* Y, TensorAddr ay, float* lse, CrossPart part);

// few rows (cross_rows.cu), and the join of pieces
int fs_cross_rows_most(int dtype);
int fs_cross_rows_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int dtype, bool* cluster);
int fs_cross_rows(fsharp_ctx* ctx, const CrossArgs& a, int dtype, void* Y, TensorAddr ay, float* lse, CrossPart part);
int fs_cross_join(fsharp_ctx* ctx, const CrossArgs& a, int dtype, void* Y, TensorAddr ay, float* lse, CrossPart part);
// multiply-add tiles (cross_fma.cu)
int fs_cross_fma_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm);
int fs_cross_fma(fsharp_ctx* ctx, const CrossArgs& a, int dtype, void* Y, TensorAddr ay, float* lse, CrossPart part);

// fp32, d and dv up to 64, on the tensor cores (tc_cross_f32.cu); scratch: the parts of the operands
int fs_tc_cross_f32_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm);
int64_t fs_tc_cross_f32_parts(const fsharp_cross_dims* dm, int backward);
int fs_tc_cross_f32(fsharp_ctx* ctx, const CrossArgs& a, void* Y, TensorAddr ay, float* lse, CrossPart part, void* scratch);

// Backward.  stat [B][H][ceil(Lq / 128)][2][128]: 128 rows' -lse log2(e), then their -D; rows that see nothing and places behind the last
// row have -inf and 0, which makes every 2^(x - lse) of theirs zero.  Partial sums of a piece: dK | dV [piece][unit][Lk][d + dv], dQ [piece][unit][R][d].
struct CrossGrad {
  const void* dY;
  TensorAddr ady;
  const float* stat;
  void *dQ, *dK, *dV;
  TensorAddr adq, adk, adv;
  float *pkv, *pq;             // null where the one piece writes the gradients themselves
  int kv_pieces, q_pieces;
};
__host__ __device__ __forceinline__ int64_t cross_stat_floats(int Lq) { return ((int64_t)Lq + 127) / 128 * 256; }
// (-lse log2(e), -D) of token i of (batch, head) bh
__device__ __forceinline__ float2 cross_stat(const float* stat, int64_t bh, int Lq, int i) {
  const float* p = stat + bh * cross_stat_floats(Lq) + (int64_t)(i >> 7) * 256 + (i & 127);
  return make_float2(p[0], p[128]);
}
// tensor cores (tc_cross_bwd.cu): bf16
void fs_tc_cross_grad_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int* kv_pieces, int* q_pieces);
int fs_tc_cross_grad(fsharp_ctx* ctx, const CrossArgs& a, const CrossGrad& gr);
void fs_tc_cross_f32_grad_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int* kv_pieces, int* q_pieces);
int fs_tc_cross_f32_grad(fsharp_ctx* ctx, const CrossArgs& a, const CrossGrad& gr, void* scratch);
void fs_cross_fma_grad_pieces(const fsharp_ctx* ctx, const fsharp_cross_dims* dm, int* kv_pieces, int* q_pieces);
int fs_cross_fma_grad(fsharp_ctx* ctx, const CrossArgs& a, int dtype, const CrossGrad& gr);
