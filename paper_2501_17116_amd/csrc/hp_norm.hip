// The joint of two blocks: norm after the one, gate, residual stream, norm before the other; and its gradients.
//
//   u = b r_a w_a, r_a = (mean b^2 + eps)^-1/2      h = s x + g u      y = h r_b w_b, r_b = (mean h^2 + eps)^-1/2
// Backward, with n = h r_b and m = b r_a:
//   t = dh + r_b (dy w_b - n mean(dy w_b n)),  dx = s t,  dg = t u (summed over the tokens that share the gate),  dw_b = sum dy n,
//   q = t g w_a,  db = r_a (q - m mean(q m)),  dw_a = sum t g m.
//
// A workgroup holds a row: each thread one or two pieces of eight channels, all loads of a row on their way together, so that every matrix is
// read once and written once.  Memory bounds both passes.
#include "hp_common.h"

#include <algorithm>

int fp4_compute_units_of_current_device();

namespace {

struct NormFwd {
  const void *w_before, *w_after, *gate, *x, *block;
  void *h, *y;
  float *r_before, *r_after;
  int64_t M, D, ld_gate, ldx, ldb, ldh, ldy;
  float scale, eps;
};
struct NormBwd {
  const void *w_before, *w_after, *gate, *dy, *dh, *h, *block;
  const float *r_before, *r_after;
  void *dx, *dblock, *dgate;            // dgate: per token
  float* part;                          // [workgroups][3][D] sums of dw_before, dw_after, dgate
  int64_t M, D, ld_gate, ld_dy, ld_dh, ldh, ldb, ld_dx, ld_db, ld_dg;
  float scale;
  int sums;                             // which of the three are wanted, bits 0 .. 2
};

// Over the workgroup; every thread gets the sum, formed in the same order.  Its own slot of LDS for each use in a row.
template <int SLOT>
FP4_D float block_sum(float v, float (&lds)[2][16]) {
  v = hp_wave_sum(v);
  const int waves = blockDim.x >> 6;
  if (waves == 1) return v;
  if ((threadIdx.x & 63) == 0) lds[SLOT][threadIdx.x >> 6] = v;
  __syncthreads();
  float s = lds[SLOT][0];
  for (int i = 1; i < waves; ++i) s += lds[SLOT][i];
  return s;
}

template <class T, int CH>
__global__ __launch_bounds__(1024) void norm_fwd_kernel(NormFwd a) {
  __shared__ float lds[2][16];
  const int64_t row = blockIdx.x;
  const int64_t D = a.D;
  const float inv = 1.0f / (float)D;
  const int64_t c0 = (int64_t)threadIdx.x * 8, stride = (int64_t)blockDim.x * 8;
  const uint8_t* const px = hp_row<T>(a.x, row, a.ldx);
  Raw8<T> x[CH], b[CH], g[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) x[i] = hp_load8<T>(px, c0 + i * stride, D);
  if (a.block) {
#pragma unroll
    for (int i = 0; i < CH; ++i) b[i] = hp_load8<T>(hp_row<T>(a.block, row, a.ldb), c0 + i * stride, D);
  }
  if (a.gate) {
#pragma unroll
    for (int i = 0; i < CH; ++i) g[i] = hp_load8<T>(hp_row<T>(a.gate, row, a.ld_gate), c0 + i * stride, D);
  }
  float h[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] = a.scale * x[i].get(e);
  if (a.block) {
    float r = 1.0f;
    if (a.w_after) {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(b[i].get(e), b[i].get(e), s);
      r = 1.0f / sqrtf(block_sum<0>(s, lds) * inv + a.eps);
      if (a.r_after && threadIdx.x == 0) a.r_after[row] = r;
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      Raw8<T> w;
      if (a.w_after) w = hp_load8<T>(a.w_after, c0 + i * stride, D);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float u = b[i].get(e);
        if (a.w_after) u = u * r * w.get(e);
        h[i][e] = a.gate ? fmaf(g[i].get(e), u, h[i][e]) : h[i][e] + u;
      }
    }
  }
  if (a.h) {
#pragma unroll
    for (int i = 0; i < CH; ++i) hp_store8<T>(hp_row<T>(a.h, row, a.ldh), c0 + i * stride, D, h[i]);
  }
  if (!a.w_before) return;
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(h[i][e], h[i][e], s);
  const float r = 1.0f / sqrtf(block_sum<1>(s, lds) * inv + a.eps);
  if (a.r_before && threadIdx.x == 0) a.r_before[row] = r;
  if (!a.y) return;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const Raw8<T> w = hp_load8<T>(a.w_before, c0 + i * stride, D);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = h[i][e] * r * w.get(e);
    hp_store8<T>(hp_row<T>(a.y, row, a.ldy), c0 + i * stride, D, y);
  }
}

template <class T, int CH>
__global__ __launch_bounds__(1024) void norm_bwd_kernel(NormBwd a) {
  __shared__ float lds[2][16];
  const int64_t D = a.D;
  const float inv = 1.0f / (float)D;
  const int64_t c0 = (int64_t)threadIdx.x * 8, stride = (int64_t)blockDim.x * 8;
  Raw8<T> wb[CH], wa[CH], gv[CH];
  float sb[CH][8], sa[CH][8], sg[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    if (a.dy) wb[i] = hp_load8<T>(a.w_before, c0 + i * stride, D);
    if (a.w_after) wa[i] = hp_load8<T>(a.w_after, c0 + i * stride, D);
    if (a.gate && a.ld_gate == 0) gv[i] = hp_load8<T>(a.gate, c0 + i * stride, D);
#pragma unroll
    for (int e = 0; e < 8; ++e) sb[i][e] = sa[i][e] = sg[i][e] = 0.0f;
  }
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    Raw8<T> dy[CH], dh[CH], h[CH], b[CH];
    const float rb = a.dy ? a.r_before[row] : 0.0f, ra = a.w_after && a.block ? a.r_after[row] : 1.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int64_t c = c0 + i * stride;
      if (a.dy) {
        dy[i] = hp_load8<T>(hp_row<T>(a.dy, row, a.ld_dy), c, D);
        h[i] = hp_load8<T>(hp_row<T>(a.h, row, a.ldh), c, D);
      }
      if (a.dh) dh[i] = hp_load8<T>(hp_row<T>(a.dh, row, a.ld_dh), c, D);
      if (a.block) b[i] = hp_load8<T>(hp_row<T>(a.block, row, a.ldb), c, D);
      if (a.gate && a.ld_gate) gv[i] = hp_load8<T>(hp_row<T>(a.gate, row, a.ld_gate), c, D);
    }
    float t[CH][8];
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][e] = a.dh ? dh[i].get(e) : 0.0f;
    if (a.dy) {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float n = h[i].get(e) * rb, d = dy[i].get(e);
          s = fmaf(d * wb[i].get(e), n, s);
          sb[i][e] = fmaf(d, n, sb[i][e]);
        }
      s = block_sum<0>(s, lds) * inv;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) t[i][e] = fmaf(rb, fmaf(-(h[i].get(e) * rb), s, dy[i].get(e) * wb[i].get(e)), t[i][e]);
    }
    if (a.dx) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = a.scale * t[i][e];
        hp_store8<T>(hp_row<T>(a.dx, row, a.ld_dx), c0 + i * stride, D, o);
      }
    }
    if (!a.block) {
      __syncthreads();   // the slots of LDS are free again
      continue;
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float dg[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float m = b[i].get(e) * ra, w = a.w_after ? wa[i].get(e) : 1.0f;
        dg[e] = t[i][e] * (m * w);
        sg[i][e] += dg[e];
        const float tg = a.gate ? t[i][e] * gv[i].get(e) : t[i][e];
        sa[i][e] = fmaf(tg, m, sa[i][e]);
        t[i][e] = tg * w;
        s = fmaf(t[i][e], m, s);
      }
      if (a.dgate) hp_store8<T>(hp_row<T>(a.dgate, row, a.ld_dg), c0 + i * stride, D, dg);
    }
    if (a.w_after) {
      s = block_sum<1>(s, lds) * inv;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) t[i][e] = ra * fmaf(-(b[i].get(e) * ra), s, t[i][e]);
    }
    if (a.dblock) {
#pragma unroll
      for (int i = 0; i < CH; ++i) hp_store8<T>(hp_row<T>(a.dblock, row, a.ld_db), c0 + i * stride, D, t[i]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int64_t c = c0 + i * stride;
    float* const p = a.part + (int64_t)blockIdx.x * 3 * D + c;
    for (int e = 0; e < 8; ++e)
      if (c + e < D) {
        if (a.sums & 1) p[e] = sb[i][e];
        if (a.sums & 2) p[D + e] = sa[i][e];
        if (a.sums & 4) p[2 * D + e] = sg[i][e];
      }
  }
}

// Columns of `rows` partial sums each, 64 columns a workgroup; sixteen waves take every sixteenth row and are joined in their order.
struct NormSums {
  const float* part;
  float* out[3];
  int64_t rows, D;
  int accumulate;
};
__global__ __launch_bounds__(1024) void norm_sums_kernel(NormSums a) {
  __shared__ float lds[16][64];
  float* const out = a.out[blockIdx.y];
  if (!out) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  float s = 0.0f;
  if (c < a.D)
    for (int64_t r = wave; r < a.rows; r += 16) s += a.part[(r * 3 + blockIdx.y) * a.D + c];
  lds[wave][lane] = s;
  __syncthreads();
  if (wave || c >= a.D) return;
  for (int i = 1; i < 16; ++i) s += lds[i][lane];
  out[c] = a.accumulate ? out[c] + s : s;
}

// Threads of a row: pieces of eight channels each, one a thread up to `single` of them, then two.
struct RowShape { int threads, pieces; };
RowShape row_shape(int64_t D, int64_t single) {
  const int64_t n = (D + 7) / 8, want = n <= single ? n : (n + 1) / 2;
  int t = 64;
  while (t < want) t *= 2;
  return {t, n <= t ? 1 : 2};
}
int64_t bwd_groups(int64_t M, const RowShape& s) { return std::min<int64_t>(M, 256 * std::max(1, 768 / s.threads)); }

}  // namespace

// Partial sums of the weight gradients: workgroups times D stays below 2^22, since their number falls as the threads of a row double.
size_t hp_norm_bwd_part(int64_t M, int64_t D) { return (size_t)std::min<int64_t>(M * D, 1 << 22) * 3 * sizeof(float); }

int hp_launch_norm_fwd(const hp_norm* n, int bf16, int64_t M, int64_t D, const void* x, int64_t ldx, const void* block, int64_t ldb, void* h, int64_t ldh,
                       void* y, int64_t ldy, float* r_before, float* r_after, hipStream_t s) {
  NormFwd a = {y || r_before ? n->w_before : nullptr, n->w_after, n->gate, x, block, h, y, r_before, r_after, M, D, n->ld_gate, ldx, ldb, ldh, ldy, n->scale, n->eps};
  const RowShape r = row_shape(D, M <= 512 ? 1024 : 128);
  const dim3 grid((unsigned)M), wg(r.threads);
  if (bf16) {
    if (r.pieces == 1) norm_fwd_kernel<BF16, 1><<<grid, wg, 0, s>>>(a);
    else norm_fwd_kernel<BF16, 2><<<grid, wg, 0, s>>>(a);
  } else {
    if (r.pieces == 1) norm_fwd_kernel<F32, 1><<<grid, wg, 0, s>>>(a);
    else norm_fwd_kernel<F32, 2><<<grid, wg, 0, s>>>(a);
  }
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}

int hp_launch_norm_bwd(const hp_norm* n, int bf16, int64_t M, int64_t D, const void* dy, int64_t ld_dy, const void* dh, int64_t ld_dh, const void* h,
                       int64_t ldh, const void* block, int64_t ldb, const float* r_before, const float* r_after, void* dx, int64_t ld_dx, void* dblock,
                       int64_t ld_db, void* dgate, int64_t ld_dg, float* dw_before, float* dw_after, int accumulate, float* part, hipStream_t s) {
  const bool shared_gate = n->ld_gate == 0;
  NormBwd a = {dy ? n->w_before : nullptr, n->w_after, n->gate, dy, dh, h, block, r_before, r_after, dx, dblock, shared_gate ? nullptr : dgate, part, M, D,
               n->ld_gate, ld_dy, ld_dh, ldh, ldb, ld_dx, ld_db, ld_dg, n->scale, 0};
  NormSums f = {part, {dw_before, dw_after, shared_gate ? (float*)dgate : nullptr}, 0, D, accumulate};
  for (int i = 0; i < 3; ++i) a.sums |= f.out[i] ? 1 << i : 0;
  const RowShape r = row_shape(D, 128);
  if (M > 0) {
    f.rows = bwd_groups(M, r);
    const dim3 grid((unsigned)f.rows), wg(r.threads);
    if (bf16) {
      if (r.pieces == 1) norm_bwd_kernel<BF16, 1><<<grid, wg, 0, s>>>(a);
      else norm_bwd_kernel<BF16, 2><<<grid, wg, 0, s>>>(a);
    } else {
      if (r.pieces == 1) norm_bwd_kernel<F32, 1><<<grid, wg, 0, s>>>(a);
      else norm_bwd_kernel<F32, 2><<<grid, wg, 0, s>>>(a);
    }
    FP4_CHECK_LAUNCH();
  }
  if (a.sums) {
    norm_sums_kernel<<<dim3((unsigned)((D + 63) / 64), 3), 1024, 0, s>>>(f);
    FP4_CHECK_LAUNCH();
  }
  return FP4_OK;
}
