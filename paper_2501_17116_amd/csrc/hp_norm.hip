// The joint of two blocks: norm after the one, gate, residual stream, norm before the other; and its gradients.
//
//   u = b r_a w_a, r_a = (mean b^2 + eps)^-1/2      h = s x + g u      y = h r_b w_b, r_b = (mean h^2 + eps)^-1/2
// Backward, with n = h r_b and m = b r_a:
//   t = dh + r_b (dy w_b - n mean(dy w_b n)),  dx = s t,  dg = t u (summed over the tokens that share the gate),  dw_b = sum dy n,
//   q = t g w_a,  db = r_a (q - m mean(q m)),  dw_a = sum t g m.
//
// A workgroup holds a row: each thread one or two pieces of eight channels, so that every matrix is read once and written once.  Memory bounds
// both passes.
#include "hp_common.h"

#include <algorithm>
#include <type_traits>

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
  float* part;                          // [workgroups][3][Dp] sums of dw_before, dw_after, dgate; Dp: D rounded up to 8
  int64_t M, D, Dp, ld_gate, ld_dy, ld_dh, ldh, ldb, ld_dx, ld_db, ld_dg;
  float scale;
  int sums;                             // which of the three are wanted, bits 0 .. 2
};

// Sums over the workgroup, every thread gets them, formed in the same order.  They take turns in two slots of LDS: a wave that writes a slot
// again has passed the barrier of the sum between, and with it every wave's reads of the slot.  The barrier is a bare one: the next row's
// elements are on their way.
struct RowSums {
  float (&lds)[2][16];
  int slot;
  FP4_D float operator()(float v) {
    v = hp_wave_sum(v);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    float (&at)[16] = lds[slot];
    slot ^= 1;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    float s = at[0];
    for (int i = 1; i < waves; ++i) s += at[i];
    return s;
  }
};

// A workgroup a row (16384 x 4096, both norms and a gate: 97 us, 5.5 TB/s).  Going from row to row, the next one's pieces requested ahead, takes longer here: 125.
template <class T, int CH>
__global__ __launch_bounds__(1024) void norm_fwd_kernel(NormFwd a) {
  __shared__ float lds[2][16];
  RowSums sum{lds, 0};
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
      r = 1.0f / sqrtf(sum(s) * inv + a.eps);
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
  const float r = 1.0f / sqrtf(sum(s) * inv + a.eps);
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

// A workgroup goes from row to row and keeps the sums of its rows; AHEAD: the next row's pieces are requested before the present one's are used.  (8192 x
// 5120: 94 us, 5.3 TB/s; with two pieces a thread, whose operands and sums spill, 1014.)
template <class T, int CH, int THREADS, bool AHEAD>
__global__ __launch_bounds__(THREADS) void norm_bwd_kernel(NormBwd a) {
  __shared__ float lds[2][16];
  RowSums sum{lds, 0};
  const int64_t D = a.D;
  const float inv = 1.0f / (float)D;
  const int64_t c0 = (int64_t)threadIdx.x * 8, stride = (int64_t)blockDim.x * 8;
  struct Row { Raw8<T> dy[CH], dh[CH], h[CH], b[CH], g[CH]; float rb, ra; };
  constexpr bool HOLD = THREADS < 1024;   // beyond 768 threads, 6144 channels, the registers do not hold them: each use reads them again
  Raw8<T> wb[CH], wa[CH], gate[CH];
  float sb[CH][8], sa[CH][8], sg[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    if (HOLD && a.dy) wb[i] = hp_load8<T>(a.w_before, c0 + i * stride, D);
    if (HOLD && a.w_after) wa[i] = hp_load8<T>(a.w_after, c0 + i * stride, D);
    if (HOLD && a.gate && a.ld_gate == 0) gate[i] = hp_load8<T>(a.gate, c0 + i * stride, D);
#pragma unroll
    for (int e = 0; e < 8; ++e) sb[i][e] = sa[i][e] = sg[i][e] = 0.0f;
  }
  const auto load = [&](Row& r, int64_t row) {
    r.rb = a.dy ? a.r_before[row] : 0.0f;
    r.ra = a.w_after ? a.r_after[row] : 1.0f;
#pragma unroll
    for (int i = 0; HOLD && i < CH; ++i) {
      const int64_t c = c0 + i * stride;
      if (a.dy) {
        r.dy[i] = hp_load8<T>(hp_row<T>(a.dy, row, a.ld_dy), c, D);
        r.h[i] = hp_load8<T>(hp_row<T>(a.h, row, a.ldh), c, D);
      }
      if (a.dh) r.dh[i] = hp_load8<T>(hp_row<T>(a.dh, row, a.ld_dh), c, D);
      if (a.block) r.b[i] = hp_load8<T>(hp_row<T>(a.block, row, a.ldb), c, D);
      if (a.gate && a.ld_gate) r.g[i] = hp_load8<T>(hp_row<T>(a.gate, row, a.ld_gate), c, D);
    }
  };
  Row next;
  if (AHEAD) load(next, blockIdx.x);
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    Row r;
    if (AHEAD) {
      r = next;
      if (row + gridDim.x < a.M) load(next, row + gridDim.x);
    } else {
      load(r, row);
    }
    const auto piece = [&](const Raw8<T> (&held)[CH], const void* x, int64_t at, int64_t ld, int i) {
      return HOLD ? held[i] : hp_load8<T>(hp_row<T>(x, at, ld), c0 + i * stride, D);
    };
    float t[CH][8], s = 0.0f;
    if (a.dy) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const Raw8<T> h = piece(r.h, a.h, row, a.ldh, i), dy = piece(r.dy, a.dy, row, a.ld_dy, i), w = piece(wb, a.w_before, 0, 0, i);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float n = h.get(e) * r.rb, d = dy.get(e);
          s = fmaf(d * w.get(e), n, s);
          sb[i][e] = fmaf(d, n, sb[i][e]);
        }
      }
      s = sum(s) * inv;
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][e] = 0.0f;
      if (a.dh) {
        const Raw8<T> dh = piece(r.dh, a.dh, row, a.ld_dh, i);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[i][e] = dh.get(e);
      }
      if (a.dy) {
        const Raw8<T> h = piece(r.h, a.h, row, a.ldh, i), dy = piece(r.dy, a.dy, row, a.ld_dy, i), w = piece(wb, a.w_before, 0, 0, i);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[i][e] = fmaf(r.rb, fmaf(-(h.get(e) * r.rb), s, dy.get(e) * w.get(e)), t[i][e]);
      }
      if (a.dx) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = a.scale * t[i][e];
        hp_store8<T>(hp_row<T>(a.dx, row, a.ld_dx), c0 + i * stride, D, o);
      }
    }
    if (!a.block) continue;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const Raw8<T> b = piece(r.b, a.block, row, a.ldb, i);
      Raw8<T> w, g;
      if (a.w_after) w = piece(wa, a.w_after, 0, 0, i);
      if (a.gate) g = a.ld_gate ? piece(r.g, a.gate, row, a.ld_gate, i) : piece(gate, a.gate, 0, 0, i);
      float dg[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float m = b.get(e) * r.ra, v = a.w_after ? w.get(e) : 1.0f;
        dg[e] = t[i][e] * (m * v);
        sg[i][e] += dg[e];
        const float tg = a.gate ? t[i][e] * g.get(e) : t[i][e];
        sa[i][e] = fmaf(tg, m, sa[i][e]);
        t[i][e] = tg * v;
        s = fmaf(t[i][e], m, s);
      }
      if (a.dgate) hp_store8<T>(hp_row<T>(a.dgate, row, a.ld_dg), c0 + i * stride, D, dg);
    }
    if (a.w_after) s = sum(s) * inv;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      if (a.w_after) {
        const Raw8<T> b = piece(r.b, a.block, row, a.ldb, i);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[i][e] = r.ra * fmaf(-(b.get(e) * r.ra), s, t[i][e]);
      }
      if (a.dblock) hp_store8<T>(hp_row<T>(a.dblock, row, a.ld_db), c0 + i * stride, D, t[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    float* const p = a.part + (int64_t)blockIdx.x * 3 * a.Dp;
    const int64_t c = c0 + i * stride;
    if (c >= D) continue;
    if (a.sums & 1) hp_store8<F32>(p, c, a.Dp, sb[i]);
    if (a.sums & 2) hp_store8<F32>(p + a.Dp, c, a.Dp, sa[i]);
    if (a.sums & 4) hp_store8<F32>(p + 2 * a.Dp, c, a.Dp, sg[i]);
  }
}

// Columns of `rows` partial sums each, 32 columns a workgroup; 32 half waves take every 32nd row and are joined in their order.
struct NormSums {
  const float* part;
  float* out[3];
  int64_t rows, D, Dp;
  int accumulate;
};
__global__ __launch_bounds__(1024) void norm_sums_kernel(NormSums a) {
  __shared__ float lds[32][32];
  float* const out = a.out[blockIdx.y];
  if (!out) return;
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  float s = 0.0f;
  if (c < a.D) {
#pragma unroll 8
    for (int64_t r = k; r < a.rows; r += 32) s += a.part[(r * 3 + blockIdx.y) * a.Dp + c];
  }
  lds[k][lane] = s;
  __syncthreads();
  if (k || c >= a.D) return;
  for (int i = 1; i < 32; ++i) s += lds[i][lane];
  out[c] = a.accumulate ? out[c] + s : s;
}

// Threads of a row, a piece of eight channels each or two.  Forward: two where there are rows enough to fill the chip.  Backward: two
// beyond 8192 channels only.
struct RowShape { int threads, pieces; };
RowShape row_shape(int64_t D, bool two) {
  const int64_t n = (D + 7) / 8;
  return two || n > 1024 ? RowShape{(int)((n + 127) / 128 * 64), 2} : RowShape{(int)((n + 63) / 64 * 64), 1};
}
RowShape fwd_shape(int64_t M, int64_t D) { return row_shape(D, M > 512 && D > 1024); }
// Backward: workgroups, as many as the registers let run at once (two bytes twelve waves a CU, four bytes eight), but no more than four a CU, whose partial
// sums have to be joined.  Twice as many, in two rounds that ask for their first rows anew: 2048 x 4096 36 against 31 us with the join, 8192 x 5120 112 against 100.
int64_t bwd_groups(int64_t M, const RowShape& s, bool two_bytes) { return std::min<int64_t>(M, 256 * std::max(1, std::min(4, (two_bytes ? 768 : 512) / s.threads))); }

template <class T>
void launch_fwd(const NormFwd& a, hipStream_t s) {
  const RowShape r = fwd_shape(a.M, a.D);
  if (r.pieces == 1) norm_fwd_kernel<T, 1><<<(unsigned)a.M, r.threads, 0, s>>>(a);
  else norm_fwd_kernel<T, 2><<<(unsigned)a.M, r.threads, 0, s>>>(a);
}
template <class T>
void launch_bwd(const NormBwd& a, hipStream_t s) {
  constexpr bool HALF = HpSize<T>::value == 2;
  const RowShape r = row_shape(a.D, false);
  const unsigned groups = (unsigned)bwd_groups(a.M, r, HALF);
  if (r.pieces == 2) norm_bwd_kernel<T, 2, 1024, false><<<groups, r.threads, 0, s>>>(a);
  else if (r.threads <= 512) norm_bwd_kernel<T, 1, 512, HALF><<<groups, r.threads, 0, s>>>(a);
  else if (r.threads <= 768) norm_bwd_kernel<T, 1, 768, HALF><<<groups, r.threads, 0, s>>>(a);
  else norm_bwd_kernel<T, 1, 1024, false><<<groups, r.threads, 0, s>>>(a);
}

}  // namespace

// Partial sums of the weight gradients: workgroups times D stays below 2^22, since their number falls as the threads of a row grow.
size_t hp_norm_bwd_part(int64_t M, int64_t D) { return (size_t)std::min<int64_t>(M * (int64_t)align_up((size_t)D, 8), 1 << 22) * 3 * sizeof(float); }

int hp_launch_norm_fwd(const hp_norm* n, int bf16, int64_t M, int64_t D, const void* x, int64_t ldx, const void* block, int64_t ldb, void* h, int64_t ldh,
                       void* y, int64_t ldy, float* r_before, float* r_after, hipStream_t s) {
  const NormFwd a = {y || r_before ? n->w_before : nullptr, n->w_after, n->gate, x, block, h, y, r_before, r_after, M, D, n->ld_gate, ldx, ldb, ldh, ldy, n->scale, n->eps};
  if (bf16) launch_fwd<BF16>(a, s);
  else launch_fwd<F32>(a, s);
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}

int hp_launch_norm_bwd(const hp_norm* n, int bf16, int64_t M, int64_t D, const void* dy, int64_t ld_dy, const void* dh, int64_t ld_dh, const void* h,
                       int64_t ldh, const void* block, int64_t ldb, const float* r_before, const float* r_after, void* dx, int64_t ld_dx, void* dblock,
                       int64_t ld_db, void* dgate, int64_t ld_dg, float* dw_before, float* dw_after, int accumulate, float* part, hipStream_t s) {
  const bool shared_gate = n->ld_gate == 0;
  const int64_t Dp = (int64_t)align_up((size_t)D, 8);
  NormBwd a = {dy ? n->w_before : nullptr, n->w_after, n->gate, dy, dh, h, block, r_before, r_after, dx, dblock, shared_gate ? nullptr : dgate, part, M, D, Dp,
               n->ld_gate, ld_dy, ld_dh, ldh, ldb, ld_dx, ld_db, ld_dg, n->scale, 0};
  NormSums f = {part, {dw_before, dw_after, shared_gate ? (float*)dgate : nullptr}, 0, D, Dp, accumulate};
  for (int i = 0; i < 3; ++i) a.sums |= f.out[i] ? 1 << i : 0;
  if (M > 0) {
    f.rows = bwd_groups(M, row_shape(D, false), bf16);
    if (bf16) launch_bwd<BF16>(a, s);
    else launch_bwd<F32>(a, s);
    FP4_CHECK_LAUNCH();
  }
  if (a.sums) {
    norm_sums_kernel<<<dim3((unsigned)((D + 31) / 32), 3), 1024, 0, s>>>(f);
    FP4_CHECK_LAUNCH();
  }
  return FP4_OK;
}
