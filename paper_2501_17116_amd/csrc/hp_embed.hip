// Embedding: rows of a table by token id, and the table's gradient, sums of the rows' gradients by id.
//
//   y[t] = s table[id_t]        dtable[v] (+)= s sum over t with id_t = v of dy[t], t ascending
//
// Gradient: (id, t) is sorted by id, stably, eight bits a pass: workgroup d of a pass takes the keys with digit d, which it counts, together with
// those of smaller digits, and then copies to their place in order; no counters in memory, no atomics, one launch a pass.  The sorted rows are then cut into
// spans of equal length, whoever they belong to, so that a frequent id costs no more than many rare ones: a workgroup adds up its span's runs of one id;
// runs within a span are done, those over a border leave partial sums, which a second launch joins in order.  Bound: memory (dy once,
// dtable once); below some thousand tokens the launches.
#include "hp_common.h"

#include <algorithm>

namespace {

template <class T>
__global__ __launch_bounds__(512) void embed_fwd_kernel(const int64_t* ids, int64_t D, int64_t V, const void* table, int64_t ldt, float scale, void* y,
                                                        int64_t ldy) {
  const int64_t row = blockIdx.x, id = ids[row];
  const bool in = id >= 0 && id < V;
  for (int64_t c = (int64_t)threadIdx.x * 8; c < D; c += (int64_t)blockDim.x * 8) {
    Raw8<T> r;
    r.zero();
    if (in) r = hp_load8<T>(hp_row<T>(table, id, ldt), c, D);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = scale * r.get(e);
    hp_store8<T>(hp_row<T>(y, row, ldy), c, D, v);
  }
}

// FIRST: keys come from ids (outside [0, V): V, behind all others), positions are the tokens' own.
template <bool FIRST>
__global__ __launch_bounds__(1024) void sort_pass_kernel(const int64_t* ids, const uint32_t* key_in, const uint32_t* pos_in, int64_t M, int64_t V, int shift,
                                                         uint32_t* key_out, uint32_t* pos_out) {
  __shared__ uint32_t less_of[16], equal_of[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t digit = blockIdx.x;
  const int64_t share = ((M + 15) / 16 + 63) / 64 * 64, from = wave * share, to = std::min(M, from + share);
  const auto key_at = [&](int64_t i) {
    if constexpr (FIRST) {
      const int64_t id = ids[i];
      return (uint32_t)(id >= 0 && id < V ? id : V);
    } else {
      return key_in[i];
    }
  };
  uint32_t less = 0, equal = 0;
  for (int64_t i = from + lane; i < to; i += 64) {
    const uint32_t d = key_at(i) >> shift & 255u;
    less += d < digit;
    equal += d == digit;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    less += __shfl_xor(less, o);
    equal += __shfl_xor(equal, o);
  }
  if (lane == 0) {
    less_of[wave] = less;
    equal_of[wave] = equal;
  }
  __syncthreads();
  int64_t at = 0;
  for (int w = 0; w < 16; ++w) at += less_of[w] + (w < wave ? equal_of[w] : 0u);
  if (equal == 0) return;
  for (int64_t i0 = from; i0 < to; i0 += 64) {
    const int64_t i = i0 + lane;
    const uint32_t key = i < to ? key_at(i) : 0u;
    const bool mine = i < to && (key >> shift & 255u) == digit;
    const uint64_t all = __ballot(mine);
    if (mine) {
      const int64_t o = at + __popcll(all & ((uint64_t{1} << lane) - 1));
      key_out[o] = key;
      pos_out[o] = FIRST ? (uint32_t)i : pos_in[i];
    }
    at += __popcll(all);
  }
}

__global__ __launch_bounds__(256) void zero_rows_kernel(float* x, int64_t D, int64_t ld) {
  float* const p = x + (int64_t)blockIdx.x * ld;
  for (int64_t c = (int64_t)threadIdx.x * 4; c < D; c += 1024) {
    if (c + 4 <= D) *reinterpret_cast<f32x4*>(p + c) = f32x4{0, 0, 0, 0};
    else
      for (int e = 0; e < 4; ++e)
        if (c + e < D) p[c + e] = 0.0f;
  }
}

struct EmbedBwd {
  const uint32_t *key, *pos;
  const void* dy;
  float *table, *part;   // part [spans][2][Dp]: the run that came in over the span's start, the one that leaves over its end
  int64_t M, D, Dp, V, ld_dy, ldt, span;
  float scale;
  int accumulate;
};

FP4_D void write_row(const EmbedBwd& a, uint32_t id, int64_t c, const float (&v)[8]) {
  float* const p = a.table + (int64_t)id * a.ldt;
  float o[8];
  Raw8<F32> old;
  old.zero();
  if (a.accumulate) old = hp_load8<F32>(p, c, a.D);
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = fmaf(a.scale, v[e], old.get(e));
  hp_store8<F32>(p, c, a.D, o);
}

template <class T>
__global__ __launch_bounds__(256) void embed_spans_kernel(EmbedBwd a) {
  const int64_t c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 8;
  const int64_t p0 = (int64_t)blockIdx.x * a.span, p1 = std::min(a.M, p0 + a.span);
  if (c >= a.D) return;
  float* const part = a.part + (int64_t)blockIdx.x * 2 * a.Dp + c;
  uint32_t id = a.key[p0];
  bool came_in = p0 > 0 && a.key[p0 - 1] == id;
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = 0.0f;
  const auto leave = [&](bool goes_on) {
    if (id == (uint32_t)a.V) return;
    if (came_in) hp_store8<F32>(part, 0, 8, s);
    else if (goes_on) hp_store8<F32>(part + a.Dp, 0, 8, s);
    else write_row(a, id, c, s);
  };
  for (int64_t p = p0; p < p1; ++p) {
    const uint32_t k = a.key[p];
    if (k == (uint32_t)a.V) {     // behind the last id
      if (id != k) leave(false);
      return;
    }
    if (k != id) {
      leave(false);
      id = k;
      came_in = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = 0.0f;
    }
    const Raw8<T> r = hp_load8<T>(hp_row<T>(a.dy, a.pos[p], a.ld_dy), c, a.D);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += r.get(e);
  }
  leave(p1 < a.M && a.key[p1] == id);
}

// Runs over borders, each by the span it begins in.
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedBwd a, int64_t spans) {
  const int64_t c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 8;
  const int64_t p0 = (int64_t)blockIdx.x * a.span, p1 = p0 + a.span;
  if (p1 >= a.M || c >= a.D) return;
  const uint32_t id = a.key[p1];
  if (id == (uint32_t)a.V || a.key[p1 - 1] != id) return;                                       // none over this border
  if (a.key[p0] == id && p0 > 0 && a.key[p0 - 1] == id) return;                                 // it began earlier
  int64_t lo = blockIdx.x + 1, hi = spans;                                                      // the spans it reaches: those that begin with it
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) / 2;
    if (a.key[mid * a.span] == id) lo = mid;
    else hi = mid;
  }
  const Raw8<F32> first = hp_load8<F32>(a.part + ((int64_t)blockIdx.x * 2 + 1) * a.Dp, c, a.Dp);
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = first.get(e);
  for (int64_t k = blockIdx.x + 1; k < hi; ++k) {
    const Raw8<F32> r = hp_load8<F32>(a.part + k * 2 * a.Dp, c, a.Dp);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += r.get(e);
  }
  write_row(a, id, c, s);
}

// Rows of a span: few enough that short batches fill the chip, and at most 1024 spans.
int64_t span_of(int64_t M) {
  int64_t s = 8;
  while (s * 1024 < M) s *= 2;
  return s;
}
int64_t spans_of(int64_t M) { return (M + span_of(M) - 1) / span_of(M); }

}  // namespace

int hp_launch_embed_fwd(const int64_t* ids, int bf16, int64_t M, int64_t D, int64_t V, const void* table, int64_t ldt, float scale, void* y, int64_t ldy,
                        hipStream_t s) {
  const int threads = (int)std::min<int64_t>(512, ((D + 7) / 8 + 63) / 64 * 64);
  if (bf16) embed_fwd_kernel<BF16><<<(unsigned)M, threads, 0, s>>>(ids, D, V, table, ldt, scale, y, ldy);
  else embed_fwd_kernel<F32><<<(unsigned)M, threads, 0, s>>>(ids, D, V, table, ldt, scale, y, ldy);
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}

// Two sets of (key, position), partial sums of at most 1024 spans.
size_t hp_embed_bwd_room(int64_t M, int64_t D) {
  return 4 * align_up((size_t)M * 4, 256) + (size_t)std::min<int64_t>(1024, (M + 7) / 8) * 2 * align_up((size_t)D, 8) * 4 + 256;
}

int hp_launch_embed_bwd(const int64_t* ids, int bf16, int64_t M, int64_t D, int64_t V, const void* dy, int64_t ld_dy, float scale, int accumulate,
                        float* table, int64_t ldt, void* workspace, hipStream_t s) {
  if (!accumulate) {
    zero_rows_kernel<<<(unsigned)V, 256, 0, s>>>(table, D, ldt);
    FP4_CHECK_LAUNCH();
  }
  if (M == 0) return FP4_OK;
  const size_t list = align_up((size_t)M * 4, 256);
  uint8_t* w = (uint8_t*)align_up((size_t)(uintptr_t)workspace, 256);
  uint32_t *key[2] = {(uint32_t*)w, (uint32_t*)(w + list)}, *pos[2] = {(uint32_t*)(w + 2 * list), (uint32_t*)(w + 3 * list)};
  int from = 0;
  for (int shift = 0; shift == 0 || V >> shift; shift += 8) {
    const int to = from ^ 1;
    if (shift == 0) sort_pass_kernel<true><<<256, 1024, 0, s>>>(ids, nullptr, nullptr, M, V, 0, key[to], pos[to]);
    else sort_pass_kernel<false><<<256, 1024, 0, s>>>(nullptr, key[from], pos[from], M, V, shift, key[to], pos[to]);
    FP4_CHECK_LAUNCH();
    from = to;
  }
  const int64_t Dp = (int64_t)align_up((size_t)D, 8), spans = spans_of(M);
  const EmbedBwd a = {key[from], pos[from], dy, table, (float*)(w + 4 * list), M, D, Dp, V, ld_dy, ldt, span_of(M), scale, accumulate};
  const dim3 grid((unsigned)spans, (unsigned)((D + 2047) / 2048));
  if (bf16) embed_spans_kernel<BF16><<<grid, 256, 0, s>>>(a);
  else embed_spans_kernel<F32><<<grid, 256, 0, s>>>(a);
  FP4_CHECK_LAUNCH();
  if (spans > 1) {
    embed_join_kernel<<<grid, 256, 0, s>>>(a, spans);
    FP4_CHECK_LAUNCH();
  }
  return FP4_OK;
}
