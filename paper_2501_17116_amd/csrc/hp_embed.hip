// Embedding: rows of a table by token id, and the table's gradient, sums of the rows' gradients by id.
//
//   y[t] = s table[id_t]        dtable[v] (+)= s sum over t with id_t = v of dy[t], t ascending
//
// Gradient: (id, t) is sorted by id, stably, eight bits a pass: workgroup d of a pass takes the keys with digit d, which it counts, together with
// those of smaller digits, and then copies to their place in order; no counters in memory, no atomics, one launch a pass (few tokens: all compared with
// all, one launch).  The sorted rows are then cut into
// spans of equal length, whoever they belong to, so that a frequent id costs no more than many rare ones: a workgroup adds up its span's runs of one id;
// runs within a span are done, those over a border leave partial sums, which a second launch joins in order.  Bound: memory (dy once,
// dtable once); below some thousand tokens the launches.
#include "hp_common.h"

#include <algorithm>
#include <type_traits>

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

// Four elements of a row from c on; zeros behind its end.  RAGGED: rows end inside a piece.
template <bool RAGGED>
FP4_D f32x4 get4(const BF16*, const uint8_t* row, int64_t c, int64_t cols) {
  const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + c;
  f32x4 v;
  if (RAGGED && c + 4 > cols) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = c + e < cols ? u2f((uint32_t)p[e] << 16) : 0.0f;
  } else {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
    v = f32x4{u2f(w.x << 16), u2f(w.x & 0xffff0000u), u2f(w.y << 16), u2f(w.y & 0xffff0000u)};
  }
  return v;
}
template <bool RAGGED>
FP4_D f32x4 get4(const F32*, const uint8_t* row, int64_t c, int64_t cols) {
  const float* p = reinterpret_cast<const float*>(row) + c;
  if (!RAGGED || c + 4 <= cols) return *reinterpret_cast<const f32x4*>(p);
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = c + e < cols ? p[e] : 0.0f;
  return v;
}
FP4_D void put4(float* row, int64_t c, int64_t cols, const f32x4& v) {
  const int64_t left = cols - c;
  if (left >= 4) *reinterpret_cast<f32x4*>(row + c) = v;
  else if (left == 3) __builtin_memcpy(__builtin_assume_aligned(row + c, 16), &v, 12);
  else if (left == 2) __builtin_memcpy(__builtin_assume_aligned(row + c, 16), &v, 8);
  else if (left == 1) row[c] = v.x;
}

// A pass of the sort by workgroups 0 .. 255, of them digit's own each; those behind clear the table's gradient, or a part of it, meanwhile.
// FIRST: keys come from ids (outside [0, V): V, behind all others), positions are the tokens' own.
struct SortPass {
  const int64_t* ids;
  const uint32_t *key_in, *pos_in;
  uint32_t *key_out, *pos_out;
  int64_t M, V;
  int shift, sorters;        // sorters: workgroups that sort
  float* table;
  int64_t D, ldt, zero_from, zero_rows;
};

template <bool FIRST, int WAVES>
FP4_D void sort_pass(const SortPass& a) {
  __shared__ uint32_t less_of[WAVES], equal_of[WAVES];
  constexpr int AT_ONCE = 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t digit = blockIdx.x;
  const int64_t share = ((a.M + WAVES - 1) / WAVES + 63) / 64 * 64, from = min(a.M, wave * share), to = min(a.M, from + share);
  const auto load = [&](int64_t i0, uint32_t (&key)[AT_ONCE]) {   // of i0 + lane + 64 k, as far as they are there
    if constexpr (FIRST) {
      int64_t id[AT_ONCE];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) id[k] = a.ids[min(i0 + lane + 64 * k, a.M - 1)];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) key[k] = (uint32_t)(id[k] >= 0 && id[k] < a.V ? id[k] : a.V);
    } else {
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) key[k] = a.key_in[min(i0 + lane + 64 * k, a.M - 1)];
    }
  };
  uint32_t less = 0, equal = 0;
  for (int64_t i0 = from; i0 < to; i0 += 64 * AT_ONCE) {
    uint32_t key[AT_ONCE];
    load(i0, key);
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const uint32_t d = key[k] >> a.shift & 255u, in = i0 + lane + 64 * k < to;
      less += in && d < digit;
      equal += in && d == digit;
    }
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
  for (int w = 0; w < WAVES; ++w) at += less_of[w] + (w < wave ? equal_of[w] : 0u);
  if (equal == 0) return;
  for (int64_t i0 = from; i0 < to; i0 += 64 * AT_ONCE) {
    uint32_t key[AT_ONCE];
    load(i0, key);
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const int64_t i = i0 + lane + 64 * k;
      const bool mine = i < to && (key[k] >> a.shift & 255u) == digit;
      const uint64_t all = __ballot(mine);
      if (mine) {
        const int64_t o = at + __popcll(all & ((uint64_t{1} << lane) - 1));
        a.key_out[o] = key[k];
        a.pos_out[o] = FIRST ? (uint32_t)i : a.pos_in[i];
      }
      at += __popcll(all);
    }
  }
}

// Few tokens: their places in the order at once, by comparing all with all, 64 tokens a workgroup whose four waves share the others; four
// cycles a comparison and wave.
FP4_D void sort_few(const SortPass& a) {
  __shared__ uint32_t before[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int M = (int)a.M, t = (int)blockIdx.x * 64 + lane;
  const auto key_at = [&](int i) {
    const int64_t id = a.ids[min(i, M - 1)];
    return (uint32_t)(id >= 0 && id < a.V ? id : a.V);
  };
  const uint32_t mine = key_at(t);
  uint32_t count = 0;
  for (int b = wave; b * 64 < M; b += 4) {
    const uint32_t theirs = b * 64 + lane < M ? key_at(b * 64 + lane) : 0xffffffffu;   // behind all keys
    if (b < (int)blockIdx.x) {
#pragma unroll
      for (int i = 0; i < 64; ++i) count += (uint32_t)__builtin_amdgcn_readlane(theirs, i) <= mine;
    } else if (b > (int)blockIdx.x) {
#pragma unroll
      for (int i = 0; i < 64; ++i) count += (uint32_t)__builtin_amdgcn_readlane(theirs, i) < mine;
    } else {
      for (int i = 0; i < 64; ++i) {
        const uint32_t k = __builtin_amdgcn_readlane(theirs, i);
        count += k < mine || (k == mine && i < lane);
      }
    }
  }
  before[wave][lane] = count;
  __syncthreads();
  if (wave || t >= M) return;
  const uint32_t at = before[0][lane] + before[1][lane] + before[2][lane] + before[3][lane];
  a.key_out[at] = mine;
  a.pos_out[at] = (uint32_t)t;
}

// One piece of four elements a thread, small workgroups: what is written together then lies together (32000 x 4096: 77 us; a workgroup of 256 a
// row 89, one of 1024 for eight rows 93).
FP4_D void zero_rows(const SortPass& a) {
  const int64_t pieces = (a.D + 3) / 4, n = a.zero_rows * pieces, step = (int64_t)(gridDim.x - a.sorters) * blockDim.x;
  for (int64_t i = (int64_t)(blockIdx.x - a.sorters) * blockDim.x + threadIdx.x; i < n; i += step) {
    const int64_t row = n >> 32 ? i / pieces : (uint32_t)i / (uint32_t)pieces, c = (i - row * pieces) * 4;
    put4(a.table + (a.zero_from + row) * a.ldt, c, a.D, f32x4{0, 0, 0, 0});
  }
}

__global__ __launch_bounds__(256) void sort_few_kernel(SortPass a) {
  if ((int)blockIdx.x < a.sorters) sort_few(a);
  else zero_rows(a);
}

template <bool FIRST, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void sort_pass_kernel(SortPass a) {
  if ((int)blockIdx.x < a.sorters) sort_pass<FIRST, WAVES>(a);
  else zero_rows(a);
}

struct EmbedBwd {
  const uint32_t *key, *pos;
  const void* dy;
  float *table, *part;   // part [spans][2][Dp]: the run that came in over the span's start, the one that leaves over its end
  int64_t M, D, Dp, V, ld_dy, ldt, span;
  float scale;
  int accumulate;
};

template <bool RAGGED>
FP4_D void write_row(const EmbedBwd& a, uint32_t id, int64_t c, const f32x4& v) {
  float* const p = a.table + (int64_t)id * a.ldt;
  f32x4 o = {0, 0, 0, 0};
  if (a.accumulate) o = get4<RAGGED>((const F32*)nullptr, (const uint8_t*)p, c, a.D);
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = fmaf(a.scale, v[e], o[e]);
  put4(p, c, a.D, o);
}

// 16384 x 4096 into 32000 rows: 75 us for 134 MB read and some 110 written, while the cleared table leaves the last-level cache; 65536 into 131072: 227 us, 4.3 TB/s.
// A thread's four columns of a span's rows, eight of which are on their way together.  (Waves, not requests a wave, hide the latencies: a run's
// store ends a wave's requests until it is done.)
template <class T, bool RAGGED>
__global__ __launch_bounds__(256) void embed_spans_kernel(EmbedBwd a) {
  constexpr int AT_ONCE = 8;
  const int64_t c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
  const int64_t p0 = (int64_t)blockIdx.x * a.span, p1 = min(a.M, p0 + a.span);
  const int lane = threadIdx.x & 63;
  const uint32_t none = (uint32_t)a.V;
  uint32_t id = a.key[p0];
  bool came_in = p0 > 0 && a.key[p0 - 1] == id;
  const bool goes_on = p1 < a.M && a.key[p1] == a.key[p1 - 1];
  const int64_t from = min(c, (a.D - 1) / 4 * 4);   // threads behind the row's end read its last piece
  const bool in = c < a.D;
  f32x4 s = {0, 0, 0, 0};
  const auto leave = [&](bool over) {
    if (id == none || !in) return;
    float* const part = a.part + (int64_t)blockIdx.x * 2 * a.Dp + c;
    if (came_in) *reinterpret_cast<f32x4*>(part) = s;
    else if (over) *reinterpret_cast<f32x4*>(part + a.Dp) = s;
    else write_row<RAGGED>(a, id, c, s);
  };
  for (int64_t q0 = p0; q0 < p1; q0 += 64) {   // keys and positions of 64 rows, a lane's each
    const int64_t q = min(q0 + lane, p1 - 1);
    const uint32_t keys = a.key[q], places = a.pos[q];
    const int n = (int)min((int64_t)64, p1 - q0);
    for (int i0 = 0; i0 < n; i0 += AT_ONCE) {
      f32x4 r[AT_ONCE];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k)
        r[k] = get4<RAGGED>((const T*)nullptr, hp_row<T>(a.dy, (uint32_t)__builtin_amdgcn_readlane(places, min(i0 + k, n - 1)), a.ld_dy), from, a.D);
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        if (i0 + k < n) {
          const uint32_t key = __builtin_amdgcn_readlane(keys, i0 + k);
          if (key != id) {
            leave(false);
            id = key;
            came_in = false;
            s = f32x4{0, 0, 0, 0};
          }
          s += r[k];
        }
      }
    }
  }
  leave(goes_on);
}

// Runs over borders, each by the span it begins in.
template <bool RAGGED>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedBwd a, int64_t spans) {
  const int64_t c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
  const int64_t p0 = (int64_t)blockIdx.x * a.span, p1 = p0 + a.span;
  if (p1 >= a.M) return;
  const uint32_t id = a.key[p1];
  if (id == (uint32_t)a.V || a.key[p1 - 1] != id) return;                                       // none over this border
  if (a.key[p0] == id && p0 > 0 && a.key[p0 - 1] == id) return;                                 // it began earlier
  int64_t hi = blockIdx.x + 2;                                                                  // behind the spans it reaches: those that begin with it
  while (true) {
    const int64_t k = hi + (threadIdx.x & 63);
    const uint64_t with = __ballot(k < spans && a.key[k * a.span] == id);   // keys ascend: the lowest lanes'
    hi += __popcll(with);
    if (~with) break;
  }
  if (c >= a.D) return;
  constexpr int AT_ONCE = 16;
  const auto at = [&](int64_t line) { return *reinterpret_cast<const f32x4*>(a.part + line * a.Dp + c); };
  f32x4 s = at((int64_t)blockIdx.x * 2 + 1);
  for (int64_t k0 = blockIdx.x + 1; k0 < hi; k0 += AT_ONCE) {
    f32x4 r[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) r[k] = at(min(k0 + k, hi - 1) * 2);
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k)
      if (k0 + k < hi) s += r[k];
  }
  write_row<RAGGED>(a, id, c, s);
}

// Rows of a span: 1024 to 2048 workgroups where there are tokens enough, each a span of some 1024 channels.
int64_t slices_of(int64_t D) { return (D + 1023) / 1024; }
int64_t span_of(int64_t M, int64_t D) {
  int64_t s = 8;
  while (s * 2048 < M * slices_of(D)) s *= 2;
  return s;
}
int64_t spans_of(int64_t M, int64_t D) { return (M + span_of(M, D) - 1) / span_of(M, D); }

}  // namespace

int hp_launch_embed_fwd(const int64_t* ids, int bf16, int64_t M, int64_t D, int64_t V, const void* table, int64_t ldt, float scale, void* y, int64_t ldy,
                        hipStream_t s) {
  const int threads = (int)std::min<int64_t>(512, ((D + 7) / 8 + 63) / 64 * 64);
  if (bf16) embed_fwd_kernel<BF16><<<(unsigned)M, threads, 0, s>>>(ids, D, V, table, ldt, scale, y, ldy);
  else embed_fwd_kernel<F32><<<(unsigned)M, threads, 0, s>>>(ids, D, V, table, ldt, scale, y, ldy);
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}

// Two sets of (key, position), partial sums of at most 2048 / slices + 1 spans of two lines of D.
size_t hp_embed_bwd_room(int64_t M, int64_t D) {
  const size_t line = align_up((size_t)D, 8) * 4;
  return 4 * align_up((size_t)M * 4, 256) + 2 * std::min((size_t)((M + 7) / 8) * line, (size_t)2048 * 1024 * 4 + line) + 256;
}

int hp_launch_embed_bwd(const int64_t* ids, int bf16, int64_t M, int64_t D, int64_t V, const void* dy, int64_t ld_dy, float scale, int accumulate,
                        float* table, int64_t ldt, void* workspace, hipStream_t s) {
  const size_t list = align_up((size_t)M * 4, 256);
  uint8_t* w = (uint8_t*)align_up((size_t)(uintptr_t)workspace, 256);
  uint32_t *key[2] = {(uint32_t*)w, (uint32_t*)(w + list)}, *pos[2] = {(uint32_t*)(w + 2 * list), (uint32_t*)(w + 3 * list)};
  // Few tokens are ordered in one launch: 8192 in some 12 us, as two passes take (16384 in 24: clearing and sorting for 16384 x 4096 into 32000 rows 94 us, by
  // two passes 89).  Up to 32768 the passes hide behind the clearing, in small workgroups as that wants them; beyond, and where nothing is
  // cleared, sixteen waves share a digit.
  const bool few = M > 0 && M <= 8192, together = !accumulate && M > 0 && M <= 32768;
  int from = 0, passes = 1;
  while (V >> (8 * passes)) ++passes;
  const auto clearing = [&](int64_t rows, int threads) { return (unsigned)std::min<int64_t>((rows * ((D + 3) / 4) + threads - 1) / threads, 1 << 22); };
  SortPass p = {ids, nullptr, nullptr, nullptr, nullptr, M, V, 0, 0, table, D, ldt, 0, 0};
  if (!accumulate && !together) {
    p.zero_rows = V;
    sort_pass_kernel<true, 4><<<clearing(V, 256), 256, 0, s>>>(p);
    FP4_CHECK_LAUNCH();
  }
  if (few) {
    p = {ids, nullptr, nullptr, key[0], pos[0], M, V, 0, (int)((M + 63) / 64), table, D, ldt, 0, accumulate ? 0 : V};
    sort_few_kernel<<<p.sorters + clearing(p.zero_rows, 256), 256, 0, s>>>(p);
    FP4_CHECK_LAUNCH();
  }
  for (int i = 0; M > 0 && !few && i < passes; ++i, from ^= 1) {
    p = {ids, key[from], pos[from], key[from ^ 1], pos[from ^ 1], M, V, 8 * i, 256, table, D, ldt, 0, 0};
    if (together) {
      p.zero_from = V * i / passes;
      p.zero_rows = V * (i + 1) / passes - p.zero_from;
      const unsigned groups = 256 + clearing(p.zero_rows, 256);
      if (i == 0) sort_pass_kernel<true, 4><<<groups, 256, 0, s>>>(p);
      else sort_pass_kernel<false, 4><<<groups, 256, 0, s>>>(p);
    } else {
      if (i == 0) sort_pass_kernel<true, 16><<<256, 1024, 0, s>>>(p);
      else sort_pass_kernel<false, 16><<<256, 1024, 0, s>>>(p);
    }
    FP4_CHECK_LAUNCH();
  }
  if (M == 0) return FP4_OK;
  const int64_t Dp = (int64_t)align_up((size_t)D, 8), spans = spans_of(M, D);
  const EmbedBwd a = {key[from], pos[from], dy, table, (float*)(w + 4 * list), M, D, Dp, V, ld_dy, ldt, span_of(M, D), scale, accumulate};
  const dim3 grid((unsigned)spans, (unsigned)slices_of(D));
  const auto launch = [&](auto ragged) {
    constexpr bool RAGGED = decltype(ragged)::value;
    if (bf16) embed_spans_kernel<BF16, RAGGED><<<grid, 256, 0, s>>>(a);
    else embed_spans_kernel<F32, RAGGED><<<grid, 256, 0, s>>>(a);
    if (spans > 1) embed_join_kernel<RAGGED><<<grid, 256, 0, s>>>(a, spans);
  };
  if (D % 4) launch(std::true_type{});
  else launch(std::false_type{});
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}
