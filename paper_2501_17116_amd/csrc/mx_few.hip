// The MX product for few tokens: y[p, q] = sum_k L[p, k] R[q, k] with few rows p, R the weights.
//
// Bound by reading the weights once: K N (1/2 + 1/32) bytes.  A workgroup of eight waves takes 16 NT rows of L x 16 NW rows of R; its waves
// share the contraction, 512 codes at a time (whole 128-byte lines of every row of R), and meet once, in LDS, where their sums are added in
// the waves' order.  Each row of R is read by one workgroup for every 16 NT tokens; the fewer columns a workgroup has, the more
// often the tokens are read.
//
// Measured (other weights each call): a launch that has next to nothing to do takes 3.4 us in a graph; one token, inputs x outputs 4096 x 4096 5.3, 4096 x 11008 9.5 - 10,
// 13824 x 5120 13.5 - 15, so beyond the launch the weights come at 3.5 - 4 TB/s.  24 tokens in 8 bits, 4096 x 11008 11.7 and 3.4 for their codes.  Tried:
// tokens and weights of two units on their way in registers, 128 bytes of a row a unit where those run short: within 2 % at 4096 x 4096 and
// 13824 x 5120, 5 - 10 % slower at 4096 x 11008; the smaller pieces cost what the waits gave.
//
// Where the tokens' codes fit a workgroup's LDS they are made there, while its first weights are on their way: one launch, and nothing but
// the weights, the tokens and the result moves.
//
// v_mfma_scale_f32_16x16x128_f8f6f4: lane (l16, g) holds 32 elements of row l16, sixteen bytes, and their scale; of 512 codes of a line
// instruction s takes chunks 4 s .. 4 s + 3, lane group g one of them, so a load takes 64 contiguous bytes of each row.  First operand: R, so
// a lane ends up with four consecutive columns of one token.
#include "mx_common.h"

#include <algorithm>

typedef int mx_i32x8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr int FW_WAVES = 8;

struct FewArgs {
  const uint8_t *L, *sL;      // codes and scales of the tokens, or
  const void* x;              // the tokens themselves
  int64_t ldx;
  const uint8_t *R, *sR;
  const float* addend;
  void* out;
  int64_t P, Q, K, ldo;
  int64_t planeL, planeR, pitch;
  int nl, nr;
};

enum { FROM_CODES, FROM_BF16, FROM_F32 };

template <int S>
FP4_D mx_f32x4 few_mfma(const u32x4& r, const u32x4& l, const mx_f32x4& c, uint32_t sr, uint32_t sl) {   // S: the byte of L's scales
  const mx_i32x8 a = {(int)r.x, (int)r.y, (int)r.z, (int)r.w, 0, 0, 0, 0}, b = {(int)l.x, (int)l.y, (int)l.z, (int)l.w, 0, 0, 0, 0};
  if constexpr (S == 0) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, 0, (int)sr, 0, (int)sl);
  else if constexpr (S == 1) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, 0, (int)sr, 1, (int)sl);
  else if constexpr (S == 2) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, 0, (int)sr, 2, (int)sl);
  else return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, 0, (int)sr, 3, (int)sl);
}

// Bytes of a token's codes / scales in LDS: sixteen tokens' chunks at one place of their rows fall on sixteen bank groups.
FP4_HD int64_t few_row(int64_t pitch) { return pitch / 2 + 16; }
FP4_HD int64_t few_scales(int64_t pitch) { return pitch / MX_BLOCK + 4; }

// Quantizes the workgroup's tokens into LDS: [plane][token] codes, then [token] scales, those of 512 codes as four words, word g the bytes
// of blocks g, 4 + g, 8 + g, 12 + g: what lane group g wants.  Four threads a block.
template <class T, int BITS>
FP4_D void few_quantize(const FewArgs& a, int64_t p0, int rows, uint8_t* codes, uint8_t* scales) {
  constexpr int P = sizeof(T) == 2 ? 1 : 2;   // 16-byte pieces of a thread's eight elements
  constexpr int FQ = P == 1 ? 8 : 4;          // times eight elements that a thread requests before it looks at the first
  const int64_t row_bytes = few_row(a.pitch), scale_bytes = few_scales(a.pitch);
  const int per_row = (int)(a.pitch / MX_PITCH), total = rows * per_row;   // a wave takes 512 elements of a token at a time
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int i0 = wave; i0 < total; i0 += FQ * FW_WAVES) {
    u32x4 w[FQ][P];
    int row[FQ], c[FQ];
    auto each = [&](bool ragged) {
#pragma unroll
      for (int n = 0; n < FQ; ++n) {
        const int i = i0 + n * FW_WAVES;
        row[n] = i / per_row;
        c[n] = (i - row[n] * per_row) * 64 + lane;
#pragma unroll
        for (int p = 0; p < P; ++p) w[n][p] = mx_load_piece<T>(a.x, p0 + row[n], p0 + rows, a.K, a.ldx, c[n] * 8 + p * 4, ragged);
      }
    };
    if (a.K % (16 / (int)sizeof(T))) each(true);
    else each(false);
#pragma unroll
    for (int n = 0; n < FQ; ++n) {
      if (row[n] >= rows) break;
      uint32_t h, l, byte;
      if constexpr (P == 1) {
        byte = mx_scale_byte<BITS>(mx_quad_max(mx_amax_bf16(w[n][0])));
        mx_encode8<BITS>(w[n][0], mx_scale_f32(byte), h, l);
      } else {
        byte = mx_scale_byte<BITS>(mx_quad_max(max(mx_amax_f32(w[n][0]), mx_amax_f32(w[n][P - 1]))));
        mx_encode8<BITS>(w[n][0], w[n][P - 1], mx_scale_f32(byte), h, l);
      }
      *reinterpret_cast<uint32_t*>(codes + row[n] * row_bytes + c[n] * 4) = h;
      if constexpr (BITS == 8) *reinterpret_cast<uint32_t*>(codes + (rows + row[n]) * row_bytes + c[n] * 4) = l;
      const int block = c[n] >> 2;
      if ((c[n] & 3) == 0) scales[row[n] * scale_bytes + (block >> 4) * 16 + (block & 3) * 4 + ((block >> 2) & 3)] = (uint8_t)byte;
    }
  }
}

// NT tiles of 16 tokens, NW of 16 columns a workgroup.
template <int SRC, int NT, int NW, bool OUT_BF16>
__global__ __launch_bounds__(FW_WAVES * 64) void mx_few_kernel(FewArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t few_smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int64_t q0 = (int64_t)blockIdx.x * (16 * NW), p0 = (int64_t)blockIdx.y * (16 * NT);
  const int rows = (int)min((int64_t)(16 * NT), a.P - p0);
  const int64_t rowb = a.pitch / 2, rows_s = a.pitch / MX_BLOCK;
  const int per_plane = (int)(a.pitch / MX_PITCH), units = per_plane * a.nr;

  // rows past the matrices' edges repeat the last one; what comes of them is not stored
  const uint8_t *w[NW], *ws[NW];
#pragma unroll
  for (int j = 0; j < NW; ++j) {
    const int64_t q = min(q0 + j * 16 + l16, a.Q - 1);
    w[j] = a.R + q * rowb + g * 16;
    ws[j] = a.sR + q * rows_s;
  }
  struct Weights {
    u32x4 c[NW][4], s[NW];
  };
  auto fetch = [&](int unit, Weights& o) {
    const int plane = unit >= per_plane ? 1 : 0, u = unit - plane * per_plane;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
#pragma unroll
      for (int s = 0; s < 4; ++s) o.c[j][s] = *reinterpret_cast<const u32x4*>(w[j] + plane * a.planeR + u * 256 + s * 64);
      o.s[j] = *reinterpret_cast<const u32x4*>(ws[j] + u * 16);
    }
  };
  Weights cur, next;
  if (wave < units) fetch(wave, cur);

  const uint8_t *lc[NT], *lsc[NT];   // this lane's rows of codes and scales
  int64_t plane_l;
  if constexpr (SRC == FROM_CODES) {
    plane_l = a.planeL;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int64_t p = p0 + min(t * 16 + l16, rows - 1);
      lc[t] = a.L + p * rowb + g * 16;
      lsc[t] = a.sL + p * rows_s;
    }
  } else {
    typedef typename std::conditional<SRC == FROM_BF16, uint16_t, float>::type T;
    const int64_t row_bytes = few_row(a.pitch), scale_bytes = few_scales(a.pitch);
    uint8_t* const scales = few_smem + rows * a.nl * row_bytes;
    if (a.nl == 1) few_quantize<T, 4>(a, p0, rows, few_smem, scales);
    else few_quantize<T, 8>(a, p0, rows, few_smem, scales);
    __syncthreads();
    plane_l = rows * row_bytes;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int p = min(t * 16 + l16, rows - 1);
      lc[t] = few_smem + p * row_bytes + g * 16;
      lsc[t] = scales + p * scale_bytes + g * 4;
    }
  }

  mx_f32x4 acc[NW][NT];
#pragma unroll
  for (int j = 0; j < NW; ++j)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[j][t] = mx_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int unit = wave; unit < units; unit += FW_WAVES) {
    if (unit + FW_WAVES < units) fetch(unit + FW_WAVES, next);
    const int plane = unit >= per_plane ? 1 : 0, u = unit - plane * per_plane;
    const uint32_t lessr = plane ? MX_EIGHTH : 0u;
    uint32_t sr[NW][4];
#pragma unroll
    for (int j = 0; j < NW; ++j)
#pragma unroll
      for (int s = 0; s < 4; ++s) sr[j][s] = (cur.s[j][s] - lessr) >> (8 * g);
    for (int pl = 0; pl < a.nl; ++pl) {
      const uint32_t lessl = pl ? MX_EIGHTH : 0u;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        u32x4 c[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) c[s] = *reinterpret_cast<const u32x4*>(lc[t] + pl * plane_l + u * 256 + s * 64);
        if constexpr (SRC == FROM_CODES) {
          const u32x4 sw = *reinterpret_cast<const u32x4*>(lsc[t] + u * 16);
          uint32_t sl[4];
#pragma unroll
          for (int s = 0; s < 4; ++s) sl[s] = (sw[s] - lessl) >> (8 * g);
#pragma unroll
          for (int j = 0; j < NW; ++j)
#pragma unroll
            for (int s = 0; s < 4; ++s) acc[j][t] = few_mfma<0>(cur.c[j][s], c[s], acc[j][t], sr[j][s], sl[s]);
        } else {
          const uint32_t sl = *reinterpret_cast<const uint32_t*>(lsc[t] + u * 16) - lessl;
#pragma unroll
          for (int j = 0; j < NW; ++j) {
            acc[j][t] = few_mfma<0>(cur.c[j][0], c[0], acc[j][t], sr[j][0], sl);
            acc[j][t] = few_mfma<1>(cur.c[j][1], c[1], acc[j][t], sr[j][1], sl);
            acc[j][t] = few_mfma<2>(cur.c[j][2], c[2], acc[j][t], sr[j][2], sl);
            acc[j][t] = few_mfma<3>(cur.c[j][3], c[3], acc[j][t], sr[j][3], sl);
          }
        }
      }
    }
    cur = next;
  }

  // The waves' sums: the last four waves' go to the first four, theirs to whoever stores; rows four floats apart from a multiple of the banks.
  constexpr int LD = 16 * NW + 4, HALF = FW_WAVES / 2;
  float* const sums = reinterpret_cast<float*>(few_smem);
  auto each = [&](auto&& f) {
#pragma unroll
    for (int j = 0; j < NW; ++j)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        f(acc[j][t], *reinterpret_cast<mx_f32x4*>(sums + (wave % HALF * (16 * NT) + t * 16 + l16) * LD + j * 16 + g * 4));
  };
  __syncthreads();   // the codes are read
  if (wave >= HALF) each([](const mx_f32x4& v, mx_f32x4& at) { at = v; });
  __syncthreads();
  if (wave < HALF) each([](const mx_f32x4& v, mx_f32x4& at) { at = v + at; });   // a lane reads and writes its own places
  __syncthreads();
  for (int i = tid; i < rows * (4 * NW); i += FW_WAVES * 64) {
    const int row = i / (4 * NW), col = (i % (4 * NW)) * 4;
    mx_f32x4 y = *reinterpret_cast<const mx_f32x4*>(sums + row * LD + col);
#pragma unroll
    for (int v = 1; v < HALF; ++v) y += *reinterpret_cast<const mx_f32x4*>(sums + (v * (16 * NT) + row) * LD + col);
    float o[4] = {y.x, y.y, y.z, y.w};
    if (q0 + col < a.Q) mx_store4<OUT_BF16>(a.out, a.addend, (p0 + row) * a.ldo + q0 + col, a.Q - q0 - col, o);
  }
}

template <int SRC, int NT, int NW>
size_t few_smem_bytes(const FewArgs& a) {
  const size_t sums = (size_t)(FW_WAVES / 2) * 16 * NT * (16 * NW + 4) * 4;
  const size_t rows = (size_t)std::min<int64_t>(16 * NT, a.P);
  return SRC == FROM_CODES ? sums : std::max(sums, rows * (size_t)(a.nl * few_row(a.pitch) + few_scales(a.pitch)));
}
template <int SRC, int NT, int NW>
void few_launch(const FewArgs& a, bool out_bf16, hipStream_t s) {
  const dim3 grid((unsigned)((a.Q + 16 * NW - 1) / (16 * NW)), (unsigned)((a.P + 16 * NT - 1) / (16 * NT)));
  const size_t lds = few_smem_bytes<SRC, NT, NW>(a);
  if (out_bf16) hipLaunchKernelGGL((mx_few_kernel<SRC, NT, NW, true>), grid, dim3(FW_WAVES * 64), lds, s, a);
  else hipLaunchKernelGGL((mx_few_kernel<SRC, NT, NW, false>), grid, dim3(FW_WAVES * 64), lds, s, a);
}
// Columns a workgroup: a workgroup a CU where there are enough of them, so that every CU has loads under way (one token, 4096 x 4096: 4.6 us
// with 16 columns, 5.5 with 32), and no more of them than that, so that the tokens are not read more often than they have to be (11008
// columns, 24 tokens of 4096: 10.2 us with 64 columns, 12.9 with 32; 5120 columns, 32 tokens of 13824: 19 us with 32, 26 with 16).
template <int SRC, int NT>
void few_columns(const FewArgs& a, bool out_bf16, int n_cu, hipStream_t s) {
  const int64_t cols = (a.Q + 15) / 16 * ((a.P + 16 * NT - 1) / (16 * NT));   // tiles of 16 columns
  if (cols <= n_cu) return few_launch<SRC, NT, 1>(a, out_bf16, s);
  if constexpr (NT <= 2) {
    if (cols > 2 * n_cu) return few_launch<SRC, NT, 4>(a, out_bf16, s);
  }
  few_launch<SRC, NT, 2>(a, out_bf16, s);
}
template <int SRC>
void few_rows(const FewArgs& a, bool out_bf16, int n_cu, hipStream_t s) {
  if (a.P <= 16) few_columns<SRC, 1>(a, out_bf16, n_cu, s);
  else if (a.P <= 32 || SRC != FROM_CODES) few_columns<SRC, 2>(a, out_bf16, n_cu, s);
  else if constexpr (SRC == FROM_CODES) few_columns<SRC, 4>(a, out_bf16, n_cu, s);
}

}  // namespace

int fp4_compute_units_of_current_device();

// Whether the tokens of a forward pass are quantized inside the product's own launch: while making their codes in every workgroup costs no
// more than the launch that it saves (about 3 us), and they fit 64 KiB of LDS.  In the product / in a launch before, 4 bits: 8 x 4096 6.7 / 8.1 us, 16 x
// 4096 8.7 / 8.4, 32 x 2048 7.9 / 7.5; the host saves a launch (about 3.5 us) besides.
bool mx_few_fuses(int64_t M, int64_t K, int bits) {
  const int64_t pitch = mx_pitch_of(K);
  return M <= 32 && M * pitch <= 65536 && M * ((bits / 4) * few_row(pitch) + few_scales(pitch)) <= 65536;
}

// Tokens as codes (x == nullptr) or as they are (then mx_few_fuses).  P, Q and the contraction are at least 1.
int mx_launch_few(const uint8_t* L, const uint8_t* sL, const void* x, int x_bf16, int64_t ldx, int bits_l, const uint8_t* R, const uint8_t* sR, int bits_r,
                  int64_t P, int64_t Q, int64_t Kc, const float* addend, void* out, int out_bf16, int64_t ldo, hipStream_t s) {
  FewArgs a;
  a.L = L; a.sL = sL;
  a.x = x;
  a.ldx = ldx;
  a.R = R; a.sR = sR;
  a.addend = addend;
  a.out = out;
  a.P = P; a.Q = Q; a.K = Kc; a.ldo = ldo;
  a.pitch = mx_pitch_of(Kc);
  a.planeL = P * (a.pitch / 2);
  a.planeR = Q * (a.pitch / 2);
  a.nl = bits_l / 4;
  a.nr = bits_r / 4;
  const int n_cu = fp4_compute_units_of_current_device();
  if (!x) few_rows<FROM_CODES>(a, out_bf16 != 0, n_cu, s);
  else if (x_bf16) few_rows<FROM_BF16>(a, out_bf16 != 0, n_cu, s);
  else few_rows<FROM_F32>(a, out_bf16 != 0, n_cu, s);
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}
