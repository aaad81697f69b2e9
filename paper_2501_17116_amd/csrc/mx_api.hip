// Host side of the microscaled entry points: argument validation, workspace carving and the sequences of the layer's passes.
// As in the rest of the library nothing here allocates, synchronizes or keeps state.
#include "mx_common.h"

#include <algorithm>
#include <climits>

int mx_launch_quantize(const void* x, int bf16, int64_t rows, int64_t cols, int64_t ld, int row_bits, uint8_t* row_codes, uint8_t* row_scales,
                       int col_bits, uint8_t* col_codes, uint8_t* col_scales, hipStream_t s);
int mx_launch_dequantize(const uint8_t* codes, const uint8_t* scales, int bits, int64_t lines, int64_t length, bool transposed, void* x, int bf16,
                         int64_t ld, hipStream_t s);
int mx_launch_gemm(const uint8_t* L, const uint8_t* sL, int bits_l, const uint8_t* R, const uint8_t* sR, int bits_r, int64_t P, int64_t Q, int64_t Kc,
                   const float* addend, void* out, int out_bf16, int64_t ldo, int tile, hipStream_t s);
int mx_launch_few(const uint8_t* L, const uint8_t* sL, const void* x, int x_bf16, int64_t ldx, int bits_l, const uint8_t* R, const uint8_t* sR, int bits_r,
                  int64_t P, int64_t Q, int64_t Kc, const float* addend, void* out, int out_bf16, int64_t ldo, hipStream_t s);
bool mx_few_fuses(int64_t M, int64_t K, int bits);

namespace {

constexpr int64_t MAX_DIM = int64_t{1} << 21;   // of any dimension: keeps every grid and every tile's byte offsets within 32 bits

bool dtype_ok(int dt) { return dt == FP4_F32 || dt == FP4_BF16; }
bool bits_ok(int bits) { return bits == 4 || bits == 8; }

// What an MX argument has to be, its lines and length given; null buffers are let through where it holds nothing.
int check_mx(const fp4_mx* t, int64_t lines, int64_t length) {
  if (!t) return FP4_ERR_NULL;
  if (!bits_ok(t->bits)) return FP4_ERR_DTYPE;
  if (t->lines != lines || t->length != length) return FP4_ERR_SHAPE;
  if (lines == 0 || length == 0) return FP4_OK;
  if (!t->codes || !t->scales) return FP4_ERR_NULL;
  return aligned16(t->codes) && aligned16(t->scales) ? FP4_OK : FP4_ERR_ARG;
}
int check_matrix(const void* x, int dt, int64_t rows, int64_t cols, int64_t ld) {
  if (!dtype_ok(dt)) return FP4_ERR_DTYPE;
  if (rows < 0 || cols < 0 || ld < cols) return FP4_ERR_SHAPE;
  if (rows > MAX_DIM || cols > MAX_DIM) return FP4_ERR_LIMIT;
  if (rows == 0 || cols == 0) return FP4_OK;
  if (!x) return FP4_ERR_NULL;
  return aligned16(x) && ld % 8 == 0 ? FP4_OK : FP4_ERR_ARG;
}

size_t code_bytes(int64_t lines, int64_t length, int bits) { return (size_t)lines * (size_t)mx_pitch_of(length) / 8 * bits; }
size_t scale_bytes(int64_t lines, int64_t length) { return (size_t)lines * (size_t)mx_pitch_of(length) / MX_BLOCK; }

struct Carve {
  uint8_t* base;
  size_t off = 0;
  explicit Carve(void* p) : base(reinterpret_cast<uint8_t*>(p)) {}
  fp4_mx take(int64_t lines, int64_t length, int bits) {
    fp4_mx t = {};
    t.lines = lines;
    t.length = length;
    t.bits = bits;
    t.codes = bytes(code_bytes(lines, length, bits));
    t.scales = bytes(scale_bytes(lines, length));
    return t;
  }
  uint8_t* bytes(size_t n) {
    uint8_t* r = base ? base + off : nullptr;
    off += align_up(n, 256);
    return r;
  }
};
void* aligned_workspace(void* w) { return reinterpret_cast<void*>(align_up((size_t)(uintptr_t)w, 256)); }

int quantize(const void* x, int dt, int64_t rows, int64_t cols, int64_t ld, const fp4_mx* r, const fp4_mx* c, hipStream_t s) {
  return mx_launch_quantize(x, dt == FP4_BF16, rows, cols, ld, r ? (int)r->bits : 0, r ? r->codes : nullptr, r ? r->scales : nullptr, c ? (int)c->bits : 0,
                            c ? c->codes : nullptr, c ? c->scales : nullptr, s);
}
int gemm(const fp4_mx& l, const fp4_mx& rt, const float* addend, void* out, int dt, int64_t ldo, hipStream_t s) {
  return mx_launch_gemm(l.codes, l.scales, l.bits, rt.codes, rt.scales, rt.bits, l.lines, rt.lines, l.length, addend, out, dt == FP4_BF16, ldo, 0, s);
}

}  // namespace

// Room for what a pass quantizes on the way, how many bits is not known: as if in 8.
size_t mx_workspace_bytes(int op, int64_t M, int64_t K, int64_t N) {
  Carve c(nullptr);
  if (op == FP4_OP_MX_FWD) c.take(M, K, 8);
  if (op == FP4_OP_MX_DGRAD || op == FP4_OP_MX_BWD) c.take(M, N, 4);
  if (op == FP4_OP_MX_WGRAD || op == FP4_OP_MX_BWD) c.take(N, M, 8);
  return c.off + 256;
}

extern "C" int64_t mx_pitch(int64_t length) { return length < 0 ? -1 : mx_pitch_of(length); }

extern "C" int mx_quantize(const void* x, fp4_dtype dt, int64_t rows, int64_t cols, int64_t ld, const fp4_mx* along_rows, const fp4_mx* along_cols,
                           void* stream) {
  int rc = check_matrix(x, dt, rows, cols, ld);
  if (rc) return rc;
  if (!along_rows && !along_cols) return FP4_ERR_NULL;
  if (along_rows && (rc = check_mx(along_rows, rows, cols))) return rc;
  if (along_cols && (rc = check_mx(along_cols, cols, rows))) return rc;
  if (rows == 0 || cols == 0) return FP4_OK;
  return quantize(x, dt, rows, cols, ld, along_rows, along_cols, (hipStream_t)stream);
}

extern "C" int mx_dequantize(const fp4_mx* t, int transposed, void* x, fp4_dtype dt, int64_t ld, void* stream) {
  if (!t) return FP4_ERR_NULL;
  const int64_t rows = transposed ? t->length : t->lines, cols = transposed ? t->lines : t->length;
  int rc = check_matrix(x, dt, rows, cols, ld);
  if (!rc) rc = check_mx(t, t->lines, t->length);
  if (rc || rows == 0 || cols == 0) return rc;
  return mx_launch_dequantize(t->codes, t->scales, t->bits, t->lines, t->length, transposed != 0, x, dt == FP4_BF16, ld, (hipStream_t)stream);
}

int mx_check_gemm(const fp4_mx* l, const fp4_mx* rt, const float* addend, const void* out, int out_dt, int64_t ldo) {
  if (!l || !rt) return FP4_ERR_NULL;
  if (l->length != rt->length || l->length < 0) return FP4_ERR_SHAPE;
  if (l->length > MAX_DIM) return FP4_ERR_LIMIT;
  int rc = check_matrix(out, out_dt, l->lines, rt->lines, ldo);
  if (!rc) rc = check_mx(l, l->lines, l->length);
  if (!rc) rc = check_mx(rt, rt->lines, rt->length);
  if (rc || l->lines == 0 || rt->lines == 0) return rc;
  return addend && !aligned16(addend) ? FP4_ERR_ARG : FP4_OK;
}

extern "C" int mx_gemm(const fp4_mx* l, const fp4_mx* rt, const float* addend, void* out, fp4_dtype out_dt, int64_t ldo, void* stream) {
  const int rc = mx_check_gemm(l, rt, addend, out, out_dt, ldo);
  return rc || l->lines == 0 || rt->lines == 0 ? rc : gemm(*l, *rt, addend, out, out_dt, ldo, (hipStream_t)stream);
}

extern "C" int mx_linear_fwd(const void* A, fp4_dtype dt, int64_t M, int64_t K, int64_t N, int64_t lda, int act_bits, const fp4_mx* W, void* Y,
                             int64_t ldy, const fp4_mx* saved, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_matrix(A, dt, M, K, lda);
  if (!rc) rc = check_matrix(Y, dt, M, N, ldy);
  if (rc) return rc;
  if (!bits_ok(act_bits)) return FP4_ERR_DTYPE;
  if ((rc = check_mx(W, N, K))) return rc;
  if (saved && (rc = check_mx(saved, K, M))) return rc;
  if (M == 0 || (N == 0 && !saved)) return FP4_OK;   // neither an output nor a checkpoint to fill
  if (!workspace || workspace_bytes < mx_workspace_bytes(FP4_OP_MX_FWD, M, K, N)) return FP4_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  if (!saved && K > 0 && N > 0 && mx_few_fuses(M, K, act_bits))
    return mx_launch_few(nullptr, nullptr, A, dt == FP4_BF16, lda, act_bits, W->codes, W->scales, W->bits, M, N, K, nullptr, Y, dt == FP4_BF16, ldy, s);
  Carve c(aligned_workspace(workspace));
  const fp4_mx a = c.take(M, K, act_bits);
  if (K > 0 && (rc = quantize(A, dt, M, K, lda, N > 0 ? &a : nullptr, saved, s))) return rc;
  return N == 0 ? FP4_OK : gemm(a, *W, nullptr, Y, dt, ldy, s);
}

namespace {
// Either gradient, or both from one read of dY.
int bwd(const void* dY, int dt, int64_t M, int64_t K, int64_t N, int64_t ldy, const fp4_mx* W, void* dA, int64_t lda, const fp4_mx* saved, int grad_bits,
        int accumulate, float* dW, int64_t ldw, int op, void* workspace, size_t workspace_bytes, void* stream) {
  const bool want_a = op != FP4_OP_MX_WGRAD, want_w = op != FP4_OP_MX_DGRAD;
  int rc = check_matrix(dY, dt, M, N, ldy);
  if (!rc && want_a) rc = check_matrix(dA, dt, M, K, lda);
  if (!rc && want_w) rc = check_matrix(dW, FP4_F32, K, N, ldw);
  if (rc) return rc;
  if (want_a && (rc = check_mx(W, K, N))) return rc;
  if (want_w && !bits_ok(grad_bits)) return FP4_ERR_DTYPE;
  if (want_w && (rc = check_mx(saved, K, M))) return rc;
  if (!workspace || workspace_bytes < mx_workspace_bytes(op, M, K, N)) return FP4_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  Carve c(aligned_workspace(workspace));
  fp4_mx along_n = {}, along_m = {};
  if (want_a) along_n = c.take(M, N, 4);
  if (want_w) along_m = c.take(N, M, grad_bits);
  if (K == 0) return FP4_OK;
  if (M > 0 && N > 0 && (rc = quantize(dY, dt, M, N, ldy, want_a ? &along_n : nullptr, want_w ? &along_m : nullptr, s))) return rc;
  if (want_a && M > 0 && (rc = gemm(along_n, *W, nullptr, dA, dt, lda, s))) return rc;
  return want_w && N > 0 ? gemm(*saved, along_m, accumulate ? dW : nullptr, dW, FP4_F32, ldw, s) : FP4_OK;
}
}  // namespace

extern "C" int mx_linear_bwd_dgrad(const void* dY, fp4_dtype dt, int64_t M, int64_t K, int64_t N, int64_t ldy, const fp4_mx* W, void* dA, int64_t lda,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  return bwd(dY, dt, M, K, N, ldy, W, dA, lda, nullptr, 0, 0, nullptr, 0, FP4_OP_MX_DGRAD, workspace, workspace_bytes, stream);
}

extern "C" int mx_linear_bwd_wgrad(const void* dY, fp4_dtype dt, int64_t M, int64_t K, int64_t N, int64_t ldy, const fp4_mx* saved, int grad_bits,
                                   int accumulate, float* dW, int64_t ldw, void* workspace, size_t workspace_bytes, void* stream) {
  return bwd(dY, dt, M, K, N, ldy, nullptr, nullptr, 0, saved, grad_bits, accumulate, dW, ldw, FP4_OP_MX_WGRAD, workspace, workspace_bytes, stream);
}

extern "C" int mx_linear_bwd(const void* dY, fp4_dtype dt, int64_t M, int64_t K, int64_t N, int64_t ldy, const fp4_mx* W, const fp4_mx* saved,
                             int grad_bits, void* dA, int64_t lda, int accumulate, float* dW, int64_t ldw, void* workspace, size_t workspace_bytes,
                             void* stream) {
  return bwd(dY, dt, M, K, N, ldy, W, dA, lda, saved, grad_bits, accumulate, dW, ldw, FP4_OP_MX_BWD, workspace, workspace_bytes, stream);
}
