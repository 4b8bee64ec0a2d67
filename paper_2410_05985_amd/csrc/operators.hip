// C ABI of the calls on the way into a linear layer: dropout, LayerNorm with
// its residual add, 8-bit quantisation and product.  Argument checks; the
// kernels are in norm_fwd.hip, norm_bwd.hip, quant_fp8.hip and gemm_fp8.hip.
#include <exception>

#include "layup_internal.h"

using namespace layup;

namespace {

struct Refused {
  layup_status st;
  std::string msg;
};

void need(bool ok, layup_status st, const char* msg) {
  if (!ok) throw Refused{st, msg};
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

size_t elem_bytes(int32_t dtype) { return dtype == LAYUP_F32 ? 4 : dtype == LAYUP_BF16 ? 2 : 1; }
bool is_wide(int32_t dtype) { return dtype == LAYUP_F32 || dtype == LAYUP_BF16; }
bool is_fp8(int32_t dtype) { return dtype == LAYUP_E4M3 || dtype == LAYUP_E5M2; }
int64_t up128(int64_t n) { return (n + 127) / 128 * 128; }

// A matrix argument: present, aligned to its elements, rows that do not overlap.
void matrix(const void* p, int64_t ld, int64_t cols, int32_t dtype, const char* null_msg) {
  need(p, LAYUP_ERR_INVALID_ARG, null_msg);
  need(ld >= cols, LAYUP_ERR_SHAPE, "leading dimension smaller than the row");
  need(aligned(p, elem_bytes(dtype)), LAYUP_ERR_ALIGN, "matrix not aligned to its elements");
}

void floats(const float* p) { need(aligned(p, 4), LAYUP_ERR_ALIGN, "float32 vector must be 4-byte aligned"); }

// Scale bytes of a matrix whose rows have k elements.
void scales(const uint8_t* p, int64_t ld, int64_t k) {
  need(p, LAYUP_ERR_INVALID_ARG, "null scale table");
  need(aligned(p, 4) && ld % 4 == 0, LAYUP_ERR_ALIGN, "scale tables must be 4-byte aligned, their rows multiples of 4");
  need(ld >= up128(k) / 128, LAYUP_ERR_SHAPE, "scale table row shorter than the row's blocks");
}

// A matrix in 8 bits: rows of k elements, filled up to a multiple of 128.
void matrix8(const void* p, int64_t ld, int64_t k) {
  need(p, LAYUP_ERR_INVALID_ARG, "null 8-bit matrix");
  need(aligned(p, 16) && ld % 16 == 0, LAYUP_ERR_ALIGN, "8-bit matrices must be 16-byte aligned, their rows multiples of 16");
  need(ld >= up128(k), LAYUP_ERR_SHAPE, "rows of 8-bit matrices are filled up to a multiple of 128");
}

Mask checked_mask(const layup_dropout_mask& m) {
  need(m.p >= 0.0f && m.p < 1.0f, LAYUP_ERR_INVALID_ARG, "dropout probability must be at least 0 and below 1");
  need(aligned(m.offset_dev, 8), LAYUP_ERR_ALIGN, "offset_dev must be 8-byte aligned");
  return make_mask(m);
}

// The stream's device is current while the call enqueues its work.
class OnDevice {
 public:
  explicit OnDevice(hipStream_t s) {
    int dev = 0;
    if (!s || hipStreamGetDevice(s, &dev) != hipSuccess || hipGetDevice(&old_) != hipSuccess || dev == old_) return;
    back_ = hipSetDevice(dev) == hipSuccess;
  }
  ~OnDevice() {
    if (back_) (void)hipSetDevice(old_);
  }

 private:
  int old_ = 0;
  bool back_ = false;
};

// Runs the checks and the launch of a call: nothing is enqueued where a check
// refuses, and no exception leaves.
template <class F>
layup_status call(const void* desc, void* stream, const char* what, F&& f) {
  try {
    need(desc, LAYUP_ERR_INVALID_ARG, "null descriptor");
    OnDevice on((hipStream_t)stream);
    const hipError_t e = f((hipStream_t)stream);
    if (e != hipSuccess) return global_fail(LAYUP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
    return LAYUP_OK;
  } catch (const Refused& r) {
    return global_fail(r.st, std::string(what) + ": " + r.msg);
  } catch (const std::exception& x) {
    return global_fail(LAYUP_ERR_INVALID_ARG, x.what());
  }
}

}  // namespace

extern "C" {

layup_status layup_dropout(const layup_dropout_desc* d, void* stream) {
  return call(d, stream, "dropout", [&](hipStream_t s) {
    need(d->rows >= 0 && d->cols >= 0 && d->rows < (1ll << 31) && d->cols < (1ll << 33), LAYUP_ERR_SHAPE,
         "rows or columns out of range");
    need(is_wide(d->dtype), LAYUP_ERR_DTYPE, "float32 or bfloat16");
    const Mask k = checked_mask(d->drop);
    if (d->rows == 0 || d->cols == 0) return hipSuccess;
    matrix(d->x, d->ldx, d->cols, d->dtype, "null x");
    matrix(d->y, d->ldy, d->cols, d->dtype, "null y");
    need(d->x != d->y || d->ldx == d->ldy, LAYUP_ERR_INVALID_ARG, "in place with another leading dimension");
    return launch_dropout(*d, k, s);
  });
}

layup_status layup_layernorm_forward(const layup_layernorm_desc* d, void* stream) {
  return call(d, stream, "layernorm forward", [&](hipStream_t s) {
    need(d->rows >= 0 && d->rows < (1ll << 31), LAYUP_ERR_SHAPE, "rows out of range");
    need(d->d >= 1 && d->d <= NORM_MAX_D, LAYUP_ERR_SHAPE, "d must be 1 to 16384");
    need(is_wide(d->x_dtype) && is_wide(d->s_dtype) && (is_wide(d->y_dtype) || is_fp8(d->y_dtype)), LAYUP_ERR_DTYPE,
         "x and s: float32 or bfloat16; y: these or 8 bits");
    need(d->eps >= 0.0f && std::isfinite(d->eps), LAYUP_ERR_INVALID_ARG, "eps must be finite and not negative");
    const Mask k = checked_mask(d->drop);
    if (d->rows == 0) return hipSuccess;
    matrix(d->x, d->ldx, d->d, d->x_dtype, "null x");
    if (d->residual) matrix(d->residual, d->ldr, d->d, d->s_dtype, "");
    if (d->sum) matrix(d->sum, d->lds, d->d, d->s_dtype, "");
    need(!d->sum || d->sum != d->residual || d->lds == d->ldr, LAYUP_ERR_INVALID_ARG, "in place with another leading dimension");
    if (is_fp8(d->y_dtype)) {
      matrix8(d->y, d->ldy, d->d);
      scales(d->y_scale, d->ld_scale, d->d);
    } else {
      matrix(d->y, d->ldy, d->d, d->y_dtype, "null y");
    }
    for (const float* p : {d->gamma, d->beta, (const float*)d->mean, (const float*)d->rstd}) floats(p);
    return launch_norm_fwd(*d, k, s);
  });
}

layup_status layup_layernorm_workspace_size(int64_t rows, int32_t d, size_t* bytes) {
  if (!bytes) return global_fail(LAYUP_ERR_INVALID_ARG, "layernorm workspace: null argument");
  if (rows < 0 || rows >= (1ll << 31) || d < 1 || d > NORM_MAX_D)
    return global_fail(LAYUP_ERR_SHAPE, "layernorm workspace: rows or d out of range");
  *bytes = (size_t)norm_partial_floats(rows, d) * sizeof(float);
  return LAYUP_OK;
}

layup_status layup_layernorm_backward(const layup_layernorm_grad_desc* d, void* stream) {
  return call(d, stream, "layernorm backward", [&](hipStream_t s) {
    need(d->rows >= 0 && d->rows < (1ll << 31), LAYUP_ERR_SHAPE, "rows out of range");
    need(d->d >= 1 && d->d <= NORM_MAX_D, LAYUP_ERR_SHAPE, "d must be 1 to 16384");
    need(is_wide(d->dy_dtype) && is_wide(d->s_dtype) && is_wide(d->dx_dtype), LAYUP_ERR_DTYPE, "float32 or bfloat16");
    const Mask k = checked_mask(d->drop);
    floats(d->dgamma);
    floats(d->dbeta);
    if (d->rows > 0) {
      matrix(d->dy, d->lddy, d->d, d->dy_dtype, "null dy");
      matrix(d->s, d->lds, d->d, d->s_dtype, "null s");
      need(d->mean && d->rstd, LAYUP_ERR_INVALID_ARG, "null statistics");
      for (const float* p : {d->mean, d->rstd, d->gamma}) floats(p);
      if (d->dsum) matrix(d->dsum, d->lddsum, d->d, d->s_dtype, "");
      if (d->dres) matrix(d->dres, d->lddres, d->d, d->s_dtype, "");
      if (d->dx) matrix(d->dx, d->lddx, d->d, d->dx_dtype, "");
      need(!d->dres || d->dres != d->dsum || d->lddres == d->lddsum, LAYUP_ERR_INVALID_ARG,
           "in place with another leading dimension");
      if (d->dgamma || d->dbeta) {
        need(d->workspace && d->workspace_bytes >= (size_t)norm_partial_floats(d->rows, d->d) * sizeof(float),
             LAYUP_ERR_INVALID_ARG, "workspace smaller than layup_layernorm_workspace_size");
        need(aligned(d->workspace, 16), LAYUP_ERR_ALIGN, "workspace must be 16-byte aligned");
      }
    }
    return launch_norm_bwd(*d, k, s);
  });
}

layup_status layup_quant_fp8(const layup_quant_desc* d, void* stream) {
  return call(d, stream, "quantise", [&](hipStream_t s) {
    need(d->rows >= 0 && d->cols >= 0 && d->rows < (1ll << 31) && d->cols < (1ll << 31), LAYUP_ERR_SHAPE,
         "rows or columns out of range");
    need(is_wide(d->x_dtype) && is_fp8(d->q_dtype), LAYUP_ERR_DTYPE, "x: float32 or bfloat16; q: 8 bits");
    need(d->block_rows == 1 || d->block_rows == 128, LAYUP_ERR_INVALID_ARG, "block_rows must be 1 or 128");
    need(d->q || d->qt, LAYUP_ERR_INVALID_ARG, "neither q nor qt given");
    if (d->rows == 0 || d->cols == 0) return hipSuccess;
    matrix(d->x, d->ldx, d->cols, d->x_dtype, "null x");
    if (d->q) {
      matrix8(d->q, d->ldq, d->cols);
      scales(d->scale, d->ld_scale, d->cols);
    }
    if (d->qt) {
      matrix8(d->qt, d->ldqt, d->rows);
      scales(d->scale_t, d->ld_scale_t, d->rows);
    }
    return launch_quant_fp8(*d, s);
  });
}

static layup_status gemm_fp8(const layup_gemm_fp8_desc* d, int cfg, int splits, void* stream,
                             int64_t max_threads = MAX_LAUNCH_THREADS) {
  return call(d, stream, "8-bit product", [&](hipStream_t s) {
    const int64_t top = 1ll << 31;
    need(d->M >= 0 && d->N >= 0 && d->K >= 0 && d->M < top && d->N < top && d->K < top, LAYUP_ERR_SHAPE,
         "dimension out of range");
    need(is_fp8(d->a_dtype) && is_fp8(d->b_dtype), LAYUP_ERR_DTYPE, "A and B: 8 bits");
    need((d->a_block == 1 || d->a_block == 128) && (d->b_block == 1 || d->b_block == 128), LAYUP_ERR_INVALID_ARG,
         "a_block and b_block must be 1 or 128");
    if (d->M == 0 || d->N == 0) return hipSuccess;
    matrix(d->C, d->ldc, d->N, d->c_f32 ? LAYUP_F32 : LAYUP_BF16, "null C");
    floats(d->bias);
    if (d->K > 0) {
      matrix8(d->A, d->lda, d->K);
      matrix8(d->B, d->ldb, d->K);
      scales(d->a_scale, d->ld_a_scale, d->K);
      scales(d->b_scale, d->ld_b_scale, d->K);
      const int64_t most = 1ll << 24;  // 32-bit offsets inside a tile
      need(d->lda <= most && d->ldb <= most && d->ld_a_scale <= most && d->ld_b_scale <= most, LAYUP_ERR_SHAPE,
           "leading dimensions above 2^24 are not supported");
    }
    need(aligned(d->workspace, 16), LAYUP_ERR_ALIGN, "workspace must be 16-byte aligned");
    return cfg < 0 ? launch_gemm_fp8(*d, s) : launch_gemm_fp8_cfg(*d, cfg, splits, s, max_threads);
  });
}

layup_status layup_gemm_fp8(const layup_gemm_fp8_desc* d, void* stream) { return gemm_fp8(d, -1, 1, stream); }

int layup_test_gemm_fp8_tile(const layup_gemm_fp8_desc* d, int32_t cfg, int32_t splits, void* stream) {
  return gemm_fp8(d, cfg, splits, stream);
}

int layup_test_gemm_fp8_slices(const layup_gemm_fp8_desc* d, int32_t cfg, int32_t splits, int64_t max_threads, void* stream) {
  return gemm_fp8(d, cfg, splits, stream, max_threads);
}

}  // extern "C"
