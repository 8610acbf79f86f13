// C-ABI entry points of the operators in four bits and of the norm with the residual's addition: argument validation and launches.
#include "fp4.cuh"
#include "kernels.h"

using namespace ssdi8;

namespace {

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned_to(p, 16); }
inline size_t elem_size(int dtype) { return dtype == 0 ? 4 : 2; }

bool sizes_supported(int32_t rows, int32_t width, int32_t block) {
  return rows >= 0 && rows <= kMaxLinearRows && width >= 32 && width <= 131072 && width % 32 == 0 && (block == 16 || block == 32);
}
ssdi8_status_t fp4_supported(const ssdi8_fp4_t* q, bool step) {
  if (!sizes_supported(q->rows, q->width, q->block)) return SSDI8_ERR_SHAPE;
  // (rows of 128 bytes of scales are counted in 32 bits, those of a tile behind the last ones too)
  if ((i64)((q->rows + 255ll) / 128) * fp4_tiles(q->width, q->block) * 4 > 0x7fff0000) return SSDI8_ERR_SHAPE;
  if (q->rows == 0) return SSDI8_OK;
  if (!q->codes || !q->scales || (step && !q->step)) return SSDI8_ERR_NULL;
  return aligned16(q->codes) && aligned16(q->scales) && aligned_to(q->step, 4) ? SSDI8_OK : SSDI8_ERR_ALIGN;
}

}  // namespace

extern "C" {

size_t ssdi8_fp4_scales_bytes(int32_t rows, int32_t width, int32_t block) {
  if (!sizes_supported(rows, width, block)) return 0;
  return (size_t)((rows + 127ll) / 128) * fp4_tiles(width, block) * kTileBytes;
}

ssdi8_status_t ssdi8_fp4_quantize(const void* x, int64_t stride_x, int32_t dtype, const ssdi8_fp4_t* q, int32_t* status, void* stream) {
  if (!q) return SSDI8_ERR_NULL;
  if (dtype < 0 || dtype > 2) return SSDI8_ERR_UNSUPPORTED;
  ssdi8_status_t s = fp4_supported(q, q->block == 16);
  if (s != SSDI8_OK || q->rows == 0) return s;
  if (!x) return SSDI8_ERR_NULL;
  if (!aligned_to(x, elem_size(dtype))) return SSDI8_ERR_ALIGN;
  if ((s = check_arch()) != SSDI8_OK) return s;
  return launch_fp4_quantize(x, stride_x, dtype, *q, status, static_cast<cudaStream_t>(stream));
}

ssdi8_status_t ssdi8_fp4_dequantize(const ssdi8_fp4_t* q, void* out, int64_t stride_out, int32_t dtype, void* stream) {
  if (!q) return SSDI8_ERR_NULL;
  if (dtype < 0 || dtype > 2) return SSDI8_ERR_UNSUPPORTED;
  ssdi8_status_t s = fp4_supported(q, false);
  if (s != SSDI8_OK) return s;
  if (q->rows > 1 && stride_out < q->width) return SSDI8_ERR_SHAPE;   // (rows that overlap)
  if (q->rows == 0) return SSDI8_OK;
  if (!out) return SSDI8_ERR_NULL;
  if (!aligned_to(out, elem_size(dtype))) return SSDI8_ERR_ALIGN;
  if ((s = check_arch()) != SSDI8_OK) return s;
  return launch_fp4_dequantize(*q, out, stride_out, dtype, static_cast<cudaStream_t>(stream));
}

ssdi8_status_t ssdi8_add_norm_quantize(const ssdi8_add_norm_args_t* a, int32_t dtype, int32_t rdtype, void* stream) {
  if (!a) return SSDI8_ERR_NULL;
  const bool streamed = a->residual || a->residual_out;
  if (dtype < 0 || dtype > 2 || (streamed && rdtype != 0 && rdtype != dtype)) return SSDI8_ERR_UNSUPPORTED;
  if (a->fp4 && (a->xq || a->scale || a->static_scale)) return SSDI8_ERR_UNSUPPORTED;
  if (a->rows < 0 || a->rows > 0x7fffffff || a->width <= 0 || a->width > kMaxNormWidth || a->width % 16 != 0) return SSDI8_ERR_SHAPE;
  if (!(a->eps >= 0.f)) return SSDI8_ERR_SHAPE;
  if (a->residual_out && a->rows > 1 && a->stride_out < a->width) return SSDI8_ERR_SHAPE;   // (rows that overlap)
  if (a->fp4) {
    if (a->fp4->rows != a->rows || a->fp4->width != a->width) return SSDI8_ERR_SHAPE;
    const ssdi8_status_t s = fp4_supported(a->fp4, true);
    if (s != SSDI8_OK) return s;
  }
  if (a->rows == 0) return SSDI8_OK;
  if (!a->x || (!a->xq && !a->fp4)) return SSDI8_ERR_NULL;
  if (!aligned16(a->weight) || !aligned16(a->xq) || !aligned_to(a->x, elem_size(dtype)) || !aligned_to(a->residual, elem_size(rdtype)) ||
      !aligned_to(a->residual_out, elem_size(rdtype)))
    return SSDI8_ERR_ALIGN;
  const ssdi8_status_t s = check_arch();
  if (s != SSDI8_OK) return s;
  return launch_add_norm(*a, dtype, streamed ? rdtype : -1, static_cast<cudaStream_t>(stream));
}

ssdi8_status_t ssdi8_fp4_linear(const ssdi8_fp4_linear_args_t* a, int32_t dtype, void* stream) {
  if (!a || !a->x || !a->w) return SSDI8_ERR_NULL;
  if (dtype < 0 || dtype > 2 || a->act < SSDI8_ACT_NONE || a->act > SSDI8_ACT_RELU2) return SSDI8_ERR_UNSUPPORTED;
  ssdi8_status_t s = fp4_supported(a->x, false);
  if (s == SSDI8_OK) s = fp4_supported(a->w, false);
  if (s != SSDI8_OK) return s;
  if (a->x->width != a->w->width || a->x->block != a->w->block || a->w->rows <= 0) return SSDI8_ERR_SHAPE;
  if (a->x->rows > 1 && a->stride_out < a->w->rows) return SSDI8_ERR_SHAPE;   // (rows that overlap)
  if (a->x->rows == 0) return SSDI8_OK;
  if (!a->out) return SSDI8_ERR_NULL;
  if (!aligned_to(a->out, elem_size(dtype)) || !aligned_to(a->residual, elem_size(dtype))) return SSDI8_ERR_ALIGN;
  if ((s = check_arch()) != SSDI8_OK) return s;
  return launch_fp4_linear(*a, dtype, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
