// C-ABI entry points of the operators around the layer: argument validation and launches.
#include "kernels.h"

using namespace ssdi8;

namespace {

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned_to(p, 16); }
inline size_t elem_size(int dtype) { return dtype == 0 ? 4 : 2; }

// dims.seqlen and dims.chunk aside
bool heads_supported(const ssdi8_dims_t* d) {
  if (d->batch <= 0 || d->nheads <= 0 || d->ngroups <= 0) return false;
  if (d->headdim != 64 || (d->dstate != 64 && d->dstate != 128)) return false;
  // (a row's channels are counted in 32 bits)
  return d->nheads % d->ngroups == 0 && (i64)d->nheads * 64 + 2 * (i64)d->ngroups * d->dstate < (1 << 28);
}

// the slots of a cache; ring: with the convolution's
ssdi8_status_t cache_supported(const ssdi8_dims_t* d, const ssdi8_cache_t* c, const int32_t* slots, bool ring) {
  if (!heads_supported(d) || c->nslots <= 0 || (!slots && c->nslots < d->batch) || (i64)d->batch * d->nheads > 0x3fffffff) return SSDI8_ERR_SHAPE;
  if (ring && (c->dtype < 0 || c->dtype > 2)) return SSDI8_ERR_UNSUPPORTED;
  if (ring && (c->width < 2 || c->width > 4)) return SSDI8_ERR_SHAPE;
  if (!c->codes || !c->scales || !c->xwin || !c->Bwin || !c->dtwin || !c->start || (ring && !c->ring)) return SSDI8_ERR_NULL;
  const void* ptrs[] = {c->codes, c->scales, c->xwin, c->Bwin, c->dtwin, c->ring};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SSDI8_ERR_ALIGN;
  return SSDI8_OK;
}

}  // namespace

extern "C" {

ssdi8_status_t ssdi8_conv_fwd(const ssdi8_dims_t* dims, const ssdi8_conv_args_t* a, int32_t dtype, int32_t width, uint32_t flags,
                              void* stream) {
  if (!dims || !a) return SSDI8_ERR_NULL;
  if ((flags & ~(uint32_t)SSDI8_FLAG_DT_SOFTPLUS) != 0 || dtype < 0 || dtype > 2) return SSDI8_ERR_UNSUPPORTED;
  if (!heads_supported(dims) || dims->seqlen < 0 || width < 2 || width > 4) return SSDI8_ERR_SHAPE;
  if (dims->seqlen == 0) return SSDI8_OK;
  if (a->ring && a->nslots <= 0) return SSDI8_ERR_SHAPE;
  if (a->ring && !a->slots && a->nslots < dims->batch) return SSDI8_ERR_SHAPE;
  if (!a->xBC || !a->weight || (a->dt && !a->dt_raw)) return SSDI8_ERR_NULL;
  if (a->xq ? !a->Bq || !a->Cq || !a->s_x || !a->s_B || !a->s_C : !a->out) return SSDI8_ERR_NULL;
  if ((a->xq && a->out) || a->out == a->xBC) return SSDI8_ERR_UNSUPPORTED;
  const void* ptrs[] = {a->weight, a->ring, a->s_x, a->xq, a->Bq, a->Cq, a->out};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SSDI8_ERR_ALIGN;
  if (!aligned_to(a->xBC, elem_size(dtype)) || !aligned_to(a->dt_raw, elem_size(dtype))) return SSDI8_ERR_ALIGN;
  const ssdi8_status_t s = check_arch();
  if (s != SSDI8_OK) return s;
  return launch_conv(make_dims(dims), *a, dtype, width, (flags & SSDI8_FLAG_DT_SOFTPLUS) != 0, static_cast<cudaStream_t>(stream));
}

ssdi8_status_t ssdi8_cache_write(const ssdi8_dims_t* dims, const ssdi8_cache_t* cache, const int32_t* slots, const int32_t* pos,
                                 const float* state, int32_t* status, void* stream) {
  if (!dims || !cache) return SSDI8_ERR_NULL;
  ssdi8_status_t s = cache_supported(dims, cache, slots, false);
  if (s != SSDI8_OK) return s;
  if (!aligned16(state)) return SSDI8_ERR_ALIGN;
  if ((s = check_arch()) != SSDI8_OK) return s;
  return launch_cache_write(make_dims(dims), *cache, slots, pos, state, status, static_cast<cudaStream_t>(stream));
}

ssdi8_status_t ssdi8_cache_read(const ssdi8_dims_t* dims, const ssdi8_cache_t* cache, const int32_t* slots, const int32_t* first,
                                const int32_t* pos, const float* A, const float* s_x, const float* s_B, float* state, int32_t* status,
                                void* stream) {
  if (!dims || !cache) return SSDI8_ERR_NULL;
  ssdi8_status_t s = cache_supported(dims, cache, slots, false);
  if (s != SSDI8_OK) return s;
  if (!pos || !A || !s_x || !s_B || !state) return SSDI8_ERR_NULL;
  if (!aligned16(state) || !aligned16(s_x)) return SSDI8_ERR_ALIGN;
  if ((s = check_arch()) != SSDI8_OK) return s;
  return launch_cache_read(make_dims(dims), *cache, slots, first, pos, A, s_x, s_B, state, status, static_cast<cudaStream_t>(stream));
}

ssdi8_status_t ssdi8_token_step(const ssdi8_dims_t* dims, const ssdi8_cache_t* cache, const ssdi8_token_args_t* a, uint32_t flags,
                                void* stream) {
  if (!dims || !cache || !a) return SSDI8_ERR_NULL;
  constexpr uint32_t y16 = SSDI8_FLAG_Y_FP16 | SSDI8_FLAG_Y_BF16;
  if ((flags & ~(y16 | (uint32_t)SSDI8_FLAG_DT_SOFTPLUS)) != 0 || (flags & y16) == y16) return SSDI8_ERR_UNSUPPORTED;
  ssdi8_status_t s = cache_supported(dims, cache, a->slots, true);
  if (s != SSDI8_OK) return s;
  if (!a->xBC || !a->weight || !a->dt_raw || !a->A || !a->s_x || !a->s_B || !a->s_C || !a->pos || !a->y) return SSDI8_ERR_NULL;
  const size_t e = elem_size(cache->dtype);
  if (!aligned16(a->weight) || !aligned16(a->s_x) || !aligned_to(a->xBC, e) || !aligned_to(a->dt_raw, e) || !aligned_to(a->y, (flags & y16) ? 2 : 4))
    return SSDI8_ERR_ALIGN;
  if ((s = check_arch()) != SSDI8_OK) return s;
  return launch_token_step(make_dims(dims), *cache, *a, (flags & SSDI8_FLAG_DT_SOFTPLUS) != 0,
                           (flags & SSDI8_FLAG_Y_FP16) ? 1 : (flags & SSDI8_FLAG_Y_BF16) ? 2 : 0, static_cast<cudaStream_t>(stream));
}

ssdi8_status_t ssdi8_norm_quantize(const ssdi8_norm_args_t* a, int32_t dtype, int32_t zdtype, void* stream) {
  if (!a) return SSDI8_ERR_NULL;
  if (dtype < 0 || dtype > 2 || (a->z && (zdtype < 0 || zdtype > 2))) return SSDI8_ERR_UNSUPPORTED;
  if (a->rows < 0 || a->rows > 0x7fffffff || a->width <= 0 || a->width > kMaxNormWidth || a->width % 16 != 0 || a->groups <= 0) return SSDI8_ERR_SHAPE;
  if (a->groups > 1 && (a->width % a->groups != 0 || (a->width / a->groups) % 128 != 0)) return SSDI8_ERR_SHAPE;
  if (!(a->eps >= 0.f)) return SSDI8_ERR_SHAPE;
  if (a->rows == 0) return SSDI8_OK;
  if (!a->x || !a->xq) return SSDI8_ERR_NULL;
  if (!aligned16(a->weight) || !aligned16(a->xq) || !aligned_to(a->x, elem_size(dtype)) || !aligned_to(a->z, elem_size(zdtype)))
    return SSDI8_ERR_ALIGN;
  const ssdi8_status_t s = check_arch();
  if (s != SSDI8_OK) return s;
  return launch_norm_quantize(*a, dtype, zdtype, static_cast<cudaStream_t>(stream));
}

ssdi8_status_t ssdi8_linear(const ssdi8_linear_args_t* a, int32_t dtype, void* stream) {
  if (!a) return SSDI8_ERR_NULL;
  if (dtype < 0 || dtype > 2 || a->act < SSDI8_ACT_NONE || a->act > SSDI8_ACT_RELU2) return SSDI8_ERR_UNSUPPORTED;
  if (a->rows > 1 && a->stride_out < a->outs) return SSDI8_ERR_SHAPE;   // (rows that overlap)
  if (a->rows > kMaxLinearRows || a->outs > kMaxLinearRows) return SSDI8_ERR_SHAPE;
  if (a->rows < 0 || a->outs <= 0 || a->inner < 16 || a->inner > 131072 || a->inner % 16 != 0) return SSDI8_ERR_SHAPE;
  if (a->rows == 0) return SSDI8_OK;
  if (!a->xq || !a->wq || !a->s_w || !a->out) return SSDI8_ERR_NULL;
  if (!aligned16(a->xq) || !aligned16(a->wq) || !aligned_to(a->out, elem_size(dtype)) || !aligned_to(a->residual, elem_size(dtype)))
    return SSDI8_ERR_ALIGN;
  const ssdi8_status_t s = check_arch();
  if (s != SSDI8_OK) return s;
  return launch_linear(*a, dtype, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
