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
  if (a->xq && a->out) return SSDI8_ERR_UNSUPPORTED;
  const void* ptrs[] = {a->weight, a->ring, a->s_x, a->xq, a->Bq, a->Cq, a->out};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SSDI8_ERR_ALIGN;
  if (!aligned_to(a->xBC, elem_size(dtype)) || !aligned_to(a->dt_raw, elem_size(dtype))) return SSDI8_ERR_ALIGN;
  const ssdi8_status_t s = check_arch();
  if (s != SSDI8_OK) return s;
  return launch_conv(make_dims(dims), *a, dtype, width, (flags & SSDI8_FLAG_DT_SOFTPLUS) != 0, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
