// Host-side helpers of the context that other translation units of the library may use.
#ifndef ZGR_HOST_INTERNAL_H_
#define ZGR_HOST_INTERNAL_H_

#include <cuda.h>
#include <stdint.h>

#include "zgr.h"
#include "zgr_internal.h"

namespace zgr {

PhiloxKeys host_make_keys(uint64_t seed);
NormalScale host_make_scale(double s, int bits);

// Read-only view of a context: descriptor of tensor l (host mirror), mixing scalars, generator mode,
// sticky error code, device ordinal the context is bound to.  Returns false if ctx is null or l is out of range.
bool host_ctx_view(const zgr_ctx* ctx, int32_t l, TensorDesc* desc, double* a, double* b, int* bits, int* sticky, int* device);

// cuTensorMapEncodeTiled through the runtime (the library does not link against libcuda); null where there is no driver that has it.
using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                   const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn();

}  // namespace zgr
#endif  // ZGR_HOST_INTERNAL_H_
