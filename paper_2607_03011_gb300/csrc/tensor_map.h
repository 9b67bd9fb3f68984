// tensor_map.h -- the CUDA driver API's encoder of tensor maps, looked up once (defined in api.cu).
#pragma once
#include <cuda.h>

namespace isoloco {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// cuTensorMapEncodeTiled; nullptr where the API has none.
EncodeTiledFn tensor_map_encoder();

}  // namespace isoloco
