// Shared by the temporal head's operators.
#pragma once
#include <cuda.h>

typedef CUresult (*SrEncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
SrEncodeTiled sr_encode_tiled();                      // the driver's cuTensorMapEncodeTiled; null: there is none
int sr_device_sms();                                  // SMs of the current device; 0: no device
int* sr_operator_error_word();                        // set to 1 by a kernel of the current device whose bounded wait expired; null: no device
