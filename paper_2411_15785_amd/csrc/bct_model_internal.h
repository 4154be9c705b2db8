// What the files behind include/bct_model.h share on the host: errors, checks of launches and of alignment.
#ifndef BCT_MODEL_INTERNAL_H
#define BCT_MODEL_INTERNAL_H

#include <hip/hip_runtime.h>

#include "../../include/bct_model.h"

namespace bct {

// Keeps msg for bctm_last_error (of this thread) and returns s.
bct_status mfail(bct_status s, const char* msg);
// BCT_OK, or BCT_ERR_HIP with the error's text if the last launch failed.
bct_status launched(const char* what, hipError_t e = hipGetLastError());

inline bool al16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace bct

#endif
