// Shared by the library's translation units; not part of the C ABI.
#ifndef TFE_INTERNAL_H
#define TFE_INTERNAL_H

#include <cuda_runtime.h>

#include "../../include/tfe.h"

// TFE_OK, or TFE_ERR_CUDA with the text kept for tfe_last_cuda_error() of this thread (the sticky error is cleared).
__attribute__((visibility("hidden"))) tfe_status tfe_note_cuda(cudaError_t e, const char *what);

#endif
