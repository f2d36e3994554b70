// Host-side set-up of the selection kernels (select.cu).
#pragma once

#include <cuda_runtime.h>

#include "../../include/ais.h"

namespace ais {

constexpr int kMaxTopLogits = AIS_TOP_MAX;      // entries of a row that top_logits returns, and of a top-k that stays a list

// Raises the dynamic shared-memory limit of every instantiation (once per device).
cudaError_t select_prepare();

}  // namespace ais
