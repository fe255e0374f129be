// The status of the launches just made, for every translation unit of the
// library: LDA_OK, or LDA_ERR_HIP with the error kept for lda_last_hip_error.
#pragma once

namespace lda {

__attribute__((visibility("hidden"))) int launch_status();

}  // namespace lda
