// Launches of the training side that do nothing, so that the host side of the C ABI can be driven through the calls that it
// takes, without a device (test infrastructure; built by tests/test_sanitizers_train.py).
#include "internal.h"

namespace reqat {

hipError_t launch_policy_loss(const PolicyArgs &, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_policy_backward(const PolicyArgs &, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_norm(const NormArgs &, bool, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_embedding(const EmbedArgs &, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_embedding_backward(const EmbedGradArgs &, const int32_t *, bool, bool, hipStream_t) { return hipSuccess; }
size_t embedding_workspace_bytes(int64_t T, int64_t, int64_t) { return T > 512 ? (size_t)T * 16 : 0; }
hipError_t launch_adamw(const AdamTensor *, int64_t, bool, bool, int, const AdamCoef &, const float *, const float *, hipStream_t) {
    return hipSuccess;
}
hipError_t launch_adamw_coef(double, double, double, double, const float *, int32_t *, float *, hipStream_t) { return hipSuccess; }
hipError_t launch_adamw_moments(const uint8_t *, const float *, const uint8_t *, const float *, int64_t, float *, float *, hipStream_t) {
    return hipSuccess;
}

}  // namespace reqat
