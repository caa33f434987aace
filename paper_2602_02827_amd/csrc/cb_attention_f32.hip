#include "cb_attention.h"
namespace cb {
hipError_t launch_attention_f32(const AttnArgs& A, const AttnPlan& P, void* out, float* lse, char* ws, hipStream_t st) {
    return launch_attention<float>(A, P, (float*)out, lse, ws, st);
}
hipError_t launch_attention_backward_f32(const AttnArgs& A, const AttnPlan& P, const AttnGrads& G, char* ws, hipStream_t st) {
    return launch_attention_backward<float>(A, P, G, ws, st);
}
}  // namespace cb
