#include "cb_attention.h"
namespace cb {
hipError_t launch_attention_bf16(const AttnArgs& A, const AttnPlan& P, void* out, float* lse, char* ws, hipStream_t st) {
    return launch_attention<__bf16, false>(A, P, (__bf16*)out, lse, ws, st);
}
hipError_t launch_attention_backward_bf16(const AttnArgs& A, const AttnPlan& P, const AttnGrads& G, char* ws, hipStream_t st) {
    return launch_attention_backward<__bf16, false>(A, P, G, ws, st);
}
}  // namespace cb
