// The paged attention over int8 codes (paged_attend_codes.cuh).
#include "paged_attend_codes.cuh"

namespace prism {

cudaError_t prepare_int8_attend(bool bf16, int D, int G) { return prepare_codes<kInt8>(bf16, D, G); }
cudaError_t start_int8_attend(const CodeAttendArgs &a, bool bf16, int D, int sms, cudaStream_t s) { return start_codes<kInt8>(a, bf16, D, sms, s); }

}  // namespace prism
