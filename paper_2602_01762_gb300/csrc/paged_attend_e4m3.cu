// The paged attention over e4m3 codes (paged_attend_codes.cuh).
#include "paged_attend_codes.cuh"

namespace prism {

cudaError_t prepare_e4m3_attend(bool bf16, int D, int G) { return prepare_codes<kE4m3>(bf16, D, G); }
cudaError_t start_e4m3_attend(const CodeAttendArgs &a, bool bf16, int D, int sms, cudaStream_t s) { return start_codes<kE4m3>(a, bf16, D, sms, s); }

}  // namespace prism
