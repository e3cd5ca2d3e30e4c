// Rows quantised to e4m3 codes (paged_codes.cuh).
#include "paged_codes.cuh"

namespace prism {

cudaError_t prepare_e4m3_store(bool bf16, int D) { return prepare_store<kE4m3>(bf16, D); }
cudaError_t start_e4m3_store(const NormRopeArgs &q, const StoreCodesArgs &a, bool bf16, int D, unsigned ctas, size_t shared, cudaStream_t s) {
    return start_store<kE4m3>(q, a, bf16, D, ctas, shared, s);
}

}  // namespace prism
