// Rows quantised to int8 codes (paged_codes.cuh).
#include "paged_codes.cuh"

namespace prism {

cudaError_t prepare_int8_store(bool bf16, int D) { return prepare_store<kInt8>(bf16, D); }
cudaError_t start_int8_store(const NormRopeArgs &q, const StoreCodesArgs &a, bool bf16, int D, unsigned ctas, size_t shared, cudaStream_t s) {
    return start_store<kInt8>(q, a, bf16, D, ctas, shared, s);
}

}  // namespace prism
