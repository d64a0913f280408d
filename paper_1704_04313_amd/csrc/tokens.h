// Host-side launch interface of the token operators' kernels (include/cbinfer_tokens.h has the formulas).  The entry
// points in tokens.hip have checked the arguments; everything here enqueues work on the given stream and
// returns the hipError_t of the launch.
#pragma once
#include "../../include/cbinfer_tokens.h"
#include "kernels.h"

namespace cbk {

// Stores a message for cbinfer_last_error() and returns the code.
int set_error(int code, const char *message) noexcept;

// A 2-byte or 4-byte element as float.
template <int DT>
struct Elem;
template <>
struct Elem<kF32> {
    typedef float type;
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <>
struct Elem<kBF16> {
    typedef unsigned short type;
    static __device__ __forceinline__ float get(unsigned short v) { return __uint_as_float((unsigned)v << 16); }
    static __device__ __forceinline__ unsigned short put(float v) { return __builtin_bit_cast(unsigned short, (__bf16)v); }
};

size_t log_probs_workspace(const cbinfer_log_probs_args &a);
hipError_t log_probs(hipStream_t st, const cbinfer_log_probs_args &a);

size_t linear_attention_workspace(const cbinfer_linear_attention_args &a);
hipError_t linear_attention(hipStream_t st, const cbinfer_linear_attention_args &a);

hipError_t quantise_weights(hipStream_t st, const void *weights, int dtype, int64_t rows, int64_t cols, int64_t row_stride,
                            int group, uint8_t *codes, uint16_t *scales);
size_t packed_weights_bytes(int64_t rows, int64_t cols, int group);
hipError_t pack_weights(hipStream_t st, const uint8_t *codes, const uint16_t *scales, int64_t rows, int64_t cols, int group,
                        void *packed);
size_t quantised_product_workspace(const cbinfer_quantised_product_args &a);
hipError_t quantised_product(hipStream_t st, const cbinfer_quantised_product_args &a);

hipError_t gated_norm(hipStream_t st, const cbinfer_gated_norm_args &a);

} // namespace cbk
