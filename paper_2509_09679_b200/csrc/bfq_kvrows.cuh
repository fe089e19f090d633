// Rows into and out of the paged low-bit key/value cache: the calls as the kernels see them.
#pragma once
#include "bfq_kv.cuh"

namespace bfq {
namespace kv {

struct AppendParams {
    Cache cache;
    Heads q, k, v, q_out;  // q.heads = 0: no queries
    const int64_t* slots;
    const int32_t* positions;  // null: no rotation by position
    const float* rope;         // [rope_rows][rope_dims]: cos of rope_dims / 2 frequencies, then sin
    const float* q_norm;
    const float* k_norm;
    const float2* tw;
    int64_t rope_rows, tokens;
    float eps;
    int rope_dims, interleaved;
    int* status;
};

struct ReadParams {
    Cache cache;
    const int64_t* slots;
    const float2* tw;
    uint8_t *k, *v;  // [tokens][heads][D]
    int64_t tokens;
    int* status;
};
// bfq_kvrows_few.cu: the same operations where rows are few
cudaError_t append_few_launch(const bfq_plan* plan, const AppendParams& p, bool f32, cudaStream_t st);
cudaError_t read_few_launch(const bfq_plan* plan, const ReadParams& p, bool f32, cudaStream_t st);

}  // namespace kv
}  // namespace bfq
