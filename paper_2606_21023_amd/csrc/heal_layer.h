// What the host and the kernels of the residual norms and of the adapters share.
#pragma once

#include <stdint.h>
#include <hip/hip_runtime.h>

namespace heal {

// N(y; weight, bias): weight NULL where there is no norm.
struct Norm {
    const float *weight, *bias;
    float eps;
    int centred;
};

struct NormArgs {
    int32_t rows, heads, dim;    // rows: all of them, rows * heads of the call
    const float *h;
    int64_t h_row, h_head;
    const float *x;
    int64_t x_row, x_head;
    Norm post, pre;
    const float *gate;
    int64_t gate_row, gate_head;
    int32_t gate_col;
    float scale;
    float *h_out;
    int64_t ho_row, ho_head;
    float *out;
    int64_t out_row, out_head;
};

hipError_t launch_block_norm(const NormArgs &a, hipStream_t stream);

struct LoraArgs {
    int32_t adapters, rank, tokens, seqs;
    int64_t K, N;
    const void *a, *b;
    const int32_t *ranks;
    const float *scales;
    const int32_t *cu, *ids;
    const float *x;
    int64_t ldx;
    const float *y;
    int64_t ldy;
    float *out;
    int64_t ldo;
    float *v;                    // parts x tokens x rank
};

int64_t lora_workspace(int64_t tokens, int64_t rank, int64_t K);   // bytes
hipError_t launch_lora(int type, const LoraArgs &a, hipStream_t stream);

}  // namespace heal
