// What the host and the kernels of the residual norms and of the adapters share.
#pragma once

#include <stdint.h>
#include <hip/hip_runtime.h>

#include "heal_kv.h"

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

// launch(first row, workgroups) for all rows, `per` of them a workgroup: 2^21 workgroups of up to 1024
// threads at a time (a dispatch counts work-items in 32 bits).
template <class F>
inline hipError_t norm_launches(int32_t rows, int per, F launch)
{
    for (int64_t r = 0; r < rows;) {
        const int64_t left = (rows - r + per - 1) / per, n = left < (1 << 21) ? left : 1 << 21;
        const hipError_t err = launch((int32_t)r, (unsigned)n);
        if (err != hipSuccess) return err;
        r += n * per;
    }
    return hipSuccess;
}

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
    float *v;                    // parts x tokens x rank, in whole 16s
};

// What a lane (row fr, place fg) has of 32 columns: of FP32 adapters' products the four from 4 fg
// on and the four 16 further on, so that the four lanes of a row ask for 64 bytes of it in one
// piece (32 bytes a lane side by side asked for every line twice); of 16-bit ones' the eight from 8
// fg on, 16 bytes. Rows may begin at any element: the loads need no alignment.
template <class T> constexpr int kNext = sizeof(T) == 4 ? 16 : 4;     // from the first four to the others
template <class T> constexpr int kLane = sizeof(T) == 4 ? 4 : 8;      // from lane to lane

// Loads of B take four elements of a row at a time, so where the rank is no multiple of four they
// run on into the rows behind it: three of them at rank 1, one otherwise. Whether they stay within
// N rows for the 32 from n0 on (the last rows of the last adapter end with the array).
HEAL_HD int32_t lora_rows_behind(int32_t rank) { return rank == 1 ? 3 : rank % 4 != 0; }
HEAL_HD bool lora_whole(int32_t n0, int32_t N, int32_t rank) { return n0 + 32 <= N - lora_rows_behind(rank); }

int64_t lora_workspace(int64_t tokens, int64_t rank, int64_t K);   // bytes
hipError_t launch_lora(int type, const LoraArgs &a, hipStream_t stream);

}  // namespace heal
