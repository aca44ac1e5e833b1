// heal_lora_add: out[t] = y[t] + s B (A x[t]) with the adapter of each token's sequence.
#include <hip/hip_fp16.h>

#include "heal_device.h"
#include "heal_layer.h"

namespace heal {

namespace {

constexpr int kThreads = 256;

template <class T> __device__ __forceinline__ float as_float(T v) { return (float)v; }
template <> __device__ __forceinline__ float as_float<uint16_t>(uint16_t v)   // bfloat16
{
    return __builtin_bit_cast(float, (uint32_t)v << 16);
}

// The sequence of token t, or -1.
__device__ __forceinline__ int32_t seq_of(const LoraArgs &a, int32_t t)
{
    if (!a.cu) return t;
    if (a.seqs == 0 || t < a.cu[0] || t >= a.cu[a.seqs]) return -1;
    int32_t lo = 0, n = a.seqs;   // the last i with cu[i] <= t
    while (n > 1) {
        const int32_t half = n / 2;
        if (a.cu[lo + half] <= t) {
            lo += half;
            n -= half;
        } else {
            n = half;
        }
    }
    return lo;
}

// The adapter of sequence i and its rank; -1 and 0 where it has none.
__device__ __forceinline__ int32_t adapter_of(const LoraArgs &a, int32_t i, int32_t *rank)
{
    const int32_t id = i >= 0 ? a.ids[i] : -1;
    *rank = 0;
    if (id < 0 || id >= a.adapters) return -1;
    const int32_t r = a.ranks ? a.ranks[id] : a.rank;
    *rank = r < 0 ? 0 : r > a.rank ? a.rank : r;
    return id;
}

// v[t][j] = A_a x[t], one token a workgroup.
template <class T>
__global__ void __launch_bounds__(kThreads) lora_down_kernel(LoraArgs a)
{
    __shared__ float part[kThreads / 64];
    const int32_t t = blockIdx.x;
    int32_t rank;
    const int32_t id = adapter_of(a, seq_of(a, t), &rank);
    for (int32_t j = 0; j < rank; ++j) {
        const T *w = (const T *)a.a + ((int64_t)id * a.rank + j) * a.K;
        float s = 0.0f;
        for (int64_t k = threadIdx.x; k < a.K; k += kThreads) s += as_float(w[k]) * a.x[t * a.ldx + k];
        for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = s;
        __syncthreads();
        if (threadIdx.x == 0) a.v[(int64_t)t * a.rank + j] = (part[0] + part[1]) + (part[2] + part[3]);
    }
}

// out[t][n] = y[t][n] + s B_a v[t], a column a thread.
template <class T>
__global__ void __launch_bounds__(kThreads) lora_up_kernel(LoraArgs a)
{
    const int32_t t = blockIdx.x, i = seq_of(a, t);
    if (i < 0) return;
    int32_t rank;
    const int32_t id = adapter_of(a, i, &rank);
    if (rank == 0 && a.out == a.y) return;
    for (int64_t n = (int64_t)blockIdx.y * kThreads + threadIdx.x; n < a.N; n += (int64_t)gridDim.y * kThreads) {
        float y = a.y[t * a.ldy + n];
        if (rank > 0) {
            const T *w = (const T *)a.b + ((int64_t)id * a.N + n) * a.rank;
            float s = 0.0f;
            for (int32_t j = 0; j < rank; ++j) s += as_float(w[j]) * a.v[(int64_t)t * a.rank + j];
            y += (a.scales ? a.scales[id] : 1.0f) * s;
        }
        a.out[t * a.ldo + n] = y;
    }
}

template <class T>
hipError_t launch(const LoraArgs &a, hipStream_t stream)
{
    lora_down_kernel<T><<<dim3((unsigned)a.tokens), dim3(kThreads), 0, stream>>>(a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const int64_t cols = (a.N + kThreads - 1) / kThreads;
    lora_up_kernel<T><<<dim3((unsigned)a.tokens, (unsigned)(cols < 64 ? cols : 64)), dim3(kThreads), 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

int64_t lora_workspace(int64_t tokens, int64_t rank, int64_t K)
{
    (void)K;
    return 4 * tokens * rank;
}

hipError_t launch_lora(int type, const LoraArgs &a, hipStream_t stream)
{
    return type == 0 ? launch<float>(a, stream) : type == 1 ? launch<uint16_t>(a, stream) : launch<_Float16>(a, stream);
}

}  // namespace heal
