// heal_block_norm: the residual stream between two blocks of a layer,
//     u = N(x; post),  h' = h + scale * gate * u,  out = N(h'; pre),
// one pass over the data: 4 bytes read for each element of h, x and a full gate, 4
// written for each of h' and out, so it is bound by HBM.  Statistics and elements
// are FP64 between the FP32 ends: a row needs no scaling against overflow, results
// are rounded once, and at four or five streams of 4 bytes an element the FP64
// instructions stay hidden.
#include "heal_device.h"
#include "heal_layer.h"

namespace heal {

namespace {

constexpr int kMaxThreads = 1024;

struct Stats {
    double shift, inv;
};

// Sums s and q over the T threads of a row, in an order that follows from T alone; every
// thread gets both.  part: LDS of 2 doubles for each wave, its own for each call.
template <int T>
__device__ __forceinline__ void row_sums(double &s, double &q, bool two, double *part)
{
#pragma unroll
    for (int off = (T < 64 ? T : 64) / 2; off > 0; off >>= 1) {
        q += __shfl_xor(q, off);
        if (two) s += __shfl_xor(s, off);
    }
    if (T > 64) {
        const int wave = threadIdx.x / 64;
        if ((threadIdx.x & 63) == 0) {
            part[2 * wave] = q;
            part[2 * wave + 1] = s;
        }
        __syncthreads();
        q = s = 0.0;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) {
            q += part[2 * w];
            if (two) s += part[2 * w + 1];
        }
    }
}

// Mean square (about the mean where centred) of a row from the sums of its elements' differences from
// `pivot`, one of its elements: the sum's square is at most dim times the sum of
// squares about the mean, so their difference keeps 52 - log2(dim) bits.
__device__ __forceinline__ Stats stats(const Norm &n, int dim, double pivot, double s, double q)
{
    const double mean = n.centred ? s / dim : 0.0;
    double square = q / dim - mean * mean;
    square = square < 0.0 ? 0.0 : square;   // (keeps what is no number)
    return Stats{pivot + mean, 1.0 / sqrt(square + (double)n.eps)};
}

struct Row {
    const float *h, *x, *gate;
    float *ho, *out;
};

__device__ __forceinline__ Row row_of(const NormArgs &a, int32_t r)
{
    int32_t i = r, j = 0;
    if (a.heads > 1) {
        i = r / a.heads;
        j = r - i * a.heads;
    }
    return Row{a.h + i * a.h_row + j * a.h_head, a.x ? a.x + i * a.x_row + j * a.x_head : nullptr,
               a.gate ? a.gate + i * a.gate_row + j * a.gate_head : nullptr,
               a.h_out ? a.h_out + i * a.ho_row + j * a.ho_head : nullptr,
               a.out ? a.out + i * a.out_row + j * a.out_head : nullptr};
}

__device__ __forceinline__ double normed(const Norm &n, const Stats &st, float y, int c)
{
    const double v = ((double)y - st.shift) * st.inv * (double)n.weight[c];
    return n.bias ? v + (double)n.bias[c] : v;
}

// h' of column c.
__device__ __forceinline__ float added(const NormArgs &a, const Row &p, const Stats &post, int c)
{
    const float h = p.h[c];
    if (!p.x) return h;
    const float x = p.x[c];
    double u = a.post.weight ? normed(a.post, post, x, c) : (double)x;
    double f = (double)a.scale;
    if (p.gate) f *= (double)p.gate[a.gate_col ? c : 0];
    return (float)((double)h + f * u);
}

// Rows of any length: one workgroup a row, which reads it once for each of its sums and once to write.
__global__ void __launch_bounds__(kMaxThreads)
norm_any_kernel(NormArgs a, int32_t row0)
{
    __shared__ double part[2][2 * kMaxThreads / 64];
    const Row p = row_of(a, row0 + blockIdx.x);
    Stats post = {0.0, 1.0}, pre = {0.0, 1.0};
    if (p.x && a.post.weight) {
        const double pivot = a.post.centred ? (double)p.x[0] : 0.0;
        double s = 0.0, q = 0.0;
        for (int c = threadIdx.x; c < a.dim; c += kMaxThreads) {
            const double d = (double)p.x[c] - pivot;
            s += d;
            q += d * d;
        }
        row_sums<kMaxThreads>(s, q, true, part[0]);
        post = stats(a.post, a.dim, pivot, s, q);
    }
    if (p.out) {
        const double pivot = a.pre.centred ? (double)added(a, p, post, 0) : 0.0;
        double s = 0.0, q = 0.0;
        for (int c = threadIdx.x; c < a.dim; c += kMaxThreads) {
            const double d = (double)added(a, p, post, c) - pivot;
            s += d;
            q += d * d;
        }
        row_sums<kMaxThreads>(s, q, true, part[1]);
        pre = stats(a.pre, a.dim, pivot, s, q);
    }
    // (an output may lie on an input: each thread reads and writes its own elements, and
    // what others read of the row, its first element, they have by now)
    for (int c = threadIdx.x; c < a.dim; c += kMaxThreads) {
        const float y = added(a, p, post, c);
        if (p.out) {
            const float o = (float)normed(a.pre, pre, y, c);
            if (p.ho) p.ho[c] = y;
            p.out[c] = o;
        } else {
            p.ho[c] = y;
        }
    }
}

}  // namespace

hipError_t launch_block_norm(const NormArgs &a, hipStream_t stream)
{
    for (int32_t r = 0; r < a.rows;) {
        const int32_t n = a.rows - r < (1 << 21) ? a.rows - r : 1 << 21;
        norm_any_kernel<<<dim3((unsigned)n), dim3(kMaxThreads), 0, stream>>>(a, r);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
        r += n;
    }
    return hipSuccess;
}

}  // namespace heal
