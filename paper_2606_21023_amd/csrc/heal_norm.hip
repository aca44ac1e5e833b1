// heal_block_norm: the residual stream between two blocks of a layer,
//     u = N(x; post),  h' = h + scale * gate * u,  out = N(h'; pre),
// one pass over the data: 4 bytes read for each element of h, x and a full gate, 4 written for each
// of h' and out, so it is bound by HBM. Statistics and elements are FP64 between the FP32 ends: a
// row needs no scaling against overflow, results are rounded once, and at four or five streams of 4
// bytes an element the FP64 instructions stay hidden.
#include "heal_device.h"
#include "heal_layer.h"

namespace heal {

namespace {

constexpr int kMaxThreads = 1024;

struct Stats {
    double shift, inv;
};

// Sums s and q over the T threads of a row, in an order that follows from T alone; every thread
// gets both. part: LDS of 2 doubles for each wave, its own for each call.
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

// Mean square (about the mean where centred) of a row from the sums of its elements' differences
// from `pivot`, one of its elements: the sum's square is at most dim times the sum of squares about
// the mean, so their difference keeps 52 - log2(dim) bits of what the sums have.
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

// T threads a row, U times four columns of it each, side by side; all of the row in registers
// between the sums and the stores: every stream is read once and written once. Rows may begin at
// any element: the 16-byte loads and stores need no alignment, and only a row's end is cut.
template <int T, int U>
struct Line {
    static __device__ __forceinline__ int column(int u, int e) { return (u * T + threadIdx.x % T) * 4 + e; }
    static __device__ __forceinline__ void load(const float *p, int dim, float (&v)[U][4])
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = column(u, 0);
            if (c + 4 <= dim) {
                __builtin_memcpy(v[u], p + c, 16);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[u][e] = c + e < dim ? p[c + e] : 0.0f;
            }
        }
    }
    static __device__ __forceinline__ void store(float *p, int dim, const float (&v)[U][4])
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = column(u, 0);
            if (c + 4 <= dim) {
                __builtin_memcpy(p + c, v[u], 16);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < dim) p[c + e] = v[u][e];
            }
        }
    }
    static __device__ __forceinline__ Stats stats_of(const Norm &n, int dim, const float (&v)[U][4], double pivot, double *part)
    {
        double s = 0.0, q = 0.0;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const double d = column(u, e) < dim ? (double)v[u][e] - pivot : 0.0;
                s += d;
                q += d * d;
            }
        row_sums<T>(s, q, n.centred, part);
        return stats(n, dim, pivot, s, q);
    }
};

// The norm of one value with its weight and bias.
__device__ __forceinline__ double normed(const Stats &st, float y, float w, float b)
{
    return ((double)y - st.shift) * st.inv * (double)w + (double)b;
}

template <int T, int U>
__global__ void __launch_bounds__(T < 256 ? 256 : T) norm_kernel(NormArgs a, int32_t row0)
{
    typedef Line<T, U> L;
    __shared__ double part[2][T > 64 ? 2 * T / 64 : 1];
    const int32_t r = (int32_t)((uint32_t)row0 + (T < 256 ? blockIdx.x * (256 / T) + threadIdx.x / T : blockIdx.x));
    if (T < 256 && (uint32_t)r >= (uint32_t)a.rows) return;   // (the last workgroup's may lie past 2^31)
    const Row p = row_of(a, r);
    float h[U][4], w[U][4], b[U][4] = {};
    L::load(p.h, a.dim, h);
    if (p.x) {
        float x[U][4], g[U][4];
        L::load(p.x, a.dim, x);
        auto rest = [&] {
            if (a.post.weight) L::load(a.post.weight, a.dim, w);
            if (a.post.bias) L::load(a.post.bias, a.dim, b);
            if (p.gate && a.gate_col) L::load(p.gate, a.dim, g);
        };
        if (U <= 4) rest();   // (longer rows' would not stay in registers)
        const double f = (double)a.scale * (p.gate && !a.gate_col ? (double)*p.gate : 1.0);
        Stats st = {0.0, 1.0};
        if (a.post.weight) st = L::stats_of(a.post, a.dim, x, a.post.centred ? (double)*p.x : 0.0, part[0]);
        if (U > 4) rest();
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const double y = a.post.weight ? normed(st, x[u][e], w[u][e], b[u][e]) : (double)x[u][e];
                const double fu = p.gate && a.gate_col ? f * (double)g[u][e] : f;
                h[u][e] = (float)((double)h[u][e] + fu * y);
            }
    }
    if (p.out) {
        if (U <= 4) {
            L::load(a.pre.weight, a.dim, w);
            if (a.pre.bias) L::load(a.pre.bias, a.dim, b);
        }
        // the pivot: the row's first element, from the thread that has it
        double pivot = 0.0;
        if (a.pre.centred) {
            if (T <= 64) {
                pivot = (double)__shfl(h[0][0], 0, T);
            } else {
                __shared__ float first;
                if (threadIdx.x == 0) first = h[0][0];
                __syncthreads();
                pivot = (double)first;
            }
        }
        const Stats st = L::stats_of(a.pre, a.dim, h, pivot, part[1]);
        float o[U][4];
        if (U > 4) {
            L::load(a.pre.weight, a.dim, w);
            if (a.pre.bias) L::load(a.pre.bias, a.dim, b);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                o[u][e] = (float)normed(st, h[u][e], w[u][e], a.pre.bias ? b[u][e] : 0.0f);
        L::store(p.out, a.dim, o);
    }
    // (an output may lie on an input: every thread writes the columns that it alone reads, and the
    // first element, which all threads of a centred row read, is written behind a sum of theirs)
    if (p.ho) L::store(p.ho, a.dim, h);
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

// Statistics of a row from y(c), column c's element. A thread's sums of dim / 1024 terms are off by as
// many roundings, and what the mean's square takes of the squares makes that larger: a first element
// of 10^6 before 2^24 threes cost 3.8e-6 of the result. So where it takes all but 2^-14 of them (the
// pivot lies more than 128 deviations off, which in rows of up to 2^14 it cannot), the sums are taken
// again about the mean.
template <class F>
__device__ __forceinline__ Stats stats_any(const Norm &n, int dim, double pivot, double *part, F y)
{
    for (int turn = 0;; ++turn) {
        double s = 0.0, q = 0.0;
        for (int c = threadIdx.x; c < dim; c += kMaxThreads) {
            const double d = y(c) - pivot;
            s += d;
            q += d * d;
        }
        row_sums<kMaxThreads>(s, q, true, part + turn * (2 * kMaxThreads / 64));
        const Stats st = stats(n, dim, pivot, s, q);
        const double mean = s / dim, square = q / dim;
        if (turn == 1 || !n.centred || !((square - mean * mean) * 16384.0 < square)) return st;
        pivot = st.shift;
    }
}

// Rows of any length: one workgroup a row, which reads it once for each of its sums and once to
// write.
__global__ void __launch_bounds__(kMaxThreads)
norm_any_kernel(NormArgs a, int32_t row0)
{
    __shared__ double part[2][2 * (2 * kMaxThreads / 64)];
    const Row p = row_of(a, row0 + blockIdx.x);
    Stats post = {0.0, 1.0}, pre = {0.0, 1.0};
    if (p.x && a.post.weight)
        post = stats_any(a.post, a.dim, a.post.centred ? (double)p.x[0] : 0.0, part[0], [&](int c) { return (double)p.x[c]; });
    if (p.out)
        pre = stats_any(a.pre, a.dim, a.pre.centred ? (double)added(a, p, post, 0) : 0.0, part[1],
                        [&](int c) { return (double)added(a, p, post, c); });
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

template <int T, int U>
hipError_t launch(const NormArgs &a, hipStream_t stream)
{
    return norm_launches(a.rows, T < 256 ? 256 / T : 1, [&](int32_t row0, unsigned n) {
        norm_kernel<T, U><<<dim3(n), dim3(T < 256 ? 256 : T), 0, stream>>>(a, row0);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_block_norm(const NormArgs &a, hipStream_t stream)
{
    if (a.dim <= 64) return launch<16, 1>(a, stream);
    if (a.dim <= 128) return launch<32, 1>(a, stream);
    if (a.dim <= 256) return launch<64, 1>(a, stream);
    if (a.dim <= 512) return launch<64, 2>(a, stream);
    if (a.dim <= 1024) return launch<256, 1>(a, stream);
    if (a.dim <= 2048) return launch<256, 2>(a, stream);
    if (a.dim <= 4096) return launch<256, 4>(a, stream);
    if (a.dim <= 8192) return launch<512, 4>(a, stream);
    if (a.dim <= 16384) return launch<512, 8>(a, stream);
    return norm_launches(a.rows, 1, [&](int32_t row0, unsigned n) {
        norm_any_kernel<<<dim3(n), dim3(kMaxThreads), 0, stream>>>(a, row0);
        return hipGetLastError();
    });
}

}  // namespace heal
