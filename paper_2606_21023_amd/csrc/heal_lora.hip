// heal_lora_add: out[t] = y[t] + s B (A x[t]) with the adapter of each token's sequence.
//
// Two kernels: v = A x in parts of K (lora_down_kernel), then the parts' sum, its product with B
// and the sum with y (lora_up_kernel).  What must move is x, y and out once and each
// adapter once; the products stay hidden behind that.
//
// Products.  An FP32 value is the exact sum of three bf16 parts (8 + 8 + 8 bits, each the
// rest of the one before it rounded), an FP16 weight of two, a bf16 weight is one.  A
// product of two values is the bf16 MFMAs of their parts i and j with i + j <= 2, up to six; the
// others are below 2^-26 of it.  So sums are FP32's in accuracy, at 16 cycles an MFMA of 32 columns
// (FP32 MFMA: 256 cycles, more than the memory takes from rank 64 on; and the compiler
// does not keep the registers of their addends from being written too early).
//
// Work units.  A unit is a tile of 64 tokens and one of the adapters in it: the first
// sequence of the tile with that adapter leads, and its workgroup takes all of the tile's rows of
// the adapter, packed into blocks of 16.  So a decode step reads an adapter once for 64
// tokens, whatever their order, and a prompt fills its tiles.
#include <string.h>

#include "heal_device.h"
#include "heal_kv.h"
#include "heal_layer.h"

namespace heal {

namespace {

constexpr int kTile = 64;                 // tokens of a unit
constexpr int kDownWaves = 8, kUpWaves = 4;
constexpr int kGroup = 128;               // ranks that a workgroup of the first kernel takes

// Depth of a part of K: the waves of a workgroup share it in runs of whole 32s.
__host__ __device__ inline int64_t part_depth(int64_t K)
{
    int64_t d = 1024;
    while (K > 8 * d) d *= 2;
    return d;
}

__host__ __device__ inline int parts_of(int64_t K) { return (int)((K + part_depth(K) - 1) / part_depth(K)); }

// Ranks of a row of v, whole 16s.
__host__ __device__ inline int32_t padded(int32_t rank) { return (rank + 15) / 16 * 16; }

struct Unit {
    int32_t first, count;     // tile, rows of it that are the unit's (0: nothing to do)
    int32_t id, rank;         // adapter (-1: none)
    int32_t row;              // lane i: the tile's row that is the i-th of the unit
};

__device__ __forceinline__ int32_t known(const LoraArgs &a, int32_t id) { return id >= 0 && id < a.adapters ? id : -1; }

__device__ __forceinline__ uint64_t bits(int32_t lo, int32_t hi)   // lo <= hi <= 64
{
    return (hi < 64 ? ((uint64_t)1 << hi) : 0) - (lo < 64 ? ((uint64_t)1 << lo) : 0);
}

// Rows of the tile at `first` that sequences of adapter id among j0 .. j0 + 63 own: lane l
// has the tokens begin .. end - 1 and the adapter of sequence j0 + l.
__device__ __forceinline__ uint64_t rows_of(int32_t first, int32_t id, int32_t begin, int32_t end, int32_t other)
{
    const int32_t lo = max(begin - first, 0), hi = min(end - first, kTile);
    uint64_t mine = __ballot(other == id && lo < hi), rows = 0;
    while (mine) {
        const int l = __builtin_ctzll(mine);
        mine &= mine - 1;
        rows |= bits(__builtin_amdgcn_readlane(lo, l), __builtin_amdgcn_readlane(hi, l));
    }
    return rows;
}

// Unit u, found by every wave for itself.
__device__ __forceinline__ Unit unit_of(const LoraArgs &a, int32_t u)
{
    const int lane = threadIdx.x & 63;
    Unit r = {0, 0, -1, 0, 0};
    uint64_t rows = 0;
    if (!a.cu) {   // a token a sequence, a unit each
        r.first = u / kTile * kTile;
        const int32_t t = r.first + lane;
        const int32_t other = t < a.tokens ? known(a, a.ids[t]) : -2;
        r.id = __builtin_amdgcn_readlane(other, u - r.first);
        rows = __ballot(other == r.id);
        if (__builtin_ctzll(rows) != u - r.first) return r;
    } else {
        // sequence i has the units first / 64 + i and on, one for each tile that it may reach
        int32_t i, begin, end, other, j0 = 0;
        auto load = [&](int32_t j) {
            const bool is = j >= 0 && j < a.seqs;
            begin = is ? kv_clamp(a.cu[j], 0, a.tokens) : a.tokens;
            end = is ? kv_clamp(a.cu[j + 1], begin, a.tokens) : a.tokens;
            other = is ? known(a, a.ids[j]) : -2;
        };
        if (a.seqs <= 64) {
            load(lane);
            const uint64_t below = __ballot(lane < a.seqs && begin / kTile + lane <= u);
            i = below ? 63 - __builtin_clzll(below) : 0;
        } else {
            i = kv_last_at_most(a.seqs, u, [&](int32_t j) { return (int64_t)kv_clamp(a.cu[j], 0, a.tokens) / kTile + j; });
            j0 = i;
            load(j0 + lane);
        }
        i = __builtin_amdgcn_readfirstlane(i);
        const int32_t at = __builtin_amdgcn_readlane(begin, i - j0), to = __builtin_amdgcn_readlane(end, i - j0);
        r.id = __builtin_amdgcn_readlane(other, i - j0);
        const int32_t tile = at / kTile + (u - (at / kTile + i));
        r.first = tile * kTile;
        if (u < at / kTile + i || r.first >= to || at >= to) return r;
        // the tile's rows from this sequence on, and whether an earlier one leads
        bool led = false;
        if (a.seqs <= 64) {
            rows = rows_of(r.first, r.id, begin, end, other);
            led = rows && __builtin_ctzll(rows) < max(at - r.first, 0);
        } else {
            for (int32_t j = j0;; j += 64) {
                if (j != j0) load(j + lane);
                rows |= rows_of(r.first, r.id, begin, end, other);
                if (__builtin_amdgcn_readlane(end, 63) >= r.first + kTile || j + 64 >= a.seqs) break;
            }
            for (int32_t j = j0 - 64; at > r.first && j > -64; j -= 64) {
                load(j + lane);
                led |= __ballot(other == r.id && begin < end && end > r.first) != 0;
                // (lane 0, or the first sequence there is)
                if (led || __builtin_amdgcn_readlane(begin, j < 0 ? -j : 0) <= r.first) break;
            }
        }
        if (led) return r;
    }
    r.count = __popcll(rows);
    // the i-th set bit to lane i, the others behind
    const int below = __popcll(rows & (((uint64_t)1 << lane) - 1));
    const int to = rows >> lane & 1 ? below : r.count + lane - below;
    r.row = __builtin_amdgcn_ds_permute(to * 4, lane);
    if (r.id >= 0) {
        const int32_t rank = a.ranks ? a.ranks[r.id] : a.rank;
        r.rank = __builtin_amdgcn_readfirstlane(rank < 0 ? 0 : rank > a.rank ? a.rank : rank);
    }
    return r;
}

__host__ __device__ inline int64_t units_of(bool ragged, int64_t tokens, int64_t seqs)
{
    return ragged ? tokens / kTile + seqs : tokens;
}

// Eight consecutive elements, of which the first n exist (the others are 0).  Rows may begin at any
// element: the loads need no alignment.
template <class T>
struct Run {
    T v[8];
};

template <class T>
__device__ __forceinline__ Run<T> load_run(const T *p, int64_t n)
{
    Run<T> r;
    if (n >= 8) {
        memcpy(&r, p, sizeof(r));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = e < n ? p[e] : T(0);
    }
    return r;
}

// The bf16 parts of eight values, operands of v_mfma_f32_16x16x32_bf16.
template <int P>
struct Parts {
    u32x4 p[P];
};

template <class T> constexpr int kParts = 3;                // FP32
template <> constexpr int kParts<uint16_t> = 1;             // bf16
template <> constexpr int kParts<_Float16> = 2;

__device__ __forceinline__ Parts<1> parts_of_run(const Run<uint16_t> &r)
{
    Parts<1> o;
    memcpy(&o, &r, sizeof(o));
    return o;
}

template <int P>
__device__ __forceinline__ Parts<P> split(const float (&v)[8])
{
    Parts<P> o;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        float a = v[e], b = v[e + 1];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
            o.p[i][e / 2] = h;
            a -= __builtin_bit_cast(float, h << 16);
            b -= __builtin_bit_cast(float, h & 0xffff0000u);
        }
    }
    return o;
}

__device__ __forceinline__ Parts<2> parts_of_run(const Run<_Float16> &r)
{
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)r.v[e];
    return split<2>(f);
}

__device__ __forceinline__ Parts<3> parts_of_run(const Run<float> &r) { return split<3>(r.v); }

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// acc[m][n] += w[n] x[m] for all products of parts i + j <= 2, the largest first.
template <int MB, int NB, int P>
__device__ __forceinline__ void products(f32x4 (&acc)[MB][NB], const Parts<3> (&x)[MB], const Parts<P> (&w)[NB])
{
#pragma unroll
    for (int sum = 0; sum <= 2; ++sum)
#pragma unroll
        for (int j = 0; j < P; ++j) {
            if (j > sum) continue;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) acc[mb][nb] = mfma(w[nb].p[j], x[mb].p[sum - j], acc[mb][nb]);
        }
}

// v of a unit's rows over one part of K, 128 ranks at most.  Eight waves take an eighth of
// the part each, 32 columns at a time straight from memory into operands (lane fr + 16
// fg: row fr, columns 8 fg .. 8 fg + 7, whole 128-byte lines of a row), then add their sums up in
// LDS, in the order of the waves.  MB: row blocks.
template <class T, int NB, int MB>
__device__ __forceinline__ void down(const LoraArgs &a, const Unit &un, int64_t depth, f32x4 (*part)[4][64])
{
    const int32_t j0 = blockIdx.z * kGroup, rank = min(un.rank - j0, 16 * NB);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), fr = lane & 15, fg = lane / 16;
    const int64_t run = depth / kDownWaves, k0 = blockIdx.y * depth + wave * run;
    const int64_t k1 = min(k0 + run, a.K);

    const float *x[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int32_t row = __shfl(un.row, mb * 16 + fr < un.count ? mb * 16 + fr : 0);
        x[mb] = a.x + (int64_t)(un.first + row) * a.ldx;
    }
    const T *w = static_cast<const T *>(a.a) + ((int64_t)un.id * a.rank + j0) * a.K;
    constexpr int N2 = NB < 2 || NB > 4 ? 1 : 2;   // weights' blocks at a time (their parts take registers)
    f32x4 acc[NB / N2][MB][N2] = {};
    auto step = [&](int64_t kk, int64_t left) {   // left: columns from kk + 8 fg on, 8 or more in whole steps
        const int64_t k = kk + 8 * fg;
        Run<float> xr[MB];
        Run<T> wr[2][N2];   // one turn ahead
        auto load = [&](int nb) {
#pragma unroll
            for (int n = 0; n < N2; ++n) {
                const int32_t j = (nb + n) * 16 + fr;
                wr[nb / N2 & 1][n] = load_run(w + (int64_t)(j < rank ? j : 0) * a.K + k, j < rank ? left : 0);
            }
        };
        load(0);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) xr[mb] = load_run(x[mb] + k, left);
        Parts<3> xp[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) xp[mb] = parts_of_run(xr[mb]);
#pragma unroll
        for (int nb = 0; nb < NB; nb += N2) {
            if (nb + N2 < NB) load(nb + N2);
            Parts<kParts<T>> wp[N2];
#pragma unroll
            for (int n = 0; n < N2; ++n) wp[n] = parts_of_run(wr[nb / N2 & 1][n]);
            products(acc[nb / N2], xp, wp);
        }
    };
    int64_t kk = k0;
    for (; kk + 32 <= k1; kk += 32) step(kk, 8);
    if (kk < k1) step(kk, a.K - kk - 8 * fg);   // (runs are whole 32s: only K's end cuts one)

    const int32_t cols = padded(a.rank);
    float *v = a.v + (int64_t)blockIdx.y * a.tokens * cols;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        if (nb > 0) __syncthreads();
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) part[wave][mb][lane] = acc[nb / N2][mb][nb % N2];
        __syncthreads();
        if (wave < MB) {   // a block of rows a wave
            f32x4 s = part[0][wave][lane];
#pragma unroll
            for (int q = 1; q < kDownWaves; ++q) s += part[q][wave][lane];
            const int32_t row = __shfl(un.row, (wave * 16 + fr) & 63);
            if (wave * 16 + fr < un.count && nb * 16 < rank)
                *reinterpret_cast<f32x4 *>(v + (int64_t)(un.first + row) * cols + j0 + nb * 16 + 4 * fg) = s;
        }
    }
}

template <class T, int NB>
__global__ void __launch_bounds__(64 * kDownWaves) lora_down_kernel(LoraArgs a, int32_t unit0, int64_t depth)
{
    __shared__ f32x4 part[kDownWaves][4][64];
    const Unit un = unit_of(a, unit0 + blockIdx.x);
    if (un.count == 0 || un.rank <= (int32_t)blockIdx.z * kGroup) return;
    if (un.count <= 16)
        down<T, NB, 1>(a, un, depth, part);
    else
        down<T, NB, 4>(a, un, depth, part);
}

// out = y + s B v for a unit's rows and a strip of columns.  The parts of v are added up in their order and split
// into LDS; then a wave takes 32 columns at a time (as the rows of the matrix
// instruction, so that a lane ends up with four columns of a token) and MB row blocks against
// them.  QB: blocks of 32 ranks, or 0 for ranks above 128, which take one row block
// at a time.
template <class T, int QB, int MB>
__device__ __forceinline__ void up(const LoraArgs &a, const Unit &un, const int32_t *rows, u32x4 *vs, int32_t parts, int32_t strip)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), fr = lane & 15, fg = lane / 16;
    const int32_t cols = padded(a.rank), held = padded(un.rank) / 8, qs = QB ? QB : (held + 3) / 4;
    const int32_t pitch = 3 * 4 * qs + 1;   // 16-byte units of a row: 4 of each part for 32 ranks
    const T *b = static_cast<const T *>(a.b) + (int64_t)un.id * a.N * a.rank;
    const float scale = a.scales ? a.scales[un.id] : 1.0f;
    const int64_t n_begin = (int64_t)blockIdx.y * strip, n_end = min(a.N, n_begin + strip);

    for (int m0 = 0; m0 < un.count; m0 += 16 * MB) {
        const int count = min(un.count - m0, 16 * MB);
        if (m0 > 0) __syncthreads();
        for (int i = threadIdx.x; i < count * 4 * qs; i += 64 * kUpWaves) {
            const int m = i / (4 * qs), j = i - m * 4 * qs;
            float s[8] = {};
            if (j < held) {
                const float *p = a.v + (int64_t)rows[m0 + m] * cols + 8 * j;
                for (int q = 0; q < parts; ++q, p += (int64_t)a.tokens * cols) {
                    const f32x4 lo = *reinterpret_cast<const f32x4 *>(p), hi = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[e] += lo[e];
                        s[4 + e] += hi[e];
                    }
                }
            }
            const Parts<3> o = split<3>(s);
#pragma unroll
            for (int e = 0; e < 3; ++e) vs[m * pitch + e * 4 * qs + j] = o.p[e];
        }
        __syncthreads();
        int64_t row[MB];   // of y and out
        int at[MB];        // of vs
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const int m = mb * 16 + fr < count ? mb * 16 + fr : 0;
            row[mb] = rows[m0 + m];
            at[mb] = m * pitch + fg;
        }

        for (int64_t n0 = n_begin + wave * 32; n0 < n_end; n0 += 32 * kUpWaves) {
            f32x4 acc[MB][2] = {};
            float y[MB][2][4];
            Run<T> br[2][2];
            auto fragment = [&](int q, Run<T> (&f)[2]) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t n = n0 + 16 * h + fr;
                    const int32_t j = 32 * q + 8 * fg;
                    f[h] = load_run(b + (n < a.N ? n : 0) * a.rank + j, un.rank - j);
                }
            };
            auto product = [&](int q, const Run<T> (&f)[2]) {
                Parts<3> vp[MB];
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int e = 0; e < 3; ++e) vp[mb].p[e] = vs[at[mb] + e * 4 * qs + 4 * q];
                const Parts<kParts<T>> bp[2] = {parts_of_run(f[0]), parts_of_run(f[1])};
                products(acc, vp, bp);
            };
            fragment(0, br[0]);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    const int64_t n = n0 + 16 * h + 4 * fg;
                    const float *p = a.y + row[mb] * a.ldy + n;
                    if (n + 4 <= a.N) {
                        memcpy(y[mb][h], p, 16);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[mb][h][e] = n + e < a.N ? p[e] : 0.0f;
                    }
                }
            if (QB == 1) {
                product(0, br[0]);
            } else {
#pragma unroll 1
                for (int q = 0; q < qs; q += 2) {   // a block of ranks ahead
                    if (q + 1 < qs) fragment(q + 1, br[1]);
                    product(q, br[0]);
                    if (q + 1 >= qs) break;
                    if (q + 2 < qs) fragment(q + 2, br[0]);
                    product(q + 1, br[1]);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    if (mb * 16 + fr >= count) continue;
                    const int64_t n = n0 + 16 * h + 4 * fg;
                    float *o = a.out + row[mb] * a.ldo + n;
                    float r[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[e] = fmaf(scale, acc[mb][h][e], y[mb][h][e]);
                    if (n + 4 <= a.N) {
                        memcpy(o, r, sizeof(r));
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (n + e < a.N) o[e] = r[e];
                    }
                }
        }
    }
}

template <class T, int QB>
__global__ void __launch_bounds__(64 * kUpWaves, 2) lora_up_kernel(LoraArgs a, int32_t unit0, int32_t parts, int32_t strip)
{
    extern __shared__ u32x4 vs[];
    __shared__ int32_t rows[kTile];
    const Unit un = unit_of(a, unit0 + blockIdx.x);
    if (un.count == 0 || (un.rank == 0 && a.out == a.y)) return;
    if (threadIdx.x < kTile) rows[threadIdx.x] = un.first + un.row;
    __syncthreads();
    if (un.rank == 0) {   // out is y
        const int64_t n_begin = (int64_t)blockIdx.y * strip, n_end = min(a.N, n_begin + strip);
        for (int m = 0; m < un.count; ++m)
            for (int64_t n = n_begin + threadIdx.x; n < n_end; n += 64 * kUpWaves)
                a.out[rows[m] * a.ldo + n] = a.y[rows[m] * a.ldy + n];
        return;
    }
    if (QB == 0 || un.count <= 16)
        up<T, QB, 1>(a, un, rows, vs, parts, strip);
    else
        up<T, QB, QB ? 4 : 1>(a, un, rows, vs, parts, strip);
}

template <class T, int NB>
hipError_t launch_down(const LoraArgs &a, int64_t units, hipStream_t stream)
{
    return in_parts(units, [&](int64_t at, unsigned n) {
        lora_down_kernel<T, NB><<<dim3(n, (unsigned)parts_of(a.K), (unsigned)((a.rank + kGroup - 1) / kGroup)),
                                  dim3(64 * kDownWaves), 0, stream>>>(a, (int32_t)at, part_depth(a.K));
    });
}

template <class T, int QB>
hipError_t launch_up(const LoraArgs &a, int64_t units, hipStream_t stream)
{
    int64_t strip = 32 * kUpWaves;
    while ((a.N + strip - 1) / strip > 32768) strip *= 2;
    const int32_t rows = QB ? (a.tokens < kTile ? a.tokens : kTile) : 16, qs = QB ? QB : (a.rank + 31) / 32;
    const size_t lds = (size_t)rows * (3 * 4 * qs + 1) * sizeof(u32x4);
    return in_parts(units, [&](int64_t at, unsigned n) {
        lora_up_kernel<T, QB><<<dim3(n, (unsigned)((a.N + strip - 1) / strip)), dim3(64 * kUpWaves), lds, stream>>>(
            a, (int32_t)at, parts_of(a.K), (int32_t)strip);
    });
}

template <class T>
hipError_t launch(const LoraArgs &a, hipStream_t stream)
{
    const int64_t units = units_of(a.cu != nullptr, a.tokens, a.seqs);
    const int blocks = a.rank < kGroup ? (a.rank + 15) / 16 : kGroup / 16;
    hipError_t err = blocks == 1   ? launch_down<T, 1>(a, units, stream)
                     : blocks == 2 ? launch_down<T, 2>(a, units, stream)
                     : blocks <= 4 ? launch_down<T, 4>(a, units, stream)
                                   : launch_down<T, 8>(a, units, stream);
    if (err != hipSuccess) return err;
    return a.rank > kGroup ? launch_up<T, 0>(a, units, stream)
           : a.rank <= 32  ? launch_up<T, 1>(a, units, stream)
           : a.rank <= 64  ? launch_up<T, 2>(a, units, stream)
                           : launch_up<T, 4>(a, units, stream);
}

}  // namespace

int64_t lora_workspace(int64_t tokens, int64_t rank, int64_t K)
{
    return 4 * parts_of(K) * tokens * padded((int32_t)rank);
}

hipError_t launch_lora(int type, const LoraArgs &a, hipStream_t stream)
{
    return type == 0 ? launch<float>(a, stream) : type == 1 ? launch<uint16_t>(a, stream) : launch<_Float16>(a, stream);
}

}  // namespace heal
