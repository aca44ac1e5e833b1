// heal_lora_add: out[t] = y[t] + s B (A x[t]) with the adapter of each token's sequence.
//
// Two kernels: v = A x in parts of K (lora_down_kernel), then the parts' sum, its product with B
// and the sum with y (lora_up_kernel). What must move is x, y and out once and each adapter once;
// the products stay hidden behind that.
//
// Products. An FP32 value is the exact sum of three bf16 parts (8 + 8 + 8 bits, each the rest of
// the one before it rounded), an FP16 weight of two, a bf16 weight is one. A product of two values
// is the bf16 MFMAs of their parts i and j with i + j <= 2, up to six; the others are below 2^-26
// of it. So sums are FP32's in accuracy, at 96 cycles for 32 columns of a 16 x 16 block. (FP32
// matrix instructions take 256, more than the memory does from rank 64 on; and as built by this
// compiler registers that one still reads as its addend were cleared: every fourth column of a
// first form was wrong at rank 64.)
//
// Tiles. A workgroup has a tile of 64 tokens, finds the adapter of each, and takes the tile's
// adapters one after another (or every n-th, where n workgroups share the tile), the rows of each
// packed into blocks of 16. So a decode step reads an adapter once for 64 tokens, whatever their
// order, and a prompt fills its tiles.
#include <string.h>

#include <algorithm>

#include "heal_device.h"
#include "heal_kv.h"
#include "heal_layer.h"

namespace heal {

namespace {

constexpr int kTile = 64;                 // tokens
constexpr int kDownWaves = 4, kUpWaves = 4;
constexpr int kGroup = 128;               // ranks that a workgroup of the first kernel takes
// Strips of the second kernel are as narrow as this many workgroups allow: 5094 tokens of 4096
// columns 44 us (512 workgroups: 63), 64 tokens with 24 adapters at 14336 columns 15 us (512: 32,
// 1024: 19).
constexpr int64_t kUpWorkgroups = 2048;

// Depth of a part of K, whole 32s for each wave; 16 parts at most (every workgroup of the second
// kernel reads them all). It follows from K alone, and so does the order of the sums.
__host__ __device__ inline int64_t part_depth(int64_t K)
{
    int64_t d = 512;
    while (K > 16 * d) d *= 2;
    return d;
}

__host__ __device__ inline int parts_of(int64_t K) { return (int)((K + part_depth(K) - 1) / part_depth(K)); }

// Ranks of a row of v, whole 16s.
__host__ __device__ inline int32_t padded(int32_t rank) { return (rank + 15) / 16 * 16; }

// The adapter of token first + lane (-1: none; -2: no such token, or of no sequence).
__device__ __forceinline__ int32_t adapter_of_lane(const LoraArgs &a, int32_t first)
{
    const int lane = threadIdx.x & 63;
    const int32_t t = first + lane;
    auto known = [&](int32_t id) { return id >= 0 && id < a.adapters ? id : -1; };
    if (!a.cu) return t < a.tokens ? known(a.ids[t]) : -2;
    // sequences j0 .. j0 + 63, from the last one that begins at the tile's first token or before it
    int32_t j0 = 0, found = -2;
    if (a.seqs > 64)
        j0 = __builtin_amdgcn_readfirstlane(
            kv_last_at_most(a.seqs, first, [&](int32_t j) { return (int64_t)kv_clamp(a.cu[j], 0, a.tokens); }));
    for (;;) {
        const int32_t j = j0 + lane;
        const bool is = j < a.seqs;
        const int32_t begin = is ? kv_clamp(a.cu[j], 0, a.tokens) : a.tokens;
        const int32_t end = is ? kv_clamp(a.cu[j + 1], begin, a.tokens) : a.tokens;
        const int32_t id = is ? known(a.ids[j]) : -2;
        int at = 0;   // the last of these sequences that begins at t or before it
#pragma unroll
        for (int step = 32; step > 0; step >>= 1) at = __shfl(begin, at + step) <= t ? at + step : at;
        const int32_t b = __shfl(begin, at), e = __shfl(end, at), other = __shfl(id, at);
        if (b <= t && t < e) found = other;
        if (__builtin_amdgcn_readlane(end, 63) >= first + kTile || j0 + 64 >= a.seqs) return found;
        j0 += 64;
    }
}

// The rows of a tile that share an adapter.
struct Group {
    int32_t first, count, id;   // tile, rows, adapter (-1: none)
    int32_t row;                // lane i: the tile's row that is the i-th of the group
};

// f for every `share`-th group of the tile, from `turn` on; every wave finds them for itself.
template <class F>
__device__ __forceinline__ void for_groups(const LoraArgs &a, int32_t first, int32_t turn, int32_t share, F f)
{
    const int lane = threadIdx.x & 63;
    const int32_t id = adapter_of_lane(a, first);
    uint64_t todo = __ballot(id != -2);
    for (int32_t n = 0; todo; ++n) {
        const int32_t mine = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
        const uint64_t rows = __ballot(id == mine);
        todo &= ~rows;
        if (n != turn) continue;
        turn += share;
        const int32_t count = __popcll(rows);
        // the i-th set bit to lane i, the others behind
        const int below = __popcll(rows & (((uint64_t)1 << lane) - 1));
        const int to = rows >> lane & 1 ? below : count + lane - below;
        f(Group{first, count, mine, __builtin_amdgcn_ds_permute(to * 4, lane)});
    }
}

__device__ __forceinline__ int32_t rank_of(const LoraArgs &a, int32_t id)
{
    const int32_t rank = id < 0 ? 0 : a.ranks ? a.ranks[id] : a.rank;
    return __builtin_amdgcn_readfirstlane(min(max(rank, 0), a.rank));
}

template <class T>
__device__ __forceinline__ int32_t column_of(int e) { return e < 4 ? e : kNext<T> + e - 4; }

template <class T>
struct Run {
    T v[8];
};

// W: the adapters' type. CHECK: only the first n elements from p on exist; the others are 0.
template <class W, bool CHECK, class T>
__device__ __forceinline__ Run<T> load_run(const T *p, int64_t n = 0)
{
    Run<T> r;
    if (!CHECK) {
        memcpy(r.v, p, 4 * sizeof(T));
        memcpy(r.v + 4, p + kNext<W>, 4 * sizeof(T));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = column_of<W>(e) < n ? p[column_of<W>(e)] : T(0);
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

// v of a group's rows over one part of K, 128 ranks at most. The waves take 32 columns of the part
// each in turn, straight from memory into operands (Run has which columns a lane takes) and a turn
// ahead, then add their sums up in LDS, in the order of the waves. MB: row blocks, from row m0 of
// the group on. Of one row block the weights are most of what is read, and all are a turn ahead; of
// more, the rows.
template <class T, int NB, int MB>
__device__ __forceinline__ void down(const LoraArgs &a, const Group &un, int m0, int64_t depth, f32x4 (*part)[4][64])
{
    constexpr bool FEW = MB == 1 && NB <= 4;
    constexpr int N2 = NB < 2 || NB > 4 ? 1 : 2;   // weights' blocks at a time (their parts take registers)
    const int count = min(un.count - m0, 16 * MB);
    const int32_t j0 = blockIdx.z * kGroup;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), fr = lane & 15, fg = lane / 16;
    constexpr int64_t stride = 32 * kDownWaves;
    const int64_t k0 = blockIdx.y * depth + wave * 32, k1 = min((blockIdx.y + 1) * depth, a.K);
    const float *x[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int32_t row = __shfl(un.row, m0 + (mb * 16 + fr < count ? mb * 16 + fr : 0));
        x[mb] = a.x + (int64_t)(un.first + row) * a.ldx + kLane<T> * fg;
    }
    struct In {
        Run<float> x[MB];
        Run<T> w[FEW ? NB : N2];   // all blocks' weights, or the first ones'
    };
    // (cut: true_type for the columns that K cuts)
    auto load_x = [&](In &o, int64_t kk, auto cut) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) o.x[mb] = load_run<T, decltype(cut)::value>(x[mb] + kk, a.K - kk - kLane<T> * fg);
    };
    const std::false_type whole;
    const std::true_type cut;
    const int64_t steps = k1 >= k0 + 32 ? (k1 - k0 - 32) / stride + 1 : 0;   // whole ones; only K's end cuts one
    In now = {};
    if (steps > 0) load_x(now, k0, whole);
    const int32_t rank = min(rank_of(a, un.id) - j0, 16 * NB);
    if (rank <= 0) return;
    const T *w = static_cast<const T *>(a.a) + ((int64_t)un.id * a.rank + j0) * a.K + kLane<T> * fg;
    // ranks that are not there read the last one's weights and are zeroed at their use
    auto load_w = [&](int nb, int64_t kk, auto cut) {
        return load_run<T, decltype(cut)::value>(w + (int64_t)min(nb * 16 + fr, rank - 1) * a.K + kk, a.K - kk - kLane<T> * fg);
    };
    auto load_ws = [&](In &o, int64_t kk, auto cut) {
#pragma unroll
        for (int n = 0; n < (FEW ? NB : N2); ++n)
            if (n == 0 || n * 16 < rank) o.w[n] = load_w(n, kk, cut);
    };
    f32x4 acc[NB / N2][MB][N2] = {};
    auto step = [&](const In &in, int64_t kk, auto cut) {
        Parts<3> xp[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) xp[mb] = parts_of_run(in.x[mb]);
        Run<T> wr[N2];
#pragma unroll
        for (int nb = 0; nb < NB; nb += N2) {
            if (nb > 0 && nb * 16 >= rank) break;
            Parts<kParts<T>> wp[N2];
#pragma unroll
            for (int n = 0; n < N2; ++n) {
                if (FEW || nb == 0) wr[n] = in.w[nb + n];
                if ((nb + n + 1) * 16 > rank && (nb + n) * 16 + fr >= rank) wr[n] = Run<T>{};
                wp[n] = parts_of_run(wr[n]);
            }
            if (!FEW && nb + N2 < NB) {
#pragma unroll
                for (int n = 0; n < N2; ++n)
                    if ((nb + N2 + n) * 16 < rank) wr[n] = load_w(nb + N2 + n, kk, cut);
            }
            products(acc[nb / N2], xp, wp);
        }
    };
    if (steps > 0) load_ws(now, k0, whole);
#pragma unroll 1
    for (int64_t i = 0; i < steps; ++i) {   // (the last one loads itself once more)
        const int64_t kk = k0 + stride * i, after = i + 1 < steps ? kk + stride : kk;
        In next = {};
        load_x(next, after, whole);
        load_ws(next, after, whole);
        step(now, kk, whole);
        now = next;
    }
    if (k0 + stride * steps < k1) {
        const int64_t kk = k0 + stride * steps;
        load_x(now, kk, cut);
        load_ws(now, kk, cut);
        step(now, kk, cut);
    }

    const int32_t cols = padded(a.rank);
    float *v = a.v + (int64_t)blockIdx.y * a.tokens * cols;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        if (nb * 16 >= rank) break;
        if (nb > 0) __syncthreads();
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) part[wave][mb][lane] = acc[nb / N2][mb][nb % N2];
        __syncthreads();
        if (wave < MB) {   // a block of rows a wave
            f32x4 s = part[0][wave][lane];
#pragma unroll
            for (int q = 1; q < kDownWaves; ++q) s += part[q][wave][lane];
            const int32_t row = __shfl(un.row, (m0 + wave * 16 + fr) & 63);
            if (wave * 16 + fr < count)
                *reinterpret_cast<f32x4 *>(v + (int64_t)(un.first + row) * cols + j0 + nb * 16 + 4 * fg) = s;
        }
    }
}

template <class T, int NB>
__global__ void __launch_bounds__(64 * kDownWaves, NB == 1 ? 3 : 2) lora_down_kernel(LoraArgs a, int32_t wg0, int32_t share, int64_t depth)
{
    __shared__ f32x4 part[kDownWaves][4][64];
    const int32_t wg = wg0 + blockIdx.x, tile = __builtin_amdgcn_readfirstlane(wg / share);
    constexpr int MB = NB <= 4 ? 4 : 2;   // (256 registers)
    bool again = false;
    for_groups(a, tile * kTile, wg - tile * share, share, [&](const Group &un) {
        if (un.id < 0) return;
        for (int m0 = 0; m0 < un.count; m0 += 16 * MB) {
            if (again) __syncthreads();   // (of one use of LDS and the next)
            again = true;
            if (un.count - m0 <= 16)
                down<T, NB, 1>(a, un, m0, depth, part);
            else
                down<T, NB, MB>(a, un, m0, depth, part);
        }
    });
}

// out = y + s B v for a group's rows and a strip of columns. The parts of v are added up in their
// order and split into LDS; then a wave takes 32 columns (as the rows of the matrix instruction, so
// that a lane ends up with four columns of a token) and MB row blocks at a time, y a turn ahead. Of
// more than 32 rows each half has waves of its own. QB: blocks of 32 ranks, or 0 for ranks above
// 128, which take 16 rows at a time.
template <class T, int QB, int MB>
__device__ __forceinline__ void up(const LoraArgs &a, const Group &un, const int32_t *rows, u32x4 *vs, int32_t rank,
                                   int32_t parts, int32_t strip, int32_t col)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), fr = lane & 15, fg = lane / 16;
    const int32_t cols = padded(a.rank), qs = QB ? QB : (a.rank + 31) / 32, q_end = (rank + 31) / 32;
    const int32_t held = padded(rank);
    const int32_t pitch = 3 * 4 * qs + 1;   // 16-byte units of a row: 4 of each part for 32 ranks
    const T *b = static_cast<const T *>(a.b) + (int64_t)un.id * a.N * a.rank;
    const float scale = a.scales ? a.scales[un.id] : 1.0f;
    const int halves = QB && un.count > 16 * MB ? 2 : 1;
    const int half = halves == 2 ? wave & 1 : 0, turns = kUpWaves >> (halves - 1);
    const int32_t N = (int32_t)a.N;   // (below 2^25)
    const int32_t n_end = (int32_t)min(a.N, ((int64_t)col + 1) * strip);

    for (int m0 = 0; m0 < un.count; m0 += 16 * MB * halves) {
        const int count = min(un.count - m0, 16 * MB * halves);   // rows in LDS
        if (m0 > 0) __syncthreads();
        auto stage = [&] {
            constexpr int PARTS = MB == 1 ? 8 : 4;
#pragma unroll 1
            for (int i = threadIdx.x; i < count * 4 * q_end; i += 64 * kUpWaves) {
                const int m = i / (4 * q_end), j = i - m * 4 * q_end;
                float s[8] = {};
                const int32_t k = j / 4 * 32 + j % 4 * kLane<T>;   // as load_run has them
                if (k < held) {
                    const bool both = k + kNext<T> < held;
                    const float *p = a.v + (int64_t)rows[m0 + m] * cols + k;
                    for (int q0 = 0; q0 < parts; q0 += PARTS) {   // so many at once; behind the last one it is read again
                        f32x4 v[PARTS][2];
#pragma unroll
                        for (int q = 0; q < PARTS; ++q) {
                            const float *r = p + (int64_t)min(q0 + q, parts - 1) * a.tokens * cols;
                            v[q][0] = *reinterpret_cast<const f32x4 *>(r);
                            v[q][1] = *reinterpret_cast<const f32x4 *>(both ? r + kNext<T> : r);
                        }
#pragma unroll
                        for (int q = 0; q < PARTS; ++q)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                s[e] += q0 + q < parts && (e < 4 || both) ? v[q][e / 4][e % 4] : 0.0f;
                    }
                }
                const Parts<3> o = split<3>(s);
#pragma unroll
                for (int e = 0; e < 3; ++e) vs[m * pitch + e * 4 * qs + j] = o.p[e];
            }
            __syncthreads();
        };
        // Results leave the matrix instructions with 16 rows of 64 bytes; whole_lines turns two of
        // them into 8 rows of 128 bytes, whole lines (half lines: 1.4 times the bytes written).
        // Those rows of y and out, and the row of vs
        int64_t row[MB][2];
        bool is[MB][2];
        int at[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const int block = half * 16 * MB + mb * 16;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int m = block + 8 * h + (fr & 7);
                is[mb][h] = m < count;
                row[mb][h] = rows[m0 + (m < count ? m : 0)];
            }
            at[mb] = (block + fr < count ? block + fr : 0) * pitch + fg;
        }
        const int32_t col4 = 16 * (fr >> 3) + 4 * fg;   // a lane's columns of 32
        constexpr int AT = QB == 2 ? 2 : 1;   // blocks of ranks read at once
        struct Out {
            float v[MB][2][4];
        };
        auto is_whole = [&](int32_t n0) { return lora_whole(n0, N, a.rank); };
        // (what the adapter lacks may be anything, up to the array's ranks in whole fours)
        auto load_w = [&](Run<T> (&w)[2], int32_t n0, int q, auto whole) {
            const int32_t j = 32 * q + kLane<T> * fg;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int32_t n = n0 + 16 * h + fr;
                if (decltype(whole)::value) {
                    const T *p = b + (int64_t)n * a.rank + j;
                    w[h] = Run<T>{};
                    if (j < a.rank) memcpy(w[h].v, p, 4 * sizeof(T));
                    if (32 * q + kNext<T> < a.rank && j + kNext<T> < a.rank) memcpy(w[h].v + 4, p + kNext<T>, 4 * sizeof(T));
                } else {
                    const T *p = b + (int64_t)min(n, N - 1) * a.rank;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int32_t k = j + column_of<T>(e);
                        const T v = p[min(k, a.rank - 1)];
                        w[h].v[e] = k < a.rank ? v : T(0);
                    }
                }
            }
        };
        const std::true_type whole;
        const std::false_type cut;
        auto load_y = [&](float (&y)[MB][2][4], int32_t n0, auto whole) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int32_t n = n0 + col4;
                    const float *p = a.y + row[mb][h] * a.ldy + n;
                    if (decltype(whole)::value) {
                        memcpy(y[mb][h], p, 16);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[mb][h][e] = p[min(n + e, N - 1) - n];
                    }
                }
        };
        // (addresses are made from n0 in each turn: kept from turn to turn they take more registers
        // than there are)
        auto load = [&](Out &o, int32_t n0) {
            asm volatile("" : "+s"(n0));
            if (is_whole(n0))
                load_y(o.v, n0, whole);
            else
                load_y(o.v, n0, cut);
        };
        auto weights = [&](Run<T> (&w)[2], int32_t n0, int q) {
            asm volatile("" : "+s"(n0));
            if (is_whole(n0))
                load_w(w, n0, q, whole);
            else
                load_w(w, n0, q, cut);
        };
        auto columns = [&](const Out &y, Run<T> (&w)[AT][2], int32_t n0) {
            asm volatile("" : "+s"(n0));
            f32x4 acc[2][MB][1] = {};
            auto turn = [&](int q, Run<T> (&w)[2]) {
                Parts<3> vp[MB];
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int e = 0; e < 3; ++e) vp[mb].p[e] = vs[at[mb] + e * 4 * qs + 4 * q];
                const int32_t j = 32 * q + kLane<T> * fg;
#pragma unroll
                for (int h = 0; h < 2; ++h) {   // (one after the other: both halves' parts take more registers than there are)
                    if ((rank < a.rank || a.rank % 4 != 0) && 32 * q + 32 > rank) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[h].v[e] = j + column_of<T>(e) < rank ? w[h].v[e] : T(0);
                    }
                    const Parts<kParts<T>> wp[1] = {parts_of_run(w[h])};
                    products(acc[h], vp, wp);
                }
            };
            turn(0, w[0]);
            if (QB == 2) {
                if (q_end > 1) turn(1, w[AT - 1]);
            } else if (QB != 1) {
#pragma unroll 1
                for (int q = 1; q < q_end; ++q) {
                    weights(w[0], n0, q);
                    turn(q, w[0]);
                }
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                f32x4 line[2];
                whole_lines(acc[0][mb][0], acc[1][mb][0], fr, line[0], line[1]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (!is[mb][h]) continue;
                    const int32_t n = n0 + col4;
                    float *o = a.out + row[mb][h] * a.ldo + n;
                    float r[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[e] = fmaf(scale, line[h][e], y.v[mb][h][e]);
                    if (n0 + 32 <= N) {
                        memcpy(o, r, sizeof(r));
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (n + e < N) o[e] = r[e];
                    }
                }
            }
        };
        const int32_t stride = 32 * turns;
        int32_t n0 = col * strip + (wave >> (halves - 1)) * 32;
        Out now = {};
        if (n0 < n_end) load(now, n0);
        stage();
#pragma unroll 1
        for (; n0 < n_end; n0 += stride) {
            Run<T> w[AT][2];
            weights(w[0], n0, 0);
            if (QB == 2 && q_end > 1) weights(w[AT - 1], n0, 1);
            Out next = {};
            if (n0 + stride < n_end) load(next, n0 + stride);
            columns(now, w, n0);
            now = next;
        }
    }
}

template <class T, int QB>
__global__ void __launch_bounds__(64 * kUpWaves, QB == 1 ? 3 : 2)
lora_up_kernel(LoraArgs a, int64_t wg0, int32_t share, int32_t parts, int32_t strip)
{
    extern __shared__ u32x4 vs[];
    __shared__ int32_t rows[kTile];
    const int32_t strips = (int32_t)((a.N + strip - 1) / strip);
    const int64_t wgi = wg0 + blockIdx.x;
    // (divisions are made by vector instructions, even of scalars)
    const int32_t wg = __builtin_amdgcn_readfirstlane((int32_t)(wgi / strips));
    const int32_t col = (int32_t)(wgi - (int64_t)wg * strips);
    const int32_t tile = __builtin_amdgcn_readfirstlane(wg / share);
    bool again = false;
    for_groups(a, tile * kTile, wg - tile * share, share, [&](const Group &un) {
        if (un.id < 0 && a.out == a.y) return;
        if (again) __syncthreads();   // (of one use of LDS and the next)
        again = true;
        if (threadIdx.x < kTile) rows[threadIdx.x] = un.first + un.row;
        __syncthreads();
        const int32_t rank = rank_of(a, un.id);
        if (rank == 0) {   // out is y
            const int64_t n_begin = (int64_t)col * strip, n_end = min(a.N, n_begin + strip);
            if (a.out != a.y)
                for (int m = 0; m < un.count; ++m)
                    for (int64_t n = n_begin + threadIdx.x; n < n_end; n += 64 * kUpWaves)
                        a.out[rows[m] * a.ldo + n] = a.y[rows[m] * a.ldy + n];
            return;
        }
        if (QB == 0 || un.count <= 16)
            up<T, QB, 1>(a, un, rows, vs, rank, parts, strip, col);
        else
            up<T, QB, QB ? 2 : 1>(a, un, rows, vs, rank, parts, strip, col);
    });
}

// Workgroups that share a tile: as many as adapters can meet there where there are few tiles (64
// tokens that decode); one where there are many (prompts, with one adapter a tile as a rule).
int64_t shares(const LoraArgs &a)
{
    const int64_t tiles = (a.tokens + kTile - 1) / kTile;
    const int64_t met = std::min({(int64_t)kTile, (int64_t)a.tokens, (int64_t)a.seqs, (int64_t)a.adapters + 1});
    return std::max<int64_t>(1, std::min(met, 64 / tiles));
}

template <class T, int NB>
hipError_t launch_down(const LoraArgs &a, hipStream_t stream)
{
    const int64_t tiles = (a.tokens + kTile - 1) / kTile, parts = parts_of(a.K);
    const int64_t share = shares(a);
    return in_parts(tiles * share, [&](int64_t at, unsigned n) {
        lora_down_kernel<T, NB><<<dim3(n, (unsigned)parts, (unsigned)((a.rank + kGroup - 1) / kGroup)), dim3(64 * kDownWaves),
                                  0, stream>>>(a, (int32_t)at, (int32_t)share, part_depth(a.K));
    });
}

template <class T, int QB>
hipError_t launch_up(const LoraArgs &a, hipStream_t stream)
{
    const int64_t tiles = (a.tokens + kTile - 1) / kTile;
    const int64_t share = shares(a);
    int64_t strip = 32 * kUpWaves;
    auto strips = [&] { return (a.N + strip - 1) / strip; };
    while (tiles * share * strips() > kUpWorkgroups && strip < 1024) strip *= 2;
    while (strips() > 32768) strip *= 2;
    const int32_t rows = QB ? (a.tokens < kTile ? a.tokens : kTile) : 16, qs = QB ? QB : (a.rank + 31) / 32;
    const size_t lds = (size_t)rows * (3 * 4 * qs + 1) * sizeof(u32x4);
    return in_parts(tiles * share * strips(), [&](int64_t at, unsigned n) {
        lora_up_kernel<T, QB><<<dim3(n), dim3(64 * kUpWaves), lds, stream>>>(
            a, at, (int32_t)share, parts_of(a.K), (int32_t)strip);
    });
}

template <class T>
hipError_t launch(const LoraArgs &a, hipStream_t stream)
{
    const int blocks = a.rank < kGroup ? (a.rank + 15) / 16 : kGroup / 16;
    hipError_t err = blocks == 1   ? launch_down<T, 1>(a, stream)
                     : blocks == 2 ? launch_down<T, 2>(a, stream)
                     : blocks <= 4 ? launch_down<T, 4>(a, stream)
                                   : launch_down<T, 8>(a, stream);
    if (err != hipSuccess) return err;
    return a.rank > kGroup ? launch_up<T, 0>(a, stream)
           : a.rank <= 32  ? launch_up<T, 1>(a, stream)
           : a.rank <= 64  ? launch_up<T, 2>(a, stream)
                           : launch_up<T, 4>(a, stream);
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
