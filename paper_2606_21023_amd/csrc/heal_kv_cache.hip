// The key/value cache's own kernels: tokens appended (with the rotation of their
// places), rows read back, and the blocks that a query should read.
#include "heal_device.h"
#include "heal_kv.h"

namespace heal {

namespace {

constexpr int kThreads = 256;

// INT8 code of one element: the real quotient 127 x / m rounded to the nearest
// integer, ties to even.  127 x is exact in FP64; the product with inv = 1 / m is off
// by less than 2^-44 and decides every quotient that is further than 2^-40 from a
// half-integer; the others take the correctly rounded FP64 quotient, which cannot
// cross a half-integer that it does not equal (x and m lie on the grid of x's last
// place, 2^-31 of m or more where a quotient reaches 1/2, so the two are 2^-33 apart
// or more).
__device__ __forceinline__ int code_i8(float x, double m, double inv)
{
    const double n = 127.0 * (double)x, p = n * inv;
    double r = __builtin_rint(p);
    if (__builtin_expect(__builtin_fabs(p - r) > 0.5 - 0x1p-40, 0)) r = __builtin_rint(n / m);
    return (int)r;
}

__device__ __forceinline__ f32x4 load4(const float *p, bool vec)
{
    if (vec) return *reinterpret_cast<const f32x4 *>(p);
    return f32x4{p[0], p[1], p[2], p[3]};
}

__device__ __forceinline__ uint32_t max_over_workgroup(uint32_t m, uint32_t *part)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) m = max(m, part[w]);
    return m;
}

// The pair (a, b) rotated: the FP64 products of FP32 values are exact and one sum of
// two is rounded once, fused or not, so the bits do not depend on contraction.
__device__ __forceinline__ void rotate(float &a, float &b, float co, float si)
{
    const double x = a, y = b, c = co, s = si;
    a = (float)(x * c - y * s);
    b = (float)(y * c + x * s);
}

// A row's columns c .. c + 3 as they lie in memory, and the rotation of rows whose
// columns are taken four pairs at a time: the first elements of the pairs and the second
// ones lie rot / 2 apart, or alternate.
struct Turn {
    int pairs;   // rot / 2
    bool interleaved;
    const float *cos, *sin;
    int64_t places;
};

// Whether rows at this address and stride can be read (written) in 16-byte units.
__device__ __forceinline__ bool units16(const float *p, int64_t token, int64_t head)
{
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)((token | head) * 4)) & 15u) == 0;
}

__device__ __forceinline__ void store4(float *p, f32x4 x, bool vec)
{
    if (vec) {
        *reinterpret_cast<f32x4 *>(p) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = x[e];
    }
}

// One row's elements, rotated if its place is in the table, four at a time: unit u of
// D / 4.  The units of the rotated part come in pairs that hold each other's partners,
// and unit u < rot / 8 does both; f(column, four elements) takes what comes out.
// Needs rot % 8 == 0.
template <class F>
__device__ __forceinline__ void turn_unit(const Turn &t, const float *src, bool vec, int u, bool turn, int64_t p, F f)
{
    const int two = t.pairs / 4;   // units that do two
    if (u >= two) {                // behind the rotated part
        const int c = 2 * t.pairs + 4 * (u - two);
        f(c, load4(src + c, vec));
        return;
    }
    const int c0 = t.interleaved ? 8 * u : 4 * u, c1 = t.interleaved ? c0 + 4 : c0 + t.pairs;
    f32x4 x = load4(src + c0, vec), y = load4(src + c1, vec);
    if (turn) {
        const float *co = t.cos + p * t.pairs + 4 * u, *si = t.sin + p * t.pairs + 4 * u;
        float a[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = t.interleaved ? 2 * e : e, j = t.interleaved ? 2 * e + 1 : e + 4;
            rotate(a[i], a[j], co[e], si[e]);
        }
        x = f32x4{a[0], a[1], a[2], a[3]};
        y = f32x4{a[4], a[5], a[6], a[7]};
    }
    f(c0, x);
    f(c1, y);
}

// ... one element, or one pair, at a time, for any even rot: unit u of D - rot / 2.
template <class F>
__device__ __forceinline__ void turn_pair(const Turn &t, const float *src, int u, bool turn, int64_t p, F f)
{
    if (u >= t.pairs) {
        f(t.pairs + u, src[t.pairs + u]);
        return;
    }
    const int c0 = t.interleaved ? 2 * u : u, c1 = t.interleaved ? c0 + 1 : c0 + t.pairs;
    float x = src[c0], y = src[c1];
    if (turn) rotate(x, y, t.cos[p * t.pairs + u], t.sin[p * t.pairs + u]);
    f(c0, x);
    f(c1, y);
}

// One block of one head, keys or values: rows staged in LDS as FP32.  Keys go in and
// out by rows, in 16-byte units; values come out by columns, four rows apart, which an
// odd row length spreads over the banks.
template <int D, int B>
struct Stage {
    union {
        float k[B][D + 4];
        float v[B][D + 1];
    };
    double sum[kThreads / D][D];
    uint32_t part[kThreads / 64];

    template <bool KEYS>
    __device__ __forceinline__ void put(int r, int c, f32x4 x)
    {
        if (KEYS) {
            *reinterpret_cast<f32x4 *>(&k[r][c]) = x;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[r][c + e] = x[e];
        }
    }
    template <bool KEYS>
    __device__ __forceinline__ float &at(int r, int c)
    {
        return KEYS ? k[r][c] : v[r][c];
    }
};

__device__ __forceinline__ uint32_t max_bits(uint32_t m, f32x4 x)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float y = x[e];
        m = max(m, __builtin_bit_cast(uint32_t, y) & 0x7fffffffu);
    }
    return m;
}

// New rows (place >= start) of block blk into the stage, rotated if they are keys, and
// the largest of m and their elements.
template <int D, int B, bool KEYS>
__device__ __forceinline__ uint32_t stage_new(Stage<D, B> &st, const KvAppendArgs &a, const KvSeq &s,
                                              int start, int head, int64_t blk, uint32_t m)
{
    const float *src = (KEYS ? a.k : a.v) + head * (KEYS ? a.k_head : a.v_head);
    const int64_t ts = KEYS ? a.k_token : a.v_token;
    const bool vec = units16(src, ts, 0);
    const int64_t p0 = blk * B;
    const int lo = p0 < start ? (int)(start - p0) : 0;
    const int hi = s.len - p0 < B ? (int)(s.len - p0) : B;
    const int64_t tok0 = (int64_t)s.first + (p0 - (s.len - s.n));
    const Turn t = {KEYS ? a.rot / 2 : 0, a.interleaved != 0, a.cos, a.sin, a.places};
    if (t.pairs % 4 == 0) {
        // threads stay in their columns: one division for all rows
        const int units = D / 4 - t.pairs / 4, step = kThreads / units, u = threadIdx.x % units;
        for (int r = lo + threadIdx.x / units; r < hi && (int)threadIdx.x < step * units; r += step)
            turn_unit(t, src + (tok0 + r) * ts, vec, u, p0 + r < t.places, p0 + r, [&](int c, f32x4 x) {
                st.template put<KEYS>(r, c, x);
                m = max_bits(m, x);
            });
    } else {
        const int units = D - t.pairs, step = kThreads / units, u = threadIdx.x % units;
        for (int r = lo + threadIdx.x / units; r < hi && (int)threadIdx.x < step * units; r += step)
            turn_pair(t, src + (tok0 + r) * ts, u, p0 + r < t.places, p0 + r, [&](int c, float x) {
                st.template at<KEYS>(r, c) = x;
                m = max(m, __builtin_bit_cast(uint32_t, x) & 0x7fffffffu);
            });
    }
    return m;
}

// The staged new rows of block blk into the sequence's ring.
template <int D, int B, bool KEYS>
__device__ __forceinline__ void store_ring(Stage<D, B> &st, const KvAppendArgs &a, const KvSeq &s, int start,
                                           int head, int64_t blk, int slot)
{
    const int64_t p0 = blk * B;
    const int lo = p0 < start ? (int)(start - p0) : 0;
    const int hi = s.len - p0 < B ? (int)(s.len - p0) : B;
    const int half = (int)(blk & 1) * B;
    const int64_t base = ((int64_t)slot * a.c.heads + head) * (2 * B * D);
    if (KEYS) {
        for (int i = lo * (D / 4) + threadIdx.x; i < hi * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4) * 4;
            *reinterpret_cast<f32x4 *>(a.c.kr + base + (half + r) * D + c) = *reinterpret_cast<const f32x4 *>(&st.k[r][c]);
        }
    } else if (hi - lo == 1) {   // one token: a thread to a column
        for (int c = threadIdx.x; c < D; c += kThreads) a.c.vr[base + c * (2 * B) + half + lo] = st.v[lo][c];
    } else {
        for (int i = threadIdx.x; i < B * D; i += kThreads) {
            const int c = i / B, r = i % B;
            if (r >= lo && r < hi) a.c.vr[base + c * (2 * B) + half + r] = st.v[r][c];
        }
    }
}

// One block of one head: the rows that the ring holds of it and the new ones, their
// maximum and mean, and, if the block is complete, its codes.
template <int D, int B, bool KEYS>
__device__ __forceinline__ void append_block(Stage<D, B> &st, const KvAppendArgs &a, int seq, int unit, int head)
{
    const KvSeq s = kv_seq(a.b, seq);
    const KvTouched t = kv_touched(s, B);
    const int64_t blk = (int64_t)t.first + unit;
    if (blk > t.last || blk >= a.b.cols) return;
    const int slot = kv_slot(a.b, seq);
    const int page = kv_page(a.b, seq, (int)blk);
    const int64_t p0 = blk * B;
    const int old = p0 < t.start ? (int)(t.start - p0) : 0;   // rows from the ring
    const int rows = s.len - p0 < B ? (int)(s.len - p0) : B;
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t m = 0u;

    // rows of the ring (zeros without one); keys by rows, values by columns
    const int64_t base = ((int64_t)slot * a.c.heads + head) * (2 * B * D);
    const int half = (int)(blk & 1) * B;
    if (KEYS) {
        for (int i = threadIdx.x; i < old * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4) * 4;
            const f32x4 x = slot >= 0 ? *reinterpret_cast<const f32x4 *>(a.c.kr + base + (half + r) * D + c) : zero;
            st.template put<KEYS>(r, c, x);
            m = max_bits(m, x);
        }
        // (zeros behind the last row add nothing to the mean)
        for (int i = rows * (D / 4) + threadIdx.x; i < B * (D / 4); i += kThreads)
            st.template put<KEYS>(i / (D / 4), i % (D / 4) * 4, zero);
    } else if (old > 0) {
        for (int i = threadIdx.x; i < D * (B / 4); i += kThreads) {
            const int c = i / (B / 4), r = i % (B / 4) * 4;
            if (r >= old) continue;
            const f32x4 x = slot >= 0 ? *reinterpret_cast<const f32x4 *>(a.c.vr + base + c * (2 * B) + half + r) : zero;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (r + e < old) {
                    const float y = x[e];
                    st.v[r + e][c] = y;
                    m = max(m, __builtin_bit_cast(uint32_t, y) & 0x7fffffffu);
                }
        }
    }
    m = stage_new<D, B, KEYS>(st, a, s, t.start, head, blk, m);
    m = max_over_workgroup(m, st.part);   // (and the rows are there for all)

    const int conflict = kv_ring_conflict(t);
    if (slot >= 0 && blk >= t.last - 1 && blk != conflict)
        store_ring<D, B, KEYS>(st, a, s, t.start, head, blk, slot);

    if (page >= 0) {
        const float mf = __builtin_bit_cast(float, m);
        const int64_t ph = (int64_t)page * a.c.heads + head;
        if (threadIdx.x == 0) a.c.scales[2 * ph + (KEYS ? 0 : 1)] = mf;
        if (rows == B) {
            const bool none = !(mf > 0.0f);
            const double md = none ? 1.0 : (double)mf, inv = 1.0 / md;
            uint32_t *out = reinterpret_cast<uint32_t *>(KEYS ? a.c.kc : a.c.vc) + ph * (B * D / 4);
            for (int i = threadIdx.x; i < B * D / 4; i += kThreads) {
                f32x4 x;
                if (KEYS) {
                    x = *reinterpret_cast<const f32x4 *>(&st.k[i / (D / 4)][i % (D / 4) * 4]);
                } else {
                    // dword i of [D][B]: value places 4 q .. 4 q + 3 of column i / (B / 4)
                    const int q = i % (B / 4), r = 16 * (q % (B / 16)) + 4 * (q / (B / 16));
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = st.v[r + e][i / (B / 4)];
                }
                uint32_t w = 0u;
#pragma unroll
                for (int e = 0; e < 4; ++e) w |= (uint32_t)(none ? 0 : code_i8(x[e], md, inv) & 0xff) << (8 * e);
                out[i] = w;
            }
        }
        if (KEYS) {
            // the mean: FP64 sums over whole parts of the block, joined in their order
            constexpr int P = kThreads / D;
            const int c = threadIdx.x % D, w = threadIdx.x / D;
            if (w < P) {
                double sum = 0.0;
                for (int r = w * (B / P); r < (w + 1) * (B / P); ++r) sum += (double)st.k[r][c];
                st.sum[w][c] = sum;
            }
            __syncthreads();
            if (threadIdx.x < D) {
                double sum = st.sum[0][threadIdx.x];
#pragma unroll
                for (int w2 = 1; w2 < P; ++w2) sum += st.sum[w2][threadIdx.x];
                a.c.mean[ph * D + threadIdx.x] = (float)(sum / (double)rows);
            }
        }
    }

    // ring rows of a later block where unit 0's old rows were
    if (unit == 0 && conflict >= 0 && conflict < a.b.cols && slot >= 0) {
        __syncthreads();
        stage_new<D, B, KEYS>(st, a, s, t.start, head, conflict, 0u);
        __syncthreads();
        store_ring<D, B, KEYS>(st, a, s, t.start, head, conflict, slot);
    }
}

// Queries of one token, rotated.
__device__ __forceinline__ void rotate_queries(const KvAppendArgs &a, int64_t token)
{
    const int seq = a.b.cu ? kv_last_at_most(a.b.seqs, token, [&](int i) { return (int64_t)kv_first(a.b, i); })
                           : (int)token;
    const KvSeq s = kv_seq(a.b, seq);
    if (token < s.first || token >= (int64_t)s.first + s.n) return;
    const int64_t p = (int64_t)s.len - s.n + (token - s.first);
    const bool turn = p >= 0 && p < a.places;
    const Turn t = {a.rot / 2, a.interleaved != 0, a.cos, a.sin, a.places};
    const float *src = a.q + token * a.q_token;
    float *dst = a.q_out + token * a.qo_token;
    const int D = a.c.dim;
    if (t.pairs % 4 == 0) {
        const bool in = units16(src, 0, a.q_head), out = units16(dst, 0, a.qo_head);
        const int units = D / 4 - t.pairs / 4, step = kThreads / units, u = threadIdx.x % units;
        for (int h = threadIdx.x / units; h < a.heads_q && (int)threadIdx.x < step * units; h += step)
            turn_unit(t, src + h * a.q_head, in, u, turn, p,
                      [&](int c, f32x4 x) { store4(dst + h * a.qo_head + c, x, out); });
    } else {
        const int units = D - t.pairs, step = kThreads / units, u = threadIdx.x % units;
        for (int h = threadIdx.x / units; h < a.heads_q && (int)threadIdx.x < step * units; h += step)
            turn_pair(t, src + h * a.q_head, u, turn, p, [&](int c, float x) { dst[h * a.qo_head + c] = x; });
    }
}

// One workgroup per (unit, head, keys or values), then one per token's queries.
// Bound by memory: a row is read once and its block staged in LDS, where the maximum, the
// mean and the codes are formed, so that they and the ring rows are written once (16018
// tokens of four prompts, 8 heads of keys and values and 32 of queries, all of 128:
// 174 us, 766 MB, 4.4 TB/s).  A token that joins a block reads the block's earlier
// rows again: one of each of 64 such sequences 11 us, bound by latency.
template <int D, int B>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(KvAppendArgs a, int64_t wg0, int64_t blocks_wg)
{
    __shared__ Stage<D, B> st;
    const int64_t wg = wg0 + blockIdx.x;
    if (wg >= blocks_wg) {
        rotate_queries(a, wg - blocks_wg);
        return;
    }
    const int64_t u = wg / (2 * a.c.heads);
    const int role = (int)(wg % (2 * a.c.heads));
    const int seq = a.b.cu ? kv_last_at_most(a.b.seqs, u, [&](int i) { return kv_unit(a.b, B, i); }) : (int)u;
    const int64_t j = u - kv_unit(a.b, B, seq);
    if (j < 0) return;
    if (role < a.c.heads)
        append_block<D, B, true>(st, a, seq, (int)j, role);
    else
        append_block<D, B, false>(st, a, seq, (int)j, role - a.c.heads);
}

// One block of one head back as FP32 rows.  Values are turned in LDS: codes with four
// bytes, FP32 rows (32 columns at a time) with one element more to a column.  Bound by
// the rows it writes (16018 tokens of 8 heads of 128, keys and values: 46 us, 131 MB).
template <int D, int B>
__global__ void __launch_bounds__(kThreads)
kv_read_kernel(KvSeqs b, KvCache c, float *k, float *v, int64_t wg0)
{
    __shared__ union {
        uint32_t codes[D][B / 4 + 1];
        float rows[32][B + 1];
    } x;
    const int64_t wg = wg0 + blockIdx.x;
    const int64_t u = wg / (2 * c.heads);
    const int role = (int)(wg % (2 * c.heads));
    const bool keys = role < c.heads;
    const int head = keys ? role : role - c.heads;
    float *out = keys ? k : v;
    if (!out) return;
    const int seq = b.cu ? kv_last_at_most(b.seqs, u, [&](int i) { return kv_unit(b, B, i); }) : (int)u;
    const int64_t j = u - kv_unit(b, B, seq);
    if (j < 0) return;
    const KvSeq s = kv_seq(b, seq);
    const KvTouched t = kv_touched(s, B);
    const int64_t ld = (int64_t)c.heads * D;
    const bool vec = (reinterpret_cast<uintptr_t>(out) & 15u) == 0;
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    out += head * D;
    if (j == 0)   // tokens before place 0 are nowhere
        for (int64_t i = threadIdx.x; i < (int64_t)(s.n - s.len) * D; i += kThreads)
            out[(s.first + i / D) * ld + i % D] = 0.0f;
    const int64_t blk = t.first + j;
    if (blk > t.last) return;
    const int64_t p0 = blk * B;
    const int lo = p0 < t.start ? (int)(t.start - p0) : 0;
    const int hi = s.len - p0 < B ? (int)(s.len - p0) : B;
    out += ((int64_t)s.first + (p0 - (s.len - s.n))) * ld;
    const int page = blk < b.cols ? kv_page(b, seq, (int)blk) : -1;
    const int slot = kv_slot(b, seq);
    const bool full = p0 + B <= s.len;
    const bool held = page >= 0 && (full || slot >= 0);
    const int64_t ph = (int64_t)page * c.heads + head;
    const int64_t ring = ((int64_t)slot * c.heads + head) * (2 * B * D);
    const int half = (int)(blk & 1) * B;
    if (held && !keys && !full) {
        for (int c0 = 0; c0 < D; c0 += 32) {
            for (int i = threadIdx.x; i < 32 * (B / 4); i += kThreads) {
                const int col = i / (B / 4), r = i % (B / 4) * 4;
                if (r >= hi) continue;
                const f32x4 y = *reinterpret_cast<const f32x4 *>(c.vr + ring + (c0 + col) * (2 * B) + half + r);
#pragma unroll
                for (int e = 0; e < 4; ++e) x.rows[col][r + e] = y[e];
            }
            __syncthreads();
            for (int i = lo * 8 + threadIdx.x; i < hi * 8; i += kThreads) {
                const int r = i / 8, col = i % 8 * 4;
                f32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = x.rows[col + e][r];
                store4(out + (int64_t)r * ld + c0 + col, y, vec);
            }
            __syncthreads();
        }
        return;
    }
    if (held && !keys) {
        const uint32_t *src = reinterpret_cast<const uint32_t *>(c.vc) + ph * (B * D / 4);
        for (int i = threadIdx.x; i < B * D / 4; i += kThreads) x.codes[i / (B / 4)][i % (B / 4)] = src[i];
        __syncthreads();
    }
    const float step = held && full ? c.scales[2 * ph + (keys ? 0 : 1)] / 127.0f : 0.0f;
    for (int i = lo * (D / 4) + threadIdx.x; i < hi * (D / 4); i += kThreads) {
        const int r = i / (D / 4), col = i % (D / 4) * 4;
        f32x4 y = zero;
        if (held && full) {
            uint32_t w;
            if (keys) {
                w = reinterpret_cast<const uint32_t *>(c.kc)[ph * (B * D / 4) + i];
            } else {
                const int at = kv_value_place(B, r);
                w = 0u;
#pragma unroll
                for (int e = 0; e < 4; ++e) w |= (x.codes[col + e][at / 4] >> (at % 4 * 8) & 0xffu) << (8 * e);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (float)(int8_t)(w >> (8 * e)) * step;
        } else if (held) {
            y = *reinterpret_cast<const f32x4 *>(c.kr + ring + (half + r) * D + col);
        }
        store4(out + (int64_t)r * ld + col, y, vec);
    }
}

// Scores in an order that unsigned integers keep: larger is better.
__device__ __forceinline__ uint64_t score_key(double x)
{
    if (!(x == x)) return 0u;   // no number: below -infinity's key, and taken like it
    uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);   // -0 counts as 0
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
constexpr uint64_t kLowest = 0x000fffffffffffffull;   // the key of -infinity

typedef double f64x4 __attribute__((ext_vector_type(4)));

// x, as a value that the compiler knows nothing of.
__device__ __forceinline__ float hidden(float x)
{
    asm volatile("" : "+v"(x));
    return x;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (uint64_t)hi << 32 | lo;
}

// The blocks of one token: the first lo, those from lo + n on, and the r best of the n
// candidates between them, whose keys are in LDS.  One wave: the r-th largest key is found
// bit by bit from the first bit in which the keys differ, ending where a threshold parts
// exactly r from the rest; then the blocks above it, and the lowest of those equal to
// it, are written in order.  A lane has candidates 64 apart, up to H of them in
// registers (H = 0: any number, read from LDS each time).
template <int H>
__device__ __forceinline__ void pick_blocks(const uint64_t *key, int lo, int n, int nb, int r, int32_t *sel)
{
    const int lane = threadIdx.x & 63;
    uint64_t held[H > 0 ? H : 1];
#pragma unroll
    for (int i = 0; i < H; ++i) held[i] = i * 64 + lane < n ? key[i * 64 + lane] : 0u;   // (no threshold is 0)
    // f(the lane's key, its candidate, whether there is one) for all of them in order
    auto each = [&](auto f) {
        if (H > 0) {
#pragma unroll
            for (int i = 0; i < H; ++i) f(held[i], i * 64 + lane, i * 64 + lane < n);
        } else {
            for (int i = lane; i - lane < n; i += 64) f(i < n ? key[i] : 0u, i, i < n);
        }
    };
    uint64_t top = 0u;
    int left = 0;
    if (r > 0) {
        auto keys_from = [&](uint64_t x) {
            int c = 0;
            each([&](uint64_t k, int, bool) { c += __popcll(__ballot(k >= x)); });
            return c;
        };
        uint64_t most = 0u, least = ~0ull;
        each([&](uint64_t k, int, bool is) {
            most = k > most ? k : most;
            least = is && k < least ? k : least;
        });
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            const uint64_t x = __shfl_xor(most, off), y = __shfl_xor(least, off);
            most = x > most ? x : most;
            least = y < least ? y : least;
        }
        most = uniform(most);
        least = uniform(least);
        top = most;
        if (most != least) {
            int bit = 63 - __builtin_clzll(most ^ least);
            top = bit == 63 ? 0u : most >> (bit + 1) << (bit + 1);
            for (; bit >= 0; --bit) {
                const uint64_t x = top | 1ull << bit;
                const int c = keys_from(x);
                if (c >= r) top = x;
                if (c == r) break;
            }
        }
        left = r - (top == ~0ull ? 0 : keys_from(top + 1));
    }
    for (int b = lane; b < lo; b += 64) sel[b] = b;
    int at = lo, equals = 0;
    if (r > 0) {
        const uint64_t before = (1ull << lane) - 1;
        each([&](uint64_t k, int i, bool is) {
            const uint64_t same = __ballot(is && k == top);
            const bool take = is && (k > top || (k == top && equals + __popcll(same & before) < left));
            const uint64_t taken = __ballot(take);
            if (take) sel[at + __popcll(taken & before)] = lo + i;
            at += __popcll(taken);
            equals += __popcll(same);
        });
    }
    for (int b = lo + n + lane; b < nb; b += 64) sel[at + b - (lo + n)] = b;
}

// One workgroup per key/value head and `slots` tokens of one sequence (1 or 4).
//
// Scores are FP64 matrix products: 16 rows of queries by 16 blocks, dim in steps of
// four that a lane has D/4 elements apart, so that its part of a mean is contiguous.
// A lane of the result holds rows lane / 16 + 4 v of one block.  With four tokens the
// row lane / 16 + 4 v is query v of token lane / 16 (queries behind the last repeat
// it), so the maximum over a token's queries is taken within the lane; with one
// token the 16 rows are its queries.  The order of the sum is the same for every block,
// so equal blocks score equally.  Bound by the latency of a workgroup's own stream of
// means and then of the search (32 sequences of up to 512 blocks 25 us, 66 MB; 777 tokens
// over up to 79 blocks 27 us).  Where waves have few tiles each (all but the sixteen-wave
// kernel) the next means are not asked for ahead: five waves fit on a SIMD instead of
// four (those 777 tokens 29.3 us with, 26.9 without).
template <int D, int SLOTS, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 1024 ? 4 : 5)
kv_select_kernel(KvSelectArgs a, int B, int64_t wg0)
{
    constexpr int slots = SLOTS;
    extern __shared__ char lds[];
    uint64_t *key = reinterpret_cast<uint64_t *>(lds);   // [slots][cols]
    const int wave = uniform((int)threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, kk = lane >> 4;
    const int64_t wg = wg0 + blockIdx.x;
    const int64_t u = wg / a.c.heads;
    const int head = (int)(wg % a.c.heads);
    int seq;
    int64_t first;   // token of slot 0
    if (slots == 1) {
        first = u;
        seq = a.b.cu ? kv_last_at_most(a.b.seqs, u, [&](int i) { return (int64_t)kv_first(a.b, i); }) : (int)u;
    } else {
        seq = kv_last_at_most(a.b.seqs, u, [&](int i) { return kv_tile(a.b, 1, 4, i); });
        first = kv_first(a.b, seq) + (u - kv_tile(a.b, 1, 4, seq)) * 4;
    }
    seq = uniform(seq);
    KvSeq s = kv_seq(a.b, seq);
    s = KvSeq{uniform(s.first), uniform(s.n), uniform(s.len)};
    if (first < s.first || first >= (int64_t)s.first + s.n) return;
    const int tokens = (int)((int64_t)s.first + s.n - first < slots ? s.first + s.n - first : slots);
    // blocks up to a token's own
    auto blocks_of = [&](int slot) {
        const int64_t place = (int64_t)s.len - s.n + (first + slot - s.first);
        const int64_t nb = place < 0 ? 0 : place / B + 1;
        return (int)(nb < a.b.cols ? nb : a.b.cols);
    };
    const int lo = a.keep_first, r = a.n_sel - a.keep_first - a.keep_last;
    const int most = blocks_of(tokens - 1), hi = most - a.keep_last;
    if (most > a.n_sel && r > 0) {
        const int per = slots == 1 ? 16 : 4;   // queries of a token in 16 rows
        for (int g0 = 0; g0 < a.group; g0 += per) {
            const int slot = slots == 1 ? 0 : col % 4, g = g0 + (slots == 1 ? col : col / 4);
            const int64_t token = first + (slot < tokens ? slot : tokens - 1);
            const float *qs = a.q + token * a.q_token + ((int64_t)head * a.group + (g < a.group ? g : a.group - 1)) * a.q_head + kk * (D / 4);
            float q[D / 4];
#pragma unroll
            for (int i = 0; i < D / 4; ++i) q[i] = qs[i];
            auto page_of = [&](int b0) { return b0 + col < hi ? kv_page(a.b, seq, b0 + col) : -1; };
            auto mean_of = [&](int page, f32x4 *m) {
                const f32x4 *src = reinterpret_cast<const f32x4 *>(a.c.mean + ((int64_t)page * a.c.heads + head) * D + kk * (D / 4));
#pragma unroll
                for (int i = 0; i < D / 16; ++i) m[i] = page >= 0 ? src[i] : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            };
            constexpr int STEP = THREADS / 64 * 16;
            constexpr bool AHEAD = THREADS == 1024;
            int b0 = lo + wave * 16;
            int page = b0 < hi ? page_of(b0) : -1;
            int next = AHEAD && b0 + STEP < hi ? page_of(b0 + STEP) : -1;
            f32x4 m[D / 16];
            if (AHEAD) mean_of(page, m);
            for (; b0 < hi; b0 += STEP) {
                // the page of the next tile is on the way, or its means and the page behind
                f32x4 m2[AHEAD ? D / 16 : 1];
                if (AHEAD)
                    mean_of(next, m2);
                else
                    mean_of(page, m);
                const int ahead = b0 + (AHEAD ? 2 : 1) * STEP;
                const int after = ahead < hi ? page_of(ahead) : -1;
                f64x4 sum = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
                for (int i = 0; i < D / 4; ++i)
                    // (q is converted here: as FP64 it would take the registers of a second wave)
                    sum = __builtin_amdgcn_mfma_f64_16x16x4f64((double)hidden(q[i]), (double)m[i / 4][i % 4], sum, 0, 0, 0);
                uint64_t best = kLowest;
                if (page >= 0) {
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const double x = sum[v];
                        const uint64_t k = score_key(x);
                        best = k > best ? k : best;
                    }
                }
                if (slots == 1) {
#pragma unroll
                    for (int off = 16; off < 64; off <<= 1) {
                        const uint64_t k = __shfl_xor(best, off);
                        best = k > best ? k : best;
                    }
                }
                if (kk < slots && b0 + col < hi) {
                    uint64_t *at = key + (int64_t)kk * a.b.cols + (b0 + col - lo);
                    *at = g0 > 0 && *at > best ? *at : best;
                }
                page = AHEAD ? next : after;
                next = after;
                if (AHEAD) {
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) m[i] = m2[AHEAD ? i : 0];
                }
            }
        }
    }
    __syncthreads();
    if (wave >= tokens) return;
    const int nb = uniform(blocks_of(wave));
    int32_t *sel = a.sel + ((first + wave) * a.c.heads + head) * a.n_sel;
    if (nb <= a.n_sel) {   // all of them
        for (int i = lane; i < a.n_sel; i += 64) sel[i] = i < nb ? i : -1;
        return;
    }
    const int n = nb - a.keep_last - lo;
    key += (int64_t)wave * a.b.cols;
    if (n <= 128)
        pick_blocks<2>(key, lo, n, nb, r, sel);
    else if (n <= 512)
        pick_blocks<8>(key, lo, n, nb, r, sel);
    else if (n <= 2048)
        pick_blocks<32>(key, lo, n, nb, r, sel);
    else
        pick_blocks<0>(key, lo, n, nb, r, sel);
}

template <int D, int B>
hipError_t append_sized(const KvAppendArgs &a, hipStream_t stream)
{
    const int64_t blocks_wg = kv_units(a.b.cu != nullptr, a.b.tokens, a.b.seqs, B) * 2 * a.c.heads;
    return in_parts(blocks_wg + (a.q ? a.b.tokens : 0), [&](int64_t at, unsigned n) {
        hipLaunchKernelGGL((kv_append_kernel<D, B>), dim3(n), dim3(kThreads), 0, stream, a, at, blocks_wg);
    });
}

template <int D, int B>
hipError_t read_sized(const KvSeqs &b, const KvCache &c, float *k, float *v, hipStream_t stream)
{
    const int64_t n = kv_units(b.cu != nullptr, b.tokens, b.seqs, B) * 2 * c.heads;
    return in_parts(n, [&](int64_t at, unsigned m) {
        hipLaunchKernelGGL((kv_read_kernel<D, B>), dim3(m), dim3(kThreads), 0, stream, b, c, k, v, at);
    });
}

template <int SLOTS, int THREADS>
hipError_t select_slots(const KvSelectArgs &a, int64_t n, size_t lds, hipStream_t stream)
{
    auto kernel = a.c.dim == 64   ? kv_select_kernel<64, SLOTS, THREADS>
                  : a.c.dim == 96 ? kv_select_kernel<96, SLOTS, THREADS>
                                  : kv_select_kernel<128, SLOTS, THREADS>;
    if (lds > 32768) {   // beyond what a kernel may ask for by itself
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)(kMaxSelectBlocks * sizeof(uint64_t)));
        if (err != hipSuccess) return err;
    }
    return in_parts(n, [&](int64_t at, unsigned m) {
        hipLaunchKernelGGL(kernel, dim3(m), dim3(THREADS), lds, stream, a, a.c.block, at);
    });
}

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs &a, hipStream_t stream)
{
    return sized(a.c.dim, a.c.block, [&](auto D, auto B) { return append_sized<D.value, B.value>(a, stream); });
}

hipError_t launch_kv_read(const KvSeqs &b, const KvCache &c, float *k, float *v, hipStream_t stream)
{
    return sized(c.dim, c.block, [&](auto D, auto B) { return read_sized<D.value, B.value>(b, c, k, v, stream); });
}

hipError_t launch_kv_select(const KvSelectArgs &a, hipStream_t stream)
{
    // four tokens of a sequence share its means, where their keys fit in LDS
    const int slots = a.b.cu && a.b.cols * 4 <= kMaxSelectBlocks ? 4 : 1;
    const int64_t n = (slots == 4 ? kv_tiles(a.b.tokens, a.b.seqs, 1, 4) : a.b.tokens) * a.c.heads;
    const size_t lds = (size_t)a.b.cols * slots * sizeof(uint64_t);
    if (slots == 4) return select_slots<4, 256>(a, n, lds, stream);
    // one token to a workgroup: sixteen waves where a compute unit has at most one workgroup
    // with much to read (32 sequences of up to 234 blocks 15.0 us, 17.9 with four waves),
    // else so few that each has a tile of 16 blocks and the next workgroups find room (256
    // sequences of 16 blocks 10.6 us with two waves, 24.8 with eight; of 62 blocks 22.2 us
    // with four, 31.1)
    if (n <= 256 && a.b.cols >= 128) return select_slots<1, 1024>(a, n, lds, stream);
    return a.b.cols <= 32 ? select_slots<1, 128>(a, n, lds, stream) : select_slots<1, 256>(a, n, lds, stream);
}

}  // namespace heal
