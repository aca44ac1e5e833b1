// Attention over the key/value cache: INT8 blocks and FP32 rows, FP32 queries and
// outputs, FP16 matrix instructions.
//
// Mathematics.  With codes c (|c| <= 127, exact in FP16) of a block whose largest key
// is m, a score is  s = scale * (m / 127) * (q . c).  A query row is scaled by the
// power of two that brings its largest element to [2^13, 2^14) and split into an FP16
// pair q = hi + lo (lo = RNE_f16(q - hi): 2^-22 of the element, and never below
// 2^-25 of 2^14), so  q . c = hi . c + lo . c  on FP16 MFMA with FP32 sums.  The
// softmax weights p in [0, 1] are multiplied by the block's value maximum, scaled by
// a power of two (below) and split alike:  o += (p_hi + p_lo) . c.  An FP32 row of
// the cache is scaled by its block's maximum and split too; the product of the two
// residuals is left out (2^-22 of 2^-11).
//
// S^T = K q^T is formed rather than S: a lane then holds four tokens in a row of one
// query, and the 16 scores it has of a 64-token tile are, as they stand, its part of
// the right operand of  o^T = V^T p^T  if the tokens of V^T are read in that same
// order -- the order in which the cache stores them.  Nothing is moved between lanes
// but the row maximum.
#include "heal_device.h"
#include "heal_kv.h"

namespace heal {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int64_t kWantedWorkgroups = 1024;
constexpr int kNoScale = -100000;   // no value block with a scale seen yet

__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Four INT8 codes as FP16: 1024 + (code + 128) is the FP16 number with the byte
// code + 128 as its last bits, and 1152 is taken off exactly.
__device__ __forceinline__ void codes4(uint32_t w, f16x2 &a, f16x2 &b)
{
    const uint32_t x = w ^ 0x80808080u;
    const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    a = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, x, 0x04010400u)) - bias;
    b = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u)) - bias;
}

__device__ __forceinline__ f16x8 codes8(uint32_t w0, uint32_t w1)
{
    f16x2 a, b, c, d;
    codes4(w0, a, b);
    codes4(w1, c, d);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight FP32 values as FP16 pairs (hi, lo).
__device__ __forceinline__ void pairs8(const float *x, f16x8 &hi, f16x8 &lo)
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const f16x2 h = __builtin_convertvector((f32x2{x[i], x[i + 1]}), f16x2);
        const f32x2 r = {x[i] - (float)h[0], x[i + 1] - (float)h[1]};
        const f16x2 l = __builtin_convertvector(r, f16x2);
        hi[i] = h[0];
        hi[i + 1] = h[1];
        lo[i] = l[0];
        lo[i + 1] = l[1];
    }
}

// e with |x| in [2^(e-1), 2^e), or kNoScale for 0 (and for what is not finite: its
// products come out as no numbers with any scale).
__device__ __forceinline__ int exponent(float x)
{
    if (!(__builtin_fabsf(x) > 0.0f) || __builtin_isinf(x)) return kNoScale;
    return __builtin_amdgcn_frexp_expf(x);
}

// A value that all lanes have.  Matrix instructions take no notice of lanes that are
// switched off, so every branch around them has to be one of the whole wave, and what
// it depends on has to be known as such.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ KvSeq uniform_seq(const KvSeqs &b, int i)
{
    const KvSeq s = kv_seq(b, i);
    return KvSeq{uniform(s.first), uniform(s.n), uniform(s.len)};
}

__device__ __forceinline__ float max_over_groups(float x)
{
    x = __builtin_fmaxf(x, __shfl_xor(x, 16));
    return __builtin_fmaxf(x, __shfl_xor(x, 32));
}

__device__ __forceinline__ float sum_over_groups(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// A row tile: 16 rows, one for each lane % 16.
struct Rows {
    KvSeq s;
    int32_t seq;
    int32_t token;   // of this lane's row, or -1 where there is none
    int32_t head_q;
    int32_t lo, hi;  // the places it sees: lo .. hi (none where hi < lo)
    int32_t first, last;   // ... one row or another
    int32_t all_lo, all_hi;   // ... all rows
};

// Finds the rows of tile u of a key/value head.  Returns false where the tile has none.
template <int R>
__device__ __forceinline__ bool find_rows(const KvAttnArgs &a, bool by_token, int64_t u, int head, int r,
                                          Rows &t)
{
    int32_t row0, rows;
    if (by_token) {
        const int per = (a.group + R - 1) / R;
        const int64_t token = u / per;
        t.seq = a.b.cu ? kv_last_at_most(a.b.seqs, token, [&](int i) { return (int64_t)kv_first(a.b, i); })
                       : (int)token;
        t.seq = uniform(t.seq);
        t.s = uniform_seq(a.b, t.seq);
        if (token < t.s.first || token >= (int64_t)t.s.first + t.s.n) return false;
        row0 = (int)(u % per) * R;
        rows = a.group - row0 < R ? a.group - row0 : R;
        row0 += (int)(token - t.s.first) * a.group;
    } else {
        t.seq = kv_last_at_most(a.b.seqs, u, [&](int i) { return kv_tile(a.b, a.group, R, i); });
        t.seq = uniform(t.seq);
        t.s = uniform_seq(a.b, t.seq);
        const int64_t j = u - kv_tile(a.b, a.group, R, t.seq);
        const int64_t n = (int64_t)t.s.n * a.group;
        if (j < 0 || j * R >= n) return false;
        row0 = (int)(j * R);
        rows = n - row0 < R ? (int)(n - row0) : R;
    }
    const int64_t end = (int64_t)a.b.cols * a.c.block;   // places that the table has
    auto bounds = [&](int row, int32_t &lo, int32_t &hi) {
        const int64_t place = (int64_t)t.s.len - t.s.n + row / a.group;
        int64_t h = a.causal ? place : t.s.len - 1, l = a.window > 0 ? place - a.window + 1 : 0;
        if (place < 0) h = -1;
        if (h >= t.s.len) h = t.s.len - 1;
        if (h >= end) h = end - 1;
        lo = (int32_t)(l < 0 ? 0 : l);
        hi = (int32_t)h;
    };
    bounds(row0, t.first, t.all_hi);
    bounds(row0 + rows - 1, t.all_lo, t.last);
    t.token = -1;
    t.lo = 0;
    t.hi = -1;
    t.head_q = 0;
    if (r < rows) {
        bounds(row0 + r, t.lo, t.hi);
        t.token = t.s.first + (row0 + r) / a.group;
        t.head_q = head * a.group + (row0 + r) % a.group;
    }
    return true;
}

// ln of the sum that the maximum m (log2 units) and the sum l stand for.
__device__ __forceinline__ float log_sum(float m, float l)
{
    return l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

__device__ __forceinline__ void store4(float *p, f32x4 x, bool vec)
{
    if (vec) {
        *reinterpret_cast<f32x4 *>(p) = x;
    } else {
        p[0] = x[0];
        p[1] = x[1];
        p[2] = x[2];
        p[3] = x[3];
    }
}

__device__ __forceinline__ float4 load16(const float *p, bool vec)
{
    if (vec) return *reinterpret_cast<const float4 *>(p);
    return float4{p[0], p[1], p[2], p[3]};
}

// The blocks of a wave's next tiles, one to a lane: a tile of 64 tokens has EPT of
// them, so the lanes hold the blocks and scales of TILES tiles, which are read in two
// round trips to memory for all of them together.
template <int B>
struct Blocks {
    static constexpr int EPT = B < 64 ? 64 / B : 1, TILES = 64 / EPT, STEP = B < 64 ? B : 64;
    int blk;     // block of the sequence, or -1 where the cache holds nothing of it
    int page;    // its page, or -1 - page where it is read from the ring
    float k, v;  // m of its keys and values

    __device__ __forceinline__ void load(const KvAttnArgs &a, const KvSeq &s, int seq, int slot, int head,
                                         const int32_t *list, int64_t first, int64_t to, int waves)
    {
        const int lane = threadIdx.x & 63;
        const int64_t tile = first + (int64_t)(lane / EPT) * waves;
        const int64_t entry = (tile * 64 + lane % EPT * STEP) / B;
        blk = page = -1;
        k = v = 0.0f;
        if (tile < to) blk = !a.sel ? (int)entry : entry < a.n_sel ? list[entry] : -1;
        if (blk >= 0) page = kv_page(a.b, seq, blk);
        const bool full = (int64_t)blk * B + B <= s.len;
        if (page < 0 || (!full && slot < 0)) blk = -1;
        if (blk >= 0) {
            const float *sc = a.c.scales + ((int64_t)page * a.c.heads + head) * 2;
            k = sc[0];
            v = sc[1];
            if (!full) page = -1 - page;
        }
    }
};

__device__ __forceinline__ int from_lane(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ __forceinline__ float from_lane(float x, int lane)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

// One tile: groups of 16 tokens, NB blocks that hold GS groups each.
template <int B>
struct Tile {
    static constexpr int NB = Blocks<B>::EPT, GS = 4 / NB;
    int blk[NB], page[NB];
    float k[NB], v[NB];
    int off;      // of its first token within the block (B > 64)
    bool coded;   // every group lies in a complete block

    __device__ __forceinline__ void take(const Blocks<B> &b, int at, int64_t kt)
    {
        off = B > 64 ? (int)(kt & 1) * 64 : 0;
        coded = true;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            blk[i] = from_lane(b.blk, at * NB + i);
            page[i] = from_lane(b.page, at * NB + i);
            k[i] = from_lane(b.k, at * NB + i);
            v[i] = from_lane(b.v, at * NB + i);
            coded = coded && blk[i] >= 0 && page[i] >= 0;
        }
    }
    // place of the first token of group s
    __device__ __forceinline__ int64_t place(int s) const
    {
        return (int64_t)blk[s / GS] * B + off + s % GS * 16;
    }
};

// Codes of a tile as they come from memory, in the registers of one lane: of keys, the
// D/4 bytes of row r of each group that belong to lanes g; of values, of row 16 n + r
// of V^T the four bytes of each group that do.
template <int D, int B>
struct Codes {
    static constexpr int N = D / 16;
    uint32_t k[4][D / 16], v[N][4];

    __device__ __forceinline__ void load_keys(const KvAttnArgs &a, const Tile<B> &t, int head, int r, int g)
    {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int8_t *src = a.c.kc + ((int64_t)t.page[s / Tile<B>::GS] * a.c.heads + head) * (B * D) +
                                (t.off + s % Tile<B>::GS * 16) * D;
            const uint32_t at = r * D + g * (D / 4);
            if constexpr (D % 64 == 0) {
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    const u32x4 w = *reinterpret_cast<const u32x4 *>(src + 16 * i + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) k[s][4 * i + e] = w[e];
                }
            } else {
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const u32x2 w = *reinterpret_cast<const u32x2 *>(src + 8 * i + at);
                    k[s][2 * i] = w[0];
                    k[s][2 * i + 1] = w[1];
                }
            }
        }
    }

    __device__ __forceinline__ void load_values(const KvAttnArgs &a, const Tile<B> &t, int head, int r, int g)
    {
#pragma unroll
        for (int i = 0; i < Tile<B>::NB; ++i) {
            const int8_t *src = a.c.vc + ((int64_t)t.page[i] * a.c.heads + head) * (B * D) + t.off / 4;
            const uint32_t at = r * B + g * (B / 4);
#pragma unroll
            for (int n = 0; n < N; ++n, src += 16 * B) {
                if constexpr (B == 16) {
                    v[n][i] = *reinterpret_cast<const uint32_t *>(src + at);
                } else if constexpr (B == 32) {
                    const u32x2 w = *reinterpret_cast<const u32x2 *>(src + at);
                    v[n][2 * i] = w[0];
                    v[n][2 * i + 1] = w[1];
                } else {
                    const u32x4 w = *reinterpret_cast<const u32x4 *>(src + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[n][e] = w[e];
                }
            }
        }
    }
};

// Keys of group s of a tile that is not coded throughout, times the queries; fk becomes
// the factor of the scores.
template <int D, int B>
__device__ __forceinline__ f32x4 scores_of_group(const KvAttnArgs &a, const Tile<B> &t, int s, int slot, int head,
                                                 int64_t len, int r, int g, const f16x8 *qh, const f16x8 *ql, float fq,
                                                 float &fk)
{
    f32x4 st = {0.0f, 0.0f, 0.0f, 0.0f};
    const int i = s / Tile<B>::GS, off = t.off + s % Tile<B>::GS * 16;
    fk = 0.0f;
    if (t.blk[i] < 0) return st;
    if (t.page[i] >= 0) {
        const int8_t *src = a.c.kc + ((int64_t)t.page[i] * a.c.heads + head) * (B * D) + (off + r) * D + g * (D / 4);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            const u32x2 w = *reinterpret_cast<const u32x2 *>(src + 8 * k);
            const f16x8 c = codes8(w[0], w[1]);
            st = mfma16(c, qh[k], st);
            st = mfma16(c, ql[k], st);
        }
        fk = t.k[i] * (1.0f / 127.0f) * fq;
        return st;
    }
    // FP32 rows; what lies behind the last one may be anything
    const float *src = a.c.kr + ((int64_t)slot * a.c.heads + head) * (2 * B * D) + ((t.blk[i] & 1) * B + off + r) * D + g * (D / 4);
    const bool there = t.place(s) + r < len;
    const int e = exponent(t.k[i]), shift = e == kNoScale ? 0 : 14 - e;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
            const f32x4 y = *reinterpret_cast<const f32x4 *>(src + 8 * k + j);
#pragma unroll
            for (int b = 0; b < 4; ++b) x[j + b] = there ? ldexpf(y[b], shift) : 0.0f;
        }
        f16x8 hi, lo;
        pairs8(x, hi, lo);
        st = mfma16(hi, qh[k], st);
        st = mfma16(hi, ql[k], st);
        st = mfma16(lo, qh[k], st);
    }
    fk = ldexpf(fq, -shift);
    return st;
}

// The lane's four values of group s in row 16 n + r of V^T as FP16 pairs.
template <int D, int B>
__device__ __forceinline__ void values_of_group(const KvAttnArgs &a, const Tile<B> &t, int s, int n, int slot, int head,
                                                int64_t len, int r, int g, f16x2 &h0, f16x2 &h1, f16x2 &l0, f16x2 &l1)
{
    const int i = s / Tile<B>::GS, off = t.off + s % Tile<B>::GS * 16;
    h0 = h1 = l0 = l1 = f16x2{(_Float16)0.0f, (_Float16)0.0f};
    if (t.blk[i] < 0) return;
    if (t.page[i] >= 0) {
        const int8_t *src = a.c.vc + ((int64_t)t.page[i] * a.c.heads + head) * (B * D) + (16 * n + r) * B + g * (B / 4) + off / 4;
        codes4(*reinterpret_cast<const uint32_t *>(src), h0, h1);
        return;
    }
    const float *src = a.c.vr + ((int64_t)slot * a.c.heads + head) * (2 * B * D) + (int64_t)(16 * n + r) * (2 * B) + (t.blk[i] & 1) * B + off + 4 * g;
    const int e = exponent(t.v[i]), shift = e == kNoScale ? 0 : 7 - e;
    const int64_t rows = len - t.place(s);
    const f32x4 y = *reinterpret_cast<const f32x4 *>(src);
    float x[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) x[b] = 4 * g + b < rows ? ldexpf(y[b], shift) : 0.0f;
    h0 = __builtin_convertvector((f32x2{x[0], x[1]}), f16x2);
    h1 = __builtin_convertvector((f32x2{x[2], x[3]}), f16x2);
    l0 = __builtin_convertvector((f32x2{x[0] - (float)h0[0], x[1] - (float)h0[1]}), f16x2);
    l1 = __builtin_convertvector((f32x2{x[2] - (float)h1[0], x[3] - (float)h1[1]}), f16x2);
}

// Attention of 16 rows by the four waves of a workgroup, each on 64-token tiles of
// its own: keys and values go from memory to registers and the matrix units without
// LDS, and the waves' results are joined at the end.  The next tile's keys are asked
// for as soon as this one's are in the matrix units, its values likewise, so that a
// wave has 16 KiB on the way while it computes.
template <int D, int B>
__global__ void __launch_bounds__(256, 2)
kv_attention_kernel(KvAttnArgs a, bool by_token, int64_t wg0)
{
    constexpr int KC = D / 32, N = D / 16, W = 4;
    using T = Tile<B>;
    __shared__ float part_o[W][16][D + 4];
    __shared__ float part_m[W][16], part_l[W][16];
    __shared__ int part_row[16], part_head[16];
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int64_t wg = wg0 + blockIdx.x;
    const int part = (int)(wg % a.parts);
    const int head = (int)(wg / a.parts % a.c.heads);
    Rows t;
    if (!find_rows<16>(a, by_token, wg / a.parts / a.c.heads, head, r, t)) return;

    // tiles of this part: of the places from the tile of the first one seen, or of
    // the listed blocks
    const int64_t listed = a.sel ? (int64_t)uniform(t.token) * a.c.heads + head : 0;
    const int32_t *list = a.sel + listed * a.n_sel;
    const int64_t base = a.sel ? 0 : t.first / 64;
    const int64_t end = a.sel ? ((int64_t)a.n_sel * B + 63) / 64 : t.last < t.first ? 0 : (int64_t)t.last / 64 + 1;
    const int64_t from = base + (int64_t)part * a.part_tiles;
    const int64_t to = from + a.part_tiles < end ? from + a.part_tiles : end;
    const int slot = uniform(kv_slot(a.b, t.seq));

    f32x4 o[N];
#pragma unroll
    for (int n = 0; n < N; ++n) o[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -__builtin_inff(), l = 0.0f;
    int ref = kNoScale;   // this row's o is in units of 2^(ref - 14) / 127

    if (from + wave < to && t.last >= t.first) {
        Blocks<B> blocks;
        blocks.load(a, t.s, t.seq, slot, head, list, from + wave, to, W);
        T cur;
        Codes<D, B> codes;
        cur.take(blocks, 0, from + wave);
        if (cur.coded) {
            codes.load_keys(a, cur, head, r, g);
            codes.load_values(a, cur, head, r, g);
        }
        // the query row: lane (r, g) holds elements g D/4 .. of row r
        f16x8 qh[KC], ql[KC];
        float fq;
        {
            float x[D / 4];
            const float *src = a.q + (int64_t)(t.token < 0 ? 0 : t.token) * a.q_token + t.head_q * a.q_head + g * (D / 4);
            float big = 0.0f;
#pragma unroll
            for (int i = 0; i < D / 4; i += 4) {
                const float4 v = t.token < 0 ? float4{0.0f, 0.0f, 0.0f, 0.0f} : load16(src + i, a.vec);
                x[i] = v.x;
                x[i + 1] = v.y;
                x[i + 2] = v.z;
                x[i + 3] = v.w;
            }
#pragma unroll
            for (int i = 0; i < D / 4; ++i) big = __builtin_fmaxf(big, __builtin_fabsf(x[i]));
            const int e = exponent(max_over_groups(big));
            const int shift = e == kNoScale ? 0 : 14 - e;
#pragma unroll
            for (int i = 0; i < D / 4; ++i) x[i] = ldexpf(x[i], shift);
#pragma unroll
            for (int k = 0; k < KC; ++k) pairs8(x + 8 * k, qh[k], ql[k]);
            fq = ldexpf(a.scale * kLog2e, -shift);
        }

        int at = 0;
        for (int64_t kt = from + wave; kt < to; kt += W) {
            T next = cur;
            const bool more = kt + W < to;
            if (more) {
                if (++at == Blocks<B>::TILES) {
                    at = 0;
                    blocks.load(a, t.s, t.seq, slot, head, list, kt + W, to, W);
                }
                next.take(blocks, at, kt + W);
            }
            const bool ask = more && next.coded;

            // scores
            f32x4 st[4];
            float fk[4];
            if (cur.coded) {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    st[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = 0; k < KC; ++k) {
                        const f16x8 c = codes8(codes.k[s][2 * k], codes.k[s][2 * k + 1]);
                        st[s] = mfma16(c, qh[k], st[s]);
                        st[s] = mfma16(c, ql[k], st[s]);
                    }
                    if (s & 1) __builtin_amdgcn_sched_barrier(0);   // (two groups' keys as FP16 at a time)
                    fk[s] = cur.k[s / T::GS] * (1.0f / 127.0f) * fq;
                }
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    st[s] = scores_of_group<D, B>(a, cur, s, slot, head, t.s.len, r, g, qh, ql, fq, fk[s]);
                    __builtin_amdgcn_sched_barrier(0);   // (rows of one group at a time in registers)
                }
            }
            if (ask) codes.load_keys(a, next, head, r, g);

            // in log2 units, and without what a row does not see
            float big = -__builtin_inff(), vm[T::NB];
            int ev = kNoScale;
            bool all = cur.coded;
#pragma unroll
            for (int i = 0; i < T::NB; ++i) {
                const int64_t p0 = cur.place(i * T::GS);
                all = all && p0 >= t.all_lo && p0 + T::GS * 16 - 1 <= t.all_hi;
                vm[i] = cur.v[i];
            }
            if (all) {
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        st[s][i] *= fk[s];
                        big = __builtin_fmaxf(big, st[s][i]);
                    }
            } else {
#pragma unroll
                for (int i = 0; i < T::NB; ++i) {
                    // (a row's units follow the blocks that it sees something of, and no others)
                    const int64_t p0 = cur.place(i * T::GS);
                    if (cur.blk[i] < 0 || p0 > t.hi || p0 + T::GS * 16 - 1 < t.lo) vm[i] = 0.0f;
                }
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int64_t p0 = cur.place(s) + 4 * g;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool seen = cur.blk[s / T::GS] >= 0 && p0 + i >= t.lo && p0 + i <= t.hi;
                        st[s][i] = seen ? st[s][i] * fk[s] : -__builtin_inff();
                        big = __builtin_fmaxf(big, st[s][i]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < T::NB; ++i) ev = max(ev, exponent(vm[i]));
            const float mn = __builtin_fmaxf(m, max_over_groups(big));
            const float mz = mn == -__builtin_inff() ? 0.0f : mn;
            const float alpha = __builtin_amdgcn_exp2f(m - mz);
            const int rn = max(ref, ev);
            // (before the first scale that is not 0, o is 0)
            const float turn = ref == kNoScale ? alpha : ldexpf(alpha, ref - rn);
            m = mn;
            ref = rn;
            if (__ballot(turn != 1.0f)) {
#pragma unroll
                for (int n = 0; n < N; ++n) o[n] *= turn;
            }
            float wv[T::NB];   // the factor of a weight for the values of a block
#pragma unroll
            for (int i = 0; i < T::NB; ++i) {
                const int e = exponent(vm[i]);
                wv[i] = cur.page[i] >= 0 ? ldexpf(vm[i], 14 - rn) : e == kNoScale ? 0.0f : ldexpf(127.0f, e + 7 - rn);
            }
            float sum = 0.0f;
            f16x8 ph[2], pl[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int s = 2 * c + i / 4;
                    const float e = __builtin_amdgcn_exp2f(st[s][i % 4] - mz);
                    sum += e;
                    p[i] = e * wv[s / T::GS];
                }
                pairs8(p, ph[c], pl[c]);
            }
            l = l * alpha + sum;

            // values
            if (cur.coded) {
#pragma unroll
                for (int n = 0; n < N; ++n) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const f16x8 v = codes8(codes.v[n][2 * c], codes.v[n][2 * c + 1]);
                        o[n] = mfma16(v, ph[c], o[n]);
                        o[n] = mfma16(v, pl[c], o[n]);
                    }
                    if (n & 1) __builtin_amdgcn_sched_barrier(0);
                }
            } else {
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        f16x2 h[4], x[4];
                        values_of_group<D, B>(a, cur, 2 * c, n, slot, head, t.s.len, r, g, h[0], h[1], x[0], x[1]);
                        values_of_group<D, B>(a, cur, 2 * c + 1, n, slot, head, t.s.len, r, g, h[2], h[3], x[2], x[3]);
                        const f16x8 vh = {h[0][0], h[0][1], h[1][0], h[1][1], h[2][0], h[2][1], h[3][0], h[3][1]};
                        const f16x8 vl = {x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
                        o[n] = mfma16(vh, ph[c], o[n]);
                        o[n] = mfma16(vh, pl[c], o[n]);
                        o[n] = mfma16(vl, ph[c], o[n]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
            if (ask) codes.load_values(a, next, head, r, g);
            cur = next;
        }
    }

    // join the waves
    l = sum_over_groups(l);
    const float unit = ref == kNoScale ? 0.0f : ldexpf(1.0f / 127.0f, ref - 14);
#pragma unroll
    for (int n = 0; n < N; ++n) *reinterpret_cast<f32x4 *>(&part_o[wave][r][16 * n + 4 * g]) = o[n] * unit;
    if (g == 0) {
        part_m[wave][r] = m;
        part_l[wave][r] = l;
        part_row[r] = t.token < 0 ? -1 : t.token;
        part_head[r] = t.head_q;
    }
    __syncthreads();
    const int rr = threadIdx.x >> 4, c0 = threadIdx.x & 15;
    const int64_t token = part_row[rr];
    if (token < 0) return;
    float top = -__builtin_inff(), total = 0.0f, w[W];
#pragma unroll
    for (int i = 0; i < W; ++i) top = __builtin_fmaxf(top, part_m[i][rr]);
    const float tz = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        w[i] = __builtin_amdgcn_exp2f(part_m[i][rr] - tz);
        total += w[i] * part_l[i][rr];
    }
    const int64_t row = token * a.c.heads * a.group + part_head[rr];
    const int64_t rows = (int64_t)a.b.tokens * a.c.heads * a.group;
    float *ml = a.ws_ml + ((int64_t)part * rows + row) * 2;
    if (a.parts > 1 && c0 == 0) {
        ml[0] = top;
        ml[1] = total;
    }
    if (a.parts > 1 && total == 0.0f) return;
    float *dst = a.parts > 1 ? a.ws_o + ((int64_t)part * rows + row) * D
                             : a.out + token * a.out_token + part_head[rr] * a.out_head;
    const bool vec = a.parts > 1 || a.vec;
    for (int c = 4 * c0; c < D; c += 64) {
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < W; ++i) x += *reinterpret_cast<const f32x4 *>(&part_o[i][rr][c]) * w[i];
        if (a.parts == 1) x = total == 0.0f ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : x / total;
        store4(dst + c, x, vec);
    }
    if (a.parts == 1 && a.lse && c0 == 0) a.lse[row] = log_sum(top, total);
}

// The parts of a row joined in ascending order, one wave to a row.  A lane holds the
// maximum and the sum of one part, and eight parts' results are asked for at once.
template <int D>
__global__ void __launch_bounds__(256)
kv_combine_kernel(KvAttnArgs a, int64_t wg0)
{
    constexpr int J = (D + 63) / 64, U = 8;
    const int lane = threadIdx.x & 63;
    const int64_t rows = (int64_t)a.b.tokens * a.c.heads * a.group;
    const int64_t row = (wg0 + blockIdx.x) * 4 + uniform(threadIdx.x >> 6);
    if (row >= rows) return;
    const int64_t token = row / (a.c.heads * a.group), head_q = row % (a.c.heads * a.group);
    if (a.b.cu && (token < kv_first(a.b, 0) || token >= kv_first(a.b, a.b.seqs))) return;
    float top = -__builtin_inff();
    for (int p = lane; p < a.parts; p += 64) top = __builtin_fmaxf(top, a.ws_ml[((int64_t)p * rows + row) * 2]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, off));
    const float tz = top == -__builtin_inff() ? 0.0f : top;
    float total = 0.0f, x[J] = {};
    for (int p0 = 0; p0 < a.parts; p0 += 64) {
        float w = 0.0f, l = 0.0f;
        if (p0 + lane < a.parts) {
            const f32x2 ml = *reinterpret_cast<const f32x2 *>(a.ws_ml + ((int64_t)(p0 + lane) * rows + row) * 2);
            w = __builtin_amdgcn_exp2f(ml[0] - tz);
            l = ml[1];
        }
        uint64_t left = __ballot(l != 0.0f);   // (a sum that is no number is one too)
        while (left) {
            int at[U];
            float y[U][J];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                at[u] = left ? __builtin_ctzll(left) : -1;
                left &= left - 1;
#pragma unroll
                for (int j = 0; j < J; ++j)
                    y[u][j] = at[u] >= 0 && j * 64 + lane < D
                                  ? a.ws_o[((int64_t)(p0 + at[u]) * rows + row) * D + j * 64 + lane]
                                  : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (at[u] < 0) continue;
                const float wu = from_lane(w, at[u]);
                total += wu * from_lane(l, at[u]);
#pragma unroll
                for (int j = 0; j < J; ++j) x[j] += wu * y[u][j];
            }
        }
    }
    float *dst = a.out + token * a.out_token + head_q * a.out_head;
#pragma unroll
    for (int j = 0; j < J; ++j)
        if (j * 64 + lane < D) dst[j * 64 + lane] = total == 0.0f ? 0.0f : x[j] / total;
    if (a.lse && lane == 0) a.lse[row] = log_sum(top, total);
}

template <int D, int B>
hipError_t attention_sized(KvAttnArgs &a, const KvPlan &plan, hipStream_t stream)
{
    const int64_t n = plan.tiles * a.c.heads * plan.parts;
    hipError_t err = in_parts(n, [&](int64_t at, unsigned m) {
        hipLaunchKernelGGL((kv_attention_kernel<D, B>), dim3(m), dim3(256), 0, stream, a, plan.by_token, at);
    });
    if (err != hipSuccess || plan.parts == 1) return err;
    const int64_t rows = (int64_t)a.b.tokens * a.c.heads * a.group;
    return in_parts((rows + 3) / 4, [&](int64_t at, unsigned m) {
        hipLaunchKernelGGL((kv_combine_kernel<D>), dim3(m), dim3(256), 0, stream, a, at);
    });
}

}  // namespace

KvPlan kv_plan(int64_t tokens, int64_t seqs, bool ragged, int heads, int group, int dim, int block,
               int64_t cols, int64_t window, int64_t n_sel, int64_t chunk)
{
    KvPlan p = {};
    p.by_token = n_sel > 0 || !ragged;
    p.tiles = p.by_token ? tokens * ((group + 15) / 16) : kv_tiles(tokens, seqs, group, 16);
    // 64-token tiles that a row tile can have to read (its rows' windows begin at up to 16 places)
    int64_t places = n_sel > 0 ? n_sel * block : cols * block;
    if (n_sel == 0 && window > 0 && window + 16 + 63 < places) places = window + 16 + 63;
    const int64_t span = (places + 63) / 64 > 0 ? (places + 63) / 64 : 1;
    int64_t part_tiles;
    if (chunk > 0) {
        part_tiles = chunk / 64;
    } else {
        // enough workgroups to fill the chip, each with a tile for every wave at least
        const int64_t wanted = (kWantedWorkgroups + p.tiles * heads - 1) / (p.tiles * heads > 0 ? p.tiles * heads : 1);
        int64_t parts = wanted < (span + 3) / 4 ? wanted : (span + 3) / 4;
        parts = parts < 1 ? 1 : parts > 64 ? 64 : parts;
        part_tiles = ((span + parts - 1) / parts + 3) / 4 * 4;
    }
    if (part_tiles > span) part_tiles = span;
    p.part_tiles = (int32_t)part_tiles;
    p.parts = (int32_t)((span + part_tiles - 1) / part_tiles);
    const double rows = (double)tokens * heads * group;
    p.bytes = p.parts == 1 ? 0 : rows * p.parts > 0x1p44 ? -1 : tokens * heads * group * p.parts * (dim + 2) * 4;
    return p;
}

hipError_t launch_kv_attention(KvAttnArgs &a, const KvPlan &plan, hipStream_t stream)
{
    a.parts = plan.parts;
    a.part_tiles = plan.part_tiles;
    return sized(a.c.dim, a.c.block,
                 [&](auto D, auto B) { return attention_sized<D.value, B.value>(a, plan, stream); });
}

}  // namespace heal
