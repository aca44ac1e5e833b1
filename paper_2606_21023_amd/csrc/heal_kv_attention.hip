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
// the cache is scaled by a power of two of its own, from its largest finite element,
// and split too (2^-22 of an element, and 2^-25 of 2^14 for keys and of 2^7 for values);
// the product of the two residuals is left out (2^-22 of 2^-11).  What a query does not
// see has the weight 0, so a value that is not finite is taken as 0 in the products and
// put into the columns of the rows that see it behind them.
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

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// Lambdas that are inlined at once: what they take by reference stays in registers.
#define HEAL_INLINE __attribute__((always_inline))

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Two workgroups of either kernel fit on a compute unit.  Parts are cut until there are
// as many (a decode step of 64 sequences 157 us; 162 with 768 or 1024, 188 with 2048; 48
// of 512 blocks of 32 sequences 54, 67, 70 and 85).
constexpr int64_t kWantedWorkgroups = 512;
// Up to so many sequences the tiles of a ragged call are counted one after another.
constexpr int64_t kCountedSeqs = 256;
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

// e with |x| in [2^(e-1), 2^e), or kNoScale for 0 (and for what is not finite: a block's
// codes times such a maximum are no numbers with any scale, nor is a row with such a key).
__device__ __forceinline__ int exponent(float x)
{
    if (!(__builtin_fabsf(x) > 0.0f) || __builtin_isinf(x)) return kNoScale;
    return __builtin_amdgcn_frexp_expf(x);
}

// A value that all lanes have.  Matrix instructions take no notice of lanes that are
// switched off, so every branch around them has to be one of the whole wave, and what
// it depends on has to be known as such.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// x, as a value that the compiler knows nothing of: what is computed from it on a path
// that is seldom taken is computed there, and not before the loop, where its results
// would take registers from the path that is.
__device__ __forceinline__ int hidden(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

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

// (without LDS: of a swap with itself one result has the lower half of the wave, or of each
// half, twice, and the other one the upper)
__device__ __forceinline__ int max_over_groups(int x)
{
    const auto h = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
    x = max((int)h[0], (int)h[1]);
    const auto q = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
    return max((int)q[0], (int)q[1]);
}

// The largest x of a lane's group of 16.
__device__ __forceinline__ uint32_t max_in_group(uint32_t x)
{
    // (row_ror: the 16 lanes turned by 8, 4, 2 and 1)
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x124, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x122, 0xf, 0xf, true));
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x121, 0xf, 0xf, true));
}

constexpr uint32_t kInfinity = 0x7f800000u;
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

__device__ __forceinline__ float sum_over_groups(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

__device__ __forceinline__ f32x4 load4(const float *p, bool vec)
{
    if (vec) return *reinterpret_cast<const f32x4 *>(p);
    return f32x4{p[0], p[1], p[2], p[3]};
}

// A row tile: R rows (token, query of the head) of one sequence.
struct Rows {
    KvSeq s;
    int32_t seq, row0, rows;   // row0: of the sequence's rows; how many the tile has
};

// Finds the rows of tile u.  Returns false where the tile has none.
template <int R>
__device__ __forceinline__ bool find_rows(const KvAttnArgs &a, bool by_token, int64_t u, Rows &t)
{
    if (by_token) {
        const int per = (a.group + R - 1) / R;
        const int64_t token = u / per;
        t.seq = uniform(a.b.cu ? kv_last_at_most(a.b.seqs, token, [&](int i) { return (int64_t)kv_first(a.b, i); })
                               : (int)token);
        t.s = uniform_seq(a.b, t.seq);
        if (token < t.s.first || token >= (int64_t)t.s.first + t.s.n) return false;
        t.row0 = (int)(u % per) * R;
        t.rows = a.group - t.row0 < R ? a.group - t.row0 : R;
        t.row0 += (int)(token - t.s.first) * a.group;
    } else {
        int64_t j;
        if (a.b.seqs <= kCountedSeqs) {
            // The tiles of each sequence are counted, so that those of the grid that are nobody's
            // come last.  Where they lie between the others, they can take every second
            // place in the order in which workgroups are dealt out, and half of the compute
            // units get nothing else (32 sequences of 128 rows over 2048 tokens: 155 us, 99 so).
            const int lane = threadIdx.x & 63;
            int64_t before = 0;
            t.seq = -1;
            for (int i0 = 0; i0 < a.b.seqs; i0 += 64) {
                const int first = i0 + lane < a.b.seqs ? kv_first(a.b, i0 + lane) : 0;
                const int next = i0 + lane < a.b.seqs ? kv_first(a.b, i0 + lane + 1) : 0;
                const int64_t own = next > first ? ((int64_t)(next - first) * a.group + R - 1) / R : 0;
                int64_t sum = own;
#pragma unroll
                for (int off = 1; off < 64; off <<= 1) {
                    const int64_t x = __shfl_up(sum, off);
                    sum += lane >= off ? x : 0;
                }
                const uint64_t past = __ballot(before + sum > u);
                if (past) {
                    const int at = __builtin_ctzll(past);
                    t.seq = uniform(i0 + at);
                    j = u - before - (__shfl(sum, at) - __shfl(own, at));
                    break;
                }
                before += __shfl(sum, 63);
            }
            if (t.seq < 0) return false;
            t.s = uniform_seq(a.b, t.seq);
        } else {
            t.seq = uniform(kv_last_at_most(a.b.seqs, u, [&](int i) { return kv_tile(a.b, a.group, R, i); }));
            t.s = uniform_seq(a.b, t.seq);
            j = u - kv_tile(a.b, a.group, R, t.seq);
        }
        j = (int64_t)uniform((int)j);
        const int64_t n = (int64_t)t.s.n * a.group;
        if (j < 0 || j * R >= n) return false;
        t.row0 = (int)(j * R);
        t.rows = n - t.row0 < R ? (int)(n - t.row0) : R;
    }
    return true;
}

// The places lo .. hi that a row of the sequence sees (none where hi < lo).
__device__ __forceinline__ void row_sees(const KvAttnArgs &a, const KvSeq &s, int row, int32_t &lo, int32_t &hi)
{
    const int64_t end = (int64_t)a.b.cols * a.c.block;   // places that the table has
    const int64_t place = (int64_t)s.len - s.n + row / a.group;
    int64_t h = a.causal ? place : s.len - 1, l = a.window > 0 ? place - a.window + 1 : 0;
    if (place < 0) h = -1;
    if (h >= s.len) h = s.len - 1;
    if (h >= end) h = end - 1;
    lo = (int32_t)(l < 0 ? 0 : l);
    hi = (int32_t)h;
}

// ... that one or another of rows row0 .. row0 + rows - 1 sees, and that all of them see.
struct Span {
    int32_t first, last, all_lo, all_hi;
};
__device__ __forceinline__ Span rows_see(const KvAttnArgs &a, const KvSeq &s, int row0, int rows)
{
    Span x;
    row_sees(a, s, row0, x.first, x.all_hi);
    row_sees(a, s, row0 + rows - 1, x.all_lo, x.last);
    return Span{uniform(x.first), uniform(x.last), uniform(x.all_lo), uniform(x.all_hi)};
}

// A query row, of which the lane takes the D/4 elements from g D/4 on, as FP16 pairs of
// the row scaled by a power of two; its scores' factor (log2 units, not negative: the
// scale's sign goes to the row).  Rows that are not there (src null) are zeros.
template <int D>
__device__ __forceinline__ float load_query(const KvAttnArgs &a, const float *src, f16x8 *qh, f16x8 *ql)
{
    float x[D / 4], big = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 4; i += 4) {
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (src) v = load4(src + i, a.vec);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i + e] = a.scale < 0.0f ? -v[e] : v[e];
    }
#pragma unroll
    for (int i = 0; i < D / 4; ++i) big = __builtin_fmaxf(big, __builtin_fabsf(x[i]));
    const int e = exponent(max_over_groups(big));
    const int shift = e == kNoScale ? 0 : 14 - e;
#pragma unroll
    for (int i = 0; i < D / 4; ++i) x[i] = ldexpf(x[i], shift);
#pragma unroll
    for (int k = 0; k < D / 32; ++k) pairs8(x + 8 * k, qh[k], ql[k]);
    return ldexpf(__builtin_fabsf(a.scale) * kLog2e, -shift);
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

// The blocks of a wave's next tiles, one to a lane: a tile of 64 tokens has EPT of
// them, so the lanes hold the blocks and scales of TILES tiles, which are read in two
// round trips to memory for all of them together.
template <int B>
struct Blocks {
    static constexpr int EPT = B < 64 ? 64 / B : 1, TILES = 64 / EPT, STEP = B < 64 ? B : 64;
    int blk;     // block of the sequence, or -1 where the cache holds nothing of it
    int page;    // its page (0 where there is none), or -1 - page where it is read from the ring
    float k, v;  // m of its keys and values (a block that is not complete goes by its rows)

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
        if (page < 0 || (!full && (slot < 0 || (int64_t)blk * B >= s.len))) {
            blk = -1;
            page = 0;   // (its codes may be read: their weights are zeros)
        }
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
    // (vectors, of which NB elements are used: arrays would end up in memory)
    i32x4 blk, page;
    f32x4 k, v;
    int off;      // of its first token within the block (B > 64)
    bool coded;   // no group is read from the ring

    // member by member: a copy of the whole struct takes its padding along, in memory
    Tile() = default;
    __device__ __forceinline__ Tile(const Tile &t) { *this = t; }
    __device__ __forceinline__ Tile &operator=(const Tile &t)
    {
        blk = t.blk;
        page = t.page;
        k = t.k;
        v = t.v;
        off = t.off;
        coded = t.coded;
        return *this;
    }

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
            coded = coded && page[i] >= 0;
        }
    }
    // the factor of the scores with coded block i, but for the query's (0 where there is none)
    __device__ __forceinline__ float key_factor(int i) const { return k[i] * (1.0f / 127.0f); }
    // place of the first token of group s
    __device__ __forceinline__ int32_t place(int s) const
    {
        return blk[s / GS] * B + off + s % GS * 16;
    }
};

// One group of 16 tokens of a tile that is not coded throughout.
struct Group {
    int blk, page;   // as in Blocks
    float k, v;
    int off;         // of its first token within the block
    int32_t place;   // of its first token

    __device__ __forceinline__ bool coded() const { return blk < 0 || page >= 0; }
};
template <int B>
__device__ __forceinline__ Group group_of(const Tile<B> &t, int s)
{
    const int i = s / Tile<B>::GS;
    return Group{t.blk[i], t.page[i], t.k[i], t.v[i], t.off + s % Tile<B>::GS * 16, t.place(s)};
}
// ... of the first of the tiles that a wave's lanes hold the blocks of; s need not be a
// constant.
template <int B>
__device__ __forceinline__ Group group_of(const Blocks<B> &b, int64_t kt, int s)
{
    const int i = s / Tile<B>::GS, off = (B > 64 ? (int)(kt & 1) * 64 : 0) + s % Tile<B>::GS * 16;
    const int blk = from_lane(b.blk, i);
    return Group{blk, from_lane(b.page, i), from_lane(b.k, i), from_lane(b.v, i), off, blk * B + off};
}

// Codes as they come from memory, in the registers of one lane: of the keys of group
// s, the D/4 bytes of row r that belong to lanes g; of row 16 n + r of V^T, the four
// bytes of each group that do.  (The block's address is the wave's, the lane's part an
// unsigned 32-bit offset, hidden so that the two are not added outside the loop: no
// 64-bit address per lane.)  ONCE: they pass the caches by.
template <bool ONCE, class X>
__device__ __forceinline__ X load_codes(const int8_t *p)
{
    const X *x = reinterpret_cast<const X *>(p);
    return ONCE ? __builtin_nontemporal_load(x) : *x;
}

template <int D, int B, bool ONCE>
__device__ __forceinline__ void load_group_keys(const KvAttnArgs &a, const Tile<B> &t, int s, int head, int r, int g,
                                                uint32_t *k)
{
    const int8_t *src = a.c.kc + ((int64_t)t.page[s / Tile<B>::GS] * a.c.heads + head) * (B * D) + (t.off + s % Tile<B>::GS * 16) * D;
    const uint32_t at = hidden(r * D + g * (D / 4));
    if constexpr (D % 64 == 0) {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const u32x4 w = load_codes<ONCE, u32x4>(src + 16 * i + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) k[4 * i + e] = w[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const u32x2 w = load_codes<ONCE, u32x2>(src + 8 * i + at);
            k[2 * i] = w[0];
            k[2 * i + 1] = w[1];
        }
    }
}

template <int D, int B, bool ONCE>
__device__ __forceinline__ void load_column_values(const KvAttnArgs &a, const Tile<B> &t, int n, int head, int r, int g,
                                                   uint32_t *v)
{
    const uint32_t at = hidden(r * B + g * (B / 4));
#pragma unroll
    for (int i = 0; i < Tile<B>::NB; ++i) {
        const int8_t *src = a.c.vc + ((int64_t)t.page[i] * a.c.heads + head) * (B * D) + t.off / 4 + n * (16 * B);
        if constexpr (B == 16) {
            v[i] = load_codes<ONCE, uint32_t>(src + at);
        } else if constexpr (B == 32) {
            const u32x2 w = load_codes<ONCE, u32x2>(src + at);
            v[2 * i] = w[0];
            v[2 * i + 1] = w[1];
        } else {
            const u32x4 w = load_codes<ONCE, u32x4>(src + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = w[e];
        }
    }
}

// The codes of a whole tile.
template <int D, int B, bool ONCE>
struct Codes {
    static constexpr int N = D / 16;
    uint32_t k[4][D / 16], v[N][4];

    __device__ __forceinline__ void load_keys(const KvAttnArgs &a, const Tile<B> &t, int head, int r, int g)
    {
#pragma unroll
        for (int s = 0; s < 4; ++s) load_group_keys<D, B, ONCE>(a, t, s, head, r, g, k[s]);
    }
    __device__ __forceinline__ void load_values(const KvAttnArgs &a, const Tile<B> &t, int head, int r, int g)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) load_column_values<D, B, ONCE>(a, t, n, head, r, g, v[n]);
    }
};

// Keys of a group, as FP16 pairs: f(k, hi, lo) for each chunk of 32 elements.  Returns the
// factor of the scores with token r, but for the query's.
template <int D, int B, class F>
__device__ __forceinline__ float keys_of_group(const KvAttnArgs &a, const Group &t, int slot, int head,
                                               int64_t len, int r, int g, F f)
{
    const f16x8 zero = {};
    const int blk = t.blk, page = t.page, off = t.off;
    if (blk < 0) {
#pragma unroll
        for (int k = 0; k < D / 32; ++k) f(k, zero, zero);
        return 0.0f;
    }
    if (page >= 0) {
        const int8_t *src = a.c.kc + ((int64_t)page * a.c.heads + head) * (B * D) + (off + r) * D + g * (D / 4);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            const u32x2 w = *reinterpret_cast<const u32x2 *>(src + 8 * k);
            f(k, codes8(w[0], w[1]), zero);
        }
        return t.k * (1.0f / 127.0f);
    }
    // FP32 rows; what lies behind the last one may be anything
    const float *src = a.c.kr + ((int64_t)slot * a.c.heads + head) * (2 * B * D) + ((blk & 1) * B + off + r) * D + g * (D / 4);
    const bool there = (int64_t)t.place + r < len;
    float x[D / 4];
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < D / 4; i += 4) {
        const f32x4 y = *reinterpret_cast<const f32x4 *>(src + i);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            x[i + b] = there ? y[b] : 0.0f;
            top = max(top, magnitude(x[i + b]));
        }
    }
    // (a key that is not finite: every score with it is no number)
    const int e = exponent(__builtin_bit_cast(float, max_over_groups((int)top))), shift = e == kNoScale ? 0 : 14 - e;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
        f16x8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[8 * k + j] = ldexpf(x[8 * k + j], shift);
        pairs8(x + 8 * k, hi, lo);
        f(k, hi, lo);
    }
    return ldexpf(1.0f, -shift);
}

// The lane's four values of a group in row 16 n + r of V^T: codes, or FP32 rows, as they
// are.
template <int D, int B>
__device__ __forceinline__ f32x4 values_of_group(const KvAttnArgs &a, const Group &t, int n, int slot, int head,
                                                 int64_t len, int r, int g)
{
    const int blk = t.blk, page = t.page, off = t.off;
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    if (blk < 0) return x;
    if (page >= 0) {
        const int8_t *src = a.c.vc + ((int64_t)page * a.c.heads + head) * (B * D) + (16 * n + r) * B + g * (B / 4) + off / 4;
        const uint32_t w = *reinterpret_cast<const uint32_t *>(src);
#pragma unroll
        for (int b = 0; b < 4; ++b) x[b] = (float)(int8_t)(w >> (8 * b));
        return x;
    }
    const float *src = a.c.vr + ((int64_t)slot * a.c.heads + head) * (2 * B * D) + (int64_t)(16 * n + r) * (2 * B) + (blk & 1) * B + off + 4 * g;
    const int64_t rows = len - t.place;
    const f32x4 y = *reinterpret_cast<const f32x4 *>(src);
#pragma unroll
    for (int b = 0; b < 4; ++b) x[b] = 4 * g + b < rows ? y[b] : 0.0f;
    return x;
}

// 0 for what is not finite.
__device__ __forceinline__ f32x4 finite(f32x4 x)
{
#pragma unroll
    for (int b = 0; b < 4; ++b) x[b] = magnitude(x[b]) < kInfinity ? x[b] : 0.0f;
    return x;
}

// The exponents of the lane's four tokens of a group, values(n) being its values in row
// 16 n + r of V^T: of an FP32 row that of its largest finite value, of a coded block that
// of its maximum.  odd: there is a value that is not finite (the wave's).
template <int N, class F>
__device__ __forceinline__ i32x4 value_exponents(const Group &t, F values, bool &odd)
{
    odd = false;
    const int eb = exponent(t.v);
    if (t.coded()) return i32x4{eb, eb, eb, eb};
    uint32_t top[4] = {};
    auto add = [&](f32x4 x) HEAL_INLINE {
#pragma unroll
        for (int b = 0; b < 4; ++b) top[b] = max(top[b], magnitude(x[b]));
    };
#pragma unroll
    for (int n = 0; n < N; ++n) add(values(n));
    odd = __ballot(max(max(top[0], top[1]), max(top[2], top[3])) >= kInfinity) != 0;
    if (__builtin_expect(odd, false)) {
        for (int b = 0; b < 4; ++b) top[b] = 0u;
#pragma unroll
        for (int n = 0; n < N; ++n) add(finite(values(n)));
    }
    i32x4 e;
#pragma unroll
    for (int b = 0; b < 4; ++b) e[b] = exponent(__builtin_bit_cast(float, max_in_group(top[b])));
    return e;
}

// Finite values as the products take them: codes as they are, FP32 rows scaled by their
// powers of two.
__device__ __forceinline__ f32x4 scaled_values(const Group &t, f32x4 x, i32x4 e)
{
    if (t.coded()) return x;
#pragma unroll
    for (int b = 0; b < 4; ++b) x[b] = ldexpf(x[b], 7 - e[b]);
    return x;
}

// 1 where a value is not finite, else 0.
__device__ __forceinline__ f32x4 odd_values(f32x4 x)
{
#pragma unroll
    for (int b = 0; b < 4; ++b) x[b] = magnitude(x[b]) < kInfinity ? 0.0f : 1.0f;
    return x;
}

__device__ __forceinline__ f16x8 to_f16(f32x4 a, f32x4 b)
{
    f16x8 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = (_Float16)a[i];
        x[4 + i] = (_Float16)b[i];
    }
    return x;
}

// No number where x counts anything.
__device__ __forceinline__ void spoil(f32x4 &o, f32x4 x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = x[i] > 0.0f ? __builtin_nanf("") : o[i];
}

// Where a row's result goes: its place in out, or in the workspace of its part.
struct Place {
    int64_t row;   // of lse
    float *dst, *ml;

    // maximum and sum
    __device__ __forceinline__ void sums(const KvAttnArgs &a, float m, float l) const
    {
        if (a.parts > 1) {
            ml[0] = m;
            ml[1] = l;
        } else if (a.lse) {
            a.lse[row] = log_sum(m, l);
        }
    }
    // columns c .. c + 3, to be divided by the sum l at the end
    __device__ __forceinline__ void store(const KvAttnArgs &a, int c, f32x4 x, float l) const
    {
        if (a.parts == 1) x = l == 0.0f ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : x / l;
        store4(dst + c, x, a.parts > 1 || a.vec);
    }
};

__device__ __forceinline__ Place place_of(const KvAttnArgs &a, int64_t token, int head_q, int part)
{
    const int64_t heads = (int64_t)a.c.heads * a.group, rows = a.b.tokens * heads;
    Place p;
    p.row = token * heads + head_q;
    const int64_t at = part * rows + p.row;
    p.ml = a.ws_ml + at * 2;
    p.dst = a.parts > 1 ? a.ws_o + at * a.c.dim : a.out + token * a.out_token + head_q * a.out_head;
    return p;
}

// One row's running softmax: the maximum of its scores (log2 units), the lane's part of
// the sum of exp2(score - m), and the units of its output, 2^(ref - 14) / 127.
struct Soft {
    float m, l;
    int ref;
};

// The scores of a tile whose blocks are all coded become weights.  st: the lane's scores, of
// tokens 4 g + i of group s, before their factors fk (one for each block).  Returns the
// weights times the blocks' value factors as FP16 pairs, in the order of the values'
// operand, and what the output so far is to be multiplied by.
template <int B>
__device__ __forceinline__ float soften(const Tile<B> &t, f32x4 *st, const float *fk, bool all, const int32_t *row_lo,
                                        const int32_t *row_hi, int g, Soft &w, f16x8 *ph, f16x8 *pl)
{
    using T = Tile<B>;
    float f[T::NB], vm[T::NB];
#pragma unroll
    for (int i = 0; i < T::NB; ++i) {
        f[i] = fk[i];
        vm[i] = t.v[i];
    }
    if (__builtin_expect(!all, false)) {
        const int32_t lo = *row_lo, hi = *row_hi;
#pragma unroll
        for (int i = 0; i < T::NB; ++i) {
            // (a row's units follow the blocks that it sees something of, and no others)
            const int32_t p0 = t.place(i * T::GS);
            const bool met = t.blk[i] >= 0 && p0 <= hi && p0 + (T::GS * 16 - 1) >= lo;
            vm[i] = met ? t.v[i] : 0.0f;
            f[i] = 1.0f;
            // what the row sees, counted from the lane's first token of the block
            const int32_t from = lo - p0 - 4 * g, to = met ? hi - p0 - 4 * g : -1;
#pragma unroll
            for (int s = i * T::GS; s < (i + 1) * T::GS; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = (s - i * T::GS) * 16 + e;
                    st[s][e] = at >= from && at <= to ? st[s][e] * fk[i] : -__builtin_inff();
                }
        }
    }
    float big = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < T::NB; ++i) {
        float top = -__builtin_inff();
#pragma unroll
        for (int s = i * T::GS; s < (i + 1) * T::GS; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = __builtin_fmaxf(top, st[s][e]);
        big = __builtin_fmaxf(big, top * f[i]);
    }
    int ev = kNoScale;
#pragma unroll
    for (int i = 0; i < T::NB; ++i) ev = max(ev, exponent(vm[i]));
    const float mn = __builtin_fmaxf(w.m, max_over_groups(big));
    const float mz = mn == -__builtin_inff() ? 0.0f : mn;
    const float alpha = __builtin_amdgcn_exp2f(w.m - mz);
    const int rn = max(w.ref, ev);
    // (before the first scale that is not 0, the output is 0)
    const float turn = w.ref == kNoScale ? alpha : ldexpf(alpha, w.ref - rn);
    float wv[T::NB];
#pragma unroll
    for (int i = 0; i < T::NB; ++i) {
        wv[i] = ldexpf(vm[i], 14 - rn);
    }
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int s = 2 * c + e / 4;
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(st[s][e % 4], f[s / T::GS], -mz));
            sum += x;
            p[e] = x * wv[s / T::GS];
        }
        pairs8(p, ph[c], pl[c]);
    }
    w.m = mn;
    w.l = w.l * alpha + sum;
    w.ref = rn;
    return turn;
}

// Whether the row that sees lo .. hi sees each of the lane's four tokens of a group.
__device__ __forceinline__ void sees_tokens(const Group &t, int32_t lo, int32_t hi, int g, bool *is)
{
    const int32_t p0 = t.place + 4 * g;
#pragma unroll
    for (int e = 0; e < 4; ++e) is[e] = t.blk >= 0 && p0 + e >= lo && p0 + e <= hi;
}

// ... as 1 and 0.
__device__ __forceinline__ f32x4 seen_tokens(const Group &t, int32_t lo, int32_t hi, int g)
{
    bool is[4];
    sees_tokens(t, lo, hi, g, is);
    f32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = is[e] ? 1.0f : 0.0f;
    return x;
}

// As soften, of a tile that may hold FP32 rows: N groups, factors(s) and exponents(s) being the
// factors and the values' exponents of the lane's tokens of group s; the tokens that the row
// sees make its units.  Leaves the weights in st.
template <int N, class F, class E>
__device__ __forceinline__ float soften_tokens(const Group *t, f32x4 *st, F factors, E exponents, int32_t lo,
                                               int32_t hi, int g, Soft &w)
{
    float big = -__builtin_inff(), vm[N];
    int ev = kNoScale;
#pragma unroll
    for (int s = 0; s < N; ++s) {
        const bool met = t[s].blk >= 0 && t[s].place <= hi && t[s].place + 15 >= lo;
        vm[s] = met ? t[s].v : 0.0f;
        if (t[s].coded()) ev = max(ev, exponent(vm[s]));
        const f32x4 fk = factors(s);
        const i32x4 ve = exponents(s);
        bool is[4];
        sees_tokens(t[s], lo, hi, g, is);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            st[s][e] = is[e] ? st[s][e] * fk[e] : -__builtin_inff();
            big = __builtin_fmaxf(big, st[s][e]);
            ev = is[e] && !t[s].coded() ? max(ev, ve[e]) : ev;
        }
    }
    const float mn = __builtin_fmaxf(w.m, max_over_groups(big));
    const float mz = mn == -__builtin_inff() ? 0.0f : mn;
    const float alpha = __builtin_amdgcn_exp2f(w.m - mz);
    const int rn = max(w.ref, max_over_groups(ev));
    const float turn = w.ref == kNoScale ? alpha : ldexpf(alpha, w.ref - rn);
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < N; ++s) {
        const i32x4 ve = exponents(s);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = __builtin_amdgcn_exp2f(st[s][e] - mz);
            sum += x;
            // (a row that is not seen may be larger than rn stands for: its x is 0)
            const float wv = t[s].coded() ? ldexpf(vm[s], 14 - rn) : ldexpf(127.0f, min(ve[e] - rn, 0) + 7);
            st[s][e] = x * wv;
        }
    }
    w.m = mn;
    w.l = w.l * alpha + sum;
    w.ref = rn;
    return turn;
}

// Four columns of a finished output out of its units.  (In two steps: the units of values
// below 2^-105 would be an FP32 number below 2^-126, which has few digits, or 0.)
__device__ __forceinline__ f32x4 from_units(f32x4 o, int ref)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = ldexpf(o[i] * (1.0f / 127.0f), ref - 14);
    return o;
}

// Attention of 16 rows by the four waves of a workgroup, each on 64-token tiles of
// its own: keys and values go from memory to registers and the matrix units without
// LDS, and the waves' results are joined at the end.  The next tile's keys are asked
// for as soon as this one's are in the matrix units, its values likewise, so that a
// wave has 16 KiB on the way while it computes.  Bound by memory where a sequence has
// one token (64 of 4096 to 8192 tokens, 8 heads of 128: 150 us, 816 MB, 5.4 TB/s), by
// latency where there is little to read (8191 tokens of one sequence 13 us).
template <int D, int B, bool ONCE>
__global__ void __launch_bounds__(256, 2)
kv_attention_kernel(KvAttnArgs a, bool by_token, int64_t wg0)
{
    constexpr int KC = D / 32, N = D / 16, W = 4;
    using T = Tile<B>;
    __shared__ float part_o[W][16][D + 4];
    __shared__ float part_m[W][16], part_l[W][16];
    // (every wave writes what it reads of these, the same values: registers are full)
    __shared__ int part_row[16], part_head[16];
    __shared__ int32_t row_lo[16], row_hi[16];
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int64_t wg = wg0 + blockIdx.x;
    const int part = (int)(wg % a.parts);
    const int head = (int)(wg / a.parts % a.c.heads);
    Rows t;
    if (!find_rows<16>(a, by_token, wg / a.parts / a.c.heads, t)) return;
    const Span span = rows_see(a, t.s, t.row0, t.rows);
    // this lane's row
    const int row = t.row0 + r;
    const int64_t token = r < t.rows ? t.s.first + row / a.group : -1;
    const int head_q = head * a.group + row % a.group;
    {
        int32_t lo = 0, hi = -1;
        if (r < t.rows) row_sees(a, t.s, row, lo, hi);
        row_lo[r] = lo;
        row_hi[r] = hi;
        part_row[r] = (int)token;
        part_head[r] = head_q;
    }

    // tiles of this part: of the places from the tile of the first one seen, or of
    // the listed blocks
    const int64_t listed = a.sel ? (int64_t)(t.s.first + t.row0 / a.group) * a.c.heads + head : 0;
    const int32_t *list = a.sel + listed * a.n_sel;
    const int64_t base = a.sel ? 0 : span.first / 64;
    const int64_t end = a.sel ? ((int64_t)a.n_sel * B + 63) / 64 : (int64_t)span.last / 64 + 1;
    const int64_t from = base + (int64_t)part * a.part_tiles;
    const int64_t to = from + a.part_tiles < end ? from + a.part_tiles : end;
    const int slot = uniform(kv_slot(a.b, t.seq));

    f32x4 o[N];
#pragma unroll
    for (int n = 0; n < N; ++n) o[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    Soft w = {-__builtin_inff(), 0.0f, kNoScale};

    if (from + wave < to && span.last >= span.first) {
        Blocks<B> blocks;
        blocks.load(a, t.s, t.seq, slot, head, list, from + wave, to, W);
        T cur;
        Codes<D, B, ONCE> codes;
        cur.take(blocks, 0, from + wave);
        if (cur.coded) {
            codes.load_keys(a, cur, head, r, g);
            codes.load_values(a, cur, head, r, g);
        }
        f16x8 qh[KC], ql[KC];
        const float fq = load_query<D>(a, token < 0 ? nullptr : a.q + token * a.q_token + head_q * a.q_head + g * (D / 4), qh, ql);

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

            if (cur.coded) {
                f32x4 st[4];
                float fk[T::NB];
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
                }
#pragma unroll
                for (int i = 0; i < T::NB; ++i) fk[i] = cur.key_factor(i) * fq;
                if (ask) codes.load_keys(a, next, head, r, g);

                bool all = true;
#pragma unroll
                for (int i = 0; i < T::NB; ++i)
                    all = all && cur.place(i * T::GS) >= span.all_lo && cur.place(i * T::GS) + T::GS * 16 - 1 <= span.all_hi;
                f16x8 ph[2], pl[2];
                const float turn = soften<B>(cur, st, fk, all, row_lo + r, row_hi + r, g, w, ph, pl);
                if (__ballot(turn != 1.0f)) {
#pragma unroll
                    for (int n = 0; n < N; ++n) o[n] *= turn;
                }
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
                if (ask) codes.load_values(a, next, head, r, g);
            } else if (ask) {
                codes.load_keys(a, next, head, r, g);
                codes.load_values(a, next, head, r, g);
            }
            cur = next;
        }
    }

    // Tiles with FP32 rows, a group of 16 tokens to each wave: all that a wave needs of
    // one is asked for at once, where one wave with the whole tile would have four times
    // the bytes of a coded tile to wait for (8191 tokens of one sequence: 17.7 us, 12.5 so).
    auto ring_tile = [&](int64_t kt) HEAL_INLINE {
        Blocks<B> blocks;
        blocks.load(a, t.s, t.seq, slot, head, list, kt, to, 1);
        const Group own = group_of(blocks, kt, wave);
        if (Blocks<B>::EPT == 1 ? own.coded() : own.blk < 0 || !__ballot(lane < Blocks<B>::EPT && blocks.page < 0))
            return;   // the loop has done it, or there is nothing
        f16x8 qh[KC], ql[KC], kh[KC], kl[KC];
        f32x4 v[N];
        const float fq = load_query<D>(a, token < 0 ? nullptr : a.q + token * a.q_token + head_q * a.q_head + g * (D / 4), qh, ql);
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = values_of_group<D, B>(a, own, n, slot, head, t.s.len, r, g);
        const float fr = keys_of_group<D, B>(a, own, slot, head, t.s.len, r, g, [&](int k, f16x8 h, f16x8 x) {
            kh[k] = h;
            kl[k] = x;
        });
        // (the lane has the scores of tokens 4 g + i, and lane r the factor of token r)
        f32x4 st = {0.0f, 0.0f, 0.0f, 0.0f}, fk;
#pragma unroll
        for (int e = 0; e < 4; ++e) fk[e] = __shfl(fr, 4 * g + e);
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            st = mfma16(kh[k], qh[k], st);
            st = mfma16(kh[k], ql[k], st);
            st = mfma16(kl[k], qh[k], st);
        }
        fk *= fq;
        bool odd;
        const i32x4 ve = value_exponents<N>(own, [&](int n) { return v[n]; }, odd);
        if (__builtin_expect(odd, false)) {
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] = finite(v[n]);
        }
        const float turn = soften_tokens<1>(
            &own, &st, [&](int) { return fk; }, [&](int) { return ve; }, row_lo[r], row_hi[r], g, w);
        f16x8 ph, pl;
        const float p[8] = {st[0], st[1], st[2], st[3]};   // (the other half of the operand is zeros)
        pairs8(p, ph, pl);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const f32x4 y = scaled_values(own, v[n], ve);
            const float x[8] = {y[0], y[1], y[2], y[3]};
            f16x8 vh, vl;
            pairs8(x, vh, vl);
            o[n] *= turn;
            o[n] = mfma16(vh, ph, o[n]);
            o[n] = mfma16(vh, pl, o[n]);
            o[n] = mfma16(vl, ph, o[n]);
        }
        if (__builtin_expect(odd, false)) {   // (the wave's)
            const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
            const int r2 = hidden(r), g2 = hidden(g);
            const f16x8 seen = to_f16(seen_tokens(own, row_lo[r2], row_hi[r2], g2), none);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const f32x4 y = values_of_group<D, B>(a, own, n, slot, head, t.s.len, r2, g2);
                spoil(o[n], mfma16(to_f16(odd_values(y), none), seen, none));
            }
        }
    };
    if (t.s.len % B != 0 && span.last >= span.first) {
        if (!a.sel) {
            for (int64_t x = kv_ring_first(t.s.len, B); x < kv_ring_end(t.s.len, B); ++x)
                if (x >= from && x < to) ring_tile(x);
        } else {
            const int32_t rb = t.s.len / B;   // the block that is not complete
            // wherever the lists have it, 64 entries at a time
            constexpr int E = B < 64 ? 64 / B : 1, P = B > 64 ? B / 64 : 1;   // entries of a tile, tiles of an entry
            for (int64_t e0 = from * E / P; e0 * P < to * E; e0 += 64) {
                const int64_t e = e0 + lane;
                uint64_t found = __ballot(e < a.n_sel && e * P < to * E && list[e] == rb);
                while (found) {
                    const int64_t at = e0 + __builtin_ctzll(found);
                    const int64_t kt = at * P / E;
                    for (int64_t x = kt; x < kt + P; ++x)
                        if (x >= from && x < to) ring_tile(x);
                    // (the other entries of that tile are done with it)
                    found &= found - 1;
                    while (found && (e0 + __builtin_ctzll(found)) * P / E == kt && P == 1) found &= found - 1;
                }
            }
        }
    }

    // join the waves
    const float sum = sum_over_groups(w.l);
#pragma unroll
    for (int n = 0; n < N; ++n) *reinterpret_cast<f32x4 *>(&part_o[wave][r][16 * n + 4 * g]) = from_units(o[n], w.ref);
    if (g == 0) {
        part_m[wave][r] = w.m;
        part_l[wave][r] = sum;
    }
    __syncthreads();
    const int rr = threadIdx.x >> 4, c0 = threadIdx.x & 15;
    const int64_t to_token = part_row[rr];
    if (to_token < 0) return;
    float top = -__builtin_inff(), total = 0.0f, share[W];
#pragma unroll
    for (int i = 0; i < W; ++i) top = __builtin_fmaxf(top, part_m[i][rr]);
    const float tz = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        share[i] = __builtin_amdgcn_exp2f(part_m[i][rr] - tz);
        total += share[i] * part_l[i][rr];
    }
    const Place to_row = place_of(a, to_token, part_head[rr], part);
    if (c0 == 0) to_row.sums(a, top, total);
    if (a.parts > 1 && total == 0.0f) return;
    for (int c = 4 * c0; c < D; c += 64) {
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < W; ++i) x += *reinterpret_cast<const f32x4 *>(&part_o[i][rr][c]) * share[i];
        to_row.store(a, c, x, total);
    }
}

// Attention of 128 rows by a workgroup whose four waves have 32 rows each, for
// prompts: keys and values are converted to FP16 once for all rows, a tile ahead, and
// wait in LDS in the order of the matrix operands (lane by lane, no bank conflicts).
// A key fragment feeds four matrix instructions (two groups of 16 rows, two parts of
// the pair) and a value fragment likewise.  Bound by instruction issue: the matrix
// units are busy 44% of the time, the vector units (exponentials, pairs, masks) 50%
// (512 tokens of 32 heads over 16001: 264 GFLOP of FP16 products in 253 us, 1.04 PFLOP/s).
template <int D, int B>
__global__ void __launch_bounds__(256, 2)
kv_prompt_kernel(KvAttnArgs a, int64_t tiles, int64_t wg0)
{
    constexpr int KC = D / 32, N = D / 16, Q = 2, R = 128, NW = (N + 3) / 4;
    using T = Tile<B>;
    // fragments of 64 lanes x 16 bytes: keys of group s and chunk k at s KC + k, values of
    // column tile n and token half c at 4 KC + 2 n + c
    __shared__ f16x8 frag[2][4 * KC + 2 * N][64];
    // what a row needs once a tile, or seldom: kept out of the registers, which are full
    __shared__ float row_factor[R];
    __shared__ int32_t row_lo[R], row_hi[R];
    // of a tile with FP32 rows: each token's factor of the scores and exponent of its values,
    // and whether a wave met a value that is not finite
    __shared__ float token_factor[64];
    __shared__ int32_t token_exponent[64], odd[4];
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int64_t wg = wg0 + blockIdx.x;
    // heads side by side, so that with eight of them each XCD has its own head's keys in
    // L2; the last rows of a sequence, which see most, first
    const int head = (int)(wg % a.c.heads);
    const int part = (int)(wg / a.c.heads % a.parts);
    Rows t;
    if (!find_rows<R>(a, false, tiles - 1 - wg / a.c.heads / a.parts, t)) return;
    const Span span = rows_see(a, t.s, t.row0, t.rows);
    const int slot = uniform(kv_slot(a.b, t.seq));
    const int64_t base = span.first / 64, end = (int64_t)span.last / 64 + 1;
    const int64_t from = base + (int64_t)part * a.part_tiles;
    const int64_t to = from + a.part_tiles < end ? from + a.part_tiles : end;

    // this wave's rows, and this lane's two
    const int mine = t.rows - 32 * wave < 32 ? t.rows - 32 * wave : 32;   // (none: <= 0)
    const Span wspan = mine > 0 ? rows_see(a, t.s, t.row0 + 32 * wave, mine) : Span{0, -1, 0, -1};
    f16x8 qh[Q][KC], ql[Q][KC];
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        const int at = 32 * wave + 16 * i + r, row = t.row0 + at;
        const bool is = at < t.rows;
        const int64_t token = t.s.first + row / a.group, head_q = head * a.group + row % a.group;
        int32_t lo = 0, hi = -1;
        if (is) row_sees(a, t.s, row, lo, hi);
        const float fq = load_query<D>(a, is ? a.q + token * a.q_token + head_q * a.q_head + g * (D / 4) : nullptr, qh[i], ql[i]);
        if (g == 0) {   // (read by this wave only)
            row_factor[at] = fq;
            row_lo[at] = lo;
            row_hi[at] = hi;
        }
    }
    f32x4 o[Q][N];
    Soft w[Q];
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        w[i] = Soft{-__builtin_inff(), 0.0f, kNoScale};
#pragma unroll
        for (int n = 0; n < N; ++n) o[i][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    if (from < to && span.last >= span.first) {
        // staging: wave w takes the keys of group w and the values of column tiles w, w + 4
        uint32_t ks[D / 16], vs[NW][4];
        auto ask = [&](const T &x) HEAL_INLINE {
            load_group_keys<D, B, false>(a, x, wave, head, r, g, ks);
#pragma unroll
            for (int j = 0; j < NW; ++j)
                if (N % 4 == 0 || wave + 4 * j < N) load_column_values<D, B, false>(a, x, wave + 4 * j, head, r, g, vs[j]);
        };
        auto keep = [&](int b) HEAL_INLINE {
#pragma unroll
            for (int k = 0; k < KC; ++k) frag[b][wave * KC + k][lane] = codes8(ks[2 * k], ks[2 * k + 1]);
#pragma unroll
            for (int j = 0; j < NW; ++j)
                if (N % 4 == 0 || wave + 4 * j < N) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        frag[b][4 * KC + 2 * (wave + 4 * j) + c][lane] = codes8(vs[j][2 * c], vs[j][2 * c + 1]);
                }
        };
        // a tile with FP32 rows (or without some of its blocks): both parts of the pairs
        auto keep_pairs = [&](const T &x, int b) HEAL_INLINE {
            const int r2 = hidden(r), g2 = hidden(g);
            const Group own = group_of(x, wave);
            const float fr = keys_of_group<D, B>(a, own, slot, head, t.s.len, r2, g2, [&](int k, f16x8 h, f16x8 l) {
                frag[b][wave * KC + k][lane] = h;
                frag[b ^ 1][wave * KC + k][lane] = l;
            });
            bool bad;
            const i32x4 ve = value_exponents<N>(
                own, [&](int n) { return values_of_group<D, B>(a, own, n, slot, head, t.s.len, r2, g2); }, bad);
            if (g == 0) token_factor[16 * wave + r] = fr;
            if (r == 0) *reinterpret_cast<i32x4 *>(&token_exponent[16 * wave + 4 * g]) = ve;
            if (lane == 0) odd[wave] = bad;
            __syncthreads();
            const bool any = uniform(odd[0] | odd[1] | odd[2] | odd[3]);
#pragma unroll 1
            for (int n = wave; n < N; n += 4)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float y[8];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const i32x4 e = *reinterpret_cast<const i32x4 *>(&token_exponent[16 * (2 * c + j) + 4 * g2]);
                        const Group of = group_of(x, 2 * c + j);
                        f32x4 v = values_of_group<D, B>(a, of, n, slot, head, t.s.len, r2, g2);
                        if (any) v = finite(v);
                        v = scaled_values(of, v, e);
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[4 * j + i] = v[i];
                    }
                    f16x8 h, l;
                    pairs8(y, h, l);
                    frag[b][4 * KC + 2 * n + c][lane] = h;
                    frag[b ^ 1][4 * KC + 2 * n + c][lane] = l;
                }
        };
        // ... and 1 for each value that is not finite, in place of the values
        auto keep_odd = [&](const T &x, int b) HEAL_INLINE {
            const int r2 = hidden(r), g2 = hidden(g);
#pragma unroll 1
            for (int n = wave; n < N; n += 4)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    frag[b][4 * KC + 2 * n + c][lane] =
                        to_f16(odd_values(values_of_group<D, B>(a, group_of(x, 2 * c), n, slot, head, t.s.len, r2, g2)),
                               odd_values(values_of_group<D, B>(a, group_of(x, 2 * c + 1), n, slot, head, t.s.len, r2, g2)));
        };

        // the tiles of the ring's block, the last ones, come after the loop
        const int64_t ring = kv_ring_first(t.s.len, B), coded_to = ring < to ? (ring > from ? ring : from) : to;
        Blocks<B> blocks;
        T cur;
        int buf = 0, at = 0;
        // the tile in LDS; residuals: with FP32 rows, whose residuals the other buffer has
        auto compute = [&](auto residuals) HEAL_INLINE {
            constexpr bool X = decltype(residuals)::value;
            // fragments are read from LDS three steps (of four matrix instructions) ahead, or one
            // where residuals take the registers
            const f16x8(*hi)[64] = frag[buf], (*res)[64] = frag[buf ^ 1];
            constexpr int A = X ? 1 : 3;
            f32x4 st[Q][4];
            f16x8 f[A + 1];
#pragma unroll
            for (int u = 0; u < A; ++u) f[u] = hi[u][lane];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
#pragma unroll
                for (int i = 0; i < Q; ++i) st[i][s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < KC; ++k) {
                    const int u = s * KC + k;
                    if (u + A < 4 * KC) f[(u + A) % (A + 1)] = hi[u + A][lane];
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < Q; ++i) st[i][s] = mfma16(f[u % (A + 1)], qh[i][k], st[i][s]);
#pragma unroll
                    for (int i = 0; i < Q; ++i) st[i][s] = mfma16(f[u % (A + 1)], ql[i][k], st[i][s]);
                    if (X) {
                        const f16x8 d = res[u][lane];
#pragma unroll
                        for (int i = 0; i < Q; ++i) st[i][s] = mfma16(d, qh[i][k], st[i][s]);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < A; ++u) f[u] = hi[4 * KC + u][lane];
            bool all = true;
#pragma unroll
            for (int i = 0; i < T::NB; ++i)
                all = all && cur.place(i * T::GS) >= wspan.all_lo && cur.place(i * T::GS) + T::GS * 16 - 1 <= wspan.all_hi;
            f16x8 ph[Q][2], pl[Q][2];
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                const int at = 32 * wave + 16 * i + r;
                const float fq = row_factor[at];
                float turn;
                if constexpr (X) {
                    const Group of[4] = {group_of(cur, 0), group_of(cur, 1), group_of(cur, 2), group_of(cur, 3)};
                    // (read from LDS when they are needed, twice: registers are full)
                    auto factors = [&](int s) HEAL_INLINE {
                        return *reinterpret_cast<const f32x4 *>(&token_factor[16 * s + hidden(4 * g)]) * fq;
                    };
                    auto exponents = [&](int s) HEAL_INLINE {
                        return *reinterpret_cast<const i32x4 *>(&token_exponent[16 * s + hidden(4 * g)]);
                    };
                    turn = soften_tokens<4>(of, st[i], factors, exponents, row_lo[at], row_hi[at], g, w[i]);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float p[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) p[e] = st[i][2 * c + e / 4][e % 4];
                        pairs8(p, ph[i][c], pl[i][c]);
                    }
                } else {
                    float fk[T::NB];
#pragma unroll
                    for (int b = 0; b < T::NB; ++b) fk[b] = cur.key_factor(b) * fq;
                    turn = soften<B>(cur, st[i], fk, all, row_lo + at, row_hi + at, g, w[i], ph[i], pl[i]);
                }
                if (__ballot(turn != 1.0f)) {
#pragma unroll
                    for (int n = 0; n < N; ++n) o[i][n] *= turn;
                }
            }
#pragma unroll
            for (int u = 0; u < 2 * N; ++u) {
                const int n = u / 2, c = u % 2;
                if (u + A < 2 * N) f[(u + A) % (A + 1)] = hi[4 * KC + u + A][lane];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < Q; ++i) o[i][n] = mfma16(f[u % (A + 1)], ph[i][c], o[i][n]);
#pragma unroll
                for (int i = 0; i < Q; ++i) o[i][n] = mfma16(f[u % (A + 1)], pl[i][c], o[i][n]);
                if (X) {
                    const f16x8 d = res[4 * KC + u][lane];
#pragma unroll
                    for (int i = 0; i < Q; ++i) o[i][n] = mfma16(d, ph[i][c], o[i][n]);
                }
            }
        };
        // (a wave whose rows see nothing of a tile only helps to stage it)
        auto sees = [&](int64_t kt) HEAL_INLINE { return kt * 64 <= wspan.last && kt * 64 + 63 >= wspan.first; };
        if (from < coded_to) {
            blocks.load(a, t.s, t.seq, slot, head, nullptr, from, coded_to, 1);
            cur.take(blocks, 0, from);
            ask(cur);
            keep(0);
            __syncthreads();
        }
        for (int64_t kt = from; kt < coded_to; ++kt) {
            T next = cur;
            const bool more = kt + 1 < coded_to;
            if (more) {
                if (++at == Blocks<B>::TILES) {
                    at = 0;
                    blocks.load(a, t.s, t.seq, slot, head, nullptr, kt + 1, coded_to, 1);
                }
                next.take(blocks, at, kt + 1);
                ask(next);
            }
            if (sees(kt)) compute(std::false_type());
            if (more) {
                keep(buf ^ 1);
                __syncthreads();
                buf ^= 1;
                cur = next;
            }
        }
#pragma unroll 1
        for (int64_t kt = coded_to; kt < to; ++kt) {
            __syncthreads();   // both buffers are written
            blocks.load(a, t.s, t.seq, slot, head, nullptr, kt, to, 1);
            cur.take(blocks, 0, kt);
            buf = 0;
            keep_pairs(cur, 0);
            __syncthreads();
            if (sees(kt)) compute(std::true_type());
            if (__builtin_expect(uniform(odd[0] | odd[1] | odd[2] | odd[3]), 0)) {   // (the workgroup's)
                __syncthreads();
                keep_odd(cur, 0);
                __syncthreads();
                if (sees(kt)) {
#pragma unroll
                    for (int i = 0; i < Q; ++i) {
                        const int at = 32 * wave + 16 * i + r;
                        f32x4 seen[4];
#pragma unroll
                        for (int s = 0; s < 4; ++s) seen[s] = seen_tokens(group_of(cur, s), row_lo[at], row_hi[at], g);
                        const f16x8 s0 = to_f16(seen[0], seen[1]), s1 = to_f16(seen[2], seen[3]);
#pragma unroll
                        for (int n = 0; n < N; ++n) {
                            const f32x4 x = mfma16(frag[0][4 * KC + 2 * n][lane], s0, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
                            spoil(o[i][n], mfma16(frag[0][4 * KC + 2 * n + 1][lane], s1, x));
                        }
                    }
                }
            }
        }
    }

#pragma unroll
    for (int i = 0; i < Q; ++i) {
        const float sum = sum_over_groups(w[i].l);
        const int at = 32 * wave + 16 * i + hidden(r), row = t.row0 + at;
        if (at >= t.rows) continue;
        const Place to_row = place_of(a, t.s.first + row / a.group, head * a.group + row % a.group, part);
        if (g == 0) to_row.sums(a, w[i].m, sum);
        if (a.parts > 1 && sum == 0.0f) continue;
#pragma unroll
        for (int n = 0; n < N; ++n) to_row.store(a, 16 * n + 4 * g, from_units(o[i][n], w[i].ref), sum);
    }
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
    // Loads pass the caches by where a sequence has one token, whose queries fit one row tile:
    // nobody else reads its blocks then, unless sequences share them (64 tokens over 4096 to
    // 8192: 141 us, 152 with ordinary loads; 32 tokens with lists of 48 of 500 blocks 49, 54;
    // with half of their 64 blocks shared by 64 sequences 78, 82, with 64 of 68 69, 66).  Not in
    // ragged calls with lists, where tokens of a sequence list the same blocks (777 tokens, 16 of
    // 79 blocks: 231 us so, 215 with ordinary loads; four drafts of 32 sequences, 48 of 500
    // blocks, the same for all four 109, 100, lists of their own 134, 133).
    hipError_t err = in_parts(n, [&](int64_t at, unsigned m) {
        if (plan.wide)
            hipLaunchKernelGGL((kv_prompt_kernel<D, B>), dim3(m), dim3(256), 0, stream, a, plan.tiles, at);
        else if (plan.by_token && !a.b.cu && a.group <= 16)
            hipLaunchKernelGGL((kv_attention_kernel<D, B, true>), dim3(m), dim3(256), 0, stream, a, true, at);
        else
            hipLaunchKernelGGL((kv_attention_kernel<D, B, false>), dim3(m), dim3(256), 0, stream, a, plan.by_token, at);
    });
    if (err != hipSuccess || plan.parts == 1) return err;
    const int64_t rows = (int64_t)a.b.tokens * a.c.heads * a.group;
    return in_parts((rows + 3) / 4, [&](int64_t at, unsigned m) {
        hipLaunchKernelGGL((kv_combine_kernel<D>), dim3(m), dim3(256), 0, stream, a, at);
    });
}

}  // namespace

namespace {

// Row tiles of a plan's kernel and the parts that each of them is cut into.
void cut(KvPlan &p, int64_t tokens, int64_t seqs, int heads, int group, int block, int64_t cols, int64_t window,
         int64_t n_sel, int64_t chunk)
{
    const int R = p.wide ? 128 : 16;
    p.tiles = p.by_token ? tokens * ((group + 15) / 16) : kv_tiles(tokens, seqs, group, R);
    // workgroups, if the sequences have equally many rows
    const int64_t each = seqs > 0 ? (tokens * group + seqs * R - 1) / (seqs * R) : 0;
    const int64_t real = p.by_token || seqs * each > p.tiles ? p.tiles : seqs * each;
    p.wgs = real * heads > 0 ? real * heads : 1;
    // 64-token tiles that a row tile can have to read (its rows' windows begin at up to R places).
    // Lengths are on the device: a table wider than they are leaves the last parts without
    // work (one token over 8191: 20 us with 128 columns, 45 with 2048)
    int64_t places = n_sel > 0 ? n_sel * block : cols * block;
    if (n_sel == 0 && window > 0 && window + R + 63 < places) places = window + R + 63;
    const int64_t span = (places + 63) / 64 > 0 ? (places + 63) / 64 : 1;
    int64_t part_tiles;
    if (chunk > 0) {
        part_tiles = chunk / 64;
    } else {
        // enough workgroups to fill the chip (of the prompts' kernel, whose workgroups take
        // equally long, no more than that), each with a tile for every wave at least
        const int64_t wanted = p.wide ? kWantedWorkgroups / p.wgs : (kWantedWorkgroups + p.wgs - 1) / p.wgs;
        int64_t parts = wanted < (span + 3) / 4 ? wanted : (span + 3) / 4;
        parts = parts < 1 ? 1 : parts > 64 ? 64 : parts;
        part_tiles = ((span + parts - 1) / parts + 3) / 4 * 4;
    }
    if (part_tiles > span) part_tiles = span;
    p.part_tiles = (int32_t)part_tiles;
    p.parts = (int32_t)((span + part_tiles - 1) / part_tiles);
}

// About how many us a plan takes: rounds of 512 workgroups, each with a fixed cost and a
// cost for each of its tiles (of the kernel for few rows: for each four), and what
// the parts' results cost.  Fitted to calls of 16 to 2048 rows of 1 to 32
// sequences over up to 8192 tokens, measured with both kernels: of 77 of them the
// faster one is found for 73, and the other four lose 11 to 29% (2048 rows of 32
// sequences over 2048 tokens: 927 us with 128-row tiles, 1807 with 16-row ones; 64 rows
// 83 and 72).
double estimate(const KvPlan &p, int64_t tokens, int heads, int group, int dim)
{
    const double rounds = (double)p.wgs * p.parts / (double)kWantedWorkgroups, d = dim / 128.0;
    const double one = p.wide ? 9.0 + p.part_tiles * (1.4 + 1.9 * d) : 6.0 + (p.part_tiles + 3) / 4 * (0.2 + 2.5 * d);
    const double join = p.parts > 1 ? 3.0 + (double)tokens * heads * group * p.parts * (dim + 2) * 2e-6 : 0.0;
    return (rounds > 1.0 ? rounds : 1.0) * one + join;
}

}  // namespace

KvPlan kv_plan(int64_t tokens, int64_t seqs, bool ragged, int heads, int group, int dim, int block,
               int64_t cols, int64_t window, int64_t n_sel, int64_t chunk)
{
    KvPlan p = {};
    p.by_token = n_sel > 0 || !ragged;
    // (a chunk of the caller's asks for sums that do not depend on the call's sizes)
    const bool either = !p.by_token && chunk == 0 && seqs > 0 && tokens > 0;
    p.wide = false;
    cut(p, tokens, seqs, heads, group, block, cols, window, n_sel, chunk);
    if (either) {
        KvPlan w = p;
        w.wide = true;
        cut(w, tokens, seqs, heads, group, block, cols, window, n_sel, chunk);
        if (estimate(w, tokens, heads, group, dim) < estimate(p, tokens, heads, group, dim)) p = w;
    }
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
