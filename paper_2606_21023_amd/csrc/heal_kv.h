// The key/value cache: what its kernels and the host share.  Everything that
// decides which row, block or workgroup a number belongs to is here, in functions
// that run on the host as well.
#pragma once

#include <stdint.h>

#include <type_traits>

#include <hip/hip_runtime.h>

namespace heal {

#define HEAL_HD __host__ __device__ __forceinline__

// Sequences of a call (heal_kv_batch_t).
struct KvSeqs {
    const int32_t *cu, *lens, *table, *slots;
    int64_t table_ld;
    int32_t seqs, tokens, cols;
    int32_t blocks, nslots;   // bounds of table and slots entries
};

// One sequence: tokens first .. first + n - 1 of the call, len tokens with them.
struct KvSeq {
    int32_t first, n, len;
};

HEAL_HD int32_t kv_clamp(int32_t x, int32_t lo, int32_t hi) { return x < lo ? lo : x > hi ? hi : x; }

HEAL_HD int32_t kv_first(const KvSeqs &b, int32_t i)
{
    return b.cu ? kv_clamp(b.cu[i], 0, b.tokens) : i;
}

HEAL_HD KvSeq kv_seq(const KvSeqs &b, int32_t i)
{
    KvSeq s;
    s.first = kv_first(b, i);
    s.n = b.cu ? kv_clamp(b.cu[i + 1], s.first, b.tokens) - s.first : 1;
    s.len = b.lens[i] > 0 ? b.lens[i] : 0;
    return s;
}

// The cache block of block blk of sequence i, or -1 where there is none.
HEAL_HD int32_t kv_page(const KvSeqs &b, int32_t i, int32_t blk)
{
    if (blk < 0 || blk >= b.cols) return -1;
    const int32_t p = b.table[(int64_t)i * b.table_ld + blk];
    return p >= 0 && p < b.blocks ? p : -1;
}

// The slot of sequence i, or -1.
HEAL_HD int32_t kv_slot(const KvSeqs &b, int32_t i)
{
    const int32_t s = b.slots ? b.slots[i] : i;
    return s >= 0 && s < b.nslots ? s : -1;
}

// Place of token t (0..B-1) among the values of a block.
HEAL_HD int kv_value_place(int B, int t) { return (t % 16) / 4 * (B / 4) + t / 16 * 4 + t % 4; }

// Work units of a call that touches blocks (append, read): sequence i owns units
// kv_unit(i) .. kv_unit(i + 1) - 1, one for each block that its n tokens can touch,
// floor((cu + n) / B) - floor(cu / B) + 2 >= floor(n / B) + 2 of them; with one
// token each a sequence has one.  Which sequence a unit belongs to is found from
// cu alone, so the grid follows from sizes that the host knows.
HEAL_HD int64_t kv_unit(const KvSeqs &b, int B, int32_t i)
{
    return b.cu ? kv_first(b, i) / B + 2 * (int64_t)i : i;
}

HEAL_HD int64_t kv_units(bool ragged, int64_t tokens, int64_t seqs, int B)
{
    return ragged ? tokens / B + 2 * seqs : seqs;
}

// Row tiles of R rows over the rows (token, query of the head) of each sequence,
// n * G of them: sequence i owns tiles kv_tile(i) and on, floor((cu + n) G / R) -
// floor(cu G / R) + 1 >= ceil(n G / R) of them.
HEAL_HD int64_t kv_tile(const KvSeqs &b, int G, int R, int32_t i)
{
    return (int64_t)kv_first(b, i) * G / R + i;
}

HEAL_HD int64_t kv_tiles(int64_t tokens, int64_t seqs, int G, int R) { return tokens * G / R + seqs; }

// The blocks of a sequence that `n` tokens at its end touch: first .. last (none
// where last < first).
struct KvTouched {
    int32_t start, first, last;   // place of the first token kept, block numbers
};

HEAL_HD KvTouched kv_touched(const KvSeq &s, int B)
{
    KvTouched t;
    t.start = s.len - s.n > 0 ? s.len - s.n : 0;
    t.first = t.start / B;
    t.last = s.n > 0 && s.len > 0 ? (s.len - 1) / B : t.first - 1;
    return t;
}

// The first 64-token tile of a sequence that has a block which is not complete, and the
// tile behind its last one (blocks of 128 tokens are two tiles, of which the second
// may have rows too); both behind every tile where the last block is complete.
HEAL_HD int64_t kv_ring_first(int32_t len, int B) { return len % B ? (int64_t)(len / B) * B / 64 : (int64_t)1 << 40; }
HEAL_HD int64_t kv_ring_end(int32_t len, int B) { return len % B ? ((int64_t)len - 1) / 64 + 1 : (int64_t)1 << 40; }

// Unit j of a sequence handles block first + j when it appends, except that the
// ring rows of a later block, which take the place of rows that unit 0 still has
// to read, are unit 0's too: the block of {last - 1, last} that lies an even
// number of blocks behind the first.  Returns that block, or -1.
HEAL_HD int32_t kv_ring_conflict(const KvTouched &t)
{
    const int32_t b = (t.last - t.first) % 2 == 0 ? t.last : t.last - 1;
    return b > t.first ? b : -1;
}

#ifdef __HIPCC__
// The largest i in [0, n) with f(i) <= u, for ascending f with f(0) <= u: 64 lanes
// look at 64 places at once, so a batch of 64 costs one load's latency and 4096 two.
template <class F>
__device__ __forceinline__ int kv_last_at_most(int n, int64_t u, F f)
{
    const int lane = threadIdx.x & 63;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) / 64;
        const int at = lane * step;
        const uint64_t below = __ballot(at < n && f(lo + at) <= u);
        int k = __popcll(below) - 1;
        k = k < 0 ? 0 : k;
        lo += k * step;
        n = n - k * step < step ? n - k * step : step;
    }
    return lo;
}
#endif

// ---- kernels -------------------------------------------------------------------

struct KvCache {
    int32_t heads, dim, block;
    int8_t *kc, *vc;
    float *scales, *mean, *kr, *vr;
};

struct KvAppendArgs {
    KvSeqs b;
    KvCache c;
    const float *k, *v;
    int64_t k_token, k_head, v_token, v_head;
    const float *cos, *sin;
    int64_t places;
    int32_t rot, interleaved;
    const float *q;
    float *q_out;
    int64_t q_token, q_head, qo_token, qo_head;
    int32_t heads_q;
};

struct KvSelectArgs {
    KvSeqs b;
    KvCache c;
    const float *q;
    int64_t q_token, q_head;
    int32_t group, n_sel, keep_first, keep_last;
    int32_t *sel;
};

struct KvAttnArgs {
    KvSeqs b;
    KvCache c;
    const float *q;
    int64_t q_token, q_head;
    float *out;
    int64_t out_token, out_head;
    float *lse;
    const int32_t *sel;
    int32_t n_sel, group;
    float scale;
    int32_t causal, window;
    int32_t parts, part_tiles;   // chunks of a row tile, 64-token tiles in each
    int32_t vec;                 // 16-byte rows of q and out
    float *ws_o, *ws_ml;         // parts x rows x dim, parts x rows x 2 (m in log2 units, l)
};

// Blocks of a sequence that heal_kv_select can score: 8 bytes of LDS each.
constexpr int64_t kMaxSelectBlocks = 16384;

// How a call of heal_kv_attention is cut (host only).
struct KvPlan {
    bool by_token;               // a row tile holds one token's queries
    bool wide;                   // 128-row tiles
    int64_t tiles;               // row tiles of the grid
    int64_t wgs;                 // workgroups for each part, about
    int32_t parts, part_tiles;
    int64_t bytes;               // of workspace
};
KvPlan kv_plan(int64_t tokens, int64_t seqs, bool ragged, int heads, int group, int dim, int block,
               int64_t cols, int64_t window, int64_t n_sel, int64_t chunk);

hipError_t launch_kv_append(const KvAppendArgs &a, hipStream_t stream);
hipError_t launch_kv_read(const KvSeqs &b, const KvCache &c, float *k, float *v, hipStream_t stream);
hipError_t launch_kv_select(const KvSelectArgs &a, hipStream_t stream);
hipError_t launch_kv_attention(KvAttnArgs &a, const KvPlan &plan, hipStream_t stream);

// A dispatch counts work-items in 32 bits: launches of at most 2^22 workgroups.
constexpr int64_t kMaxWorkgroups = (int64_t)1 << 22;

template <class F>
inline hipError_t in_parts(int64_t n, F launch)
{
    for (int64_t at = 0; at < n; at += kMaxWorkgroups) {
        launch(at, (unsigned)(n - at < kMaxWorkgroups ? n - at : kMaxWorkgroups));
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

// f of the constants dim and block.
template <class F>
inline hipError_t sized(int dim, int block, F f)
{
#define HEAL_KV_BLOCKS(D)                                                                             \
    switch (block) {                                                                                  \
    case 16: return f(std::integral_constant<int, D>(), std::integral_constant<int, 16>());           \
    case 32: return f(std::integral_constant<int, D>(), std::integral_constant<int, 32>());           \
    case 64: return f(std::integral_constant<int, D>(), std::integral_constant<int, 64>());           \
    case 128: return f(std::integral_constant<int, D>(), std::integral_constant<int, 128>());         \
    }                                                                                                 \
    break;
    switch (dim) {
    case 64: HEAL_KV_BLOCKS(64)
    case 96: HEAL_KV_BLOCKS(96)
    case 128: HEAL_KV_BLOCKS(128)
    }
#undef HEAL_KV_BLOCKS
    return hipErrorInvalidValue;
}

}  // namespace heal
