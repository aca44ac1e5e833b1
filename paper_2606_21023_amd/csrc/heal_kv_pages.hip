// The pages of a cache: which sequences hold which blocks (heal_kv_release, _fork, _reserve,
// _compact) and copies of blocks and slots (heal_kv_copy). Tables and counts are 32-bit integers;
// every result follows from sums and minima of integers, so it does not depend on the order in
// which workgroups run.
#include "heal_device.h"
#include "heal_kv.h"

namespace heal {

namespace {

constexpr int kThreads = 256, kWide = 1024;

__device__ __forceinline__ bool is_page(const KvPages &p, int32_t page) { return page >= 0 && page < p.blocks; }

__device__ __forceinline__ int32_t blocks_of(const KvPages &p, int32_t row)
{
    const int32_t len = p.lens[row] > 0 ? p.lens[row] : 0;
    return (int32_t)(((int64_t)len + p.block - 1) / p.block);
}

// ---- release, fork ---------------------------------------------------------------

// A workgroup takes 1024 entries of a row.
__global__ void __launch_bounds__(kThreads) kv_release_kernel(KvPages p, int64_t wg0, int32_t parts)
{
    const int64_t wg = wg0 + blockIdx.x;
    const int32_t row = (int32_t)(wg / parts), part = (int32_t)(wg - (int64_t)row * parts);
    const int32_t held = blocks_of(p, row);
    int32_t *table = p.table + row * p.table_ld;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t b = (int64_t)part * 1024 + j * kThreads + threadIdx.x;
        if (b < held || b >= p.cols) continue;
        const int32_t page = table[b];
        if (is_page(p, page)) atomicSub(p.refs + page, 1);
        if (page != -1) table[b] = -1;
    }
}

// One pair a workgroup. No pair's child is a parent, so the rows that are read are not written by
// the call; and each row that is written has one pair.
__global__ void __launch_bounds__(kThreads)
kv_fork_kernel(KvPages p, const int32_t *parents, const int32_t *children, int32_t pairs)
{
    const int32_t j = blockIdx.x, from = parents[j], to = children[j];
    if (from < 0 || from >= p.rows || to < 0 || to >= p.rows) return;
    bool out = false;
    for (int32_t i = threadIdx.x; i < pairs; i += kThreads) out |= parents[i] == to || (i < j && children[i] == to);
    if (__syncthreads_or(out)) return;
    const int32_t held = blocks_of(p, from);
    const int32_t *src = p.table + from * p.table_ld;
    int32_t *dst = p.table + to * p.table_ld;
    for (int64_t b = threadIdx.x; b < p.cols; b += kThreads) {
        const int32_t old = dst[b];
        int32_t page = b < held ? src[b] : -1;
        if (!is_page(p, page)) page = -1;
        if (is_page(p, old)) atomicSub(p.refs + old, 1);
        if (page >= 0) atomicAdd(p.refs + page, 1);
        dst[b] = page;
    }
}

// ---- reserve ---------------------------------------------------------------------

// Units of a call that one workgroup has a thread each for; a ragged call, of two units for each
// sequence and more, has kSmallSeqs sequences then, whose cu are kept in LDS.
constexpr int kSmallUnits = kWide, kSmallSeqs = kSmallUnits / 2;
constexpr int kSlots = 2 * kSmallUnits;      // of the table of their blocks
constexpr int32_t kMark = -2147483647 - 1;   // kMark + unit: the unit keeps the block

// The place of the threads with `mine` among all of the workgroup's, counted on from base, which every
// thread has a copy of and moves on alike; part: 16 words of LDS, not those of the call before.
__device__ __forceinline__ int32_t place_of(bool mine, int32_t &base, int32_t *part)
{
    const uint64_t all = __ballot(mine);
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    if (lane == 0) part[wave] = __popcll(all);
    __syncthreads();
    int32_t at = base + __popcll(all & (((uint64_t)1 << lane) - 1)), sum = 0;
#pragma unroll
    for (int w = 0; w < kWide / 64; ++w) {
        at += w < wave ? part[w] : 0;
        sum += part[w];
    }
    base += sum;
    return at;
}

struct Unit {
    int32_t seq, block;   // block -1: none
};

template <class F>
__device__ __forceinline__ Unit unit_of(const KvSeqs &b, int B, int32_t u, F cu)
{
    int32_t i = u;
    KvSeq s;
    if (b.cu) {
        int32_t lo = 0, n = b.seqs;   // the last i with kv_unit(i) <= u
        while (n > 1) {
            const int32_t half = n / 2;
            if ((int64_t)cu(lo + half) / B + 2 * (int64_t)(lo + half) <= u) {
                lo += half;
                n -= half;
            } else {
                n = half;
            }
        }
        i = lo;
        s.first = cu(i);
        const int32_t end = cu(i + 1);
        s.n = end > s.first ? end - s.first : 0;
        u -= s.first / B + 2 * i;
    } else {
        s.first = i;
        s.n = 1;
        u = 0;
    }
    s.len = b.lens[i] > 0 ? b.lens[i] : 0;
    const KvTouched t = kv_touched(s, B);
    const int32_t blk = t.first + u;
    return Unit{i, u >= 0 && blk <= t.last && blk < b.cols ? blk : -1};
}

// The first `need` free blocks into fresh, 4096 counts a turn, the next turn's on the way; returns
// how many there are, or more than need.
__device__ __forceinline__ int32_t find_free(const KvPages &p, int32_t need, int32_t *fresh, int32_t *part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const uint64_t lower = ((uint64_t)1 << lane) - 1;
    auto load = [&](int64_t at) {
        u32x4 r = {1, 1, 1, 1};
        if (at + 4 <= p.blocks) {
            __builtin_memcpy(&r, p.refs + at, sizeof(r));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (at + j < p.blocks) r[j] = p.refs[at + j];
        }
        return r;
    };
    int32_t found = 0;
    int turn = 0;
    u32x4 r = load(threadIdx.x * 4);
    for (int64_t p0 = 0; p0 < p.blocks && found < need; p0 += 4 * kWide, turn ^= 1) {
        const int64_t at = p0 + threadIdx.x * 4;
        const u32x4 next = load(at + 4 * kWide);
        int32_t place = 0, all = 0;
        bool free[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            free[j] = (int32_t)r[j] <= 0 && (int32_t)r[j] > kMark / 2;
            const uint64_t b = __ballot(free[j]);
            place += __popcll(b & lower);
            all += __popcll(b);
        }
        if (lane == 0) part[32 * turn + wave] = all;
        __syncthreads();
        place += found;
#pragma unroll
        for (int w = 0; w < kWide / 64; ++w) {
            place += w < wave ? part[32 * turn + w] : 0;
            found += part[32 * turn + w];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (free[j] && place < need) fresh[place] = (int32_t)(at + j);
            place += free[j];
        }
        r = next;
    }
    return found;
}

// Up to 1024 units, one workgroup, a thread each. The touched blocks meet in a table in LDS, which
// counts their entries and keeps the lowest unit of each; so counts are read once and written once,
// and nothing is written where the free blocks do not suffice.
__global__ void __launch_bounds__(kWide) kv_reserve_kernel(KvPages p, KvSeqs b, int32_t units, int32_t *missing)
{
    __shared__ int32_t s_cu[kSmallSeqs + 1], key[kSlots], count[kSlots], first[kSlots], fresh[kSmallUnits], part[64];
    const int32_t u = threadIdx.x;
    if (b.cu)
        for (int32_t i = u; i <= b.seqs; i += kWide) s_cu[i] = kv_first(b, i);
    for (int32_t i = u; i < kSlots; i += kWide) {
        key[i] = -1;
        count[i] = 0;
        first[i] = kSmallUnits;
    }
    __syncthreads();
    auto cu = [&](int32_t i) { return s_cu[i]; };
    Unit at = {0, -1};
    int32_t *entry = nullptr, page = -1, was = 0, slot = 0;
    if (u < units) at = unit_of(b, p.block, u, cu);
    if (at.block >= 0) {
        entry = p.table + at.seq * p.table_ld + at.block;
        page = *entry;
        if (is_page(p, page)) was = p.refs[page];
        if (was >= 1) {
            slot = (uint32_t)page * 2654435761u >> 21;   // (of 2048; at most half of them are taken)
            for (;;) {
                const int32_t old = atomicCAS(&key[slot], -1, page);
                if (old == -1 || old == page) break;
                slot = (slot + 1) % kSlots;
            }
            atomicAdd(&count[slot], 1);
            atomicMin(&first[slot], u);
        }
    }
    __syncthreads();
    const bool leads = was >= 1 && first[slot] == u, all_here = was >= 1 && count[slot] >= was;
    const bool take = at.block >= 0 && !(leads && all_here);
    int32_t need = 0;
    const int32_t place = place_of(take, need, part);
    __syncthreads();
    const int32_t found = need > 0 ? find_free(p, need, fresh, part) : 0;
    if (u == 0) *missing = found < need ? need - found : 0;
    if (found < need) return;
    __syncthreads();
    if (leads) p.refs[page] = all_here ? 1 : was - count[slot];
    if (take) {
        *entry = fresh[place];
        p.refs[fresh[place]] = 1;
    }
}

// More units: one workgroup with its state in the workspace. Every touched entry takes one off the
// count of its block; where the count comes to 0 all holders are here, and the lowest unit of them
// marks the block as kept. So an entry needs a new block unless its unit is in the mark. Nothing
// but counts of touched blocks has changed by then, and they are put back if the free blocks do not
// suffice.
__global__ void __launch_bounds__(kWide) kv_reserve_many_kernel(KvPages p, KvSeqs b, int32_t units, int32_t *ws, int32_t *missing)
{
    __shared__ int32_t part[64];
    int32_t *pages = ws, *was = ws + units, *fresh = ws + 2 * (int64_t)units;
    const int tid = threadIdx.x;
    auto cu = [&](int32_t i) { return kv_first(b, i); };
    auto load = [](const int32_t *q) { return __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };

    // (-2: no block; -1: an entry that holds nothing)
    for (int32_t u = tid; u < units; u += kWide) {
        const Unit at = unit_of(b, p.block, u, cu);
        int32_t page = -2, r = 0;
        if (at.block >= 0) {
            page = p.table[at.seq * p.table_ld + at.block];
            if (is_page(p, page)) r = p.refs[page];
            if (r < 1) page = -1;
        }
        pages[u] = page;
        was[u] = r;
    }
    __threadfence();
    __syncthreads();
    for (int32_t u = tid; u < units; u += kWide)
        if (pages[u] >= 0) atomicSub(p.refs + pages[u], 1);
    __threadfence();
    __syncthreads();
    for (int32_t u = tid; u < units; u += kWide)
        if (pages[u] >= 0 && load(p.refs + pages[u]) <= 0) atomicMin(p.refs + pages[u], kMark + u);
    __threadfence();
    __syncthreads();

    int32_t need = 0;   // units that take a new block
    int turn = 0;
    for (int32_t u0 = 0; u0 < units; u0 += kWide, turn ^= 1) {
        const int32_t u = u0 + tid, page = u < units ? pages[u] : -2;
        const bool keep = page >= 0 && load(p.refs + page) == kMark + u;
        (void)place_of(page != -2 && !keep, need, part + 32 * turn);
    }
    __syncthreads();
    // (counts that this kernel has changed are no free blocks', before or after)
    const int32_t found = need > 0 ? find_free(p, need, fresh, part) : 0;
    if (tid == 0) *missing = found < need ? need - found : 0;
    const bool fine = found >= need;
    __threadfence();
    __syncthreads();
    int32_t taken = 0;
    for (int32_t u0 = 0; u0 < units; u0 += kWide, turn ^= 1) {
        const int32_t u = u0 + tid, page = u < units ? pages[u] : -2;
        const bool keep = page >= 0 && load(p.refs + page) == kMark + u;
        const bool take = page != -2 && !keep;
        const int32_t at = place_of(take, taken, part + 32 * turn);
        if (fine && take) {
            const Unit un = unit_of(b, p.block, u, cu);
            p.table[un.seq * p.table_ld + un.block] = fresh[at];
            p.refs[fresh[at]] = 1;
        }
        if (fine && keep) pages[u] = -3 - page;   // its mark is what the others compare with until all have
    }
    __syncthreads();
    for (int32_t u = tid; u < units; u += kWide) {
        const int32_t page = pages[u];
        if (page <= -3) p.refs[-3 - page] = 1;
        if (!fine && page >= 0) p.refs[page] = was[u];
    }
}

// ---- compact -----------------------------------------------------------------------

constexpr int kSegment = 4096;   // blocks a workgroup looks at, 4 a thread

struct CompactArgs {
    KvPages p;
    int32_t *src, *dst, *count;
    int32_t *to;        // [blocks]: the move that a block is the source of, or -1
    int32_t *held;      // [segments]: held blocks of each
    int32_t segments;
};

__device__ __forceinline__ int32_t sum_over_wide(int32_t x, int32_t *part)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int w = 0; w < kWide / 64; ++w) x += part[w];
    return x;
}

__global__ void __launch_bounds__(kWide) kv_count_kernel(CompactArgs a)
{
    __shared__ int32_t part[16];
    const int64_t at = (int64_t)blockIdx.x * kSegment + threadIdx.x * 4;
    int32_t n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (at + j >= a.p.blocks) break;
        n += a.p.refs[at + j] > 0;
        if (at + j < a.p.blocks / 2) a.src[at + j] = a.dst[at + j] = -1;
    }
    n = sum_over_wide(n, part);
    if (threadIdx.x == 0) a.held[blockIdx.x] = n;
}

// The k-th held block from the back, k from 0, at or behind n is the source of move k, the k-th
// hole below n its destination: there are as many of the one as of the other.
__global__ void __launch_bounds__(kWide) kv_moves_kernel(CompactArgs a)
{
    __shared__ int32_t part[3][16];
    int32_t before = 0, all = 0;
    for (int32_t s = threadIdx.x; s < a.segments; s += kWide) {
        const int32_t h = a.held[s];
        all += h;
        before += s < (int32_t)blockIdx.x ? h : 0;
    }
    all = sum_over_wide(all, part[0]);
    before = sum_over_wide(before, part[1]);
    const int64_t at = (int64_t)blockIdx.x * kSegment + threadIdx.x * 4;
    bool held[4];
    int32_t mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        held[j] = at + j < a.p.blocks && a.p.refs[at + j] > 0;
        mine += held[j];
    }
    int32_t upto = mine;   // of the wave's lanes up to this one
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int32_t v = __shfl_up(upto, off);
        if ((int)(threadIdx.x & 63) >= off) upto += v;
    }
    if ((threadIdx.x & 63) == 63) part[2][threadIdx.x / 64] = upto;
    __syncthreads();
    before += upto - mine;
#pragma unroll
    for (int w = 0; w < kWide / 64; ++w) before += w < (int)(threadIdx.x / 64) ? part[2][w] : 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = at + j;
        if (i >= a.p.blocks) break;
        if (i == all) *a.count = all - before;
        const int32_t move = all - before - 1;
        a.to[i] = held[j] && i >= all ? move : -1;
        if (held[j] && i >= all) a.src[move] = (int32_t)i;
        if (!held[j] && i < all) a.dst[(int32_t)i - before] = (int32_t)i;
        before += held[j];
    }
    if (all == a.p.blocks && blockIdx.x == 0 && threadIdx.x == 0) *a.count = 0;
}

// Counts of the moves, then the tables' entries, 1024 a workgroup.
__global__ void __launch_bounds__(kThreads) kv_moved_kernel(CompactArgs a, int64_t wg0, int64_t ref_wgs, int32_t parts)
{
    const int64_t wg = wg0 + blockIdx.x;
    if (wg < ref_wgs) {
        const int64_t j = wg * kThreads + threadIdx.x;
        if (j >= a.p.blocks / 2 || a.src[j] < 0) return;
        a.p.refs[a.dst[j]] = a.p.refs[a.src[j]];
        a.p.refs[a.src[j]] = 0;
        return;
    }
    const int64_t row = (wg - ref_wgs) / parts;
    const int32_t at = (int32_t)(wg - ref_wgs - row * parts);
    int32_t *table = a.p.table + row * a.p.table_ld;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t b = (int64_t)at * 1024 + j * kThreads + threadIdx.x;
        if (b >= a.p.cols) continue;
        const int32_t page = table[b], move = is_page(a.p, page) ? a.to[page] : -1;
        if (move >= 0) table[b] = a.dst[move];
    }
}

// All of it in one workgroup, for pools and tables that are small, the moves in LDS: one launch of
// 3.5 us (1220 blocks) to 5.5 (3300) instead of three that take 8.5 to 11 and the host 3.6 apiece.
constexpr int kSmallPool = 8192, kSmallTable = 8192;

__global__ void __launch_bounds__(kWide) kv_compact_kernel(CompactArgs a)
{
    constexpr int SEGMENTS = kSmallPool / kSegment;
    __shared__ uint16_t to[kSmallPool], src[kSmallPool / 2], dst[kSmallPool / 2];
    __shared__ int32_t part[SEGMENTS][kWide / 64], moves;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const uint64_t lower = ((uint64_t)1 << lane) - 1;
    int32_t refs[SEGMENTS][4], before[SEGMENTS];
#pragma unroll
    for (int g = 0; g < SEGMENTS; ++g) {
        int32_t all = 0;
        before[g] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int32_t i = g * kSegment + threadIdx.x * 4 + j;
            refs[g][j] = i < a.p.blocks ? a.p.refs[i] : 0;
            const uint64_t held = __ballot(refs[g][j] > 0);
            before[g] += __popcll(held & lower);
            all += __popcll(held);
        }
        if (lane == 0) part[g][wave] = all;
    }
    if (threadIdx.x == 0) moves = 0;
    __syncthreads();
    int32_t all = 0;
#pragma unroll
    for (int g = 0; g < SEGMENTS; ++g) {
        before[g] += all;
#pragma unroll
        for (int w = 0; w < kWide / 64; ++w) {
            before[g] += w < wave ? part[g][w] : 0;
            all += part[g][w];
        }
    }
#pragma unroll
    for (int g = 0; g < SEGMENTS; ++g) {
        int32_t n = before[g];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int32_t i = g * kSegment + threadIdx.x * 4 + j, move = all - n - 1;
            const bool held = refs[g][j] > 0;
            if (i >= a.p.blocks) break;
            if (i == all) moves = all - n;
            to[i] = held && i >= all ? (uint16_t)move : (uint16_t)0xffff;
            if (held && i >= all) src[move] = (uint16_t)i;
            if (!held && i < all) dst[i - n] = (uint16_t)i;
            n += held;
        }
    }
    __syncthreads();
#pragma unroll
    for (int g = 0; g < SEGMENTS; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int32_t i = g * kSegment + threadIdx.x * 4 + j;
            if (i >= a.p.blocks || to[i] == 0xffff) continue;
            a.p.refs[dst[to[i]]] = refs[g][j];
            a.p.refs[i] = 0;
        }
    for (int32_t j = threadIdx.x; j < a.p.blocks / 2; j += kWide) {
        a.src[j] = j < moves ? src[j] : -1;
        a.dst[j] = j < moves ? dst[j] : -1;
    }
    if (threadIdx.x == 0) *a.count = moves;
    const int32_t entries = a.p.rows * a.p.cols;
    for (int32_t e = threadIdx.x; e < entries; e += kWide) {
        const int32_t row = e / a.p.cols;
        int32_t *entry = a.p.table + row * a.p.table_ld + (e - row * a.p.cols);
        const int32_t page = *entry;
        if (is_page(a.p, page) && to[page] != 0xffff) *entry = dst[to[page]];
    }
}

// ---- copy --------------------------------------------------------------------------

constexpr int kCopyBytes = 16384;   // of one array, by a workgroup at a time

// n pairs of entries of up to three arrays (16-byte units) and of one that goes with the first part
// of the last one (8-byte units).
struct CopyArgs {
    const int32_t *src, *dst, *count;
    int64_t n;
    int32_t bound, parts;        // entries of the arrays; workgroups' turns for a pair
    char *at[3];
    int64_t bytes[3];
    char *more;
    int64_t more_bytes;
};

__global__ void __launch_bounds__(kThreads) kv_copy_kernel(CopyArgs a)
{
    int64_t n = a.n;
    if (a.count) n = *a.count < 0 ? 0 : *a.count < n ? *a.count : n;
    for (int64_t u = blockIdx.x; u < n * a.parts; u += gridDim.x) {
        const int64_t pair = u / a.parts;
        int64_t part = u - pair * a.parts;
        const int32_t from = a.src[pair], to = a.dst[pair];
        if (from < 0 || from >= a.bound || to < 0 || to >= a.bound || from == to) continue;
        int r = 0;
        while (r < 2 && part * kCopyBytes >= a.bytes[r]) {
            part -= (a.bytes[r] + kCopyBytes - 1) / kCopyBytes;
            ++r;
        }
        const int64_t first = part * kCopyBytes, size = a.bytes[r];
        const char *s = a.at[r] + from * size;
        char *d = a.at[r] + to * size;
#pragma unroll
        for (int j = 0; j < kCopyBytes / 16 / kThreads; ++j) {
            const int64_t off = first + (j * kThreads + threadIdx.x) * 16;
            if (off < size) *reinterpret_cast<u32x4 *>(d + off) = *reinterpret_cast<const u32x4 *>(s + off);
        }
        if (a.more && r == 2 && part == 0)
            for (int64_t off = threadIdx.x * 8; off < a.more_bytes; off += kThreads * 8)
                *reinterpret_cast<u32x2 *>(a.more + to * a.more_bytes + off) =
                    *reinterpret_cast<const u32x2 *>(a.more + from * a.more_bytes + off);
    }
}

hipError_t launch_copy(CopyArgs a, hipStream_t stream)
{
    a.parts = 0;
    for (int64_t size : a.bytes) a.parts += (int32_t)((size + kCopyBytes - 1) / kCopyBytes);
    const int64_t units = a.n * a.parts;
    kv_copy_kernel<<<dim3((unsigned)(units < 4096 ? units : 4096)), dim3(kThreads), 0, stream>>>(a);
    return hipGetLastError();
}

int32_t row_parts(const KvPages &p) { return (p.cols + 1023) / 1024; }

}  // namespace

hipError_t launch_kv_release(const KvPages &p, hipStream_t stream)
{
    const int32_t parts = row_parts(p);
    return in_parts((int64_t)p.rows * parts, [&](int64_t at, unsigned n) {
        kv_release_kernel<<<dim3(n), dim3(kThreads), 0, stream>>>(p, at, parts);
    });
}

hipError_t launch_kv_fork(const KvPages &p, int32_t pairs, const int32_t *parents, const int32_t *children,
                          hipStream_t stream)
{
    kv_fork_kernel<<<dim3((unsigned)pairs), dim3(kThreads), 0, stream>>>(p, parents, children, pairs);
    return hipGetLastError();
}

int64_t kv_reserve_bytes(int64_t units) { return units <= kSmallUnits ? 0 : (12 * units + 15) / 16 * 16; }

hipError_t launch_kv_reserve(const KvPages &p, const KvSeqs &b, int64_t units, void *workspace, int32_t *missing,
                             hipStream_t stream)
{
    int32_t *ws = static_cast<int32_t *>(workspace);
    if (units <= kSmallUnits)
        kv_reserve_kernel<<<dim3(1), dim3(kWide), 0, stream>>>(p, b, (int32_t)units, missing);
    else
        kv_reserve_many_kernel<<<dim3(1), dim3(kWide), 0, stream>>>(p, b, (int32_t)units, ws, missing);
    return hipGetLastError();
}

int64_t kv_compact_bytes(int64_t blocks) { return (4 * (blocks + (blocks + kSegment - 1) / kSegment) + 15) / 16 * 16; }

hipError_t launch_kv_compact(const KvPages &p, int32_t *src, int32_t *dst, int32_t *count, void *workspace,
                             hipStream_t stream)
{
    CompactArgs a = {p, src, dst, count, static_cast<int32_t *>(workspace), nullptr, 0};
    a.held = a.to + p.blocks;
    a.segments = (int32_t)(((int64_t)p.blocks + kSegment - 1) / kSegment);
    if (p.blocks <= kSmallPool && (int64_t)p.rows * p.cols <= kSmallTable) {
        kv_compact_kernel<<<dim3(1), dim3(kWide), 0, stream>>>(a);
        return hipGetLastError();
    }
    kv_count_kernel<<<dim3((unsigned)a.segments), dim3(kWide), 0, stream>>>(a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    kv_moves_kernel<<<dim3((unsigned)a.segments), dim3(kWide), 0, stream>>>(a);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
    const int64_t ref_wgs = (p.blocks / 2 + kThreads - 1) / kThreads;
    const int32_t parts = row_parts(p);
    return in_parts(ref_wgs + (int64_t)p.rows * parts, [&](int64_t at, unsigned n) {
        kv_moved_kernel<<<dim3(n), dim3(kThreads), 0, stream>>>(a, at, ref_wgs, parts);
    });
}

hipError_t launch_kv_copy(const KvCache &c, const KvCopy &l, int32_t blocks, int32_t slots, hipStream_t stream)
{
    const int64_t rows = (int64_t)c.heads * c.dim;
    if (l.blocks > 0) {
        const CopyArgs a = {l.block_src, l.block_dst, l.count, l.blocks, blocks, 0,
                            {(char *)c.kc, (char *)c.vc, (char *)c.mean}, {rows * c.block, rows * c.block, rows * 4},
                            (char *)c.scales, (int64_t)c.heads * 8};
        const hipError_t err = launch_copy(a, stream);
        if (err != hipSuccess) return err;
    }
    if (l.slots > 0) {
        const CopyArgs a = {l.slot_src, l.slot_dst, nullptr, l.slots, slots, 0,
                            {(char *)c.kr, (char *)c.vr, nullptr}, {rows * c.block * 8, rows * c.block * 8, 0},
                            nullptr, 0};
        return launch_copy(a, stream);
    }
    return hipSuccess;
}

}  // namespace heal
