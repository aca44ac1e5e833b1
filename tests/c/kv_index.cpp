// The index functions of the key/value cache, checked on the host: every block and
// row belongs to one workgroup, and whatever the tables hold nothing leads outside
// an array.  Prints "ok".
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "heal.h"
#include "heal_kv.h"

using namespace heal;

#define CHECK(c)                                                    \
    do {                                                            \
        if (!(c)) {                                                 \
            printf("line %d: %s (round %d)\n", __LINE__, #c, round); \
            return 1;                                               \
        }                                                           \
    } while (0)

static unsigned long long state = 88172645463325252ull;
static int rnd(int n)
{
    state ^= state << 13;
    state ^= state >> 7;
    state ^= state << 17;
    return (int)(state % (unsigned long long)n);
}

// what kv_last_at_most finds, one place after another
template <class F>
static int last_at_most(int n, int64_t u, F f)
{
    int at = 0;
    for (int i = 1; i < n; ++i)
        if (f(i) <= u) at = i;
    return at;
}

int main()
{
    int round = 0;
    for (int B : {16, 32, 64, 128}) {
        std::vector<int> seen(B);
        for (int t = 0; t < B; ++t) {
            const int at = kv_value_place(B, t);
            CHECK(at >= 0 && at < B);
            ++seen[at];
            // groups of four tokens lie together, aligned
            CHECK(at % 4 == t % 4);
            if (t % 4) CHECK(at == kv_value_place(B, t - 1) + 1);
        }
        for (int c : seen) CHECK(c == 1);
    }
    // every tile before the first one of the ring has complete blocks only, every row of an
    // incomplete block lies in a tile from that one to the end
    for (int B : {16, 32, 64, 128})
        for (int len = 0; len < 1000; ++len) {
            const int64_t first = kv_ring_first(len, B), end = kv_ring_end(len, B);
            for (int64_t kt = 0; kt * 64 < len; ++kt) {
                bool ring = false;
                for (int64_t p = kt * 64; p < kt * 64 + 64 && p < len; ++p) ring |= (p / B + 1) * B > len;
                CHECK(ring == (kt >= first));
                CHECK(kt < end);
            }
            CHECK(len % B == 0 || (end - 1) * 64 < len);
        }
    const int blocks[] = {16, 32, 64, 128}, groups[] = {1, 2, 3, 4, 7, 16, 17, 64};
    for (round = 0; round < 3000; ++round) {
        const int B = blocks[rnd(4)], G = groups[rnd(8)], R = rnd(2) ? 16 : 128, seqs = 1 + rnd(9);
        const bool ragged = rnd(4) != 0;
        std::vector<int32_t> cu(seqs + 1), lens(seqs);
        for (int i = 0; i < seqs; ++i) {
            const int n = ragged ? (rnd(4) ? rnd(3 * B) : rnd(3)) : 1;
            cu[i + 1] = cu[i] + n;
            lens[i] = rnd(8) ? n + rnd(4 * B) : rnd(n + 1);
        }
        KvSeqs b = {};
        b.cu = ragged ? cu.data() : nullptr;
        b.lens = lens.data();
        b.seqs = seqs;
        b.tokens = cu[seqs];
        b.cols = 100;
        // units
        std::vector<std::vector<int>> units(seqs, std::vector<int>(64));
        const int64_t total = kv_units(ragged, b.tokens, seqs, B);
        for (int64_t u = 0; u < total; ++u) {
            const int i = last_at_most(seqs, u, [&](int k) { return kv_unit(b, B, k); });
            const int64_t j = u - kv_unit(b, B, i);
            CHECK(j >= 0);
            if (j < 64) ++units[i][j];
        }
        for (int i = 0; i < seqs; ++i) {
            const KvSeq s = kv_seq(b, i);
            const KvTouched t = kv_touched(s, B);
            CHECK(s.first >= 0 && s.n >= 0 && s.first + s.n <= b.tokens);
            for (int j = 0; j < 64 && t.first + j <= t.last; ++j) CHECK(units[i][j] == 1);
            // the ring: rows written by other units than 0 never lie where unit 0 reads
            if (t.last < t.first) continue;
            const int c = kv_ring_conflict(t);
            const int old_lo = t.first * B, old_hi = t.start;   // places that unit 0 reads from the ring
            for (int blk = t.last - 1; blk <= t.last; ++blk) {
                if (blk <= t.first || blk == c) continue;
                for (int p = blk * B; p < blk * B + B && p < s.len; ++p)
                    for (int o = old_lo; o < old_hi; ++o) CHECK(p % (2 * B) != o % (2 * B));
            }
            CHECK(c == -1 || (c > t.first && (c == t.last || c == t.last - 1)));
        }
        // row tiles
        std::vector<std::vector<int>> tiles(seqs, std::vector<int>(8192));
        const int64_t rt = kv_tiles(b.tokens, seqs, G, R);
        for (int64_t u = 0; u < rt; ++u) {
            const int i = last_at_most(seqs, u, [&](int k) { return kv_tile(b, G, R, k); });
            const int64_t j = u - kv_tile(b, G, R, i);
            CHECK(j >= 0 && j < 8192);
            ++tiles[i][j];
        }
        for (int i = 0; i < seqs; ++i) {
            const int64_t rows = (int64_t)kv_seq(b, i).n * G;
            for (int64_t j = 0; j * R < rows; ++j) CHECK(tiles[i][j] == 1);
        }
    }
    // tables, slots and cu that hold anything
    for (round = 0; round < 2000; ++round) {
        const int seqs = 1 + rnd(5), cols = rnd(6);
        std::vector<int32_t> cu(seqs + 1), lens(seqs), table(seqs * 8), slots(seqs);
        auto any = [&]() { return rnd(3) ? rnd(40) - 8 : (int32_t)((unsigned)rnd(1 << 30) * 4u + 3u); };
        for (auto *v : {&cu, &lens, &table, &slots})
            for (auto &x : *v) x = any();
        KvSeqs b = {};
        b.cu = cu.data();
        b.lens = lens.data();
        b.table = table.data();
        b.slots = slots.data();
        b.table_ld = 8;
        b.seqs = seqs;
        b.tokens = rnd(40);
        b.cols = cols;
        b.blocks = 1 + rnd(20);
        b.nslots = 1 + rnd(4);
        for (int i = 0; i < seqs; ++i) {
            const KvSeq s = kv_seq(b, i);
            CHECK(s.first >= 0 && s.n >= 0 && s.len >= 0 && (int64_t)s.first + s.n <= b.tokens);
            const int slot = kv_slot(b, i);
            CHECK(slot >= -1 && slot < b.nslots);
            CHECK(slot == -1 || slot == slots[i]);
            for (int blk : {-2147483647, -1, 0, cols - 1, cols, 7, 2147483647}) {
                const int p = kv_page(b, i, blk);
                CHECK(p >= -1 && p < b.blocks);
                CHECK(p == -1 || (blk >= 0 && blk < cols && p == table[i * 8 + blk]));
            }
        }
    }
    puts("ok");
}
