// The loads of B in the adapters' second kernel, checked on the host: where they are made without
// a check, all that they ask for lies within the adapter's N rows.  Prints "ok".
#include <cstdio>

#include "heal_layer.h"

using namespace heal;

// The element behind the last one that the 32 rows from n0 on ask for.
template <class T>
static long last_asked(int n0, int rank)
{
    long end = 0;
    for (int q = 0; q < (rank + 31) / 32; ++q)
        for (int lane = 0; lane < 64; ++lane)
            for (int h = 0; h < 2; ++h) {
                const int n = n0 + 16 * h + lane % 16, j = 32 * q + kLane<T> * (lane / 16);
                for (int from : {j, j + kNext<T>})
                    if (from < rank && (long)n * rank + from + 4 > end) end = (long)n * rank + from + 4;
            }
    return end;
}

template <class T>
static bool sweep()
{
    for (int rank = 1; rank <= 512; ++rank)
        for (int N = 1; N <= 70; ++N)
            for (int n0 = 0; n0 < N; n0 += 32) {
                if (!lora_whole(n0, N, rank)) {
                    // no more of them are checked than have to be
                    if (n0 + 32 <= N && last_asked<T>(n0, rank) <= (long)N * rank) {
                        printf("rank %d, N %d, n0 %d need no check (elements of %d bytes)\n", rank, N, n0, (int)sizeof(T));
                        return false;
                    }
                    continue;
                }
                if (last_asked<T>(n0, rank) > (long)N * rank) {
                    printf("rank %d, N %d, n0 %d: %ld of %ld elements (of %d bytes)\n", rank, N, n0,
                           last_asked<T>(n0, rank), (long)N * rank, (int)sizeof(T));
                    return false;
                }
            }
    return true;
}

int main()
{
    if (!sweep<float>() || !sweep<uint16_t>()) return 1;
    // the whole range of N, with the rows' bound alone
    for (int rank = 1; rank <= 512; ++rank)
        for (int N = (1 << 24) - 70; N <= 1 << 24; ++N) {
            const int n0 = (N - 32) / 32 * 32;
            if (lora_whole(n0, N, rank) && (long)(n0 + 31) * rank + (rank + 3) / 4 * 4 > (long)N * rank) {
                printf("rank %d, N %d\n", rank, N);
                return 1;
            }
        }
    printf("ok\n");
    return 0;
}
