// The launches of a norm of many rows, checked on the host: they cover every row once, in order, and
// none has more workgroups than a launch takes.  Prints "ok".
#include <cstdio>

#include "heal_layer.h"

int main()
{
    const int64_t most = ((int64_t)1 << 31) - 1, full = 1 << 21;
    for (int per : {1, 4, 8, 16})
        for (int64_t rows : {(int64_t)1, (int64_t)per, per + (int64_t)1, full * per - 1, full * per, full * per + 1,
                             full * per + per + 1, 3 * full * per - per, most - per, most - 1, most}) {
            if (rows > most) continue;
            int64_t next = 0;
            const hipError_t err = heal::norm_launches((int32_t)rows, per, [&](int32_t row0, unsigned n) {
                if (row0 != next || n < 1 || n > full) return hipErrorInvalidValue;
                // (every workgroup has a row, and only the last one may have some missing)
                if (row0 + ((int64_t)n - 1) * per >= rows) return hipErrorInvalidValue;
                next = row0 + (int64_t)n * per;
                return hipSuccess;
            });
            if (err != hipSuccess || next < rows || next - rows >= per) {
                printf("%lld rows, %d a workgroup: ends at %lld\n", (long long)rows, per, (long long)next);
                return 1;
            }
        }
    // the first launch that fails is the last
    int calls = 0;
    if (heal::norm_launches(1 << 30, 1, [&](int32_t, unsigned) { return ++calls == 3 ? hipErrorInvalidValue : hipSuccess; }) !=
            hipErrorInvalidValue || calls != 3)
        return 1;
    printf("ok\n");
    return 0;
}
