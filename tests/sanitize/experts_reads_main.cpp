// Host-only model of what a product's requests read of an operand stored across k: every unit of every stage that is read by whole
// units has to lie inside the operand's storage (tests/test_experts_reads.py builds and runs it; no GPU is touched).
#include <stdint.h>
#include <stdio.h>

#include "experts_internal.h"

int main()
{
    long cases = 0, outside = 0;
    for (int es = 1; es <= 2; ++es) {
        const int bk = 128 / es, e = 16 / es;
        for (int lines = 1; lines <= 40; ++lines)
            for (int apart = 0; apart <= 12; apart = apart < 4 ? apart + 1 : apart + 4)
                for (int k = 1; k <= 5 * bk + 20; k += k % bk < 20 || k % bk > bk - 3 ? 1 : 7) {
                    const int64_t pitch = (int64_t)(lines + apart) * es, row = (int64_t)lines * es, end = (k - 1) * pitch + row;
                    int whole = k / bk;
                    if (lines % e != 0) whole = amulet::stages_of_whole_units(whole, bk, k, row, pitch);
                    ++cases;
                    if (whole < 0 || whole < k / bk - 1) { printf("too few: es %d lines %d pitch %d k %d: %d\n", es, lines, (int)pitch, k, whole); return 1; }
                    for (int r = 0; r < whole * bk; ++r)
                        for (int c = 0; c < lines; c += e)
                            if (r * pitch + (int64_t)c * es + 16 > end) {
                                if (outside++ < 5) printf("outside: es %d lines %d pitch %d k %d: row %d, bytes to %ld of %ld\n", es, lines, (int)pitch, k, r, (long)(r * pitch + c * es + 16), (long)end);
                                r = whole * bk;
                                break;
                            }
                }
    }
    printf("%ld cases, %ld read outside\n", cases, outside);
    return outside ? 1 : 0;
}
