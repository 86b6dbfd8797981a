// Which products of rows the kernels over small matrices take, and in how many runs, for every size: the library's own rules,
// called on the host.  Prints "columns sums fits runs" a line.
#include <stdio.h>

#include "grouped_kernels.h"

int main()
{
    for (unsigned cols = 1; cols <= 130; ++cols)
        for (unsigned sums = 1; sums <= 130; ++sums) {
            lmk::RowsArgs r = {};
            r.lda = r.ldw = sums;
            r.ldo = r.cols = cols;
            r.sums = sums;
            r.blocks = 1;
            r.rows = 1u << 26;
            const bool fits = lmk::narrow_rows_fit(r);
            // the grid counts two ends of blocks more
            printf("%u %u %d %llu\n", cols, sums, fits ? 1 : 0, (unsigned long long)lmk::narrow_rows_threads(r) / 256 - 3);
        }
    return 0;
}
