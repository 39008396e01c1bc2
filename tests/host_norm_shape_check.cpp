// Shapes of the passes over rows (paper_2605_28691_amd/csrc/norm_shape.h) on the host.  Reads rows, cols, one pair a line; prints the forward shape for 2, 4 and 8 bytes read a channel and the backward one:
// span, pieces of a lane, lanes of a row, threads (and parts).  Built and run by tests/test_norm_shape.py.
#include <cstdio>

#include "../paper_2605_28691_amd/csrc/norm_shape.h"

using namespace skiparse;

int main() {
    unsigned rows, cols;
    while (scanf("%u %u", &rows, &cols) == 2) {
        for (unsigned read : {2u, 4u, 8u}) {
            const NormShape s = norm_shape(rows, cols, read);
            printf("%d %d %u %u ", s.span, s.ch, s.lanes, s.threads);
        }
        const NormBwdShape b = norm_bwd_shape(rows, cols);
        printf("%d %d %u %u %u\n", b.span, b.ch, b.lanes, b.threads, b.parts);
    }
}
