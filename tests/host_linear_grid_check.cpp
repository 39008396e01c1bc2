// How many workgroups products of the linear layer take (paper_2605_28691_amd/csrc/linear_plan.h), without a look at each: for sizes up to those that the library takes.  Reads M N K, one product a
// line; prints whether a result of M x N fits one launch, the workgroups of the product's, and the rows of a part and workgroups of the pass over M rows of N channels.  Built and run by
// tests/test_linear_grid.py.
#include <cstdio>

#include "../paper_2605_28691_amd/csrc/linear_plan.h"

using namespace skiparse;

int main() {
    unsigned M, N, K;
    while (scanf("%u %u %u", &M, &N, &K) == 3) {
        const LinearPlan p = plan_linear(M, N, K);
        const unsigned per = linear_rows_per_part(M, N);
        printf("%d %llu %u %llu\n", (int)linear_fits(M, N), p.whole + (unsigned long long)p.rest * p.parts, per, (unsigned long long)linear_rows_parts(M, N) * ((N + 255u) / 256u));
    }
}
