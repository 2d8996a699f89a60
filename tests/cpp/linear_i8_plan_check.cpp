// Prints the kernel that an 8-bit product is planned by, for every "m n k dtype cus direct residual" on standard input.
#include <cstdio>

#include "decode_ops.h"

int main()
{
    int m, n, k, dtype, cus, direct, residual;
    while (scanf("%d %d %d %d %d %d %d", &m, &n, &k, &dtype, &cus, &direct, &residual) == 7) {
        const sgprs_linear_i8_desc_t d = {m, n, k, dtype, SGPRS_ACT_NONE, 0, k, k, n, n};
        printf("%d\n", sgprs::plan_linear_i8(d, cus, direct != 0, residual != 0));
    }
    return 0;
}
