// How many steps a piece of a tile of the many-row attention has (csrc/fbq_attend_plan.h): one line on stdout for each line "twice tiles kv_heads blocks" on stdin.
#include <cstdio>
#include <iostream>

#include "fbq_attend_plan.h"

int main()
{
    unsigned long long twice;
    int tiles, kv_heads, blocks;
    while (std::cin >> twice >> tiles >> kv_heads >> blocks) printf("%d\n", fbq::share_of_steps(twice, tiles, kv_heads, blocks));
    return 0;
}
