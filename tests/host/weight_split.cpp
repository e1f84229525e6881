// Prints how weight gradients are split: for every line "rows width outputs dtype" of the input, "tile parts steps workspace bytes".
#include <cstdio>

#include "adasum_layers.h"

int main() {
    long long rows, width, outputs;
    int dtype;
    while (std::scanf("%lld %lld %lld %d", &rows, &width, &outputs, &dtype) == 4) {
        const adasum::WeightSplit s = adasum::weight_split(rows, width, outputs, dtype);
        std::printf("%d %lld %lld %zu\n", s.tile, static_cast<long long>(s.parts), static_cast<long long>(s.steps), s.total);
    }
    return 0;
}
