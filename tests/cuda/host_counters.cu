// Two operators' counts of waits that ran out (csrc/a2sgd_train.cu), asked for on the same streams, on the runtime of fake_runtime.cpp: no GPU.
#include "a2sgd_train.cuh"

#include <cstdio>

using namespace a2sgd_train;

static int failures = 0;
#define EXPECT(cond) do { if (!(cond)) { std::printf("FAILED line %d: %s\n", __LINE__, #cond); ++failures; } } while (0)

int main()
{
    const cudaStream_t a = reinterpret_cast<cudaStream_t>(0x1000), b = reinterpret_cast<cudaStream_t>(0x2000);
    const int one = 0, two = 0; // whose addresses say which counter is meant
    // equal counts: each is told of, once
    EXPECT(count_moved(0, a, 1, &one) && count_moved(0, a, 1, &two));
    EXPECT(!count_moved(0, a, 1, &one) && !count_moved(0, a, 1, &two));
    // different ones, asked for in turn: not told of again
    EXPECT(count_moved(0, a, 5, &two));
    for (int i = 0; i < 3; ++i) EXPECT(!count_moved(0, a, 1, &one) && !count_moved(0, a, 5, &two));
    // another stream, and another device, for each
    EXPECT(count_moved(0, b, 5, &one) && count_moved(0, b, 5, &two) && !count_moved(0, b, 5, &one) && !count_moved(0, b, 5, &two));
    EXPECT(count_moved(1, a, 5, &one) && count_moved(1, a, 5, &two) && !count_moved(1, a, 5, &one));
    std::printf("%s\n", failures ? "FAILED" : "ok");
    return failures ? 1 : 0;
}
