// The host's notes of the training operators (csrc/a2sgd_train.cu) on the runtime of fake_runtime.cpp: two devices, no GPU.
#include "a2sgd_train.cuh"

#include <cstdio>
#include <thread>

using namespace a2sgd_train;

extern "C" int current_device, occupancy_questions; // of the runtime in fake_runtime.cpp

static int failures = 0;
#define EXPECT(cond) do { if (!(cond)) { std::printf("FAILED line %d: %s\n", __LINE__, #cond); ++failures; } } while (0)

int main(int argc, char **argv)
{
    const char *part = argc > 1 ? argv[1] : "";
    if (part[0] == 'c') { // count
        const cudaStream_t a = reinterpret_cast<cudaStream_t>(0x1000), b = reinterpret_cast<cudaStream_t>(0x2000), own = cudaStreamPerThread;
        EXPECT(!count_moved(0, a, 0) && !count_moved(0, b, 0) && !count_moved(0, nullptr, 0));
        // a wait runs out while b's caller is not looking: a is told once, and b all the same
        EXPECT(count_moved(0, a, 1));
        EXPECT(!count_moved(0, a, 1));
        EXPECT(count_moved(0, b, 1));
        EXPECT(!count_moved(0, b, 1) && !count_moved(0, a, 1));
        EXPECT(count_moved(0, nullptr, 1) && !count_moved(0, nullptr, 1));
        // two more between two questions: told again, once
        EXPECT(count_moved(0, b, 3) && !count_moved(0, b, 3) && count_moved(0, a, 3) && !count_moved(0, a, 3));
        // another device has its own count
        EXPECT(!count_moved(1, a, 0) && count_moved(1, a, 1) && !count_moved(0, a, 3));
        // each thread's own default stream goes by the same handle
        EXPECT(count_moved(0, own, 3) && !count_moved(0, own, 3));
        bool other = false, again = true;
        std::thread([&] { other = count_moved(0, own, 3), again = count_moved(0, own, 3); }).join();
        EXPECT(other && !again);
    } else { // occupancy
        EXPECT(sm_count(0) == 100 && sm_count(1) == 101);
        const void *fn = &failures;
        EXPECT(resident_ctas(fn, 128, 0, 0) == 2 && resident_ctas(fn, 128, 0, 0) == 2 && occupancy_questions == 1);
        current_device = 1;
        EXPECT(resident_ctas(fn, 128, 0, 1) == 3 && resident_ctas(fn, 128, 0, 1) == 3 && occupancy_questions == 2);
        current_device = 0;
        EXPECT(resident_ctas(fn, 128, 0, 0) == 2 && occupancy_questions == 2);
        EXPECT(resident_ctas(fn, 128, 1024, 0) == 2 && occupancy_questions == 3);
    }
    std::printf("%s\n", failures ? "FAILED" : "ok");
    return failures ? 1 : 0;
}
