// a2sgd_gated_ffn_status with the kernels' count set by hand: every stream is told of a wait that ran out, once.
#include "a2sgd_gated_ffn.cu"

#include <cstdio>

static int failures = 0;
#define EXPECT(cond) do { if (!(cond)) { std::printf("FAILED line %d: %s\n", __LINE__, #cond); ++failures; } } while (0)

static int ask(cudaStream_t s)
{
    int status = 77;
    EXPECT(a2sgd_gated_ffn_status(0, &status, s) == A2SGD_OK);
    return status;
}
static void run_out(unsigned int times) { EXPECT(cudaMemcpyToSymbol(g_waits_run_out, &times, sizeof times) == cudaSuccess); }

int main()
{
    cudaStream_t a, b;
    EXPECT(cudaStreamCreateWithFlags(&a, cudaStreamNonBlocking) == cudaSuccess);
    EXPECT(cudaStreamCreate(&b) == cudaSuccess);
    EXPECT(ask(a) == A2SGD_OK && ask(b) == A2SGD_OK && ask(nullptr) == A2SGD_OK);
    run_out(2);
    EXPECT(ask(a) == A2SGD_ERR_TIMEOUT && ask(a) == A2SGD_OK);
    EXPECT(ask(b) == A2SGD_ERR_TIMEOUT && ask(b) == A2SGD_OK && ask(a) == A2SGD_OK);
    run_out(3);
    EXPECT(ask(nullptr) == A2SGD_ERR_TIMEOUT && ask(nullptr) == A2SGD_OK);
    EXPECT(ask(b) == A2SGD_ERR_TIMEOUT && ask(a) == A2SGD_ERR_TIMEOUT && ask(a) == A2SGD_OK);
    std::printf("%s\n", failures ? "FAILED" : "ok");
    return failures ? 1 : 0;
}
