// a2sgd_window_attention_status and a2sgd_gated_ffn_status asked for side by side, with the kernels' counts set by hand.  Two translation units, as in
// the library: with FEED_FORWARD the feed-forward block's, else the attention's and the program.
#ifdef FEED_FORWARD
#include "a2sgd_gated_ffn.cu"

bool feed_forward_ran_out(unsigned int times) { return cudaMemcpyToSymbol(g_waits_run_out, &times, sizeof times) == cudaSuccess; }
#else
#include "a2sgd_window_attention.cu"

#include <cstdio>

bool feed_forward_ran_out(unsigned int times);
static bool attention_ran_out(unsigned int times) { return cudaMemcpyToSymbol(g_waits_run_out, &times, sizeof times) == cudaSuccess; }

static int failures = 0;
#define EXPECT(cond) do { if (!(cond)) { std::printf("FAILED line %d: %s\n", __LINE__, #cond); ++failures; } } while (0)

static int attention(cudaStream_t s)
{
    int status = 77;
    EXPECT(a2sgd_window_attention_status(0, &status, s) == A2SGD_OK);
    return status;
}
static int feed_forward(cudaStream_t s)
{
    int status = 77;
    EXPECT(a2sgd_gated_ffn_status(0, &status, s) == A2SGD_OK);
    return status;
}

int main()
{
    cudaStream_t a;
    EXPECT(cudaStreamCreateWithFlags(&a, cudaStreamNonBlocking) == cudaSuccess);
    EXPECT(attention(a) == A2SGD_OK && feed_forward(a) == A2SGD_OK);
    EXPECT(feed_forward_ran_out(1) && feed_forward(a) == A2SGD_ERR_TIMEOUT && attention(a) == A2SGD_OK);
    EXPECT(attention_ran_out(1) && attention(a) == A2SGD_ERR_TIMEOUT); // the same count as the other's
    EXPECT(attention(a) == A2SGD_OK && feed_forward(a) == A2SGD_OK);
    EXPECT(attention_ran_out(2) && attention(a) == A2SGD_ERR_TIMEOUT);
    for (int i = 0; i < 3; ++i) EXPECT(feed_forward(a) == A2SGD_OK && attention(a) == A2SGD_OK); // different ones, in turn
    EXPECT(feed_forward(nullptr) == A2SGD_ERR_TIMEOUT && attention(nullptr) == A2SGD_ERR_TIMEOUT && feed_forward(nullptr) == A2SGD_OK);
    std::printf("%s\n", failures ? "FAILED" : "ok");
    return failures ? 1 : 0;
}
#endif
