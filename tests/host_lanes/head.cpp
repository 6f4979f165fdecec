// The vocabulary head's launches (HEAD_LOSS: head_loss.hip with each launch as a call of
// lanes::launch) as C functions of host memory.
#include "lanes.h"
#include HEAD_LOSS

extern "C" void host_order(int early, int backwards)
{
    lanes::early = early != 0;
    lanes::backwards = backwards != 0;
}
extern "C" size_t host_head_workspace(int64_t B, int64_t T, int64_t D, int64_t V, int64_t sb, int64_t st,
                                      int64_t ld, int dtype, int backward)
{
    return cdk::head_workspace_bytes({nullptr, nullptr, B, T, D, V, sb, st, ld, dtype}, backward != 0);
}
extern "C" void host_head(const void *h, const void *w, int64_t B, int64_t T, int64_t D, int64_t V, int64_t sb,
                          int64_t st, int64_t ld, int dtype, const int32_t *tokens, float temperature,
                          float *logprob, float *entropy, void *saved, void *ws)
{
    cdk::launch_head_forward({h, w, B, T, D, V, sb, st, ld, dtype}, tokens, temperature, logprob, entropy,
                             static_cast<cdk::ScoreRow *>(saved), ws, nullptr);
}
extern "C" void host_head_grad(const void *h, const void *w, int64_t B, int64_t T, int64_t D, int64_t V,
                               int64_t sb, int64_t st, int64_t ld, int dtype, const int32_t *tokens,
                               float temperature, const void *saved, const float *gl, const float *ge,
                               void *gh, void *gw, void *ws)
{
    cdk::launch_head_backward({h, w, B, T, D, V, sb, st, ld, dtype}, tokens, temperature,
                              static_cast<const cdk::ScoreRow *>(saved), gl, ge, gh, gw, ws, nullptr);
}
