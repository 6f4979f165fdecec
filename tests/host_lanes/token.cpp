// The token losses' launches (TOKEN_LOSS: token_loss.hip with each launch as a call of
// lanes::launch) as C functions of host memory.
#include "lanes.h"
#include TOKEN_LOSS

extern "C" size_t host_workspace(int64_t R, int64_t V, int dtype, int top)
{
    return cdk::rows_workspace_bytes(R, V, dtype, top);
}
extern "C" void host_score(const void *x, int64_t B, int64_t T, int64_t V, int64_t sb, int64_t st, int dtype,
                           const int32_t *tokens, float temperature, int top, float *logprob, float *entropy,
                           float *top_logprob, int32_t *top_token, void *saved, void *ws)
{
    cdk::launch_score_forward({x, B, T, V, sb, st, dtype}, tokens, temperature, top, logprob, entropy,
                              top_logprob, top_token, static_cast<cdk::ScoreRow *>(saved), ws, nullptr);
}
extern "C" void host_score_grad(const void *x, int64_t B, int64_t T, int64_t V, int64_t sb, int64_t st,
                                int dtype, const int32_t *tokens, float temperature, const void *saved,
                                const float *gl, const float *ge, void *gx)
{
    cdk::launch_score_backward({x, B, T, V, sb, st, dtype}, tokens, temperature,
                               static_cast<const cdk::ScoreRow *>(saved), gl, ge, gx, nullptr);
}
extern "C" void host_distill(const void *x, int64_t B, int64_t T, int64_t V, int64_t sb, int64_t st, int dtype,
                             int K, const int32_t *ids, const void *teacher, int teacher_dtype,
                             float temperature, float *loss, void *saved, void *ws)
{
    cdk::launch_distill_forward({x, B, T, V, sb, st, dtype}, K, ids, teacher, teacher_dtype, temperature, loss,
                                static_cast<cdk::DistillRow *>(saved), ws, nullptr);
}
extern "C" void host_distill_grad(const void *x, int64_t B, int64_t T, int64_t V, int64_t sb, int64_t st,
                                  int dtype, int K, const int32_t *ids, const void *teacher,
                                  int teacher_dtype, float temperature, const void *saved, const float *g,
                                  void *gx)
{
    cdk::launch_distill_backward({x, B, T, V, sb, st, dtype}, K, ids, teacher, teacher_dtype, temperature,
                                 static_cast<const cdk::DistillRow *>(saved), g, gx, nullptr);
}
