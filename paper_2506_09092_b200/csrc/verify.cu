// Entry point of include/cudallm_cache.h for drafted tokens: validation, the split over the vocabulary, launch.
#include "../../include/cudallm_cache.h"

#include <algorithm>

#include "runtime.h"
#include "draft_verify.cuh"

using namespace cudallm;

namespace {

constexpr int64_t kMaxDim = (int64_t(1) << 31) - 1024;
constexpr int64_t kMaxElems = int64_t(1) << 46;
constexpr int64_t kPlanSms = 148;

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool off(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// wide: all rows begin on 16 bytes
template <typename T> int launch(const VerifyParams &v, bool wide, dim3 grid, cudaStream_t stream)
{
    return rt_launch_cluster(wide ? draft_verify_kernel<T, 16 / (int)sizeof(T)> : draft_verify_kernel<T, 1>, grid, (unsigned)v.cluster,
                             kVerifyThreads, 0, stream, v);
}

}  // namespace

extern "C" int cudallm_draft_verify(const void *p, const void *q, const int32_t *drafts, const int32_t *draft_lens, const float *u,
                                    int32_t *tokens, int32_t *accepted, int64_t batch, int64_t n, int64_t vocab, int64_t ldp,
                                    int64_t ldq, int dtype, void *stream_v)
{
    if (dtype != CUDALLM_F32 && dtype != CUDALLM_BF16 && dtype != CUDALLM_F16) return CUDALLM_ERR_INVALID_DTYPE;
    if (batch < 0 || n < 0 || n > kMaxDim || vocab < 1 || vocab > kMaxDim || batch > kMaxDim / (n + 1)) return CUDALLM_ERR_INVALID_DIM;
    if (batch == 0) return CUDALLM_OK;
    if (ldp < vocab || (q && n > 0 && ldq < vocab)) return CUDALLM_ERR_INVALID_LD;
    if ((long double)ldp * batch * (n + 1) > (long double)kMaxElems || (q && (long double)ldq * batch * n > (long double)kMaxElems))
        return CUDALLM_ERR_INVALID_DIM;
    if (!p || (n > 0 && !drafts) || !u || !tokens || !accepted) return CUDALLM_ERR_INVALID_POINTER;
    const int es = dtype == CUDALLM_F32 ? 4 : 2;
    if (off(p, es) || off(q, es) || off(drafts, 4) || off(draft_lens, 4) || off(u, 4) || off(tokens, 4) || off(accepted, 4))
        return CUDALLM_ERR_MISALIGNED;
    int dev = 0, sms = 0;
    const int st = rt_current_device(&dev, &sms);
    if (st != CUDALLM_OK) return st;
    VerifyParams v{};
    v.p = p; v.q = n > 0 ? q : nullptr; v.drafts = drafts; v.draft_lens = draft_lens; v.u = u; v.tokens = tokens; v.accepted = accepted;
    v.ldp = ldp; v.ldq = ldq; v.n = (int)n; v.vocab = (int)vocab;
    // CTAs of a sequence: two an SM in all, and four chunks of 512 at least for one.  (One row of 4000, 16000, 32000, 128000 fp32
    // values on one CTA 5.5, 7.1, 11.5, 29.1 us, on eight 6.3, 5.5, 6.8, 8.4; 64 rows of 128000 on 1, 2, 4, 8: 33.8, 24.1, 16.4, 21.1.)
    const int64_t want = std::min<int64_t>({int64_t(kVerifyCluster), 2 * kPlanSms / batch, vocab / (4 * kVerifyChunk)});
    v.cluster = (int)std::max<int64_t>(want, 1);
    v.chunk = (int)(kVerifyChunk * cdiv(vocab, (int64_t)kVerifyChunk * kVerifyChunks * v.cluster));
    v.chunks = (int)cdiv(cdiv(vocab, v.chunk), v.cluster);
    if (batch * v.cluster > kMaxDim) return CUDALLM_ERR_INVALID_DIM;
    const dim3 grid((unsigned)(batch * v.cluster));
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    const bool wide = !off(p, 16) && !off(v.q, 16) && ldp * es % 16 == 0 && (!v.q || ldq * es % 16 == 0);
    if (dtype == CUDALLM_F32) return launch<float>(v, wide, grid, stream);
    return dtype == CUDALLM_BF16 ? launch<__nv_bfloat16>(v, wide, grid, stream) : launch<__half>(v, wide, grid, stream);
}
