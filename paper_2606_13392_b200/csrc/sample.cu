// C ABI of the choice of the next token (see include/msa.h): argument validation and dispatch; the arithmetic is in sample.cuh.
#include <cmath>

#include "sample.cuh"

using namespace msa;

template <class T>
static msa_status_t launch_sample(const SampleArgs& a, int64_t rows, cudaStream_t st) {
    StageScope sc(kStageNone, st);
    sample_kernel<T><<<(unsigned)rows, kSampleThreads, 0, st>>>(a);
    return launch_status();
}

extern "C" {

msa_status_t msa_sample(const msa_sampling_t* settings, const void* logits, int32_t logits_type, int64_t stride, int64_t n_rows,
                        int32_t vocab, const float* uniform, int64_t* token, float* logprob, msa_stream_t stream) {
    auto aligned = [](const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
    if (settings == nullptr || n_rows < 0 || vocab <= 0 || stride < vocab) return MSA_ERR_INVALID_ARG;
    if (logits_type < MSA_BF16 || logits_type > MSA_FP32) return MSA_ERR_INVALID_ARG;
    if (vocab > (1 << 21) || n_rows > 2147483647LL) return MSA_ERR_UNSUPPORTED;
    const msa_sampling_t& p = *settings;
    if (std::isnan(p.temperature) || std::isnan(p.top_p) || std::isnan(p.min_p)) return MSA_ERR_INVALID_ARG;
    if (n_rows == 0) return MSA_OK;
    if (!logits || !aligned(logits, logits_type == MSA_FP32 ? 4 : 2) || !uniform || !aligned(uniform, 4) || !token || !aligned(token, 8) ||
        !aligned(logprob, 4) || !aligned(p.temperatures, 4) || !aligned(p.top_ks, 4) || !aligned(p.top_ps, 4) || !aligned(p.min_ps, 4))
        return MSA_ERR_INVALID_ARG;
    const SampleArgs a{logits, stride, vocab, uniform, p.temperatures, p.top_ks, p.top_ps, p.min_ps,
                       p.temperature, p.top_k, p.top_p, p.min_p, token, logprob};
    cudaStream_t st = (cudaStream_t)stream;
    switch (logits_type) {
        case MSA_BF16: return launch_sample<__nv_bfloat16>(a, n_rows, st);
        case MSA_FP16: return launch_sample<__half>(a, n_rows, st);
        default: return launch_sample<float>(a, n_rows, st);
    }
}

}  // extern "C"
