// C ABI of the choice of the next token (see include/msa.h): argument validation and dispatch; the arithmetic is in sample.cuh.
#include <algorithm>
#include <cmath>

#include "sample.cuh"

using namespace msa;

// CTAs of a row: as many as are resident at once (two per SM) and have some 8 KB of it each.
static int sample_ctas(int dev, int64_t rows, int64_t row_bytes) {
    static int sms[64] = {0};  // per device
    if (sms[dev] == 0 && cudaDeviceGetAttribute(&sms[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cuda_failed();
        sms[dev] = 148;
    }
    return (int)std::max<int64_t>(1, std::min<int64_t>({kSampleCtas, 2 * (int64_t)sms[dev] / rows, row_bytes / 8192}));
}

template <class T>
static msa_status_t launch_sample(const SampleArgs& a, int64_t rows, cudaStream_t st) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) cuda_failed();
    dev = dev < 0 || dev >= 64 ? 0 : dev;
    static bool attr_set[64] = {false};  // per device
    if (!attr_set[dev]) {
        if (cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SampleSmem)) != cudaSuccess)
            return cuda_failed();
        attr_set[dev] = true;
    }
    const int ctas = sample_ctas(dev, rows, (int64_t)a.vocab * (int64_t)sizeof(T));
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = ctas;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * ctas));
    cfg.blockDim = dim3(kSampleThreads);
    cfg.dynamicSmemBytes = sizeof(SampleSmem);
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    StageScope sc(kStageNone, st);
    return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a) == cudaSuccess ? MSA_OK : cuda_failed();
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
