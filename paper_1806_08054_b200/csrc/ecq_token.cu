// C ABI of the token log-probability operators: argument checks and launches.
#include <cfloat>
#include <cstdint>

#include <cuda_runtime.h>

#include "../../include/ecq.h"
#include "ecq_host.h"
#include "ecq_token.cuh"

using namespace ecq;

namespace {

template <typename T, bool ENT, int NT>
int launch_forward(const TokenForward& P, uint64_t rows, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)(rows << P.cluster_log2));
    cfg.blockDim = dim3(NT);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 1u << P.cluster_log2;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = P.cluster_log2 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, token_logprob_kernel<T, ENT, NT>, P) != cudaSuccess) {
        cudaGetLastError();
        return ECQ_ERR_CUDA;
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return ECQ_OK;
}

template <typename T>
int launch_forward(const TokenForward& P, uint64_t rows, bool stream, cudaStream_t st) {
    if (stream) return P.entropy ? launch_forward<T, true, kTokStream>(P, rows, st) : launch_forward<T, false, kTokStream>(P, rows, st);
    return P.entropy ? launch_forward<T, true, kTokThreads>(P, rows, st) : launch_forward<T, false, kTokThreads>(P, rows, st);
}

template <typename T>
int launch_backward(const TokenBackward& P, cudaStream_t st) {
    const uint64_t tasks = P.rows * P.chunks;
    const uint32_t grid = tasks < 0x7FFFFFFFull ? (uint32_t)tasks : 0x7FFFFFFFu;
    if (P.d_entropy) token_logprob_grad_kernel<T, true><<<grid, kTokGradThreads, 0, st>>>(P);
    else token_logprob_grad_kernel<T, false><<<grid, kTokGradThreads, 0, st>>>(P);
    if (cudaGetLastError() != cudaSuccess) return ECQ_ERR_CUDA;
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return ECQ_OK;
}

// The kernels take it times log2(e).
bool positive(float x) { return x > 0.f && x * kLog2e <= FLT_MAX; }

bool bad_logits(const void* logits, int dtype, uint64_t rows, uint32_t vocab, uint64_t stride) {
    const uint32_t es = dtype_bytes(dtype);
    if (!es || !logits || !aligned_to(logits, es) || !vocab || vocab > 0x40000000u) return true;
    return rows > 0x10000000ull || (rows > 1 && (stride < vocab || stride > 0x100000000ull));
}

}  // namespace

extern "C" {

int ecq_token_logprob(const void* logits, int dtype, uint64_t rows, uint32_t vocab, uint64_t row_stride,
                      const int64_t* targets, float inv_temperature, uint32_t top, float* logprob,
                      float* entropy, float* lse, float* top_logprob, int32_t* top_index,
                      void* cuda_stream) {
    if (rows == 0) return dtype_bytes(dtype) ? ECQ_OK : ECQ_ERR_ARG;
    if (bad_logits(logits, dtype, rows, vocab, row_stride) || !positive(inv_temperature)) return ECQ_ERR_ARG;
    if (top > ECQ_TOKEN_MAX_TOP || top > vocab) return ECQ_ERR_ARG;
    if ((logprob != nullptr) != (targets != nullptr) || (top != 0) != (top_logprob != nullptr) ||
        (top != 0) != (top_index != nullptr) || (!logprob && !entropy && !lse && !top))
        return ECQ_ERR_ARG;
    if (!aligned_to(targets, 8) || !aligned_to(logprob, 4) || !aligned_to(entropy, 4) || !aligned_to(lse, 4) ||
        !aligned_to(top_logprob, 4) || !aligned_to(top_index, 4))
        return ECQ_ERR_ARG;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return ECQ_ERR_CUDA;
    TokenForward P = {logits, row_stride, targets, logprob, entropy, lse, top_logprob, top_index,
                      vocab, top, 0, inv_temperature};
    // Vectors of 16 bytes that a thread has of a row.  A row of 12 or more is split over a cluster of
    // CTAs, as long as 3 are left for each thread and there is no more than a CTA an SM, or, with 24
    // left, three.  In us, on 1, 2, 4 and 8 CTAs, with top 5 (one row: 20) and entropy:
    //     bf16   1 x 16384    6.0   6.5   6.6   7.1       200 x 50257   11.6  12.7  18.3  26.1
    //            1 x 50257   10.1   8.7   7.4   7.2       60 x 128001   14.5  10.9  10.4  12.6
    //           24 x 50257    8.9   8.2   7.3   8.0      200 x 128001   24.2  20.1  26.0  32.8
    //           60 x 50257    9.0   8.4   8.9  10.9      400 x 128001   30.7  37.3  42.1  60.0
    const uint32_t held = vocab / (16 / (uint32_t)dtype_bytes(dtype)) / kTokThreads;
    if (held >= 12)
        for (uint32_t c = 1; (1u << c) <= (uint32_t)kTokMaxCluster && held >> c >= 3; ++c)
            if (rows << c <= (uint64_t)(held >> c >= 24 ? 3 : 1) * (uint64_t)sms) P.cluster_log2 = c;
    // Half the threads a CTA where the rows are more than fit the GPU at once (2047 x 50257, top 8: 59.2
    // against 62.6 us; 400 x 50257: 20.5 against 17.2) or short (400 x 4096: 6.8 against 7.7).
    const bool stream = !P.cluster_log2 && (rows > (uint64_t)(1024 / kTokThreads) * (uint64_t)sms || held < 4);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    switch (dtype) {
        case ECQ_F32: return launch_forward<float>(P, rows, stream, st);
        case ECQ_BF16: return launch_forward<__nv_bfloat16>(P, rows, stream, st);
        default: return launch_forward<__half>(P, rows, stream, st);
    }
}

int ecq_token_logprob_grad(const void* logits, int dtype, uint64_t rows, uint32_t vocab, uint64_t row_stride,
                           const int64_t* targets, float inv_temperature, const float* lse,
                           const float* entropy, const float* d_logprob, const float* d_entropy,
                           void* d_logits, uint64_t d_row_stride, void* cuda_stream) {
    if (rows == 0) return dtype_bytes(dtype) ? ECQ_OK : ECQ_ERR_ARG;
    if (bad_logits(logits, dtype, rows, vocab, row_stride) || bad_logits(d_logits, dtype, rows, vocab, d_row_stride) ||
        !positive(inv_temperature))
        return ECQ_ERR_ARG;
    if (!lse || (d_logprob != nullptr) != (targets != nullptr) || (d_entropy && !entropy) || (!d_logprob && !d_entropy))
        return ECQ_ERR_ARG;
    if (!aligned_to(targets, 8) || !aligned_to(lse, 4) || !aligned_to(entropy, 4) || !aligned_to(d_logprob, 4) ||
        !aligned_to(d_entropy, 4))
        return ECQ_ERR_ARG;
    if (logits == d_logits && row_stride != d_row_stride && rows > 1) return ECQ_ERR_ARG;
    TokenBackward P = {logits, d_logits, rows, row_stride, d_row_stride, targets, lse, entropy, d_logprob,
                       d_entropy, vocab, 1, inv_temperature};
    const uint32_t per = kTokGradThreads * kTokGradUnroll * (16u / dtype_bytes(dtype));
    P.chunks = (vocab + per - 1) / per;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    switch (dtype) {
        case ECQ_F32: return launch_backward<float>(P, st);
        case ECQ_BF16: return launch_backward<__nv_bfloat16>(P, st);
        default: return launch_backward<__half>(P, st);
    }
}

}  // extern "C"
