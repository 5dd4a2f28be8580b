// osd_topk.cu -- the K largest logits of a row with their ids, and the log of the mass of
// all other entries: the compact form in which the buffer R of Algorithm 1 keeps a
// target row.
//
// One CTA per row.  Logits are compared as 32-bit keys of the same order; the K-th
// largest key T is found bit by bit (the largest T that at least K entries reach), the
// entries above it are collected in any order and those equal to it in index order, and
// each entry's place is the number of entries that come before it.
#include <climits>
#include <cmath>
#include <cstdint>

#include "osd.h"
#include "osd_device.cuh"
#include "osd_host.hpp"

namespace osd {

constexpr int kTopThreads = 256;

struct TopParams {
    const void* logits;
    int P, V;
    long long sg, sp;
    const uint8_t* mask;
    int K;
    float c;        // log2(e) / tau
    float tau;
    float* values;
    int32_t* ids;
    float* rest;
};

// Unsigned keys in the order of the floats; -0 and 0 have the same.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}

template <typename In>
__global__ void __launch_bounds__(kTopThreads) topk_kernel(TopParams p) {
    using E = Elem<In>;
    __shared__ uint32_t s_key[OSD_TOPK_MAX_K];
    __shared__ int s_id[OSD_TOPK_MAX_K];
    __shared__ int s_n, s_red[kTopThreads / 32];
    __shared__ float s_sum[kTopThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long row = blockIdx.x;
    grid_dependency_sync();
    if (p.mask && !p.mask[row]) return;
    const int V = p.V, K = p.K;
    const In* x = static_cast<const In*>(p.logits) + (row / p.P) * p.sg + (row % p.P) * p.sp;
    auto count = [&](auto pred) {
        int n = 0;
        for (int j = tid; j < V; j += kTopThreads) n += pred(key_of(E::load(x + j))) ? 1 : 0;
        return block_reduce<kTopThreads>(n, [](int a, int b) { return a + b; }, s_red);
    };
    uint32_t T = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t at = T | (1u << bit);
        if (count([at](uint32_t k) { return k >= at; }) >= K) T = at;
    }
    if (tid == 0) s_n = 0;
    __syncthreads();
    for (int j = tid; j < V; j += kTopThreads) {
        const uint32_t k = key_of(E::load(x + j));
        if (k > T) {
            const int at = atomicAdd(&s_n, 1);
            s_key[at] = k;
            s_id[at] = j;
        }
    }
    __syncthreads();
    if (warp == 0) {  // entries equal to T, the lowest indices
        int n = s_n;
        for (int c = 0; c < V && n < K; c += 32) {
            const bool eq = c + lane < V && key_of(E::load(x + c + lane)) == T;
            const unsigned m = __ballot_sync(0xffffffffu, eq);
            const int at = n + __popc(m & ((1u << lane) - 1u));
            if (eq && at < K) {
                s_key[at] = T;
                s_id[at] = c + lane;
            }
            n += __popc(m);
        }
    }
    __syncthreads();
    for (int i = tid; i < K; i += kTopThreads) {
        const uint32_t k = s_key[i];
        const int id = s_id[i];
        int r = 0;
        for (int j = 0; j < K; ++j) r += (s_key[j] > k || (s_key[j] == k && s_id[j] < id)) ? 1 : 0;
        p.values[row * K + r] = value_of(k);
        p.ids[row * K + r] = id;
    }
    if (!p.rest) return;
    // the others: everything below T, and the entries equal to it that were not taken;
    // the reference of the sum is the largest of them
    uint32_t top = 0;
    int reach = 0;
    for (int j = tid; j < V; j += kTopThreads) {
        const uint32_t k = key_of(E::load(x + j));
        reach += k >= T ? 1 : 0;
        if (k < T) top = max(top, k);
    }
    reach = block_reduce<kTopThreads>(reach, [](int a, int b) { return a + b; }, s_red);
    top = block_reduce<kTopThreads>(top, [](uint32_t a, uint32_t b) { return max(a, b); }, reinterpret_cast<uint32_t*>(s_red));
    const int left = reach - K;  // equal to T and not taken
    const float m = value_of(left > 0 ? T : top);
    if (m == kNegInf || (left <= 0 && top == 0)) {
        if (tid == 0) p.rest[row] = kNegInf;
        return;
    }
    float s = 0.f;
    for (int j = tid; j < V; j += kTopThreads) {
        const float v = E::load(x + j);
        if (key_of(v) < T) s += ex2((v - m) * p.c);
    }
    s = block_reduce<kTopThreads>(s, [](float a, float b) { return a + b; }, s_sum);
    if (tid == 0) {
        s += static_cast<float>(max(left, 0));
        p.rest[row] = fmaf(log2f(s), kLn2, __fdiv_rn(m, p.tau));
    }
}

}  // namespace osd

extern "C" osd_status osd_topk(const void* logits, osd_dtype dtype, int G, int P, int V, int64_t stride_g,
                               int64_t stride_p, const uint8_t* mask, int K, float temperature, float* values,
                               int32_t* ids, float* rest, int32_t* status, void* stream) {
    using namespace osd;
    if (dtype != OSD_F32 && dtype != OSD_BF16) return OSD_ERR_INVALID_ARG;
    if (!(temperature > 0.f) || !std::isfinite(temperature)) return OSD_ERR_INVALID_ARG;
    if (G < 0 || P < 0 || V < 1 || K < 1 || K > V) return OSD_ERR_INVALID_ARG;
    if (stride_g < 0 || stride_p < 0) return OSD_ERR_INVALID_ARG;
    if (K > OSD_TOPK_MAX_K || V > OSD_VERIFY_MAX_V) return OSD_ERR_UNSUPPORTED;
    if (!aligned_to(status, 4)) return OSD_ERR_INVALID_ARG;
    const long long rows = static_cast<long long>(G) * P;
    if (rows > INT_MAX) return OSD_ERR_UNSUPPORTED;
    if (rows > 0) {
        if (!logits || !values || !ids) return OSD_ERR_INVALID_ARG;
        if (!aligned_to(logits, dtype_size(dtype)) || !aligned_to(values, 4) || !aligned_to(ids, 4) || !aligned_to(rest, 4))
            return OSD_ERR_INVALID_ARG;
    }
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (status && cudaMemsetAsync(status, 0, sizeof(int32_t), s) != cudaSuccess) return OSD_ERR_CUDA;
    if (rows == 0) return OSD_OK;
    const TopParams tp = {logits, P, V, stride_g, stride_p, mask, K,
                          static_cast<float>(1.4426950408889634074 / static_cast<double>(temperature)),
                          temperature, values, ids, rest};
    const dim3 grid(static_cast<unsigned>(rows)), block(kTopThreads);
    return from_cuda(dtype == OSD_BF16 ? launch_ex(true, topk_kernel<__nv_bfloat16>, grid, block, 0, s, 1, tp)
                                       : launch_ex(true, topk_kernel<float>, grid, block, 0, s, 1, tp));
}
