// osd_verify_probs.cu -- speculative-sampling verification (Section 3 and
// Appendix A.1 of the paper) against probabilities the caller has made, with
// drafts of different lengths and drafts without a distribution.
//
// The tests u q(y) < p(y) need two entries a position, all fetched at once; the
// first failure (or the last draft) says which one pair of rows the extra token is
// drawn from, and only that pair is read.
//
// Every probability counts as an integer multiple of 2^-62, so the weights
// max(0, p - q) and all their sums are integers: exact, in any order.
#include <climits>
#include <cstdint>

#include "osd.h"
#include "osd_device.cuh"
#include "osd_host.hpp"

namespace osd {

constexpr int kProbThreads = 256;
constexpr int kProbWarps = kProbThreads / 32;

struct ProbParams {
    const void* draft;   // nullable
    const void* target;
    int k, V;
    long long dsb, dsi, tsb, tsi;
    const int32_t* tokens;
    const int32_t* lens;  // nullable
    const float* uniforms;
    int32_t* accepted;
    int32_t* out_tokens;
    uint8_t* mask;
};

// x in [0, 2) as a multiple of 2^-62, rounded to nearest, ties to even (0 for others).
__device__ __forceinline__ unsigned long long fix62(float x) {
    const uint32_t bits = __float_as_uint(x);
    const int e = static_cast<int>(bits >> 23);  // with the sign: negative values have e >= 256
    if (e == 0 || e > 127) return 0ull;          // below 2^-126, or 2 and above
    const unsigned long long m = (bits & 0x7fffffu) | 0x800000u;
    const int sh = e - 150 + 62;                 // x = m 2^(e - 150)
    if (sh >= 0) return m << sh;
    if (sh < -25) return 0ull;
    const unsigned long long half = 1ull << (-sh - 1), v = m >> -sh, rem = m & ((half << 1) - 1);
    return v + ((rem > half || (rem == half && (v & 1ull))) ? 1ull : 0ull);
}

template <typename In>
__global__ void __launch_bounds__(kProbThreads) verify_probs_kernel(ProbParams p) {
    using E = Elem<In>;
    __shared__ unsigned long long s_warp[kProbWarps];
    __shared__ int s_a, s_n, s_y;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.x, k = p.k, V = p.V;
    grid_dependency_sync();
    const In* target = static_cast<const In*>(p.target) + b * p.tsb;
    const In* draft = p.draft ? static_cast<const In*>(p.draft) + b * p.dsb : nullptr;
    const int32_t* y = p.tokens + size_t(b) * k;
    const float* u = p.uniforms + size_t(b) * (k + 1);
    int32_t* out = p.out_tokens + size_t(b) * (k + 1);
    if (warp == 0) {
        const int n = p.lens ? p.lens[b] : k;
        bool bad = n < 0 || n > k;
        int a = n;
        for (int c = 0; c < n && !bad; c += 32) {
            const int i = c + lane;
            bool fail = false, off = false;
            if (i < n) {
                const int t = y[i];
                off = t < 0 || t >= V;
                if (!off) {
                    const float py = E::load(target + i * p.tsi + t), qy = draft ? E::load(draft + i * p.dsi + t) : 1.f;
                    fail = !(static_cast<double>(u[i]) * static_cast<double>(qy) < static_cast<double>(py));  // exact
                }
            }
            bad = __any_sync(0xffffffffu, off);
            const unsigned f = __ballot_sync(0xffffffffu, fail);
            if (f && a == n) a = c + __ffs(f) - 1;
        }
        if (lane == 0) {
            s_a = bad ? -1 : a;
            s_n = n;
            s_y = (!bad && a < n) ? y[a] : -1;
        }
    }
    __syncthreads();
    const int a = s_a, n = s_n;
    if (tid == 0) p.accepted[b] = a;
    for (int i = tid; i <= k; i += kProbThreads)
        if (i != a) out[i] = i < a ? y[i] : -1;
    for (int i = tid; i < k; i += kProbThreads) p.mask[size_t(b) * k + i] = (i == a && a < n) ? 1 : 0;
    if (a < 0) return;
    const In* prow = target + a * p.tsi;
    const In* qrow = (draft && a < n) ? draft + a * p.dsi : nullptr;
    const int hot = draft ? -1 : s_y;  // the entry a draft without a distribution holds
    auto weight = [&](int j) -> unsigned long long {
        const unsigned long long P = fix62(E::load(prow + j));
        const unsigned long long Q = qrow ? fix62(E::load(qrow + j)) : (j == hot ? 1ull << 62 : 0ull);
        return P > Q ? P - Q : 0ull;
    };
    const int per = (V + kProbWarps - 1) / kProbWarps;
    const int j0 = min(V, warp * per), j1 = min(V, j0 + per);
    unsigned long long mine = 0ull;
    for (int j = j0 + lane; j < j1; j += 32) mine += weight(j);
    mine = warp_sum_u64(mine);
    if (lane == 0) s_warp[warp] = mine;
    __syncthreads();
    unsigned long long W = 0ull, base = 0ull;
    for (int w = 0; w < kProbWarps; ++w) W += s_warp[w];
    const unsigned long long tau = fix_scale(u[k], W);
    int owner = -1;
    if (W > 0ull && tau < W) {
        // (bounded: the sums of rows outside the domain may wrap)
        for (owner = 0; owner < kProbWarps - 1 && base + s_warp[owner] <= tau; ++owner) base += s_warp[owner];
    }
    if (owner >= 0 ? warp == owner : warp == 0) {
        int token = -1;
        if (owner >= 0) {
            for (int c = j0; c < j1 && token < 0; c += 32) {
                const unsigned long long w = c + lane < j1 ? weight(c + lane) : 0ull;
                const unsigned long long incl = base + warp_incl_scan_u64(w);
                const unsigned hit = __ballot_sync(0xffffffffu, incl > tau);
                if (hit) token = c + __ffs(hit) - 1;
                base = __shfl_sync(0xffffffffu, incl, 31);
            }
        } else if (W > 0ull) {  // u >= 1: the largest entry with weight
            for (int j = lane; j < V; j += 32)
                if (weight(j)) token = j;
            token = warp_reduce(token, [](int x, int z) { return max(x, z); });
        } else {  // no weight anywhere: the first maximum of p_a
            MaxIdx acc{kNegInf, INT_MAX};
            for (int j = lane; j < V; j += 32) {
                const float x = E::load(prow + j);
                if (x > acc.m) acc = MaxIdx{x, j};
            }
            acc = warp_reduce(acc, [](MaxIdx x, MaxIdx z) { return merge_mi(x, z); });
            token = acc.i;
        }
        if (lane == 0) out[a] = (token >= 0 && token < V) ? token : 0;
    }
}

}  // namespace osd

extern "C" osd_status osd_verify_probs(const void* draft_probs, const void* target_probs, osd_dtype dtype, int B, int k,
                                       int V, int64_t d_stride_b, int64_t d_stride_i, int64_t t_stride_b,
                                       int64_t t_stride_i, const int32_t* draft_tokens, const int32_t* draft_lens,
                                       const float* uniforms, int32_t* accepted, int32_t* out_tokens,
                                       uint8_t* mismatch_mask, void* stream) {
    using namespace osd;
    if (dtype != OSD_F32 && dtype != OSD_BF16) return OSD_ERR_INVALID_ARG;
    if (B < 0 || k < 0 || V < 1) return OSD_ERR_INVALID_ARG;
    if (d_stride_b < 0 || d_stride_i < 0 || t_stride_b < 0 || t_stride_i < 0) return OSD_ERR_INVALID_ARG;
    if (k > OSD_VERIFY_MAX_K || V > OSD_VERIFY_MAX_V) return OSD_ERR_UNSUPPORTED;
    if (B == 0) return OSD_OK;
    if (!target_probs || !uniforms || !accepted || !out_tokens) return OSD_ERR_INVALID_ARG;
    if (k > 0 && (!draft_tokens || !mismatch_mask)) return OSD_ERR_INVALID_ARG;
    const size_t es = dtype_size(dtype);
    if (!aligned_to(target_probs, es) || (draft_probs && !aligned_to(draft_probs, es)) || !aligned_to(draft_tokens, 4) ||
        !aligned_to(draft_lens, 4) || !aligned_to(uniforms, 4) || !aligned_to(accepted, 4) || !aligned_to(out_tokens, 4))
        return OSD_ERR_INVALID_ARG;
    ProbParams pp = {draft_probs, target_probs, k, V, d_stride_b, d_stride_i, t_stride_b, t_stride_i,
                     draft_tokens, draft_lens, uniforms, accepted, out_tokens, mismatch_mask};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid(static_cast<unsigned>(B)), block(kProbThreads);
    return from_cuda(dtype == OSD_BF16 ? launch_ex(true, verify_probs_kernel<__nv_bfloat16>, grid, block, 0, s, 1, pp)
                                       : launch_ex(true, verify_probs_kernel<float>, grid, block, 0, s, 1, pp));
}
