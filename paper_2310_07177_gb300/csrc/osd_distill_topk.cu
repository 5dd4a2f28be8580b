// osd_distill_topk.cu -- per-position distillation loss and gradient (Eq. 2-3 of the
// paper) against compact target rows: K kept tokens, and all other tokens as one class.
//
// With c over the K + 1 classes, p from the kept values and the log-mass of the rest, and
// q_c the draft's mass in class c, the loss is D(p || q) over the classes and its
// gradient, with g_c = dD/dq_c,
//
//   dl/dz_j = q_j (g_c(j) - sum_c q_c g_c) / tau,
//
// one factor for all the other tokens and one value for each kept token.  So a row
// needs the sum of its other entries' exponentials (summed on its own: 1 - sum of the kept
// ones would cancel), K + 1 classes' worth of arithmetic, and one scaled exponential an entry.
#include <climits>
#include <cmath>
#include <cstdint>

#include "osd.h"
#include "osd_device.cuh"
#include "osd_host.hpp"

namespace osd {

constexpr int kDtThreads = 256;
constexpr int kDtMaxV = 393216;

struct DtParams {
    const void* draft;
    int P, V;
    long long dsg, dsp;
    const float* values;
    const int32_t* ids;
    const float* rest;
    int K;
    const uint8_t* mask;
    float beta;
    float c;           // log2(e) / tau
    float c_hi, c_lo;  // the same as a pair, for the K + 1 classes
    float inv_tau;
    float* loss;
    float* dlogits;
    int32_t* status;
};

// log2 of exp(rest) against exp(v / tau), rest and v / tau of any size: each product keeps
// the rounding of its leading part, so only the difference is rounded.
__device__ __forceinline__ float rest_minus(float rest, float v, float c_hi, float c_lo) {
    constexpr float kLog2eLo = 1.92596303e-8f;  // log2(e) - kLog2e
    const float a = __fmul_rn(v, c_hi), b = __fmul_rn(rest, kLog2e);
    const float ea = fmaf(v, c_lo, fmaf(v, c_hi, -a)), eb = fmaf(rest, kLog2eLo, fmaf(rest, kLog2e, -b));
    return __fadd_rn(__fadd_rn(b, -a), __fadd_rn(eb, -ea));
}

// What one class adds to the row's sums: the loss (fkl, rkl in bits with the masses' difference in
// nats apart; jsd the two divergences in bits; tvd |p - q| and q by the sign of q - p).
template <int kKind>
__device__ __forceinline__ float3 class_terms(float p, float lp, float q, float lq, float beta) {
    if constexpr (kKind == OSD_FKL || kKind == OSD_CE) {
        return make_float3(p > 0.f ? p * (lp - lq) : 0.f, q - p, 0.f);
    } else if constexpr (kKind == OSD_RKL) {
        return make_float3(q > 0.f ? q * (lq - lp) : 0.f, p - q, 0.f);
    } else if constexpr (kKind == OSD_JSD) {
        const float lm = log2f(fmaxf(fmaf(beta, p, (1.f - beta) * q), 1.17549435e-38f));
        return make_float3(p > 0.f ? p * (lp - lm) : 0.f, q > 0.f ? q * (lq - lm) : 0.f, 0.f);
    } else {
        return make_float3(fabsf(p - q), q > p ? q : 0.f, q < p ? q : 0.f);
    }
}
template <int kKind>
__device__ __forceinline__ float class_loss(float3 s, float beta) {
    if constexpr (kKind == OSD_JSD) return kLn2 * (beta * s.x + (1.f - beta) * s.y);
    if constexpr (kKind == OSD_TVD) return 0.5f * s.x;
    // sum of p log(p/q) + q - p: the last two cancel what the rounding of a normaliser
    // does to all classes alike
    return s.x == __int_as_float(0x7f800000) ? s.x : fmaf(kLn2, s.x, s.y);
}
// g_c - sum q g in nats (FKL and CE: times q, see there)
template <int kKind>
__device__ __forceinline__ float class_factor(float p, float lp, float q, float lq, float3 s, float loss, float beta) {
    if constexpr (kKind == OSD_RKL) return kLn2 * (lq - lp) - loss;
    if constexpr (kKind == OSD_JSD) {
        const float lm = log2f(fmaxf(fmaf(beta, p, (1.f - beta) * q), 1.17549435e-38f));
        return (1.f - beta) * kLn2 * ((lq - lm) - s.y);
    }
    // TVD, s_c = sign(q - p) / 2: s_c - sum q s by the masses on the two sides and on neither, so that
    // nothing cancels when one side holds almost everything
    const float eq = fmaxf(1.f - s.y - s.z, 0.f);
    return q > p ? s.z + 0.5f * eq : (q < p ? -(s.y + 0.5f * eq) : 0.5f * (s.z - s.y));
}

template <typename In, int kKind>
__global__ void __launch_bounds__(kDtThreads) distill_topk_kernel(DtParams p) {
    using E = Elem<In>;
    extern __shared__ uint32_t s_bits[];  // which entries are kept
    __shared__ float s_v[OSD_TOPK_MAX_K], s_z[OSD_TOPK_MAX_K];
    __shared__ int s_id[OSD_TOPK_MAX_K];
    __shared__ int s_bad;
    __shared__ float s_red[kDtThreads / 32];
    __shared__ float3 s_red3[kDtThreads / 32];
    __shared__ MaxIdx s_redi[kDtThreads / 32];
    const int tid = threadIdx.x;
    const long long row = blockIdx.x;
    const int V = p.V, K = p.K;
    grid_dependency_sync();
    if (p.mask && !p.mask[row]) {
        if (tid == 0) p.loss[row] = 0.f;
        return;
    }
    const In* x = static_cast<const In*>(p.draft) + (row / p.P) * p.dsg + (row % p.P) * p.dsp;
    float* out = p.dlogits + row * V;
    auto add = [](float a, float b) { return a + b; };
    auto most = [](float a, float b) { return fmaxf(a, b); };
    if (tid == 0) s_bad = 0;
    for (int i = tid; i < (V + 31) / 32; i += kDtThreads) s_bits[i] = 0u;
    __syncthreads();
    MaxIdx best{kNegInf, INT_MAX};  // the largest value, with the lowest id
    for (int i = tid; i < K; i += kDtThreads) {
        const int id = p.ids[row * K + i];
        const float v = p.values[row * K + i];
        s_id[i] = id;
        s_v[i] = v;
        if (id < 0) continue;
        if (id >= V) {
            s_bad = 1;
            continue;
        }
        if (atomicOr(&s_bits[id >> 5], 1u << (id & 31)) >> (id & 31) & 1u) s_bad = 1;
        s_z[i] = E::load(x + id);
        best = merge_mi(best, MaxIdx{v, id});
    }
    best = block_reduce<kDtThreads>(best, [](MaxIdx a, MaxIdx b) { return merge_mi(a, b); }, s_redi);
    const bool bad = s_bad;
    const float vref = best.m, rest = (p.rest && kKind != OSD_CE) ? p.rest[row] : kNegInf;
    if (bad || fmaxf(vref, rest) == kNegInf) {  // a bad row, or no target mass
        for (int j = tid; j < V; j += kDtThreads) out[j] = 0.f;
        if (tid == 0) {
            p.loss[row] = bad ? __int_as_float(0x7fc00000) : 0.f;
            if (bad && p.status) atomicExch(p.status, static_cast<int32_t>(OSD_ERR_INVALID_ARG));
        }
        return;
    }
    // ---- the target: t_c = log2 of the class's weight against the largest kept value's
    const float c = p.c, ch = p.c_hi, cl = p.c_lo;
    const float tr = rest == kNegInf ? kNegInf : (vref == kNegInf ? 0.f : rest_minus(rest, vref, ch, cl));
    const float mt = vref == kNegInf ? tr : fmaxf(0.f, tr);
    auto t_of = [&](int i) { return (s_v[i] == kNegInf) ? kNegInf : mul_c(s_v[i] - vref, ch, cl) - mt; };
    float L = 0.f;
    for (int i = tid; i < K; i += kDtThreads)
        if (s_id[i] >= 0) L += ex2(t_of(i));
    L = block_reduce<kDtThreads>(L, add, s_red) + ex2(tr - mt);
    const float lgL = log2f(L), inv_L = 1.f / L;
    // ---- the draft: the sum of the others against their largest, m
    auto kept = [&](int j) { return (s_bits[j >> 5] >> (j & 31)) & 1u; };
    float m = kNegInf;
    for (int j = tid; j < V; j += kDtThreads)
        if (!kept(j)) m = fmaxf(m, E::load(x + j));
    m = block_reduce<kDtThreads>(m, most, s_red);
    const bool others = m != kNegInf;
    float zmax = kNegInf;
    for (int i = tid; i < K; i += kDtThreads)
        if (s_id[i] >= 0) zmax = fmaxf(zmax, s_z[i]);
    zmax = block_reduce<kDtThreads>(zmax, most, s_red);
    if (!others) m = zmax;
    float S = 0.f;
    if (others)
        for (int j = tid; j < V; j += kDtThreads)
            if (!kept(j)) S += ex2((E::load(x + j) - m) * c);
    S = block_reduce<kDtThreads>(S, add, s_red);
    const float mx = fmaxf(others ? 0.f : kNegInf, mul_c(zmax - m, ch, cl));
    float Z = 0.f;
    for (int i = tid; i < K; i += kDtThreads)
        if (s_id[i] >= 0) Z += ex2(mul_c(s_z[i] - m, ch, cl) - mx);
    Z = block_reduce<kDtThreads>(Z, add, s_red) + S * ex2(-mx);
    const float lgZ = log2f(Z), inv_Z = 1.f / Z;
    // ---- the classes
    const float lqr = others ? (log2f(S) - mx) - lgZ : kNegInf, qr = S * ex2(-mx) * inv_Z;
    const float lpr = kKind == OSD_CE ? kNegInf : (tr - mt) - lgL, pr = kKind == OSD_CE ? 0.f : ex2(tr - mt) * inv_L;
    auto target = [&](int i, float& pc, float& lp) {
        if constexpr (kKind == OSD_CE) {
            pc = s_id[i] == best.i ? 1.f : 0.f;
            lp = pc > 0.f ? 0.f : kNegInf;
        } else {
            const float t = t_of(i);
            pc = ex2(t) * inv_L;
            lp = t - lgL;
        }
    };
    auto draft = [&](int i, float& qc, float& lq) {
        const float e = mul_c(s_z[i] - m, ch, cl) - mx;
        qc = ex2(e) * inv_Z;
        lq = e - lgZ;
    };
    float3 s = tid == 0 ? class_terms<kKind>(pr, lpr, qr, lqr, p.beta) : make_float3(0.f, 0.f, 0.f);
    for (int i = tid; i < K; i += kDtThreads) {
        if (s_id[i] < 0) continue;
        float pc, lp, qc, lq;
        target(i, pc, lp);
        draft(i, qc, lq);
        const float3 t = class_terms<kKind>(pc, lp, qc, lq, p.beta);
        s = make_float3(s.x + t.x, s.y + t.y, s.z + t.z);
    }
    s = block_reduce<kDtThreads>(s, [](float3 a, float3 b) { return make_float3(a.x + b.x, a.y + b.y, a.z + b.z); }, s_red3);
    const float loss = class_loss<kKind>(s, p.beta);
    if (tid == 0) p.loss[row] = loss;
    const bool dead = kKind == OSD_RKL && !(loss < __int_as_float(0x7f800000));  // +inf: no gradient
    // ---- the gradient: others first, then the kept entries over them
    float coef = 0.f;
    if (others && !dead) {
        const float w = ex2(-mx) * inv_Z;
        if constexpr (kKind == OSD_FKL || kKind == OSD_CE) coef = w - pr / S;  // q_j - p_R q_j / q_R
        else coef = w * class_factor<kKind>(pr, lpr, qr, lqr, s, loss, p.beta);
        coef *= p.inv_tau;
    }
    for (int j = tid; j < V; j += kDtThreads)
        if (!kept(j)) out[j] = others ? coef * ex2((E::load(x + j) - m) * c) : 0.f;
    for (int i = tid; i < K; i += kDtThreads) {
        if (s_id[i] < 0) continue;
        float pc, lp, qc, lq, g = 0.f;
        target(i, pc, lp);
        draft(i, qc, lq);
        if constexpr (kKind == OSD_FKL || kKind == OSD_CE) g = qc - pc;
        else if (qc > 0.f && !dead) g = qc * class_factor<kKind>(pc, lp, qc, lq, s, loss, p.beta);
        out[s_id[i]] = g * p.inv_tau;
    }
}

template <typename In>
static cudaError_t launch_distill_topk(osd_loss kind, const DtParams& dp, unsigned rows, cudaStream_t s) {
    const size_t smem = size_t((dp.V + 31) / 32) * 4;
    const dim3 grid(rows), block(kDtThreads);
    auto go = [&](auto* kernel) -> cudaError_t {
        if (smem > 24 * 1024) {
            const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kDtMaxV / 8);
            if (e != cudaSuccess) return e;
        }
        return launch_ex(true, kernel, grid, block, smem, s, 1, dp);
    };
    switch (kind) {
        case OSD_FKL: return go(distill_topk_kernel<In, OSD_FKL>);
        case OSD_RKL: return go(distill_topk_kernel<In, OSD_RKL>);
        case OSD_JSD: return go(distill_topk_kernel<In, OSD_JSD>);
        case OSD_TVD: return go(distill_topk_kernel<In, OSD_TVD>);
        default: return go(distill_topk_kernel<In, OSD_CE>);
    }
}

}  // namespace osd

extern "C" osd_status osd_distill_topk(const void* draft_logits, osd_dtype dtype, int G, int P, int V, int64_t d_stride_g,
                                       int64_t d_stride_p, const float* values, const int32_t* ids, const float* rest,
                                       int K, const uint8_t* mask, osd_loss kind, float beta, float temperature,
                                       float* loss, float* dlogits, int32_t* status, void* stream) {
    using namespace osd;
    if (dtype != OSD_F32 && dtype != OSD_BF16) return OSD_ERR_INVALID_ARG;
    if (kind < OSD_FKL || kind > OSD_CE) return OSD_ERR_INVALID_ARG;
    if (!(temperature > 0.f) || !std::isfinite(temperature)) return OSD_ERR_INVALID_ARG;
    if (G < 0 || P < 0 || V < 1 || K < 1 || d_stride_g < 0 || d_stride_p < 0) return OSD_ERR_INVALID_ARG;
    if (kind == OSD_JSD && !(beta >= 0.f && beta <= 1.f)) return OSD_ERR_INVALID_ARG;
    if (kind == OSD_RKL && !rest && K < V) return OSD_ERR_INVALID_ARG;  // every row's loss would be +inf
    if (K > OSD_TOPK_MAX_K || V > kDtMaxV) return OSD_ERR_UNSUPPORTED;
    if (!aligned_to(status, 4)) return OSD_ERR_INVALID_ARG;
    const long long rows = static_cast<long long>(G) * P;
    if (rows > INT_MAX) return OSD_ERR_UNSUPPORTED;
    if (rows > 0) {
        if (!draft_logits || !values || !ids || !loss || !dlogits) return OSD_ERR_INVALID_ARG;
        if (!aligned_to(draft_logits, dtype_size(dtype)) || !aligned_to(values, 4) || !aligned_to(ids, 4) ||
            !aligned_to(rest, 4) || !aligned_to(loss, 4) || !aligned_to(dlogits, 4))
            return OSD_ERR_INVALID_ARG;
    }
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (status && cudaMemsetAsync(status, 0, sizeof(int32_t), s) != cudaSuccess) return OSD_ERR_CUDA;
    if (rows == 0) return OSD_OK;
    DtParams dp = {};
    dp.draft = draft_logits; dp.P = P; dp.V = V; dp.dsg = d_stride_g; dp.dsp = d_stride_p;
    dp.values = values; dp.ids = ids; dp.rest = rest; dp.K = K; dp.mask = mask; dp.beta = beta;
    split_scale(temperature, &dp.c_hi, &dp.c_lo);
    dp.c = static_cast<float>(1.4426950408889634074 / static_cast<double>(temperature));
    dp.inv_tau = static_cast<float>(1.0 / static_cast<double>(temperature));
    dp.loss = loss; dp.dlogits = dlogits; dp.status = status;
    return from_cuda(dtype == OSD_BF16 ? launch_distill_topk<__nv_bfloat16>(kind, dp, static_cast<unsigned>(rows), s)
                                       : launch_distill_topk<float>(kind, dp, static_cast<unsigned>(rows), s));
}
