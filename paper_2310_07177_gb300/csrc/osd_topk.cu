// osd_topk.cu -- the K largest logits of a row with their ids, and the log of the mass of
// all other entries: the compact form in which the buffer R of Algorithm 1 keeps a
// target row.
//
// One thread-block cluster per row, each CTA with a span of it that is read twice, the second time
// from L2:
//
//   sweep 1  the maximum of each of several K groups of 16-byte chunks; theta, which K of these
//            reach and few more, from a histogram: K entries at least are theta or larger,
//            and few more where large entries lie anyhow;
//   sweep 2  the sum of the exponentials of the chunks below theta, and a list of the
//            others, whose entries are then taken one by one: those from theta on are the
//            candidates;
//   finish   one CTA ranks the candidates (value, then index) by a histogram of their values.
//            Those past the K-th join the sum.
//
// Rows with more candidates than there is room for (many equal entries, or large ones
// crowded in few groups) go on to the exact K-th largest value, counted bit by bit over the
// row, and take the entries equal to it in index order.
//
// @@
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "osd.h"
#include "osd_device.cuh"
#include "osd_host.hpp"

namespace osd {

#ifndef TOPK_C
#define TOPK_T 256
#define TOPK_R 1280
#define TOPK_C(bytes, rows) int((bytes + 72 * 1024 - 1) / (72 * 1024)) * (rows <= 152 ? 4 : 1)
#endif

constexpr int kTopMaxCluster = 8;
constexpr int kTopBins = 512;        // bins of a histogram over a range of keys
constexpr int kTopCrowd = 48;        // candidates of one bin that are ranked by comparing; with more all are sorted
// Exponentials (at most 1) of candidates, whose order is that of atomics, are added as whole multiples
// of 2^-40, so that the sum does not depend on it.
constexpr float kTopFix = 0x1p40f;

struct TopParams {
    const void* logits;
    int P, V;
    long long sg, sp;
    const uint8_t* mask;
    int K;
    float c;  // log2(e) / tau
    float tau;
    float* values;
    int32_t* ids;
    float* rest;
    int csize;    // CTAs per row
    int span;     // positions per CTA: whole chunks
    int room;     // candidates a CTA can hold, a power of two
    int groups;   // maxima per thread
};

// Unsigned keys in the order of the floats; -0 and 0 have the same.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}
constexpr float kLn2Lo = -1.90465421e-9f;  // ln 2 - kLn2
constexpr uint32_t kKeyNegInf = 0x007fffffu;

// What the CTAs of a cluster tell each other at one point.
struct TopPart {
    int n;      // candidates, or a count
    int m;      // another count
    float s;    // a sum
    float top;  // a maximum
};

// Where bin b lies: a lane of the scan reads 8 or 16 neighbouring bins, and the lanes' first ones
// fall on different banks.
__device__ __forceinline__ int top_slot(int b) { return b + (b >> 4); }

template <int kWarps> struct TopSmem {
    TopPart parts[2][kTopMaxCluster];  // slot r from CTA r; alternately
    TopPart mine;
    int n, crowd;
    uint32_t T, kmax;
    int bin, reach, above;  // of a histogram: the bin of the K-th largest, entries from it on, past it
    float ref;
    unsigned long long left;
    int warp_i[kWarps];
    float warp_f[kWarps];
    uint32_t warp_hi[kWarps], warp_lo[kWarps];
    int hist[kTopBins + 32], base[kTopBins + 32];  // entries per bin, and in the bins above it (at top_slot)
};

__device__ __forceinline__ void st_dsmem_v4(uint32_t addr, int a, int b, float c, float d) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(__float_as_int(c)),
                 "r"(__float_as_int(d)) : "memory");
}
__device__ __forceinline__ void st_dsmem_u32(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void st_dsmem_u64(uint32_t addr, unsigned long long v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive_release() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}

// Whether either half of a pair of bf16 numbers is at least that of another.
__device__ __forceinline__ bool any_ge2(uint32_t a, uint32_t b) {
    uint32_t ok;
    asm("{\n .reg .pred p, q;\n setp.ge.bf16x2 p|q, %1, %2;\n or.pred p, p, q;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(a), "r"(b));
    return ok != 0;
}

template <typename In, bool kRest, int kT>
__global__ void __launch_bounds__(kT, TOPK_R / kT) topk_kernel(TopParams p) {
    using E = Elem<In>;
    constexpr int kW = E::kVec, kWarps = kT / 32;
    extern __shared__ __align__(128) unsigned char dsm[];
    __shared__ __align__(16) TopSmem<kWarps> sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int csize = p.csize, rank = csize > 1 ? static_cast<int>(cluster_rank()) : 0;
    const unsigned row = csize > 1 ? blockIdx.x / static_cast<unsigned>(csize) : blockIdx.x;
    const int V = p.V, K = p.K;
    grid_dependency_sync();
    if (p.mask && !p.mask[row]) return;  // the cluster alike
    if (csize > 1) cluster_arrive_relaxed();  // (no CTA writes to one that has not started)
    unsigned group = row, pos = 0;
    if (p.P > 1) {
        group = row / static_cast<unsigned>(p.P);
        pos = row - group * static_cast<unsigned>(p.P);
    }
    const In* x = static_cast<const In*>(p.logits) + group * p.sg + pos * p.sp;
    float* values = p.values + size_t(row) * K;
    int32_t* ids = p.ids + size_t(row) * K;
    // entry j counts as position j + ph: chunks of positions are 16-byte vectors of the row
    const int ph = static_cast<int>((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(In));
    const int p0 = rank * p.span, p1 = min(p0 + p.span, V + ph);  // this CTA's positions,
    const int first = max(p0 - ph, 0), end = max(first, p1 - ph); // its entries,
    const int c0 = (first + ph + kW - 1) / kW, c1 = max(c0, (end + ph) / kW);  // its whole chunks [c0, c1),
    const int head = min(end, c0 * kW - ph), tail = min(end, max(head, c1 * kW - ph));  // and the entries before and after them
    const int singles = (head - first) + (end - tail);
    const In* body = x - ph;  // chunk v starts at body + v kW
    unsigned long long* cand = reinterpret_cast<unsigned long long*>(dsm);
    unsigned long long* sorted = cand + p.room;
    // chunks with an entry from theta on, a part for every warp; later the candidates' places
    const int list_room = 2 * p.room / kWarps;
    uint32_t* lists = reinterpret_cast<uint32_t*>(sorted + p.room);
    uint32_t* list = lists + warp * list_room;
    uint32_t* maxima = lists + 2 * p.room;
    if (tid == 0) {
        sh.n = 0;
        sh.left = 0ull;
    }
    auto single = [&](int i) { return i < head - first ? first + i : tail + (i - (head - first)); };
    unsigned turn = 0;
    // this CTA's part (thread 0's) to every CTA of the cluster; the parts are in the result for every thread
    auto exchange = [&](TopPart mine) -> const TopPart* {
        TopPart* slots = sh.parts[turn & 1u];
        ++turn;
        if (csize == 1) {
            __syncthreads();
            if (tid == 0) slots[0] = mine;
            __syncthreads();
            return slots;
        }
        if (tid == 0) sh.mine = mine;
        __syncthreads();
        if (tid < csize) {
            const TopPart v = sh.mine;
            st_dsmem_v4(map_rank(&slots[rank], static_cast<uint32_t>(tid)), v.n, v.m, v.s, v.top);
        }
        cluster_arrive_release();
        cluster_wait();
        return slots;
    };

    // the larger of each word of two chunks (bf16: of each half)
    auto max_into = [](uint4& a, const uint4& b) {
        if constexpr (sizeof(In) == 2) {
            a = make_uint4(bmax2(a.x, b.x), bmax2(a.y, b.y), bmax2(a.z, b.z), bmax2(a.w, b.w));
        } else {
            a = make_uint4(__float_as_uint(fmaxf(__uint_as_float(a.x), __uint_as_float(b.x))),
                           __float_as_uint(fmaxf(__uint_as_float(a.y), __uint_as_float(b.y))),
                           __float_as_uint(fmaxf(__uint_as_float(a.z), __uint_as_float(b.z))),
                           __float_as_uint(fmaxf(__uint_as_float(a.w), __uint_as_float(b.w))));
        }
    };
    // ---- sweep 1: group maxima of all CTAs, into every CTA
    const int g = p.groups, mine_at = rank * kT * g;
    for (int k = 0; k < g; ++k) {
        const int step = kT * g, at = c0 + tid + k * kT;
        uint4 m = ninf_raw<In>();
        int v = at;
        for (; v + 3 * step < c1; v += 4 * step) {  // (four loads in flight)
            uint4 r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = ldg_stream(body + size_t(v + i * step) * kW);
#pragma unroll
            for (int i = 0; i < 4; ++i) max_into(m, r[i]);
        }
        if (v < c1) {
            uint4 r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = ldg_stream(body + size_t(min(v + i * step, c1 - 1)) * kW);  // (the last again)
#pragma unroll
            for (int i = 0; i < 4; ++i) max_into(m, v + i * step < c1 ? r[i] : m);
        }
        float top = E::max_raw(m);
        bool any = at < c1;
        if (k == 0 && tid < singles) {
            top = fmaxf(top, E::load(x + single(tid)));
            any = true;
        }
        maxima[mine_at + k * kT + tid] = any ? key_of(top) : 0u;
    }
    if (csize > 1) {
        cluster_wait();
        for (int i = tid; i < kT * g; i += kT) {
            const uint32_t v = maxima[mine_at + i];
            for (int r = 0; r < csize; ++r)
                if (r != rank) st_dsmem_u32(map_rank(&maxima[mine_at + i], static_cast<uint32_t>(r)), v);
        }
        cluster_arrive_release();
        cluster_wait();
    }
    const int total = kT * g * csize;
    // 2^bits bins over a range of keys
    const int bits = K <= 128 ? 8 : 9;
    auto shift_of = [bits](uint32_t range) { return max(0, 32 - __clz(range) - bits); };
    // The two histograms are the work of a team: one warp where it has little to do (the others would spend as
    // many instructions on nothing), else the whole CTA.
    auto team_sync = [&](auto all) {
        if constexpr (decltype(all)::value) __syncthreads();
        else __syncwarp();
    };
    auto clear_bins = [&](auto all) {
        constexpr bool kAll = decltype(all)::value;
        for (int i = kAll ? tid : lane; i < top_slot(1 << bits); i += kAll ? kT : 32) sh.hist[i] = 0;
    };
    // one warp: from the histogram the highest bin from which on there are `need` entries, and, where wanted, the
    // entries in the bins above each and the fullest bin
    auto scan_bins = [&](int need, auto bases) {
        constexpr bool kBases = decltype(bases)::value;
        const int per = (1 << bits) / 32;
        int sum = 0, most = 0;
        for (int i = 0; i < per; ++i) {
            const int h = sh.hist[top_slot(lane * per + i)];
            sum += h;
            most = max(most, h);
        }
        int incl = sum;  // of this lane's bins and all above
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_down_sync(0xffffffffu, incl, o);
            if (lane + o < 32) incl += y;
        }
        int above = incl - sum;
        const bool mine = above < need && incl >= need;
        if (kBases || mine) {
            for (int i = per - 1; i >= 0; --i) {
                const int at = top_slot(lane * per + i), h = sh.hist[at];
                if constexpr (kBases) sh.base[at] = above;
                if (above < need && above + h >= need) {
                    sh.bin = lane * per + i;
                    sh.reach = above + h;
                    sh.above = above;
                }
                above += h;
            }
        }
        if constexpr (kBases) {
            most = __reduce_max_sync(0xffffffffu, most);
            if (lane == 0) sh.crowd = most;
        } else {
            if (!__any_sync(0xffffffffu, mine) && lane == 0) sh.bin = -1;
        }
    };
    // T: reached by K maxima or more, and by few more, from a histogram over the range of the maxima, refined in
    // the bin of the K-th largest where that holds many (a row with a few entries far above the others)
    auto find_theta = [&](auto all) {
        constexpr bool kAll = decltype(all)::value;
        const int t0 = kAll ? tid : lane, step = kAll ? kT : 32;
        uint32_t hi = 0u, lo = 0xffffffffu, T = 0u;  // the largest, and the smallest of a group that has entries
        for (int i = t0; i < total; i += step) {
            const uint32_t k = maxima[i];
            hi = max(hi, k);
            if (k) lo = min(lo, k);
        }
        hi = __reduce_max_sync(0xffffffffu, hi);
        lo = __reduce_min_sync(0xffffffffu, lo);
        clear_bins(all);
        if constexpr (kAll) {
            if (lane == 0) {
                sh.warp_hi[warp] = hi;
                sh.warp_lo[warp] = lo;
            }
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                hi = max(hi, sh.warp_hi[w]);
                lo = min(lo, sh.warp_lo[w]);
            }
        } else {
            __syncwarp();
        }
        if (kAll ? tid == 0 : lane == 0) sh.kmax = hi;
        int above = 0;
        while (lo <= hi) {
            const int shift = shift_of(hi - lo);
            for (int i = t0; i < total; i += step) {
                const uint32_t k = maxima[i];
                if (k >= lo && k <= hi) atomicAdd(&sh.hist[top_slot(static_cast<int>((k - lo) >> shift))], 1);
            }
            team_sync(all);
            if (!kAll || warp == 0) scan_bins(K - above, std::false_type());
            team_sync(all);
            const int bin = sh.bin, reach = sh.reach, past = sh.above;
            if (bin < 0) break;  // fewer than K groups
            T = lo + (static_cast<uint32_t>(bin) << shift);
            if (above + reach <= K + K / 8 + 4 || shift == 0) break;
            above += past;
            lo = T;
            hi = min(hi, T + ((1u << shift) - 1u));
            clear_bins(all);
            team_sync(all);
        }
        return max(T, kKeyNegInf);
    };
    uint32_t T;
    if (total <= 512) {
        __syncthreads();
        if (warp == 0) {
            T = find_theta(std::false_type());
            if (lane == 0) sh.T = T;
        }
        __syncthreads();
        T = sh.T;
    } else {
        T = find_theta(std::true_type());
    }
    const float theta = value_of(T);

    // ---- sweep 2: the sum below theta and the candidates.  Each warp lists the chunks with an entry from theta
    // on as it meets them and takes their entries afterwards, one a lane: the sum depends on no order
    // but that of the row
    // (exponents x c - M as one FMA, M = rn(theta c): one rounding, after the cancellation, and M belongs to the
    // sum.  They stay below 1: x < theta)
    const float c = p.c, M = theta == kNegInf ? 0.f : __fmul_rn(theta, c);
    float S = 0.f;
    bool over = false;
    auto append = [&](float v, int j) {
        const int at = atomicAdd(&sh.n, 1);
        if (at < p.room)
            cand[at] = (static_cast<unsigned long long>(key_of(v)) << 32) | (0xffffffffu - static_cast<uint32_t>(j));
    };
    // whether a chunk has an entry from theta on (bf16: packed, theta rounded up to the entries' grid)
    const uint32_t theta2 = __byte_perm(__float_as_uint(theta < 0.f ? theta : __uint_as_float((__float_as_uint(theta) + 0xffffu) & 0xffff0000u)), 0u, 0x3232);
    auto reaches = [&](const uint4& r) {
        if constexpr (sizeof(In) == 2) {
            const uint32_t m = bmax2(bmax2(r.x, r.y), bmax2(r.z, r.w));
            return any_ge2(m, theta2);
        } else {
            return E::max_raw(r) >= theta;
        }
    };
    {
        float2 acc = f2(0.f);
        int hits = 0;
        auto chunk = [&](const uint4& raw, int v, auto whole) {
            const bool in = decltype(whole)::value || v < c1, hit = in && reaches(raw);
            if constexpr (kRest) {
                float y[kW];
                E::unpack(raw, y);
                float2 d[kW / 2];
#pragma unroll
                for (int e = 0; e < kW / 2; ++e) {
                    const float2 a = fma2(make_float2(y[2 * e], y[2 * e + 1]), f2(c), f2(-M));
                    d[e] = make_float2(ex2(a.x), ex2(a.y));
                }
#pragma unroll
                for (int w = kW / 4; w > 0; w /= 2)
#pragma unroll
                    for (int e = 0; e < w; ++e) d[e] = add2(d[e], d[e + w]);
                if (in && !hit) acc = add2(acc, d[0]);
            }
            const unsigned m = __ballot_sync(0xffffffffu, hit);
            if (m) {
                const int at = hits + __popc(m & ((1u << lane) - 1u));
                if (hit && at < list_room) list[at] = static_cast<uint32_t>(v);
                hits += __popc(m);
            }
        };
        int v0 = c0 + warp * 32;
        for (; v0 + 3 * kT + 32 <= c1; v0 += 4 * kT) {  // (four loads in flight)
            uint4 raw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[i] = ldg_stream(body + size_t(v0 + i * kT + lane) * kW);
#pragma unroll
            for (int i = 0; i < 4; ++i) chunk(raw[i], v0 + i * kT + lane, std::true_type());
        }
        if (v0 < c1) {
            uint4 raw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[i] = ldg_stream(body + size_t(min(v0 + i * kT + lane, c1 - 1)) * kW);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v0 + i * kT < c1) chunk(raw[i], v0 + i * kT + lane, std::false_type());
        }
        __syncwarp();
        over |= hits > list_room;
        hits = min(hits, list_room);
        S += acc.x + acc.y;
        // a listed chunk a lane, then, in the first warp, the single entries
        for (int i = lane; i < hits; i += 32) {
            const int v = static_cast<int>(list[i]);
            float y[kW];
            E::unpack(ldg_stream(body + size_t(v) * kW), y);
#pragma unroll
            for (int e = 0; e < kW; ++e) {
                if (y[e] >= theta) append(y[e], v * kW + e - ph);
                else if (kRest) S += ex2(fmaf(y[e], c, -M));
            }
        }
        if (warp == 0 && lane < singles) {
            const int j = single(lane);
            const float v = E::load(x + j);
            if (v >= theta) append(v, j);
            else if (kRest) S += ex2(fmaf(v, c, -M));
        }
    }
    if constexpr (kRest) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
    }
    if (lane == 0) {
        sh.warp_f[warp] = S;
        if (over) atomicAdd(&sh.n, 1 << 24);  // (above any room)
    }
    __syncthreads();
    int n = sh.n, before = 0;
    bool slow = n > p.room;
    S = sh.warp_f[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) S += sh.warp_f[w];
    const TopPart* parts;
    if (csize > 1) {
        parts = exchange(TopPart{min(n, 1 << 24), slow ? 1 : 0, S, 0.f});
        n = 0;
        S = 0.f;
        for (int r = 0; r < csize; ++r) {
            before += r < rank ? parts[r].n : 0;
            n += parts[r].n;
            S += parts[r].s;
            slow |= parts[r].m != 0;
        }
    }
    slow |= n > p.room;
    float log_ref = mul_c(M, kLn2, kLn2Lo);  // the logarithm of what the sum is against
    // the sum of the entries' exponentials below `bound` over the cluster, against the largest of them, m
    auto below = [&](float bound, float& m) {
        float mx = kNegInf;
#pragma unroll 8
        for (int j = first + tid; j < end; j += kT) {
            const float v = E::load(x + j);
            if (v < bound) mx = fmaxf(mx, v);
        }
        mx = block_reduce<kT>(mx, [](float a, float b) { return fmaxf(a, b); }, sh.warp_f);
        const TopPart* q = exchange(TopPart{0, 0, 0.f, mx});
        for (int r = 0; r < csize; ++r) mx = fmaxf(mx, q[r].top);
        float sum = 0.f;
        if (mx != kNegInf) {
#pragma unroll 8
            for (int j = first + tid; j < end; j += kT) {
                const float v = E::load(x + j);
                if (v < bound) sum += ex2((v - mx) * c);
            }
        }
        sum = block_reduce<kT>(sum, [](float a, float b) { return a + b; }, sh.warp_f);
        q = exchange(TopPart{0, 0, sum, 0.f});
        m = mx;
        sum = 0.f;
        for (int r = 0; r < csize; ++r) sum += q[r].s;
        return sum;
    };
    if (slow) {
        // the exact K-th largest key: theta itself if fewer than K entries lie above it
        auto block_sum = [&](int v) { return block_reduce<kT>(v, [](int a, int b) { return a + b; }, sh.warp_i); };
        auto count = [&](auto pred) {
            int m = 0;
#pragma unroll 8
            for (int j = first + tid; j < end; j += kT) m += pred(key_of(E::load(x + j))) ? 1 : 0;
            m = block_sum(m);
            const TopPart* q = exchange(TopPart{m, 0, 0.f, 0.f});
            m = 0;
            for (int r = 0; r < csize; ++r) m += q[r].n;
            return m;
        };
        uint32_t kth = T;
        if (sizeof(In) == 2 && !(T & 0x80000000u)) kth |= 0xffffu;  // (negative bf16 keys end in ones)
        const uint32_t least = kth;
        if (count([least](uint32_t k) { return k > least; }) >= K) {
            kth = 0u;
            for (int bit = 31; bit >= 0; --bit) {
                const uint32_t at = kth | (1u << bit);
                if (count([at](uint32_t k) { return k >= at; }) >= K) kth = at;
            }
        }
        T = kth;
        // the entries above it, then those equal to it, in index order: warps own runs of entries
        if (tid == 0) sh.n = 0;
        __syncthreads();
        int equal = 0;
        for (int j0 = first + warp * 32; j0 < end; j0 += kT) {
            const bool in = j0 + lane < end;
            const float v = in ? E::load(x + j0 + lane) : 0.f;
            const uint32_t k = key_of(v);
            if (in && k > kth) append(v, j0 + lane);
            equal += in && k == kth ? 1 : 0;
        }
        __syncthreads();
        const int above = min(sh.n, p.room);
        equal = block_sum(equal);
        parts = exchange(TopPart{above, equal, 0.f, 0.f});
        int lower = 0, all_above = 0, all_equal = 0;  // equal entries in lower CTAs
        for (int r = 0; r < csize; ++r) {
            lower += r < rank ? parts[r].m : 0;
            all_above += parts[r].n;
            all_equal += parts[r].m;
        }
        const int quota = max(0, min(equal, K - all_above - lower));  // how many of the equal ones here are taken
        {
            const int per = ((end - first + kWarps - 1) / kWarps + 31) / 32 * 32;
            const int lo = min(end, first + warp * per), hi = min(end, lo + per);
            auto is = [&](int j) { return j < hi && key_of(E::load(x + j)) == kth; };
            int mine = 0;
            for (int j = lo; j < hi; j += 32) mine += __popc(__ballot_sync(0xffffffffu, is(j + lane)));
            __syncthreads();
            if (lane == 0) sh.warp_i[warp] = mine;
            __syncthreads();
            int at = 0;
            for (int w = 0; w < warp; ++w) at += sh.warp_i[w];
            for (int j = lo; j < hi && at < quota; j += 32) {
                const bool eq = is(j + lane);
                const unsigned m = __ballot_sync(0xffffffffu, eq);
                if (eq && at + __popc(m & ((1u << lane) - 1u)) < quota) append(value_of(kth), j + lane);
                at += __popc(m);
            }
            __syncthreads();
        }
        n = min(sh.n, p.room);
        parts = exchange(TopPart{n, 0, 0.f, 0.f});
        before = n = 0;
        for (int r = 0; r < csize; ++r) {
            before += r < rank ? parts[r].n : 0;
            n += parts[r].n;
        }
        if constexpr (kRest) {
            const float v = value_of(kth);
            float m;
            S = below(v, m);
            const int left = all_above + all_equal - K;  // equal entries that were not taken
            if (left > 0 && v != kNegInf) {
                S = (S > 0.f ? S * ex2((m - v) * c) : 0.f) + static_cast<float>(left);
                m = v;
            }
            log_ref = __fdiv_rn(m, p.tau);
        }
    } else if (kRest && n <= K && !(S > 0x1p-10f)) {  // all others lie below theta by far
        float m;
        S = below(theta, m);
        log_ref = __fdiv_rn(m, p.tau);
    }
    // ---- finish: all candidates to the first CTA
    n = min(n, p.room);
    if (csize > 1) {
        const int have = min(sh.n, p.room);
        if (rank > 0)
            for (int i = tid; i < have && before + i < p.room; i += kT)
                st_dsmem_u64(map_rank(&cand[before + i], 0u), cand[i]);
        cluster_arrive_release();
        if (rank > 0) return;
        cluster_wait();
    }
    // By the bin of each candidate's value; those of one bin compare with each other.  T and the largest maximum
    // bound the values, but for NaN, which goes to the last bin.
    const uint32_t range = sh.kmax > T ? sh.kmax - T : 0u;
    const int shift = shift_of(range);
    auto bin_of = [&](unsigned long long k) {
        const uint32_t v = static_cast<uint32_t>(k >> 32);
        return top_slot(static_cast<int>(min(v > T ? v - T : 0u, range) >> shift));
    };
    unsigned short* place = reinterpret_cast<unsigned short*>(lists);
    auto finish = [&](auto all) {
        constexpr bool kAll = decltype(all)::value;
        const int t0 = kAll ? tid : lane, step = kAll ? kT : 32;
        auto emit = [&](unsigned long long k, int r) {
            if (r < K) {
                values[r] = value_of(static_cast<uint32_t>(k >> 32));
                ids[r] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(k));
            } else if (r == K) {
                sh.ref = value_of(static_cast<uint32_t>(k >> 32));
            }
        };
        clear_bins(all);
        team_sync(all);
        for (int i = t0; i < n; i += step)
            place[i] = static_cast<unsigned short>(atomicAdd(&sh.hist[bin_of(cand[i])], 1));  // in its bin
        team_sync(all);
        if (!kAll || warp == 0) scan_bins(K, std::true_type());
        team_sync(all);
        if (sh.crowd <= kTopCrowd) {
            for (int i = t0; i < n; i += step) sorted[sh.base[bin_of(cand[i])] + place[i]] = cand[i];
            team_sync(all);
            for (int i = t0; i < n; i += step) {
                const unsigned long long k = sorted[i];
                const int slot = bin_of(k), from = sh.base[slot], to = from + sh.hist[slot];
                int at = from;
                for (int j = from; j < to; ++j) at += sorted[j] > k ? 1 : 0;
                emit(k, at);
                place[i] = static_cast<unsigned short>(at);
            }
        } else {  // many equal values: a bitonic sort
            int size = 1;
            while (size < n) size <<= 1;  // <= room
            for (int i = t0; i < size; i += step) sorted[i] = i < n ? cand[i] : 0ull;
            for (int k = 2; k <= size; k <<= 1) {
                for (int j = k >> 1; j > 0; j >>= 1) {
                    team_sync(all);
                    for (int t = t0; t < size / 2; t += step) {
                        const int a = 2 * t - (t & (j - 1)), b = a + j;
                        const unsigned long long va = sorted[a], vb = sorted[b];
                        const bool descending = (a & k) == 0;
                        if ((va < vb) == descending) {
                            sorted[a] = vb;
                            sorted[b] = va;
                        }
                    }
                }
            }
            team_sync(all);
            for (int i = t0; i < n; i += step) {
                emit(sorted[i], i);
                place[i] = static_cast<unsigned short>(i);
            }
        }
        for (int i = n + t0; i < K; i += step) {  // fewer than K numbers in the row
            values[i] = kNegInf;
            ids[i] = -1;
        }
        if constexpr (kRest) {
            if (n > K) {  // the candidates that were not taken, against the largest of them
                team_sync(all);
                const float v = sh.ref;
                unsigned long long left = 0ull;
                for (int i = t0; i < n; i += step)
                    if (place[i] >= K)
                        left += __float2ull_rn(ex2((value_of(static_cast<uint32_t>(sorted[i] >> 32)) - v) * c) * kTopFix);
                if (__any_sync(0xffffffffu, left != 0ull)) {
                    left = warp_sum_u64(left);
                    if (kAll && lane == 0) atomicAdd(&sh.left, left);
                }
                if constexpr (kAll) {
                    __syncthreads();
                    left = sh.left;
                }
                S = (S > 0.f ? S * ex2(fmaf(-v, c, M)) : 0.f) + __ull2float_rn(left) * (1.f / kTopFix);
                log_ref = __fdiv_rn(v, p.tau);
            }
            if (t0 == 0) p.rest[row] = S > 0.f ? fmaf(log2f(S), kLn2, log_ref) : kNegInf;
        }
    };
    if (n <= 128) {
        __syncthreads();
        if (warp == 0) finish(std::false_type());
    } else {
        finish(std::true_type());
    }
}

template <typename In, int kT>
static osd_status launch_topk(TopParams tp, long long rows, int c, cudaStream_t s) {
    constexpr int kW = Elem<In>::kVec;
    const int positions = tp.V + kW - 1;  // a row starts up to kW - 1 positions into the grid
    c = std::max(1, std::min(c, kTopMaxCluster));
    tp.span = ((positions + c - 1) / c + 63) / 64 * 64;
    tp.csize = (positions + tp.span - 1) / tp.span;
    tp.room = 256;
    while (tp.room < tp.K + tp.K / 2 + 128) tp.room *= 2;
    const int per = (tp.span / kW + kT - 1) / kT;  // chunks per thread
    tp.groups = std::max(1, std::min(per, (4 * tp.K + tp.csize * kT - 1) / (tp.csize * kT)));
    const size_t smem = size_t(tp.room) * 24 + size_t(tp.csize) * kT * tp.groups * 4;
    if (rows * tp.csize > INT_MAX) return OSD_ERR_UNSUPPORTED;
    auto go = [&](auto kernel_tag) -> osd_status {
        constexpr bool kRest = decltype(kernel_tag)::value;
        if (ctas_per_sm<topk_kernel<In, kRest, kT>, kT>(smem) < 1) return OSD_ERR_CUDA;  // (opts in for the size)
        return from_cuda(launch_ex(true, topk_kernel<In, kRest, kT>, dim3(static_cast<unsigned>(rows * tp.csize)), dim3(kT),
                                   smem, s, tp.csize, tp));
    };
    return tp.rest ? go(std::true_type()) : go(std::false_type());
}

template <typename In>
static osd_status launch_topk_dtype(const TopParams& tp, long long rows, cudaStream_t s) {
    const long long bytes = (long long)tp.V * (long long)sizeof(In);
    const int c = TOPK_C(bytes, rows);
    switch (TOPK_T) {
        case 128: return launch_topk<In, 128>(tp, rows, c, s);
        case 256: return launch_topk<In, 256>(tp, rows, c, s);
        default: return launch_topk<In, 512>(tp, rows, c, s);
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
    TopParams tp = {};
    tp.logits = logits; tp.P = P; tp.V = V; tp.sg = stride_g; tp.sp = stride_p; tp.mask = mask; tp.K = K;
    tp.c = static_cast<float>(1.4426950408889634074 / static_cast<double>(temperature));
    tp.tau = temperature;
    tp.values = values; tp.ids = ids; tp.rest = rest;
    return dtype == OSD_BF16 ? launch_topk_dtype<__nv_bfloat16>(tp, rows, s) : launch_topk_dtype<float>(tp, rows, s);
}
