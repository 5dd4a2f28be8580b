// osd_topk.cu -- the K largest logits of a row with their ids, and the log of the mass of
// all other entries: the compact form in which the buffer R of Algorithm 1 keeps a
// target row.
//
// One thread-block cluster per row, each CTA with its span of the row in shared memory
// (one bulk copy), so that a row is read once:
//
//   sweep 1  the maximum of each of several K groups of 16-byte chunks; the K-th
//            largest of these, theta, found bit by bit, is reached by K entries at
//            least, and by few more where large entries lie anyhow;
//   sweep 2  the sum of the exponentials of the chunks below theta, and a list of the
//            others, whose entries are then taken one by one: those from theta on are the
//            candidates;
//   finish   one CTA ranks the candidates (value, then index).  Those past the K-th join
//            the sum.
//
// Rows with more candidates than there is room for (many equal entries, or large ones
// crowded in few groups) go on to the exact K-th largest value, counted bit by bit over the
// staged row, and take the entries equal to it in index order.
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
#define TOPK_C(bytes, rows) int((bytes + 72 * 1024 - 1) / (72 * 1024)) * (rows <= 152 ? 4 : 1)
#endif

constexpr int kTopThreads = 256;
constexpr int kTopMaxCluster = 8;
constexpr int kTopBins = 512;        // bins of a histogram over a range of keys
constexpr int kTopCrowd = 48;        // candidates of one bin that are ranked by comparing; with more all are sorted
// Exponentials (at most 1) of candidates, whose order is that of atomics, are added as whole multiples
// of 2^-40, so that the sum does not depend on it.
constexpr float kTopFix = 0x1p40f;
constexpr uint64_t kTopWaitNs = 1000000000ull;  // bound on the wait for the bulk copies

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
    int32_t* status;
    int csize;    // CTAs per row
    int span;     // positions per CTA: whole chunks
    int section;  // positions staged at a time: the span, or what fits
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
constexpr uint32_t kKeyNegInf = 0x007fffffu;

// What the CTAs of a cluster tell each other at one point.
struct TopPart {
    int n;      // candidates, or a count
    int m;      // another count
    float s;    // a sum
    float top;  // a maximum
};

struct TopSmem {
    TopPart parts[2][kTopMaxCluster];  // slot r from CTA r; alternately
    TopPart mine;
    uint64_t bar;
    int n, err, crowd;
    int bin, reach, above;  // of a histogram: the bin of the K-th largest, entries from it on, past it
    float ref;
    unsigned long long left;
    int warp_i[kTopThreads / 32];
    float warp_f[kTopThreads / 32];
    uint32_t warp_hi[kTopThreads / 32], warp_lo[kTopThreads / 32];
    __align__(16) int hist[kTopBins], base[kTopBins];  // entries per bin, and in the bins above it
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

template <typename In, bool kRest>
__global__ void __launch_bounds__(kTopThreads, 3) topk_kernel(TopParams p) {
    using E = Elem<In>;
    constexpr int kW = E::kVec, kT = kTopThreads, kWarps = kT / 32;
    extern __shared__ __align__(128) unsigned char dsm[];
    __shared__ __align__(16) TopSmem sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int csize = p.csize, rank = csize > 1 ? static_cast<int>(cluster_rank()) : 0;
    const long long row = blockIdx.x / csize;
    const int V = p.V, K = p.K;
    if (tid == 0) mbar_init(&sh.bar, 1);
    grid_dependency_sync();
    if (p.mask && !p.mask[row]) return;  // the cluster alike
    if (csize > 1) cluster_arrive_relaxed();  // (no CTA writes to one that has not started)
    const In* x = static_cast<const In*>(p.logits) + (row / p.P) * p.sg + (row % p.P) * p.sp;
    // entry j counts as position j + ph: chunks of positions are 16-byte vectors of the row
    const int ph = static_cast<int>((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(In));
    const int p0 = rank * p.span, p1 = min(p0 + p.span, V + ph);  // this CTA's positions
    In* staged = reinterpret_cast<In*>(dsm);
    unsigned long long* cand = reinterpret_cast<unsigned long long*>(dsm + size_t(p.section) * sizeof(In));
    unsigned long long* sorted = cand + p.room;
    // chunks with an entry from theta on, a part for every warp
    const int list_room = p.room / 4;
    unsigned short* list = reinterpret_cast<unsigned short*>(sorted + p.room) + warp * list_room;
    uint32_t* maxima = reinterpret_cast<uint32_t*>(sorted + p.room) + p.room;
    const int sections = max(1, (p1 - p0 + p.section - 1) / p.section);  // (a CTA past the row's end has an empty one)
    unsigned parity = 0;
    if (tid == 0) {
        sh.err = 0;
        sh.n = 0;
        sh.left = 0ull;
    }
    __syncthreads();

    // Positions [s0, s0 + section) of this CTA into shared memory; what lies outside the row reads as -inf.
    // Returns the number of chunks.
    auto stage = [&](int sec) -> int {
        const int s0 = p0 + sec * p.section, s1 = min(s0 + p.section, p1);
        const int n = max(0, (s1 - s0 + kW - 1) / kW);
        const int c0 = s0 < ph ? 1 : 0;                                   // whole chunks [c0, c1)
        const int c1 = max(c0, (s0 + n * kW > V + ph) ? n - 1 : n);
        if (tid == 0 && c1 > c0) {
            const uint32_t bytes = static_cast<uint32_t>(c1 - c0) * 16u;
            mbar_arrive_expect_tx(&sh.bar, bytes);
            bulk_g2s(staged + c0 * kW, x + (s0 + c0 * kW - ph), bytes, &sh.bar);
        }
        for (int i = tid; i < n * kW; i += kT) {
            if (i >= c0 * kW && i < c1 * kW) {  // on to the last chunk
                i += ((c1 * kW - i + kT - 1) / kT) * kT - kT;
                continue;
            }
            const int j = s0 + i - ph;
            E::store(staged + i, j >= 0 && j < V ? E::load(x + j) : kNegInf);
        }
        if (c1 > c0) {
            if (!mbar_wait_bounded(&sh.bar, parity, kTopWaitNs)) {
                sh.err = 1;
                mbar_wait_bounded(&sh.bar, parity, kTopWaitNs);  // give the copy in flight a last chance to land
            }
            parity ^= 1u;
        }
        __syncthreads();
        return n;
    };
    int chunks = stage(0);
    // f(chunks, first position) on each section in turn; the only one stays staged
    auto sweep = [&](auto&& f) {
        for (int sec = 0; sec < sections; ++sec) {
            if (sections > 1) {
                fence_proxy_async_smem();  // (the accesses of the section before)
                __syncthreads();
                chunks = stage(sec);
            }
            f(chunks, p0 + sec * p.section);
        }
    };
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
    auto block_sum_f = [&](float v) {
        return block_reduce<kT>(v, [](float a, float b) { return a + b; }, sh.warp_f);
    };
    auto block_max_f = [&](float v) {
        return block_reduce<kT>(v, [](float a, float b) { return fmaxf(a, b); }, sh.warp_f);
    };
    auto block_sum_i = [&](int v) { return block_reduce<kT>(v, [](int a, int b) { return a + b; }, sh.warp_i); };

    // ---- sweep 1: group maxima of all CTAs, into every CTA
    const int g = p.groups, mine_at = rank * kT * g;
    for (int i = tid; i < kT * g; i += kT) maxima[mine_at + i] = 0u;
    sweep([&](int n, int) {
        for (int k = 0; k < g; ++k) {
            float m = kNegInf;
            const int first = tid + k * kT, step = kT * g;
            int v = first;
            for (; v + 3 * step < n; v += 4 * step) {  // (four loads in flight)
                uint4 r[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] = lds_v4(staged + (v + i * step) * kW);
#pragma unroll
                for (int i = 0; i < 4; ++i) m = fmaxf(m, E::max_raw(r[i]));
            }
            for (; v < n; v += step) m = fmaxf(m, E::max_raw(lds_v4(staged + v * kW)));
            if (first < n) {
                uint32_t& at = maxima[mine_at + first];
                at = max(at, key_of(m));
            }
        }
    });
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
    uint32_t kmax, kmin;  // the largest, and the smallest of a group that has entries
    {
        uint32_t hi = 0u, lo = 0xffffffffu;
        for (int i = tid; i < total; i += kT) {
            const uint32_t k = maxima[i];
            hi = max(hi, k);
            if (k) lo = min(lo, k);
        }
        hi = __reduce_max_sync(0xffffffffu, hi);
        lo = __reduce_min_sync(0xffffffffu, lo);
        if (lane == 0) {
            sh.warp_hi[warp] = hi;
            sh.warp_lo[warp] = lo;
        }
        for (int i = tid; i < kTopBins; i += kT) sh.hist[i] = 0;
        __syncthreads();
        kmax = sh.warp_hi[0];
        kmin = sh.warp_lo[0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) {
            kmax = max(kmax, sh.warp_hi[w]);
            kmin = min(kmin, sh.warp_lo[w]);
        }
    }
    auto shift_of = [](uint32_t range) { return max(0, 32 - __clz(range) - 9); };  // range >> it < 512 bins
    // warp 0: from the histogram, the entries in the bins above each (base), the highest bin from which on there are
    // `need`, and the fullest bin
    auto scan_bins = [&](int need) {
        constexpr int kPer = kTopBins / 32;
        int h[kPer], sum = 0, most = 0;
#pragma unroll
        for (int i = 0; i < kPer; i += 4) {
            const int4 v = *reinterpret_cast<const int4*>(&sh.hist[lane * kPer + i]);
            h[i] = v.x; h[i + 1] = v.y; h[i + 2] = v.z; h[i + 3] = v.w;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            sum += h[i];
            most = max(most, h[i]);
        }
        int incl = sum;  // of this lane's bins and all above
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_down_sync(0xffffffffu, incl, o);
            if (lane + o < 32) incl += y;
        }
        int above = incl - sum, bin = -1, reach = 0, past = 0;
#pragma unroll
        for (int i = kPer - 1; i >= 0; --i) {
            sh.base[lane * kPer + i] = above;
            if (above < need && above + h[i] >= need) {
                bin = lane * kPer + i;
                reach = above + h[i];
                past = above;
            }
            above += h[i];
        }
        most = __reduce_max_sync(0xffffffffu, most);
        const unsigned has = __ballot_sync(0xffffffffu, bin >= 0);
        if (lane == (has ? __ffs(has) - 1 : 0)) {
            sh.bin = bin;
            sh.reach = reach;
            sh.above = past;
            sh.crowd = most;
        }
    };
    // T: reached by K maxima or more, and by few more, from a histogram over the range of the maxima, refined in
    // the bin of the K-th largest where that holds many (a row with a few entries far above the others)
    uint32_t T = 0u;
    {
        uint32_t lo = kmin, hi = kmax;
        int above = 0;
        while (lo <= hi) {
            const int shift = shift_of(hi - lo);
            for (int i = tid; i < total; i += kT) {
                const uint32_t k = maxima[i];
                if (k >= lo && k <= hi) atomicAdd(&sh.hist[(k - lo) >> shift], 1);
            }
            __syncthreads();
            if (warp == 0) scan_bins(K - above);
            __syncthreads();
            const int bin = sh.bin;
            if (bin < 0) break;  // fewer than K groups
            T = lo + (static_cast<uint32_t>(bin) << shift);
            if (above + sh.reach <= K + K / 8 + 4 || shift == 0) break;
            above += sh.above;
            lo = T;
            hi = min(hi, T + ((1u << shift) - 1u));
            for (int i = tid; i < kTopBins; i += kT) sh.hist[i] = 0;
            __syncthreads();
        }
        T = max(T, kKeyNegInf);
    }
    const float theta = value_of(T);

    // ---- sweep 2: the sum below theta and the candidates.  Each warp lists the chunks with an entry from theta
    // on as it meets them and takes their entries afterwards, one a lane: the sum depends on no order
    // but that of the row
    const float c = p.c;
    float S = 0.f;
    bool over = false;
    auto append = [&](bool is, float v, int j) {  // by whole warps
        const unsigned m = __ballot_sync(0xffffffffu, is);
        if (!m) return;
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh.n, __popc(m));
        at = __shfl_sync(0xffffffffu, at, 0) + __popc(m & ((1u << lane) - 1u));
        if (is && at < p.room)
            cand[at] = (static_cast<unsigned long long>(key_of(v)) << 32) | (0xffffffffu - static_cast<uint32_t>(j));
    };
    sweep([&](int n, int s0) {
        float2 acc = f2(0.f);
        int hits = 0;
        auto chunk = [&](const uint4& r, int v, bool in) {
            const bool hit = in && E::max_raw(r) >= theta;
            if constexpr (kRest) {
                float2 d[kW / 2], e = f2(0.f);
                E::minus(r, theta, d);
#pragma unroll
                for (int i = 0; i < kW / 2; ++i) {
                    const float2 a = mul2(d[i], f2(c));
                    e = add2(e, make_float2(ex2(a.x), ex2(a.y)));
                }
                acc = add2(acc, (hit || !in) ? f2(0.f) : e);
            }
            const unsigned m = __ballot_sync(0xffffffffu, hit);
            if (m) {
                const int at = hits + __popc(m & ((1u << lane) - 1u));
                if (hit && at < list_room) list[at] = static_cast<unsigned short>(v);
                hits += __popc(m);
            }
        };
        const uint4 none = ninf_raw<In>();
        for (int v0 = warp * 32; v0 < n; v0 += 2 * kT) {
            const int va = v0 + lane, vb = va + kT;
            const uint4 ra = va < n ? lds_v4(staged + va * kW) : none, rb = vb < n ? lds_v4(staged + vb * kW) : none;
            chunk(ra, va, va < n);
            if (v0 + kT < n) chunk(rb, vb, vb < n);
        }
        __syncwarp();
        over |= hits > list_room;
        hits = min(hits, list_room);
        S += acc.x + acc.y;
        for (int i0 = 0; i0 < hits * kW; i0 += 32) {
            const int i = i0 + lane;
            const bool in = i < hits * kW;
            const int at = in ? static_cast<int>(list[i / kW]) * kW + i % kW : 0;
            const float v = E::lds(staged + at);
            const int j = s0 + at - ph;
            const bool is = in && v >= theta;
            if (kRest && in && !is) S += ex2((v - theta) * c);
            append(is && j >= 0 && j < V, v, j);  // (not the -inf from outside the row)
        }
        __syncwarp();
    });
    if constexpr (kRest) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
    }
    if (lane == 0) {
        sh.warp_f[warp] = S;
        sh.warp_i[warp] = over ? 1 : 0;
    }
    __syncthreads();
    int n = sh.n, before = 0;
    bool slow = false, err = sh.err != 0;
    S = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        S += sh.warp_f[w];
        slow |= sh.warp_i[w] != 0;
    }
    const TopPart* parts;
    if (csize > 1) {
        parts = exchange(TopPart{n, slow || n > p.room ? 1 : 0, S, err ? 1.f : 0.f});
        n = 0;
        S = 0.f;
        for (int r = 0; r < csize; ++r) {
            before += r < rank ? parts[r].n : 0;
            n += parts[r].n;
            S += parts[r].s;
            slow |= parts[r].m != 0;
            err |= parts[r].top != 0.f;
        }
    }
    slow |= n > p.room;
    if (err) {  // a copy did not arrive in time
        if (rank == 0) {
            for (int i = tid; i < K; i += kT) {
                p.values[row * K + i] = kNegInf;
                p.ids[row * K + i] = -1;
            }
            if (tid == 0) {
                if (p.rest) p.rest[row] = kNegInf;
                if (p.status) atomicExch(p.status, static_cast<int32_t>(OSD_ERR_TIMEOUT));
            }
        }
        return;
    }
    float ref = theta;
    // the largest entry below `bound` and the sum of 2^((x - it) c) of all entries below, over the cluster
    auto below = [&](float bound, float& m, float& s) {
        float mx = kNegInf;
        sweep([&](int nc, int) {
            for (int i = tid; i < nc * kW; i += kT) {
                const float v = E::lds(staged + i);
                if (v < bound) mx = fmaxf(mx, v);
            }
        });
        mx = block_max_f(mx);
        const TopPart* q = exchange(TopPart{0, 0, 0.f, mx});
        for (int r = 0; r < csize; ++r) mx = fmaxf(mx, q[r].top);
        float sum = 0.f;
        if (mx != kNegInf)
            sweep([&](int nc, int) {
                for (int i = tid; i < nc * kW; i += kT) {
                    const float v = E::lds(staged + i);
                    if (v < bound) sum += ex2((v - mx) * c);
                }
            });
        sum = block_sum_f(sum);
        q = exchange(TopPart{0, 0, sum, 0.f});
        sum = 0.f;
        for (int r = 0; r < csize; ++r) sum += q[r].s;
        m = mx;
        s = sum;
    };
    if (slow) {
        // the exact K-th largest key: theta itself if fewer than K entries lie above it
        auto count = [&](auto pred) {
            int m = 0;
            sweep([&](int nc, int s0) {
                for (int i = tid; i < nc * kW; i += kT) {
                    const int j = s0 + i - ph;
                    m += (j >= 0 && j < V && pred(key_of(E::lds(staged + i)))) ? 1 : 0;
                }
            });
            m = block_sum_i(m);
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
        // the entries above it, then those equal to it, in index order: warps own runs of positions
        if (tid == 0) sh.n = 0;
        __syncthreads();
        int equal = 0;
        sweep([&](int nc, int s0) {
            for (int i0 = warp * 32; i0 < nc * kW; i0 += kT) {
                const int i = i0 + lane, j = s0 + i - ph;
                const bool in = i < nc * kW && j >= 0 && j < V;
                const float v = in ? E::lds(staged + i) : 0.f;
                const uint32_t k = key_of(v);
                append(in && k > kth, v, j);
                equal += in && k == kth ? 1 : 0;
            }
        });
        __syncthreads();
        const int above = min(sh.n, p.room);
        equal = block_sum_i(equal);
        parts = exchange(TopPart{above, equal, 0.f, 0.f});
        int first = 0, all_above = 0, all_equal = 0;  // equal entries in lower CTAs
        for (int r = 0; r < csize; ++r) {
            first += r < rank ? parts[r].m : 0;
            all_above += parts[r].n;
            all_equal += parts[r].m;
        }
        int quota = max(0, min(equal, K - all_above - first));  // how many of the equal ones here are taken
        sweep([&](int nc, int s0) {
            const int per = (nc * kW + kWarps * 32 - 1) / (kWarps * 32) * 32;
            const int lo = min(nc * kW, warp * per), hi = min(nc * kW, lo + per);
            auto is = [&](int i) {
                const int j = s0 + i - ph;
                return i < hi && j >= 0 && j < V && key_of(E::lds(staged + i)) == kth;
            };
            int mine = 0;
            for (int i = lo; i < hi; i += 32) mine += __popc(__ballot_sync(0xffffffffu, is(i + lane)));
            __syncthreads();
            if (lane == 0) sh.warp_i[warp] = mine;
            __syncthreads();
            int at = 0, here = 0;
            for (int w = 0; w < kWarps; ++w) {
                at += w < warp ? sh.warp_i[w] : 0;
                here += sh.warp_i[w];
            }
            for (int i = lo; i < hi && at < quota; i += 32) {
                const bool eq = is(i + lane);
                const unsigned m = __ballot_sync(0xffffffffu, eq);
                append(eq && at + __popc(m & ((1u << lane) - 1u)) < quota, value_of(kth), s0 + i + lane - ph);
                at += __popc(m);
            }
            quota = max(0, quota - here);
            __syncthreads();
        });
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
            below(v, m, S);
            const int left = all_above + all_equal - K;  // equal entries that were not taken
            ref = m;
            if (left > 0 && v != kNegInf) {
                S = (m == kNegInf ? 0.f : S * ex2((m - v) * c)) + static_cast<float>(left);
                ref = v;
            }
        }
    } else if (kRest && n <= K && !(S > 0x1p-10f)) {
        below(theta, ref, S);  // all others lie below theta by far: their sum against their own largest
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
    auto emit = [&](unsigned long long k, int r) {
        if (r < K) {
            p.values[row * K + r] = value_of(static_cast<uint32_t>(k >> 32));
            p.ids[row * K + r] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(k));
        } else if (r == K) {
            sh.ref = value_of(static_cast<uint32_t>(k >> 32));
        }
    };
    // By the bin of each candidate's value; those of one bin compare with each other.  T and kmax bound the
    // values, but for NaN, which goes to the last bin.
    const uint32_t range = kmax > T ? kmax - T : 0u;
    const int shift = shift_of(range);
    auto bin_of = [&](unsigned long long k) {
        const uint32_t v = static_cast<uint32_t>(k >> 32);
        return static_cast<int>(min(v > T ? v - T : 0u, range) >> shift);
    };
    for (int i = tid; i < kTopBins; i += kT) sh.hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kT) {
        const unsigned long long k = cand[i];
        sorted[i] = static_cast<unsigned long long>(atomicAdd(&sh.hist[bin_of(k)], 1));  // its place in the bin
    }
    __syncthreads();
    if (warp == 0) scan_bins(K);
    __syncthreads();
    constexpr int kMostPer = 2048 / kT;  // candidates per thread: room <= 2048
    int r[kMostPer];
    if (sh.crowd <= kTopCrowd) {
#pragma unroll
        for (int u = 0; u < kMostPer; ++u) {
            const int i = tid + u * kT;
            if (i < n) r[u] = sh.base[bin_of(cand[i])] + static_cast<int>(sorted[i]);
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kMostPer; ++u) {
            const int i = tid + u * kT;
            if (i < n) sorted[r[u]] = cand[i];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kMostPer; ++u) {
            const int i = tid + u * kT;
            if (i >= n) continue;
            const unsigned long long k = sorted[i];
            const int bin = bin_of(k), first = sh.base[bin], last = first + sh.hist[bin];
            int at = first;
            for (int j = first; j < last; ++j) at += sorted[j] > k ? 1 : 0;
            emit(k, at);
            r[u] = at;
        }
    } else {  // many equal values: a bitonic sort
        int size = 1;
        while (size < n) size <<= 1;  // <= room
        for (int i = tid; i < size; i += kT) sorted[i] = i < n ? cand[i] : 0ull;
        for (int k = 2; k <= size; k <<= 1) {
            for (int j = k >> 1; j > 0; j >>= 1) {
                __syncthreads();
                for (int t = tid; t < size / 2; t += kT) {
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
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kMostPer; ++u) {
            const int i = tid + u * kT;
            r[u] = i;
            if (i < n) emit(sorted[i], i);
        }
    }
    for (int i = n + tid; i < K; i += kT) {  // fewer than K numbers in the row
        p.values[row * K + i] = kNegInf;
        p.ids[row * K + i] = -1;
    }
    if constexpr (kRest) {
        if (n > K) {  // the candidates that were not taken
            __syncthreads();
            const float m = sh.ref;
#pragma unroll
            for (int u = 0; u < kMostPer; ++u) {
                const int i = tid + u * kT;
                if (i < n && r[u] >= K)
                    atomicAdd(&sh.left, __float2ull_rn(ex2((value_of(static_cast<uint32_t>(sorted[i] >> 32)) - m) * c) * kTopFix));
            }
            __syncthreads();
            if (tid == 0) S = fmaf(S, ex2((ref - m) * c), __ull2float_rn(sh.left) * (1.f / kTopFix));
            ref = m;
        }
        if (tid == 0) p.rest[row] = S > 0.f ? fmaf(log2f(S), kLn2, __fdiv_rn(ref, p.tau)) : kNegInf;
    }
}

// Shared memory per CTA beside the section.
static size_t top_extra(int room, int csize, int groups) {
    return size_t(room) * 20 + size_t(csize) * kTopThreads * groups * 4;
}

template <typename In>
static osd_status launch_topk(TopParams tp, long long rows, cudaStream_t s) {
    constexpr int kW = Elem<In>::kVec;
    constexpr size_t es = sizeof(In);
    constexpr size_t kMost = 200 * 1024;
    const int positions = tp.V + kW - 1;  // a row starts up to kW - 1 positions into the grid
    const long long bytes = (long long)positions * (long long)es;
    int c = TOPK_C(bytes, rows);
    c = std::max(1, std::min(c, kTopMaxCluster));
    tp.span = ((positions + c - 1) / c + 63) / 64 * 64;
    tp.csize = (positions + tp.span - 1) / tp.span;
    tp.room = 256;
    while (tp.room < tp.K + tp.K / 2 + 128) tp.room *= 2;
    const int per = (tp.span / kW + kTopThreads - 1) / kTopThreads;  // chunks per thread
    tp.groups = std::max(1, std::min(per, (4 * tp.K + tp.csize * kTopThreads - 1) / (tp.csize * kTopThreads)));
    const size_t extra = top_extra(tp.room, tp.csize, tp.groups);
    tp.section = static_cast<int>(std::min<size_t>(tp.span, (kMost - extra) / es / 64 * 64));
    const size_t smem = size_t(tp.section) * es + extra;
    if (rows * tp.csize > INT_MAX) return OSD_ERR_UNSUPPORTED;
    auto go = [&](auto kernel_tag) -> osd_status {
        constexpr bool kRest = decltype(kernel_tag)::value;
        if (ctas_per_sm<topk_kernel<In, kRest>, kTopThreads>(smem) < 1) return OSD_ERR_CUDA;  // (opts in for the size)
        return from_cuda(launch_ex(true, topk_kernel<In, kRest>, dim3(static_cast<unsigned>(rows * tp.csize)), dim3(kTopThreads),
                                   smem, s, tp.csize, tp));
    };
    return tp.rest ? go(std::true_type()) : go(std::false_type());
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
    tp.values = values; tp.ids = ids; tp.rest = rest; tp.status = status;
    return dtype == OSD_BF16 ? launch_topk<__nv_bfloat16>(tp, rows, s) : launch_topk<float>(tp, rows, s);
}
