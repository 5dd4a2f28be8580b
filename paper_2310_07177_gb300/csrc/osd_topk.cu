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
constexpr int kTopCountMost = 384;   // candidates ranked by counting; more are sorted
// Exponentials at most 1 of entries whose order is that of atomics are added as whole multiples of
// 2^-40, so that the sums do not depend on it.
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
    int counts[33];
    int n, hits, err, total;
    uint32_t kmax, kmin;
    float ref;
    int warp_i[kTopThreads / 32];
    float warp_f[kTopThreads / 32];
    unsigned long long warp_u[kTopThreads / 32];
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
    uint32_t* list = reinterpret_cast<uint32_t*>(cand + p.room);
    uint32_t* maxima = list + p.room;
    const int sections = max(1, (p1 - p0 + p.section - 1) / p.section);  // (a CTA past the row's end has an empty one)
    unsigned parity = 0;
    if (tid == 0) {
        sh.err = 0;
        sh.n = 0;
        sh.kmax = 0u;
        sh.kmin = 0xffffffffu;
    }
    if (tid < 33) sh.counts[tid] = 0;
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
            bool any = false;
            for (int v = tid + k * kT; v < n; v += kT * g) {
                m = fmaxf(m, E::max_raw(lds_v4(staged + v * kW)));
                any = true;
            }
            if (any) {
                uint32_t& at = maxima[mine_at + k * kT + tid];
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
    {
        uint32_t hi = 0u, lo = 0xffffffffu;
        for (int i = tid; i < total; i += kT) {
            hi = max(hi, maxima[i]);
            lo = min(lo, maxima[i]);
        }
        hi = __reduce_max_sync(0xffffffffu, hi);
        lo = __reduce_min_sync(0xffffffffu, lo);
        if (lane == 0) {
            atomicMax(&sh.kmax, hi);
            atomicMin(&sh.kmin, lo);
        }
        __syncthreads();
    }
    // the largest T that K maxima reach, from the highest bit in which they differ on, until few more reach it
    uint32_t T;
    {
        const uint32_t diff = sh.kmax ^ sh.kmin;
        const int top = diff ? 31 - __clz(diff) : -1;
        T = top >= 0 ? sh.kmin & ~((2u << top) - 1u) : sh.kmin;
        if (total < K) T = 0u;
        constexpr int kLast = sizeof(In) == 2 ? 16 : 0;
        for (int bit = top; bit >= kLast && total >= K; --bit) {
            const uint32_t at = T | (1u << bit);
            int n = 0;
            for (int i = tid; i < total; i += kT) n += maxima[i] >= at ? 1 : 0;
            n = __reduce_add_sync(0xffffffffu, n);
            if (lane == 0 && n) atomicAdd(&sh.counts[bit], n);
            __syncthreads();
            n = sh.counts[bit];
            if (n >= K) {
                T = at;
                if (n <= K + K / 8 + 4) break;
            }
        }
        T = max(T, kKeyNegInf);
    }
    const float theta = value_of(T);

    // ---- sweep 2: the sum below theta and the candidates
    const float c = p.c;
    float S = 0.f;
    unsigned long long fixed = 0ull;
    bool over = false;
    auto append = [&](float v, int j) {
        const int at = atomicAdd(&sh.n, 1);
        if (at < p.room) cand[at] = (static_cast<unsigned long long>(key_of(v)) << 32) | (0xffffffffu - static_cast<uint32_t>(j));
    };
    sweep([&](int n, int s0) {
        if (tid == 0) sh.hits = 0;
        __syncthreads();
        float2 acc = f2(0.f);
#pragma unroll 2
        for (int v = tid; v < n; v += kT) {
            const uint4 r = lds_v4(staged + v * kW);
            const bool hit = E::max_raw(r) >= theta;
            if constexpr (kRest) {
                float2 d[kW / 2], e = f2(0.f);
                E::minus(r, theta, d);
#pragma unroll
                for (int i = 0; i < kW / 2; ++i) {
                    const float2 a = mul2(d[i], f2(c));
                    e = add2(e, make_float2(ex2(a.x), ex2(a.y)));
                }
                acc = add2(acc, hit ? f2(0.f) : e);
            }
            if (hit) {
                const int at = atomicAdd(&sh.hits, 1);
                if (at < p.room) list[at] = static_cast<uint32_t>(v);
            }
        }
        __syncthreads();
        const int hits = sh.hits;
        over |= hits > p.room;
        S += acc.x + acc.y;
        for (int i = tid; i < min(hits, p.room) * kW; i += kT) {
            const int at = static_cast<int>(list[i / kW]) * kW + i % kW;
            const float v = E::lds(staged + at);
            const int j = s0 + at - ph;
            if (v >= theta) {
                if (j >= 0 && j < V) append(v, j);  // (-inf from outside the row)
            } else if (kRest) {
                fixed += __float2ull_rn(ex2((v - theta) * c) * kTopFix);
            }
        }
        __syncthreads();
    });
    auto block_sum_fixed = [&](unsigned long long v) {
        v = block_reduce<kT>(v, [](unsigned long long a, unsigned long long b) { return a + b; }, sh.warp_u);
        return __ull2float_rn(v) * (1.f / kTopFix);
    };
    if constexpr (kRest) S = block_sum_f(S) + block_sum_fixed(fixed);
    int n = sh.n;
    TopPart part = {n, (over || n > p.room) ? 1 : 0, S, sh.err ? 1.f : 0.f};
    const TopPart* parts = exchange(part);
    int before = 0;
    bool slow = false, err = false;
    n = 0;
    S = 0.f;
    for (int r = 0; r < csize; ++r) {
        before += r < rank ? parts[r].n : 0;
        n += parts[r].n;
        S += parts[r].s;
        slow |= parts[r].m != 0;
        err |= parts[r].top != 0.f;
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
        // the entries above it, then those equal to it, in index order: warps own runs of positions
        if (tid == 0) sh.n = 0;
        __syncthreads();
        int equal = 0;
        sweep([&](int nc, int s0) {
            for (int i = tid; i < nc * kW; i += kT) {
                const int j = s0 + i - ph;
                if (j < 0 || j >= V) continue;
                const float v = E::lds(staged + i);
                const uint32_t k = key_of(v);
                if (k > kth) append(v, j);
                equal += k == kth ? 1 : 0;
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
                if (eq && at + __popc(m & ((1u << lane) - 1u)) < quota) append(value_of(kth), s0 + i + lane - ph);
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
    unsigned long long left = 0ull;
    auto emit = [&](unsigned long long k, int r) {
        if (r < K) {
            p.values[row * K + r] = value_of(static_cast<uint32_t>(k >> 32));
            p.ids[row * K + r] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(k));
        }
    };
    if (n <= kTopCountMost) {
        constexpr int kPer = (kTopCountMost + kT - 1) / kT;
        int r[kPer];
        unsigned long long k[kPer];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int i = tid + u * kT;
            r[u] = 0;
            k[u] = i < n ? cand[i] : 0ull;
            if (i - lane < n) {
#pragma unroll 4
                for (int j = 0; j < n; ++j) r[u] += cand[j] > k[u] ? 1 : 0;
            }
            if (i < n) {
                emit(k[u], r[u]);
                if (r[u] == K) sh.ref = value_of(static_cast<uint32_t>(k[u] >> 32));
            }
        }
        if (kRest && n > K) {
            __syncthreads();
            const float m = sh.ref;
#pragma unroll
            for (int u = 0; u < kPer; ++u)
                if (tid + u * kT < n && r[u] >= K)
                    left += __float2ull_rn(ex2((value_of(static_cast<uint32_t>(k[u] >> 32)) - m) * c) * kTopFix);
        }
    } else {
        int size = 1;
        while (size < n) size <<= 1;  // <= room
        for (int i = n + tid; i < size; i += kT) cand[i] = 0ull;
        for (int k = 2; k <= size; k <<= 1) {
            for (int j = k >> 1; j > 0; j >>= 1) {
                __syncthreads();
                for (int t = tid; t < size / 2; t += kT) {
                    const int a = 2 * t - (t & (j - 1)), b = a + j;
                    const unsigned long long va = cand[a], vb = cand[b];
                    const bool descending = (a & k) == 0;
                    if ((va < vb) == descending) {
                        cand[a] = vb;
                        cand[b] = va;
                    }
                }
            }
        }
        __syncthreads();
        for (int i = tid; i < min(n, K); i += kT) emit(cand[i], i);
        if (kRest && n > K) {
            const float m = value_of(static_cast<uint32_t>(cand[K] >> 32));
            if (tid == 0) sh.ref = m;
            for (int i = K + tid; i < n; i += kT)
                left += __float2ull_rn(ex2((value_of(static_cast<uint32_t>(cand[i] >> 32)) - m) * c) * kTopFix);
        }
    }
    for (int i = n + tid; i < K; i += kT) {  // fewer than K numbers in the row
        p.values[row * K + i] = kNegInf;
        p.ids[row * K + i] = -1;
    }
    if constexpr (kRest) {
        if (n > K) {
            const float others = block_sum_fixed(left), m = sh.ref;
            S = fmaf(S, ex2((ref - m) * c), others);
            ref = m;
        }
        if (tid == 0) p.rest[row] = S > 0.f ? fmaf(log2f(S), kLn2, __fdiv_rn(ref, p.tau)) : kNegInf;
    }
}

// Shared memory per CTA beside the section.
static size_t top_extra(int room, int csize, int groups) {
    return size_t(room) * 12 + size_t(csize) * kTopThreads * groups * 4;
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
