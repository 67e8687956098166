// Tokens from logits: temperature, top-k, top-p, min-p, then the token whose interval of the cumulative weights holds u.
//
// With m the largest logit, a token weighs w = 2^(-(m - x) log2(e) / T).  All three filters keep a prefix of the tokens in
// descending order (equal logits: the lowest index first): the first k; those in front of which less than p * Z_k has
// gathered, Z_k the sum over the first k; those with w >= min_p.  The token is the first kept one, by index, at which the sum of
// kept weights exceeds u * (their sum).
//
// A row is read once: the CTAs of a cluster (one to eight) hold it in shared memory and go over it there.  Nothing is sorted but the
// members of one bin: (m - x) / T in units of 1/32 is a bin number that falls as x rises, one pass sums counts and weights
// per bin, the bins' sums say in which bin a prefix ends, and only that bin's members (some hundreds of 131071) are put in order.
// A bin with more members than fit (many equal logits) is bisected instead.
//
// A token on the wrong side of a border is another token, so that weights are summed as integers, in units of 2^-40 (no order
// of additions matters), and formed to about 1e-9 of themselves: fp32 steps on a difference m - x that is kept in two parts.  Tokens
// more than 28 nats below the top weigh less than half a unit, and nothing.
#include <cooperative_groups.h>

#include "gdn_attn.cuh"
#include "gdn_sample.cuh"

namespace cg = cooperative_groups;

namespace gdn {

namespace {

constexpr int SA_THREADS = 512, SA_WARPS = SA_THREADS / 32;
constexpr int SA_BINS = 1024;           // the last one: everything that weighs nothing
constexpr float SA_PER_NAT = 32.f;
constexpr int SA_SORT = 2048;           // members of a bin that are sorted
constexpr int SA_UNIT = 40;             // weights in units of 2^-40
typedef unsigned long long u64;

struct SampleShared {
    u64 table[32];                      // 2^(-j/32) in units
    u64 sorted[SA_SORT];
    float table_16[32];                 // the same in units of 16
    u64 mass[SA_BINS];                  // of the CTA; then, for the bins of this rank's share, of the cluster
    uint32_t count[SA_BINS];
    u64 sum[2][SA_WARPS + 1];           // of the CTA's warps, then of the CTA (read by the cluster), in turn
    uint32_t number[2][SA_WARPS + 1];
    float top[SA_WARPS + 1];
    int members;                        // rank 0: entries of `sorted`
    u64 cut_key, cut_mass;              // rank 0: where a prefix ends inside a bin, and what it weighs up to there
    uint32_t scan_n[SA_WARPS];
    u64 scan_w[SA_WARPS];
    int bin;                            // where a prefix ends
    uint32_t before_n;
    u64 before_w;
    int picked;
};

// In units, of the token whose logit is d + lo below the top; per = 32 log2(e) / T in two parts.
struct Weigh {
    float m, per_hi, per_lo;
    bool finite;
    const u64 *table;
    const float *table_16;
    __device__ __forceinline__ u64 operator()(float x) const
    {
        const float d = fmaxf(m - x, 0.f);
        const float t = __fmul_rn(d, per_hi);   // (rounded here, whatever is added to it: err is what this loses)
        if (!(t < 28.f * 1.4426950408889634f * 32.f && d < INFINITY)) return 0;
        // m - x = d + lo exactly
        const float back = d - m;
        const float lo = finite ? (m - (d - back)) + (-x - back) : 0.f;
        const float err = fmaf(d, per_hi, -t) + fmaf(d, per_lo, lo * per_hi);
        const float shifted = t + 12582912.f;               // 1.5 * 2^23: rounds t to a whole number
        const int n = __float_as_int(shifted) - 0x4B400000;
        const float r = -((t - (shifted - 12582912.f)) + err) * 0.021660849392498290f;   // ln(2) / 32
        // e^r - 1 of |r| <= 0.011: the terms of its series
        const float q = r * fmaf(r, fmaf(r, fmaf(r, 0.041666666666666664f, 0.16666666666666666f), 0.5f), 1.f);
        const u64 w = table[n & 31];
        // (the correction is below 2^40 * 0.011 < 2^34: in units of 16 it fits a 32-bit number)
        const long long c = (long long)__float2int_rn(table_16[n & 31] * q) * 16;
        const u64 v = w + (u64)c;
        const int down = n >> 5;
        return down ? (v + (1ull << (down - 1))) >> down : v;
    }
};

__device__ __forceinline__ uint32_t ordered(float x)   // as unsigned numbers in the order of x
{
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);   // (-0 and 0 are equal)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ u64 key_of(float x, int index) { return (u64)(~ordered(x)) << 32 | (uint32_t)index; }
__device__ __forceinline__ float logit_of(u64 key)
{
    const uint32_t u = ~(uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}

template <typename T> struct Quad;   // four logits
template <> struct Quad<float> {
    static __device__ __forceinline__ float4 get(const float *p) { return *reinterpret_cast<const float4 *>(p); }
};
template <> struct Quad<__nv_bfloat16> {
    static __device__ __forceinline__ float4 get(const __nv_bfloat16 *p)
    {
        const uint2 u = *reinterpret_cast<const uint2 *>(p);
        return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                           __uint_as_float(u.y & 0xFFFF0000u));
    }
};

template <typename T> __global__ void __launch_bounds__(SA_THREADS) sample_kernel(const SampleParams p, int chunk, int places)
{
    extern __shared__ __align__(16) unsigned char sa_smem[];
    SampleShared &sh = *reinterpret_cast<SampleShared *>(sa_smem);
    T *x_s = reinterpret_cast<T *>(sa_smem + (sizeof(SampleShared) + 15) / 16 * 16);   // [places], a multiple of 128 per warp
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row = (int)blockIdx.x / ranks;
    constexpr int PIECE = 16 / (int)sizeof(T);

    if (tid < 32) {
        const double w = exp2((double)SA_UNIT - tid / 32.0);
        sh.table[tid] = (u64)(w + 0.5);
        sh.table_16[tid] = (float)(w / 16.0);
    }
    wait_for_previous_kernel();

    // ---- the row's part [first, first + n) of this CTA, at places shift ... of x_s: 16-byte pieces of both line up
    const int first = min(rank * chunk, p.vocab), n = min(chunk, p.vocab - first);
    const T *src = static_cast<const T *>(p.logits) + (size_t)row * p.row_stride + first;
    const int shift = (int)((reinterpret_cast<uintptr_t>(src) / sizeof(T)) % PIECE);
    float top = -INFINITY;
    auto one = [&](int place) {   // a place outside the part holds no logit; no number is none either
        const int i = place - shift;
        float x = i >= 0 && i < n ? load_as_float(src + i) : -INFINITY;
        x = fmaxf(x, -INFINITY);
        top = fmaxf(top, x);
        if constexpr (sizeof(T) == 4) x_s[place] = x;
        else x_s[place] = __float2bfloat16_rn(x);
    };
    {
        // pieces that lie wholly inside: [1 or 0, whole)
        const int begin = shift ? 1 : 0, whole = (shift + n) / PIECE;
        const uint4 *from = reinterpret_cast<const uint4 *>(src - shift);
        uint4 *to = reinterpret_cast<uint4 *>(x_s);
#pragma unroll 8
        for (int i = begin + tid; i < whole; i += SA_THREADS) {
            uint4 u = __ldg(from + i);
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float x = fmaxf(__uint_as_float((&u.x)[k]), -INFINITY);
                    top = fmaxf(top, x);
                    (&u.x)[k] = __float_as_uint(x);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float a = fmaxf(__uint_as_float((&u.x)[k] << 16), -INFINITY), b = fmaxf(__uint_as_float((&u.x)[k] & 0xFFFF0000u), -INFINITY);
                    top = fmaxf(top, fmaxf(a, b));
                    (&u.x)[k] = __float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xFFFF0000u);
                }
            }
            to[i] = u;
        }
        const int behind = max(whole, begin) * PIECE;
        if (tid < begin * PIECE) one(tid);
        for (int i = behind + tid; i < places; i += SA_THREADS) one(i);
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    if (lane == 0) sh.top[warp] = top;
    for (int i = tid; i < SA_BINS; i += SA_THREADS) {
        sh.count[i] = 0;
        sh.mass[i] = 0;
    }
    if (tid == 0) sh.members = 0;
    __syncthreads();
    if (tid < 32) {
        float t = lane < SA_WARPS ? sh.top[lane] : -INFINITY;
#pragma unroll
        for (int off = 16; off; off >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, off));
        if (lane == 0) sh.top[SA_WARPS] = t;
    }
    cluster.sync();
    float m = -INFINITY;
    for (int r = 0; r < ranks; ++r) m = fmaxf(m, *cluster.map_shared_rank(&sh.top[SA_WARPS], r));

    const float T_row = p.temperature ? p.temperature[row] : 1.f;
    const bool greedy = !(T_row > 0.f);
    int k = p.top_k ? p.top_k[row] : 0;
    if (k >= p.vocab) k = 0;
    const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
    const bool by_k = k > 0, by_p = top_p < 1.f;
    const double per = fmin(32.0 * 1.4426950408889634 / (double)T_row, 1e30);
    const Weigh weigh{m, (float)per, (float)(per - (double)(float)per), m < INFINITY, sh.table, sh.table_16};
    const float to_bin = (float)fmin((double)SA_PER_NAT / (double)T_row, 1e30);
    auto place_of = [&](float x) { return fmaxf(m - x, 0.f) * to_bin; };   // its whole part is the bin (no number: the last)

    // every four logits of the CTA's part, in rising order for one warp: a warp has `places / SA_WARPS` places
    const int per_warp = places / SA_WARPS, from_place = warp * per_warp;
    auto index_at = [&](int place) { return first + place - shift; };
    int turn = 0;
    // sums over the cluster of (w, c) of all threads; before_w: of the ranks and warps in front of this warp
    auto cluster_sum = [&](u64 w, uint32_t c, u64 &all_w, uint32_t &all_c, u64 *before_w) {
#pragma unroll
        for (int off = 16; off; off >>= 1) {
            w += __shfl_xor_sync(0xffffffffu, w, off);
            c += __shfl_xor_sync(0xffffffffu, c, off);
        }
        if (lane == 0) {
            sh.sum[turn][warp] = w;
            sh.number[turn][warp] = c;
        }
        __syncthreads();
        if (tid == 0) {
            u64 a = 0;
            uint32_t b = 0;
            for (int i = 0; i < SA_WARPS; ++i) {
                a += sh.sum[turn][i];
                b += sh.number[turn][i];
            }
            sh.sum[turn][SA_WARPS] = a;
            sh.number[turn][SA_WARPS] = b;
        }
        cluster.sync();
        all_w = 0;
        all_c = 0;
        u64 front = 0;
        for (int r = 0; r < ranks; ++r) {
            const u64 a = *cluster.map_shared_rank(&sh.sum[turn][SA_WARPS], r);
            if (r < rank) front += a;
            all_w += a;
            all_c += *cluster.map_shared_rank(&sh.number[turn][SA_WARPS], r);
        }
        if (before_w) {
            for (int i = 0; i < warp; ++i) front += sh.sum[turn][i];
            *before_w = front;
        }
        turn ^= 1;   // (the next sum's barrier lies between these reads and the sum after it)
    };

    if (m == -INFINITY || greedy) {   // nothing to choose from, or the first of the largest
        int best = 0x7fffffff;
        if (m > -INFINITY)
            for (int i = from_place + lane * 4; i < from_place + per_warp; i += 128) {
                const float4 v = Quad<T>::get(x_s + i);
#pragma unroll
                for (int j = 3; j >= 0; --j)
                    if ((&v.x)[j] == m) best = min(best, index_at(i + j));
            }
#pragma unroll
        for (int off = 16; off; off >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, off));
        if (lane == 0) sh.number[0][warp] = (uint32_t)best;
        __syncthreads();
        if (tid == 0) {
            for (int i = 0; i < SA_WARPS; ++i) best = min(best, (int)sh.number[0][i]);
            sh.number[0][SA_WARPS] = (uint32_t)best;
        }
        cluster.sync();
        if (rank == 0 && tid == 0) {
            for (int r = 0; r < ranks; ++r) best = min(best, (int)*cluster.map_shared_rank(&sh.number[0][SA_WARPS], r));
            p.token[row] = m > -INFINITY ? best : -1;
            if (p.prob) p.prob[row] = m > -INFINITY ? 1.f : 0.f;
        }
        cluster.sync();   // (nobody leaves while its shared memory is read)
        return;
    }

    // ---- where the kept prefix ends: tokens of bins in front of `cut_bin`, and of that bin those with keys up to `cut_key`
    int cut_bin = SA_BINS - 1;
    u64 cut_key = ~0ull;
    if (by_k || by_p) {
        for (int i = from_place + lane * 4; i < from_place + per_warp; i += 128) {
            const float4 v = Quad<T>::get(x_s + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x = (&v.x)[j], b = place_of(x);
                if (b < (float)(SA_BINS - 1)) {
                    if (by_k) atomicAdd(&sh.count[(int)b], 1u);
                    if (by_p) atomicAdd(&sh.mass[(int)b], weigh(x));
                }
            }
        }
        // bins' sums over the cluster: each rank those of its share, then everybody reads all of them
        cluster.sync();
        const int share = SA_BINS / ranks;
        for (int i = rank * share + tid; i < (rank + 1) * share; i += SA_THREADS) {
            uint32_t c = 0;
            u64 w = 0;
            for (int r = 0; r < ranks; ++r) {
                if (by_k) c += *cluster.map_shared_rank(&sh.count[i], r);
                if (by_p) w += *cluster.map_shared_rank(&sh.mass[i], r);
            }
            sh.count[i] = c;   // (of this bin no other rank reads this copy)
            sh.mass[i] = w;
        }
        cluster.sync();
        // this thread's two bins, and the sums over all in front of them
        uint32_t c2[2], cb;
        u64 w2[2], wb;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = 2 * tid + j;
            c2[j] = *cluster.map_shared_rank(&sh.count[i], i / share);
            w2[j] = *cluster.map_shared_rank(&sh.mass[i], i / share);
        }
        {
            uint32_t c = c2[0] + c2[1];
            u64 w = w2[0] + w2[1];
            const uint32_t c_own = c;
            const u64 w_own = w;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const uint32_t cu = __shfl_up_sync(0xffffffffu, c, off);
                const u64 wu = __shfl_up_sync(0xffffffffu, w, off);
                if (lane >= off) {
                    c += cu;
                    w += wu;
                }
            }
            if (lane == 31) {
                sh.scan_n[warp] = c;
                sh.scan_w[warp] = w;
            }
            __syncthreads();
            cb = c - c_own;
            wb = w - w_own;
            for (int i = 0; i < warp; ++i) {
                cb += sh.scan_n[i];
                wb += sh.scan_w[i];
            }
        }
        u64 z = 0;   // weight of the first k (all, where k is off)
        for (int i = 0; i < SA_WARPS; ++i) z += sh.scan_w[i];

        // The end of a prefix inside bin `bin`: the smallest key there up to which `enough` holds of the (count, weight) of the
        // bin's members with keys up to it; and that weight.
        auto end_in_bin = [&](int bin, auto enough, u64 &key, u64 &weight) {
            auto in_bin = [&](float x) {
                const float b = place_of(x);
                return b >= (float)bin && b < (float)(bin + 1);
            };
            int *members = cluster.map_shared_rank(&sh.members, 0);
            u64 *list = cluster.map_shared_rank(sh.sorted, 0);
            for (int i = from_place + lane * 4; i < from_place + per_warp; i += 128) {
                const float4 v = Quad<T>::get(x_s + i);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (in_bin((&v.x)[j])) {
                        const int at = atomicAdd(members, 1);
                        if (at < SA_SORT) list[at] = key_of((&v.x)[j], index_at(i + j));
                    }
            }
            cluster.sync();
            const int have = *members;
            if (have <= SA_SORT) {
                if (rank == 0) {   // in order by exchanges at distances that are powers of two
                    int size = 32;
                    while (size < have) size *= 2;
                    for (int i = have + tid; i < size; i += SA_THREADS) sh.sorted[i] = ~0ull;
                    __syncthreads();
                    for (int run = 2; run <= size; run *= 2)
                        for (int apart = run / 2; apart; apart /= 2) {
                            for (int i = tid; i < size / 2; i += SA_THREADS) {
                                const int a = 2 * i - (i & (apart - 1)), b = a + apart;
                                const u64 ka = sh.sorted[a], kb = sh.sorted[b];
                                if ((ka > kb) == ((a & run) == 0)) {
                                    sh.sorted[a] = kb;
                                    sh.sorted[b] = ka;
                                }
                            }
                            __syncthreads();
                        }
                    // the first member up to which it is enough, by one warp, 32 members at a time
                    if (warp == 0) {
                        u64 sum = 0;
                        bool found = false;
                        for (int i = 0; i < have && !found; i += 32) {
                            const bool there = i + lane < have;
                            const u64 own_key = sh.sorted[min(i + lane, have - 1)];
                            u64 w = there ? weigh(logit_of(own_key)) : 0;
#pragma unroll
                            for (int off = 1; off < 32; off <<= 1) {
                                const u64 up = __shfl_up_sync(0xffffffffu, w, off);
                                if (lane >= off) w += up;
                            }
                            const unsigned yes = __ballot_sync(0xffffffffu, there && enough((uint32_t)(i + lane + 1), sum + w));
                            const int at = yes ? __ffs(yes) - 1 : min(31, have - 1 - i);
                            const u64 upto = sum + __shfl_sync(0xffffffffu, w, at), k_at = __shfl_sync(0xffffffffu, own_key, at);
                            found = yes != 0;
                            if (lane == 0) {
                                sh.cut_key = k_at;
                                sh.cut_mass = upto;
                            }
                            sum += __shfl_sync(0xffffffffu, w, 31);
                        }
                    }
                }
                cluster.sync();
                if (rank == 0 && tid == 0) sh.members = 0;   // (everybody has read it)
                key = *cluster.map_shared_rank(&sh.cut_key, 0);
                weight = *cluster.map_shared_rank(&sh.cut_mass, 0);
                cluster.sync();   // (before the list is used again)
                return;
            }
            // too many of them: the key bit by bit, each with a pass over the row
            key = ~0ull;
            weight = 0;
            u64 lo = 0, hi = ~0ull;
            while (lo < hi) {
                const u64 mid = lo + (hi - lo) / 2;
                u64 w = 0, w_all;
                uint32_t c = 0, c_all;
                for (int i = from_place + lane * 4; i < from_place + per_warp; i += 128) {
                    const float4 v = Quad<T>::get(x_s + i);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (in_bin((&v.x)[j]) && key_of((&v.x)[j], index_at(i + j)) <= mid) {
                            ++c;
                            w += weigh((&v.x)[j]);
                        }
                }
                cluster_sum(w, c, w_all, c_all, nullptr);
                if (c_all && enough(c_all, w_all)) {
                    hi = mid;
                    weight = w_all;
                } else
                    lo = mid + 1;
            }
            key = lo;
            if (rank == 0 && tid == 0) sh.members = 0;
            cluster.sync();
        };
        // which bin: its sums are in one thread
        auto end_in = [&](auto enough, u64 &weight) {
            if (tid == 0) sh.bin = SA_BINS - 1;
            __syncthreads();
            uint32_t c = cb;
            u64 w = wb;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const bool was = (c > 0 || w > 0) && enough(c, w);   // (an empty prefix is never enough: one token is kept)
                c += c2[j];
                w += w2[j];
                if (!was && (c2[j] || w2[j]) && enough(c, w)) {
                    sh.bin = 2 * tid + j;
                    sh.before_n = c - c2[j];
                    sh.before_w = w - w2[j];
                }
            }
            __syncthreads();
            const int bin = sh.bin;
            const uint32_t bn = sh.before_n;
            const u64 bw = sh.before_w;
            u64 key = ~0ull;
            if (bin < SA_BINS - 1) {
                u64 inside;
                end_in_bin(bin, [&](uint32_t cc, u64 ww) { return enough(bn + cc, bw + ww); }, key, inside);
                weight = bw + inside;
            }
            __syncthreads();
            if (bin < cut_bin || (bin == cut_bin && key < cut_key)) {
                cut_bin = bin;
                cut_key = key;
            }
        };
        if (by_k) end_in([&](uint32_t c, u64) { return c >= (uint32_t)k; }, z);
        if (by_p) {
            const double goal = (double)top_p * (double)z;
            u64 unused = 0;
            end_in([&](uint32_t, u64 w) { return (double)w >= goal; }, unused);
        }
    }

    // ---- the kept weights: of each warp, of the warps in front, of all
    const u64 least = min_p > 0.f ? (u64)ceil(fmin((double)min_p, 1.0) * (double)(1ull << SA_UNIT)) : 0;
    auto kept = [&](float x, int place) -> u64 {
        const float b = place_of(x);
        if (b < (float)cut_bin || (b < (float)(cut_bin + 1) && key_of(x, index_at(place)) <= cut_key)) {
            const u64 w = weigh(x);
            return w >= least ? w : 0;
        }
        return 0;
    };
    u64 w = 0, z, before;
    uint32_t unused;
    for (int i = from_place + lane * 4; i < from_place + per_warp; i += 128) {
        const float4 v = Quad<T>::get(x_s + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) w += kept((&v.x)[j], i + j);
    }
    cluster_sum(w, 0, z, unused, &before);
    double u = (double)p.uniform[row];
    u = u >= 0.0 ? u : 0.0;   // (no number: 0)
    const double at = u * (double)z;
    const u64 goal = at < (double)z ? min((u64)at, z - 1) : z - 1;
#pragma unroll
    for (int off = 16; off; off >>= 1) w += __shfl_xor_sync(0xffffffffu, w, off);
    if (before <= goal && goal < before + w) {   // this warp alone
        u64 sum = before;
        for (int i = from_place; i < from_place + per_warp; i += 128) {
            const float4 v = Quad<T>::get(x_s + i + lane * 4);
            u64 own[4], four = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) four += own[j] = kept((&v.x)[j], i + lane * 4 + j);
            u64 upto = four;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const u64 up = __shfl_up_sync(0xffffffffu, upto, off);
                if (lane >= off) upto += up;
            }
            const u64 all = __shfl_sync(0xffffffffu, upto, 31);
            if (goal < sum + all) {
                u64 s = sum + upto - four;
                bool mine = false;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (!mine && s <= goal && goal < s + own[j]) {
                        p.token[row] = index_at(i + lane * 4 + j);
                        if (p.prob) p.prob[row] = (float)((double)own[j] / (double)z);
                        mine = true;
                    }
                    s += own[j];
                }
                break;
            }
            sum += all;
        }
    }
    cluster.sync();   // (nobody leaves while its shared memory is read)
}

}  // namespace

cudaError_t launch_sample(const SampleParams &p, bool bf16, cudaStream_t stream)
{
    // CTAs of a row: as many as keep the SMs busy, up to eight, none with less than 4096 logits
    int ranks = 1;
    while (ranks < 8 && p.vocab > 4096 * ranks && (p.n_rows * ranks < 2 * 148 || p.vocab > 16384 * ranks)) ranks *= 2;
    const int chunk = ((p.vocab + ranks - 1) / ranks + 7) / 8 * 8;
    const int step = 128 * SA_WARPS, places = (chunk + 8 + step - 1) / step * step;
    const size_t smem = (sizeof(SampleShared) + 15) / 16 * 16 + (size_t)places * (bf16 ? 2 : 4);
    static PerContext seen[2];
    const auto kernel = bf16 ? sample_kernel<__nv_bfloat16> : sample_kernel<float>;
    int sms = 0;
    const cudaError_t e = device_sms(seen[bf16], reinterpret_cast<const void *>(kernel), 220 << 10, &sms);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(p.n_rows * ranks));
    cfg.blockDim = dim3(SA_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ranks;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, p, chunk, places);
}

}  // namespace gdn
