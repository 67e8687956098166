// Tokens from logits: temperature, top-k, top-p, min-p, then the token whose interval of the cumulative weights holds u.
//
// With m the largest logit, a token weighs w = 2^(-(m - x) log2(e) / T).  All three filters keep a prefix of the tokens in
// descending order (equal logits: the lowest index first): the first k; those in front of which less than p * Z_k has
// gathered, Z_k the sum over the first k; those with w >= min_p.  The token is the first kept one, by index, at which the sum of
// kept weights exceeds u * (their sum).
//
// A row belongs to the CTAs of a cluster (one to eight).  They go over it two to four times: from shared memory where a CTA's part is
// small (few rows: what counts is the time of a pass), else from where the first reading left it: L2, while the rows at work at one time
// fit there (many rows: what counts is how many CTAs an SM holds.  Up to 592 rows are at work at once; 256 of 131071 fp32 logits, 134 MB,
// take 0.90 us each with top-p, 600 of them 0.84: instructions decide, not where a pass reads from).  Nothing is sorted but the
// members of one bin: (m - x) / T in units of 1/64 is a bin number that falls as x rises, and one pass counts the tokens of each bin.
// The first k end in a bin that the counts tell.  Where the p end the counts nearly tell: a count times the weight at the bin's middle
// is off by a percent at most, so that the next pass, which sums the weights for good, sums them up to that bin, in it and
// its neighbours, and altogether, and sees whether it is one of the three (else the estimate starts again from these sums).  Only that bin's members (some hundreds
// of 131071) are put in order; a bin with more members than fit (many equal logits) is bisected instead.  What the pass summed up
// to the bin, warp by warp, also says where the token lies.
// The first k of a row, k up to two thousand, are put in order at once, and the row is done with.
//
// A token on the wrong side of a border is another token, so that weights are formed in 64 bits (to 2e-12 of themselves) and summed as
// integers, in units of 2^-45, where no order of additions matters: 2^18 weights of 1 just fit.  Each is rounded to whole units, which makes
// the sum of n of them wrong by n 2^-46 at most (equal logits), as a rule by sqrt(n) 2^-47; less than half a unit is nothing.  (In fp32 a
// weight is off by up to 2^-24 of itself, and the sum of many that are alike by as much.)
#include <cooperative_groups.h>

#include "gdn_attn.cuh"
#include "gdn_sample.cuh"

namespace cg = cooperative_groups;

namespace gdn {

namespace {

constexpr int SA_THREADS = 256, SA_WARPS = SA_THREADS / 32, SA_CTAS = 4;
constexpr int SA_BINS = 2048, SA_OWN = SA_BINS / SA_THREADS;   // bins, of a thread
constexpr int SA_HELD = 32 << 10;       // bytes of a row that a CTA holds in shared memory
constexpr float SA_PER_NAT = 64.f;
constexpr int SA_SORT = 2048;           // members of a bin that are sorted; more are bisected, some 40 passes: 131071 equal logits, top-p, take 0.9 ms (256 rows: 6 ms)
constexpr int SA_UNIT = 45;             // weights in units of 2^-45
constexpr double SA_DEEP = 60.0;        // logits further below the largest than this many powers of two count as that far: weights of nothing
typedef unsigned long long u64;

struct SampleShared {
    u64 sorted[SA_SORT];                // members of a bin; of rank 0, those of all ranks
    uint32_t count[SA_BINS + 32];       // of the CTA; then, for the bins of this rank's share, of the cluster; 32 for what lies behind all bins
    u64 sum[2][5][SA_WARPS + 1];        // of the CTA's warps, then of the CTA (read by the cluster), in turn
    float top[SA_WARPS + 1];
    int best[SA_WARPS + 1];
    int members;                        // entries of `sorted`, of this rank alone
    u64 cut_key;                        // rank 0: where a prefix ends inside a bin
    uint32_t scan_n[SA_WARPS];
    float scan_a[SA_WARPS];
    int bin;
    uint32_t before_n;
    bool few;                           // tokens down to the end of `bin`
};

// 2^(d per) in units, d per in [-62, 0]: n + r with r in [-1/2, 1/2], 2^r by the polynomial of degree 8 with p(0) = 1 and the least relative
// error there, 1.1e-12 (fitted to 2^r), n into the exponent; a number so large that its last bit is a unit rounds to whole units and leaves
// them in the low bits.  (Doubles run at half of fp32's rate, but need half the instructions that fp32 in two parts, to 8e-8, did: 256 x
// 131071 logits without filters 105 us instead of 153, with top-p 230 either way.)
__device__ __forceinline__ u64 units_of_power(double d, double per)
{
    constexpr double whole = 6755399441055744.0;                             // 1.5 * 2^52
    constexpr double unit = 1.5 * (double)(1ull << (52 - SA_UNIT));
    const double n = fma(d, per, whole), r = fma(d, per, whole - n);
    double y = 1.3344183484134179e-06;
    y = fma(y, r, 1.5314209223349525e-05);
    y = fma(y, r, 0.0001540309828656179);
    y = fma(y, r, 0.0013333434157560176);
    y = fma(y, r, 0.009618129558838935);
    y = fma(y, r, 0.05550410959228811);
    y = fma(y, r, 0.2402265069474259);
    y = fma(y, r, 0.6931471805412327);
    y = fma(y, r, 1.0);
    y = __hiloint2double(__double2hiint(y) + (__double2loint(n) << 20), __double2loint(y));
    return (u64)(__double_as_longlong(y + unit) - __double_as_longlong(unit));
}

// Weight in units of any logit, where the largest is so large, or weights fall so slowly or so fast, that Weigh's bound is none.  A
// function of its own, as the other steps that are taken now and then are: inlined wherever they are called they make code that few rows
// never find in the instruction cache.
__device__ __noinline__ u64 weigh_any(float x, double m, double per)
{
    if (!(x > -INFINITY)) return 0;   // (no number, too)
    const double d = (double)x - m;
    if (d == 0.0) return 1ull << SA_UNIT;   // (a short way for rows of equal logits, whose last bin is bisected)
    return d * per > -SA_DEEP ? units_of_power(d, per) : 0;
}

// The same without the unit's rounding, of one token that weighs something.
__device__ __noinline__ double weigh_exactly(float x, double m, double per)
{
    return exp(((double)x - m) * per * 0.6931471805599453) * (double)(1ull << SA_UNIT);
}

// By a whole CTA: `have` keys in rising order, by exchanges at distances that are powers of two; the greatest number stands behind them
// up to such a power.
__device__ __noinline__ void sort_keys(u64 *keys, int have)
{
    const int tid = threadIdx.x;
    int size = 32;
    while (size < have) size *= 2;
    for (int i = have + tid; i < size; i += SA_THREADS) keys[i] = ~0ull;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2)
        for (int apart = run / 2; apart; apart /= 2) {
            for (int i = tid; i < size / 2; i += SA_THREADS) {
                const int a = 2 * i - (i & (apart - 1)), b = a + apart;
                const u64 ka = keys[a], kb = keys[b];
                if ((ka > kb) == ((a & run) == 0)) {
                    keys[a] = kb;
                    keys[b] = ka;
                }
            }
            __syncthreads();
        }
}

// Weights in units of tokens with given logits.
struct Weigh {
    double m, per;   // the largest logit; log2(e) / T
    float deep;      // logits below count as this one, which weighs nothing
    bool any;        // no such bound: see weigh_any

    __device__ __forceinline__ u64 one(float x) const { return weigh_any(x, m, per); }
    __device__ __forceinline__ void four(const float4 &x, u64 (&w)[4]) const
    {
        if (any) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = one((&x.x)[j]);
            return;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = units_of_power((double)fmaxf((&x.x)[j], deep) - m, per);   // (of a number and none, the number)
    }
    __device__ __forceinline__ double exactly(float x) const { return weigh_exactly(x, m, per); }
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

template <typename T, bool HELD> __global__ void __launch_bounds__(SA_THREADS, HELD ? 3 : SA_CTAS) sample_kernel(const SampleParams p, int chunk, int places)
{
    extern __shared__ __align__(16) unsigned char sa_smem[];
    SampleShared &sh = *reinterpret_cast<SampleShared *>(sa_smem);
    T *x_s = reinterpret_cast<T *>(sa_smem + (sizeof(SampleShared) + 15) / 16 * 16);   // [places], a multiple of 8 per warp
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row = (int)blockIdx.x / ranks;
    constexpr int PIECE = 16 / (int)sizeof(T);

    if (tid == 0) sh.members = 0;
    for (int i = tid; i < SA_BINS; i += SA_THREADS) sh.count[i] = 0;
    wait_for_previous_kernel();

    // ---- the row's part [first, first + n) of this CTA, at places shift, shift + 1, ...: place 0 is on a 16-byte boundary
    const int first = min(rank * chunk, p.vocab), n = min(chunk, p.vocab - first);
    const T *src = static_cast<const T *>(p.logits) + (size_t)row * p.row_stride + first;
    const int shift = (int)((reinterpret_cast<uintptr_t>(src) / sizeof(T)) % PIECE), end = shift + n;
    // a warp goes over its share of the places, four neighbouring ones per lane
    const int from_place = warp * (places / SA_WARPS), to_place = min(from_place + places / SA_WARPS, (end + 3) / 4 * 4);
    auto index_at = [&](int place) { return first + place - shift; };
    const int in0 = (shift + 3) / 4 * 4, in1 = end / 4 * 4;   // [in0, in1): fours of places that lie wholly inside
    auto from_row = [&](int i, int warp_at) {   // four logits where they come from; the warp is at places warp_at ... + 127
        if (warp_at >= in0 && warp_at + 128 <= in1) return Quad<T>::get(src - shift + i);
        float4 v;   // a place outside the part holds none
#pragma unroll
        for (int j = 0; j < 4; ++j) (&v.x)[j] = i + j >= shift && i + j < end ? load_as_float(src - shift + i + j) : -INFINITY;
        return v;
    };
    bool infinite = false;   // the largest logit is +inf: those that are count as 0, all others as none
    auto quad = [&](int i, int warp_at) {
        if constexpr (HELD) return Quad<T>::get(x_s + i);
        else return from_row(i, warp_at);
    };
    auto as_finite = [&](float4 &v) {
        if (infinite) {
#pragma unroll
            for (int j = 0; j < 4; ++j) (&v.x)[j] = (&v.x)[j] == INFINITY ? 0.f : -INFINITY;
        }
    };
    // f(four logits, place) for this lane's fours of places [from, to) (of the whole warp), the next ones on their way meanwhile
    auto each = [&](int from, int to, auto f) {
        if (from >= to) return;
        const int mine = lane * 4;
        float4 next = from + mine < to ? quad(from + mine, from) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        for (int at = from; at < to; at += 128) {
            float4 v = next;
            if (at + 128 + mine < to) next = quad(at + 128 + mine, at + 128);
            as_finite(v);
            if (at + mine < to) f(v, at + mine);
        }
    };
    // the same for an f too short to wait behind: eight loads on their way
    auto each_short = [&](int from, int to, auto f) {
        constexpr int N = HELD ? 1 : 8;
        for (int at = from; at < to; at += N * 128) {
            float4 v[N];
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (at + k * 128 + lane * 4 < to) v[k] = quad(at + k * 128 + lane * 4, at + k * 128);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                as_finite(v[k]);
                if (at + k * 128 + lane * 4 < to) f(v[k], at + k * 128 + lane * 4);
            }
        }
    };
    float top = -INFINITY;
    auto take = [&](const float4 &v, int i) {
        top = fmaxf(fmaxf(fmaxf(top, v.x), v.y), fmaxf(v.z, v.w));   // (of a number and none, the number)
        if constexpr (HELD) {
            if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(x_s + i) = v;
            else *reinterpret_cast<uint2 *>(x_s + i) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
        }
    };
    {
        int at = from_place;
        for (; at < to_place && at < in0; at += 128)
            if (at + lane * 4 < to_place) take(from_row(at + lane * 4, at), at + lane * 4);
        for (; at + 8 * 128 <= min(to_place, in1); at += 8 * 128) {   // eight loads on their way
            float4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = Quad<T>::get(src - shift + at + k * 128 + lane * 4);
#pragma unroll
            for (int k = 0; k < 8; ++k) take(v[k], at + k * 128 + lane * 4);
        }
#pragma unroll 4
        for (; at < to_place; at += 128)
            if (at + lane * 4 < to_place) take(from_row(at + lane * 4, at), at + lane * 4);
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    if (lane == 0) sh.top[warp] = top;
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
    const bool here = sh.top[SA_WARPS] == m;   // this CTA has it
    infinite = m == INFINITY;
    if (infinite) m = 0.f;

    const float T_row = p.temperature ? p.temperature[row] : 1.f;
    const bool greedy = !(T_row > 0.f);

    if (m == -INFINITY || greedy) {   // nothing to choose from, or the first of the largest
        int best = 0x7fffffff;
        if (m > -INFINITY && here)
            each_short(from_place, to_place, [&](const float4 &v, int i) {
#pragma unroll
                for (int j = 3; j >= 0; --j)
                    if ((&v.x)[j] == m) best = min(best, index_at(i + j));
            });
#pragma unroll
        for (int off = 16; off; off >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, off));
        if (lane == 0) sh.best[warp] = best;
        __syncthreads();
        if (tid == 0) {
            for (int i = 0; i < SA_WARPS; ++i) best = min(best, sh.best[i]);
            sh.best[SA_WARPS] = best;
        }
        cluster.sync();
        if (rank == 0 && tid == 0) {
            for (int r = 0; r < ranks; ++r) best = min(best, *cluster.map_shared_rank(&sh.best[SA_WARPS], r));
            p.token[row] = m > -INFINITY ? best : -1;
            if (p.prob) p.prob[row] = m > -INFINITY ? 1.f : 0.f;
        }
        cluster.sync();   // (nobody leaves while its shared memory is read)
        return;
    }

    int k = p.top_k ? p.top_k[row] : 0;
    if (k >= p.vocab) k = 0;
    const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
    const bool by_k = k > 0, by_p = top_p < 1.f;
    const double per = 1.4426950408889634 / (double)T_row;
    const float d_deep = (float)(SA_DEEP / per);
    // (the bound can be told from m, and is finite)
    const Weigh weigh{m, per, m - d_deep, !(fabsf(m) * 2.4e-7f < 0.1f * d_deep && fabsf(m) + d_deep < 1e37f)};
    const float to_bin = (float)fmin((double)SA_PER_NAT / (double)T_row, 1e30);
    auto place_of = [&](float x) { return (m - x) * to_bin; };   // its whole part is the bin; it falls as x rises (no number: in no bin)

    int turn = 0;
    // sums of up to five numbers over the cluster; before: of the first one, of the ranks and warps in front of this warp
    auto cluster_sum = [&](auto &a, auto &all, u64 *before) {
        constexpr int N = (int)(sizeof(a) / sizeof(u64));
#pragma unroll
        for (int off = 16; off; off >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) a[i] += __shfl_xor_sync(0xffffffffu, a[i], off);
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) sh.sum[turn][i][warp] = a[i];
        __syncthreads();
        if (tid < N) {
            u64 s = 0;
            for (int i = 0; i < SA_WARPS; ++i) s += sh.sum[turn][tid][i];
            sh.sum[turn][tid][SA_WARPS] = s;
        }
        cluster.sync();
        u64 front = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) all[i] = 0;
        for (int r = 0; r < ranks; ++r) {
#pragma unroll
            for (int i = 0; i < N; ++i) all[i] += *cluster.map_shared_rank(&sh.sum[turn][i][SA_WARPS], r);
            if (before && r + 1 == rank) front = all[0];
        }
        if (before) {
            for (int i = 0; i < warp; ++i) front += sh.sum[turn][0][i];
            *before = front;
        }
        turn ^= 1;   // (the next sum's barrier lies between these reads and the sum after it)
    };

    // ---- where the kept prefix ends: tokens of bins in front of `cut_bin`, and of that bin those with keys up to `cut_key`
    int cut_bin = SA_BINS;
    u64 cut_key = ~0ull;
    auto inside = [&](float b, float x, int place) {   // of the prefix
        return b < (float)cut_bin || (b < (float)(cut_bin + 1) && key_of(x, index_at(place)) <= cut_key);
    };
    const u64 least = min_p > 0.f ? (u64)ceil(fmin((double)min_p, 1.0) * (double)(1ull << SA_UNIT)) : 0;
    u64 w = 0;              // this thread's share of the kept weights
    bool summed = false;    // where it is known already
    if (by_k || by_p) {
        each_short(from_place, to_place, [&](const float4 &v, int) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float b = place_of((&v.x)[j]);
                atomicAdd(&sh.count[b < (float)SA_BINS ? (int)b : SA_BINS + lane], 1u);   // (behind the bins: no two lanes meet)
            }
        });
        cluster.sync();
        // bins' counts over the cluster: each rank those of its share, then everybody reads all of them
        const int share = SA_BINS / ranks;
        for (int i = rank * share + tid; i < (rank + 1) * share; i += SA_THREADS) {
            uint32_t c = 0;
            for (int r = 0; r < ranks; ++r) c += *cluster.map_shared_rank(&sh.count[i], r);
            sh.count[i] = c;   // (of this bin no other rank reads this copy)
        }
        cluster.sync();
        uint32_t own[SA_OWN], mine = 0, cb;   // this thread's bins, their sum, and the counts of all in front of them
#pragma unroll
        for (int j = 0; j < SA_OWN; ++j) mine += own[j] = *cluster.map_shared_rank(&sh.count[SA_OWN * tid + j], (SA_OWN * tid + j) / share);
        {
            uint32_t c = mine;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const uint32_t up = __shfl_up_sync(0xffffffffu, c, off);
                if (lane >= off) c += up;
            }
            if (lane == 31) sh.scan_n[warp] = c;
            if (tid == 0) sh.bin = SA_BINS;
            __syncthreads();
            cb = c - mine;
            for (int i = 0; i < warp; ++i) cb += sh.scan_n[i];
        }
        auto in_bin = [&](float b, int bin) { return b >= (float)bin && b < (float)(bin + 1); };
        // the members of a bin, those of the prefix so far, to this rank's list
        auto keep_key = [&](float x, int place) {
            const int at = atomicAdd(&sh.members, 1);
            if (at < SA_SORT) sh.sorted[at] = key_of(x, index_at(place));
        };
        auto gather = [&](float b, float x, int place, int bin) {
            if (in_bin(b, bin) && inside(b, x, place)) keep_key(x, place);
        };
        // behind a barrier of the cluster: all ranks' lists to rank 0's; how many members there are (more than SA_SORT: nothing is moved)
        auto collect = [&]() {
            int in_front = 0, total = 0;
            for (int r = 0; r < ranks; ++r) {
                const int c = *cluster.map_shared_rank(&sh.members, r);
                if (r < rank) in_front += c;
                total += c;
            }
            if (rank != 0 && total <= SA_SORT) {
                u64 *list = cluster.map_shared_rank(sh.sorted, 0);
                for (int i = tid; i < sh.members; i += SA_THREADS) list[in_front + i] = sh.sorted[i];
            }
            cluster.sync();
            return total;
        };
        // The smallest key of the bin's members in the list up to which `enough` holds of the (count, weight) of those with keys up to it;
        // where they were too many for the list, found bit by bit, each with a pass over the row.  After a barrier of the cluster.
        auto end_in_list = [&](int bin, int have, bool weights, auto enough) {
            u64 key = ~0ull;
            if (have <= SA_SORT) {
                if (rank == 0) {
                    sort_keys(sh.sorted, have);
                    // the first member up to which it is enough: some neighbouring ones per thread, and the sums in front of them
                    constexpr int OWN = SA_SORT / SA_THREADS;
                    u64 own_w[OWN], upto = 0;
#pragma unroll
                    for (int j = 0; j < OWN; ++j) {
                        own_w[j] = weights && tid * OWN + j < have ? weigh.one(logit_of(sh.sorted[tid * OWN + j])) : 0;
                        upto += own_w[j];
                    }
                    u64 sum = upto;
#pragma unroll
                    for (int off = 1; off < 32; off <<= 1) {
                        const u64 up = __shfl_up_sync(0xffffffffu, upto, off);
                        if (lane >= off) upto += up;
                    }
                    u64 *parts = sh.sum[turn][0];   // (this rank alone; the next sum of the cluster lies behind a barrier)
                    if (lane == 31) parts[warp] = upto;
                    if (tid == 0) sh.cut_key = have ? sh.sorted[have - 1] : ~0ull;
                    __syncthreads();
                    sum = upto - sum;
                    for (int i = 0; i < warp; ++i) sum += parts[i];
#pragma unroll
                    for (int j = 0; j < OWN; ++j) {
                        const int i = tid * OWN + j;
                        const bool was = i > 0 && enough((uint32_t)i, sum);
                        sum += own_w[j];
                        if (i < have && !was && enough((uint32_t)(i + 1), sum)) sh.cut_key = sh.sorted[i];
                    }
                }
                cluster.sync();
                key = *cluster.map_shared_rank(&sh.cut_key, 0);
            } else {
                // (from the ends of the bin, a little further apart than rounding can put them)
                u64 lo = 0, hi = ~0ull;
                const float above = m - (float)bin / to_bin, below = m - (float)(bin + 1) / to_bin, more = (fabsf(above) + fabsf(below) + fabsf(m)) * 1e-5f;
                if (below - more > -3e38f && above + more < 3e38f) {
                    lo = key_of(above + more, 0);
                    hi = key_of(below - more, -1);
                }
                while (lo < hi) {
                    const u64 mid = lo + (hi - lo) / 2;
                    u64 a[2] = {0, 0}, all[2];
                    each(from_place, to_place, [&](const float4 &v, int i) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float x = (&v.x)[j], b = place_of(x);
                            if (in_bin(b, bin) && key_of(x, index_at(i + j)) <= mid && inside(b, x, i + j)) {
                                ++a[1];
                                if (weights) a[0] += weigh.one(x);
                            }
                        }
                    });
                    cluster_sum(a, all, nullptr);
                    if (all[1] && enough((uint32_t)all[1], all[0])) hi = mid;
                    else lo = mid + 1;
                }
                key = lo;
            }
            return key;
        };
        auto empty_list = [&]() {
            cluster.sync();   // (everybody has read it)
            if (tid == 0) sh.members = 0;
            __syncthreads();
        };

        if (by_k) {   // the bin in which the k-th token lies, and its key
            uint32_t c = cb;
#pragma unroll
            for (int j = 0; j < SA_OWN; ++j) {
                if (c < (uint32_t)k && (uint32_t)k <= c + own[j]) {
                    sh.bin = SA_OWN * tid + j;
                    sh.before_n = c;
                    sh.few = c + own[j] <= SA_SORT;
                }
                c += own[j];
            }
            __syncthreads();
            const int bin = sh.bin;
            if (k <= SA_SORT && bin < SA_BINS && sh.few) {
                // all tokens down to that bin fit the list: the rest goes on there, without the row
                each_short(from_place, to_place, [&](const float4 &v, int i) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (place_of((&v.x)[j]) < (float)(bin + 1)) keep_key((&v.x)[j], i + j);
                });
                cluster.sync();
                const int have = collect();
                if (rank != 0) return;   // (nobody reads its shared memory any more)
                sort_keys(sh.sorted, have);
                // weights' sums in falling order, by one warp; how many are kept of the first k
                int kept_n = k;
                if (warp == 0) {
                    u64 total = 0;
                    for (int pass = 0; pass < 2; ++pass) {   // the sum of the first k, then the prefix
                        const double goal = (double)top_p * (double)total;
                        u64 sum = 0;
                        bool over = false;
                        for (int i = 0; i < k && !over; i += 32) {
                            const bool there = i + lane < k;
                            u64 upto = there ? weigh.one(logit_of(sh.sorted[i + lane])) : 0;
                            const u64 own_w = upto;
#pragma unroll
                            for (int off = 1; off < 32; off <<= 1) {
                                const u64 up = __shfl_up_sync(0xffffffffu, upto, off);
                                if (lane >= off) upto += up;
                            }
                            if (pass == 1) {
                                const bool ends = there && ((by_p && (i + lane > 0) && (double)(sum + upto - own_w) >= goal) || own_w < least || own_w == 0);
                                const unsigned yes = __ballot_sync(0xffffffffu, ends);
                                if (yes) {
                                    kept_n = i + __ffs(yes) - 1;
                                    over = true;
                                }
                            }
                            sum += __shfl_sync(0xffffffffu, upto, 31);
                        }
                        if (pass == 0) total = sum;
                    }
                    if (lane == 0) sh.members = kept_n;
                }
                __syncthreads();
                kept_n = sh.members;
                // by index: the place in the falling order stands in the lower half of a key meanwhile
                for (int i = tid; i < kept_n; i += SA_THREADS) {
                    const u64 key = sh.sorted[i];
                    sh.sorted[i] = key << 32 | key >> 32;
                }
                __syncthreads();
                sort_keys(sh.sorted, kept_n);
                if (warp == 0) {
                    auto logit_at = [&](int i) { return logit_of(sh.sorted[i] << 32); };
                    u64 z = 0;
                    for (int i = lane; i < kept_n; i += 32) z += weigh.one(logit_at(i));
#pragma unroll
                    for (int off = 16; off; off >>= 1) z += __shfl_xor_sync(0xffffffffu, z, off);
                    double u = (double)p.uniform[row];
                    u = u >= 0.0 ? u : 0.0;
                    const double at = u * (double)z;
                    const u64 goal = at < (double)z ? min((u64)at, z - 1) : z - 1;
                    u64 sum = 0;
                    for (int i = 0; i < kept_n; i += 32) {
                        const float x = i + lane < kept_n ? logit_at(i + lane) : -INFINITY;
                        const u64 own_w = i + lane < kept_n ? weigh.one(x) : 0;
                        u64 upto = own_w;
#pragma unroll
                        for (int off = 1; off < 32; off <<= 1) {
                            const u64 up = __shfl_up_sync(0xffffffffu, upto, off);
                            if (lane >= off) upto += up;
                        }
                        if (sum + upto - own_w <= goal && goal < sum + upto) {
                            p.token[row] = (int)(sh.sorted[i + lane] >> 32);
                            if (p.prob) p.prob[row] = (float)(weigh.exactly(x) / (double)z);
                        }
                        sum += __shfl_sync(0xffffffffu, upto, 31);
                    }
                }
                return;
            }
            if (bin < SA_BINS) {   // (else all that weigh anything are among the first k)
                const uint32_t wanted = (uint32_t)k - sh.before_n;
                each_short(from_place, to_place, [&](const float4 &v, int i) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) gather(place_of((&v.x)[j]), (&v.x)[j], i + j, bin);
                });
                cluster.sync();
                const int have = collect();
                const u64 key = end_in_list(bin, have, false, [&](uint32_t cc, u64) { return cc >= wanted; });
                empty_list();
                cut_bin = bin;
                cut_key = key;
            }
        }
        if (by_p) {
            // weights by the counts, in units; of the prefix so far, whose last bin counts as far as it belongs to it
            float about[SA_OWN], ab, a_mine = 0.f;
            {
                uint32_t c = cb;
#pragma unroll
                for (int j = 0; j < SA_OWN; ++j) {
                    const int bin = SA_OWN * tid + j;
                    const float in = bin < cut_bin ? (float)own[j] : bin == cut_bin ? (float)((uint32_t)k - c) : 0.f;
                    a_mine += about[j] = in * exp2f((float)SA_UNIT - ((float)bin + 0.5f) * (1.4426950408889634f / SA_PER_NAT));
                    c += own[j];
                }
                float a = a_mine;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const float up = __shfl_up_sync(0xffffffffu, a, off);
                    if (lane >= off) a += up;
                }
                if (lane == 31) sh.scan_a[warp] = a;
                __syncthreads();
                ab = __shfl_up_sync(0xffffffffu, a, 1);
                if (lane == 0) ab = 0.f;
                for (int i = 0; i < warp; ++i) ab += sh.scan_a[i];
            }
            float estimate = 0.f;   // of everything
            for (int i = 0; i < SA_WARPS; ++i) estimate += sh.scan_a[i];
            // the first bin in (from, to) that has members of the prefix and up to whose end about `goal` has gathered; else the last, or -1
            auto search = [&](int from, int to, float goal) {
                __syncthreads();
                if (tid == 0) {
                    sh.bin = SA_BINS;
                    sh.best[0] = -1;
                }
                __syncthreads();
                float a = ab;
#pragma unroll
                for (int j = 0; j < SA_OWN; ++j) {
                    const int bin = SA_OWN * tid + j;
                    a += about[j];
                    if (bin > from && bin < to && own[j] && bin <= cut_bin) {
                        if (a >= goal) atomicMin(&sh.bin, bin);
                        atomicMax(&sh.best[0], bin);
                    }
                }
                __syncthreads();
                return sh.bin < SA_BINS ? sh.bin : sh.best[0];
            };
            int low = -1, high = SA_BINS, bin = search(low, high, top_p * estimate);
            bool found = false;
            u64 up = 0, z = 0;
            while (bin >= 0) {   // ends: the bins between low and high get fewer
                // the weights up to the bin in front of this one, in that one, in this one and in the next; of all of the prefix
                u64 a[5] = {0, 0, 0, 0, 0}, all[5], keep[3] = {0, 0, 0};
                const float to = (float)(bin - 1), this_one = (float)bin, next = (float)(bin + 1), behind = (float)(bin + 2);
                each(from_place, to_place, [&](const float4 &v, int i) {
                    u64 w4[4];
                    weigh.four(v, w4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float x = (&v.x)[j], b = place_of(x);
                        if (by_k && !inside(b, x, i + j)) continue;
                        a[4] += w4[j];
                        if (b < to) {
                            a[0] += w4[j];
                            if (least && w4[j] >= least) keep[0] += w4[j];
                        } else if (b < behind) {
                            const u64 kept = w4[j] >= least ? w4[j] : 0;
                            if (b < this_one) {
                                a[1] += w4[j];
                                keep[1] += kept;
                            } else if (b < next) {
                                a[2] += w4[j];
                                keep[2] += kept;
                                gather(b, x, i + j, bin);
                            } else
                                a[3] += w4[j];
                        }
                    }
                });
                if (!least) keep[0] = a[0];
                cluster_sum(a, all, nullptr);
                z = all[4];
                const double goal = (double)top_p * (double)z;
                const u64 to1 = all[0] + all[1], to2 = to1 + all[2], to3 = to2 + all[3];
                if (all[0] > 0 && (double)all[0] >= goal) high = bin - 1;             // it ends further in front
                else if ((double)to3 < goal) low = bin + 1;                            // or further behind
                else {
                    found = true;
                    // (an empty prefix is never enough)
                    const int step = to1 > 0 && (double)to1 >= goal ? -1 : to2 > 0 && (double)to2 >= goal ? 0 : 1;
                    up = step < 0 ? all[0] : step == 0 ? to1 : to2;
                    w = keep[0] + (step >= 0 ? keep[1] : 0) + (step > 0 ? keep[2] : 0);
                    if (step != 0) {
                        bin += step;
                        empty_list();
                        each_short(from_place, to_place, [&](const float4 &v, int i) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) gather(place_of((&v.x)[j]), (&v.x)[j], i + j, bin);
                        });
                        cluster.sync();
                    }
                    break;
                }
                empty_list();
                // the estimate again, from the sums that are now known: the threads' prefix sums are compared with a goal that is moved
                if (tid == max(bin - 1, 0) / SA_OWN) {
                    float e = ab;
#pragma unroll
                    for (int j = 0; j < SA_OWN; ++j) {
                        if (j == max(bin - 1, 0) % SA_OWN) sh.scan_a[0] = e;           // estimated up to the bin in front
                        e += about[j];
                    }
                }
                __syncthreads();
                bin = search(low, high, (float)(goal - (double)all[0]) + sh.scan_a[0]);
            }
            if (found) {
                const double goal = (double)top_p * (double)z;
                const int have = collect();
                const u64 key = end_in_list(bin, have, true, [&](uint32_t, u64 ww) { return (double)(up + ww) >= goal; });
                cut_bin = bin;
                cut_key = key;
                summed = have <= SA_SORT;
                if (!summed) w = 0;
                else {   // the kept members of the bin that lie in this warp's share
                    const u64 *list = cluster.map_shared_rank(sh.sorted, 0);
                    for (int i = lane; i < have; i += 32) {
                        const u64 member = list[i];
                        const int index = (int)(uint32_t)member;
                        if (member <= key && index >= index_at(from_place) && index < index_at(to_place) && index >= first && index < first + n) {
                            const u64 ww = weigh.one(logit_of(member));
                            if (ww >= least) w += ww;
                        }
                    }
                }
            }
        }
    }

    // ---- the kept weights: of each warp, of the warps in front, of all
    const bool some = cut_bin < SA_BINS;   // not all are kept
    const float cut_from = (float)cut_bin, cut_behind = some ? (float)(cut_bin + 1) : INFINITY;
    auto kept_four = [&](const float4 &v, int place, u64 (&own)[4]) {
        if (some) {   // (as a rule few are kept)
            const float x = fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w));
            if (!(place_of(x) < cut_behind)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) own[j] = 0;
                return;
            }
        }
        weigh.four(v, own);
        if (some) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float b = place_of((&v.x)[j]);
                if (!(b < cut_from || (b < cut_behind && key_of((&v.x)[j], index_at(place + j)) <= cut_key))) own[j] = 0;
            }
        }
        if (least) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (own[j] < least) own[j] = 0;
        }
    };
    if (!summed)
        each(from_place, to_place, [&](const float4 &v, int i) {
            u64 own[4];
            kept_four(v, i, own);
#pragma unroll
            for (int j = 0; j < 4; ++j) w += own[j];
        });
    u64 sums[1] = {w}, all[1], before;
    cluster_sum(sums, all, &before);
    const u64 z = all[0];
    double u = (double)p.uniform[row];
    u = u >= 0.0 ? u : 0.0;   // (no number: 0)
    const double at = u * (double)z;
    const u64 goal = at < (double)z ? min((u64)at, z - 1) : z - 1;
    // whose share holds the token: a warp's, then, all warps of its CTA over that one, an eighth of it, which one warp goes through
    const u64 *parts = sh.sum[turn ^ 1][0];   // the warps' sums
    u64 at_warp = before;
    for (int i = 0; i < warp; ++i) at_warp -= parts[i];
    const bool in_cta = at_warp <= goal && goal < at_warp + parts[SA_WARPS];
    if (in_cta) {
        int chosen = 0;
        while (goal >= at_warp + parts[chosen]) at_warp += parts[chosen++];
        const int share = places / SA_WARPS, part = (share / 8 + SA_WARPS - 1) / SA_WARPS * 8;   // (of places: a multiple of 8)
        const int lo = chosen * share, hi = min(lo + share, (end + 3) / 4 * 4);
        const int from = min(lo + warp * part, hi), to = min(from + part, hi);
        u64 mine = 0;
        each(from, to, [&](const float4 &v, int i) {
            u64 own[4];
            kept_four(v, i, own);
            mine += (own[0] + own[1]) + (own[2] + own[3]);
        });
#pragma unroll
        for (int off = 16; off; off >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, off);
        u64 *eighths = sh.sum[turn][0];
        if (lane == 0) eighths[warp] = mine;
        __syncthreads();
        u64 sum = at_warp;
        for (int i = 0; i < warp; ++i) sum += eighths[i];
        if (sum <= goal && goal < sum + mine)
            for (int at = from; at < to; at += 128) {
                const int i = at + lane * 4;
                u64 own[4] = {0, 0, 0, 0};
                float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                if (i < to) {
                    v = quad(i, at);
                    as_finite(v);
                    kept_four(v, i, own);
                }
                const u64 four = own[0] + own[1] + own[2] + own[3];
                u64 upto = four;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const u64 up = __shfl_up_sync(0xffffffffu, upto, off);
                    if (lane >= off) upto += up;
                }
                const u64 quads = __shfl_sync(0xffffffffu, upto, 31);
                if (goal < sum + quads) {
                    u64 s = sum + upto - four;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (s <= goal && goal < s + own[j]) {
                            p.token[row] = index_at(i + j);
                            if (p.prob) p.prob[row] = (float)(weigh.exactly((&v.x)[j]) / (double)z);
                        }
                        s += own[j];
                    }
                    break;
                }
                sum += quads;
            }
    }
    cluster.sync();   // (nobody leaves while its shared memory is read)
}

}  // namespace

cudaError_t launch_sample(const SampleParams &p, bool bf16, cudaStream_t stream)
{
    // CTAs of a row: as many as are resident at once for all rows together (up to 592), one to eight, none with less than about 1024 logits (more
    // than 2048 are cut into two).
    int ranks = 1;
    while (ranks < 8 && p.vocab > 2048 * ranks && (long long)p.n_rows * ranks * 2 <= SA_CTAS * AT_SMS) ranks *= 2;
    const int chunk = ((p.vocab + ranks - 1) / ranks + 7) / 8 * 8;
    const int step = 8 * SA_WARPS, places = (chunk + 8 + step - 1) / step * step;   // (up to seven in front of a row's part: 16-byte boundaries)
    const bool held = (size_t)places * (bf16 ? 2 : 4) <= SA_HELD;
    const size_t smem = (sizeof(SampleShared) + 15) / 16 * 16 + (held ? (size_t)places * (bf16 ? 2 : 4) : 0);
    static PerContext seen[4];
    using Kernel = void (*)(const SampleParams, int, int);
    static const Kernel kernels[4] = {sample_kernel<float, false>, sample_kernel<float, true>, sample_kernel<__nv_bfloat16, false>,
                                      sample_kernel<__nv_bfloat16, true>};
    const int which = (bf16 ? 2 : 0) + (held ? 1 : 0);
    int sms = 0;
    const cudaError_t e = device_sms(seen[which], reinterpret_cast<const void *>(kernels[which]), (sizeof(SampleShared) + 15) / 16 * 16 + SA_HELD, &sms);
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
    return cudaLaunchKernelEx(&cfg, kernels[which], p, chunk, places);
}

}  // namespace gdn
