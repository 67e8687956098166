// New rows on their way to a paged cache: keys rotated by position, values as they are, queries rotated beside them.
//
// A pair (a, b) of a head's components at position t becomes (a cos - b sin, b cos + a sin) with the table's row t; pairs are
// (i, i + R/2) of the R rotated components, or (2i, 2i + 1).  The products are formed in fp32 and rounded once.
// Memory decides: every element is read once and written once.  A warp has a row, or a part of one where rows are few (one
// token of one sequence: 48 heads of 128 components over 8 warps), and moves 16 components of a lane at a time.
#include "gdn_attn.cuh"

namespace gdn {

struct AppendParams {
    AttnParams a;                        // q, caches, page_table, seq_lens, row_offsets, parent, status
    const void *k, *v;
    long long k_stride, v_stride;
    const float *rope;                   // [>= max_len][rope_dim]: cos of the rope_dim / 2 angles, then sin
    int rope_dim, interleaved;
    void *q_out, *k_out, *v_out;
    const int32_t *path, *path_offsets;  // the rows of accepted paths alone, null: all rows
};

namespace {

constexpr int KA_WARPS = 8;

template <typename T> struct Piece;   // 8 components
template <> struct Piece<float> {
    float x[8];
    __device__ __forceinline__ void load(const float *p)
    {
        *reinterpret_cast<float4 *>(x) = *reinterpret_cast<const float4 *>(p);
        *reinterpret_cast<float4 *>(x + 4) = *reinterpret_cast<const float4 *>(p + 4);
    }
    __device__ __forceinline__ void store(float *p) const
    {
        *reinterpret_cast<float4 *>(p) = *reinterpret_cast<const float4 *>(x);
        *reinterpret_cast<float4 *>(p + 4) = *reinterpret_cast<const float4 *>(x + 4);
    }
};
template <> struct Piece<__nv_bfloat16> {
    float x[8];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p)
    {
        const uint4 u = *reinterpret_cast<const uint4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float((&u.x)[i] << 16);
            x[2 * i + 1] = __uint_as_float((&u.x)[i] & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const
    {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
};

// The last of the ascending offsets[0 .. n - 1] that is at most x, -1 where the first is not (by a whole warp).
__device__ __forceinline__ int warp_search(const int32_t *offsets, int n, int x, int lane)
{
    int lo = 0, hi = n;
    if (offsets[0] > x) return -1;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, i = lo + lane * step;
        const unsigned le = __ballot_sync(0xffffffffu, i < hi && offsets[i] <= x);
        if (le == 0) return -1;   // (offsets that do not ascend)
        const int top = 31 - __clz((int)le);
        lo += top * step;
        hi = min(lo + step, hi);
    }
    return lo;
}

template <typename T> __device__ __forceinline__ void rotate_pair(T &a, T &b, const float *cs, int half, bool interleaved)
{
    if (interleaved) {   // a: components 0 .. 7, b: 8 .. 15 of sixteen; pair i has the angle i
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float *x = i < 4 ? &a.x[2 * i] : &b.x[2 * (i - 4)];
            const float c = __ldg(cs + i), s = __ldg(cs + half + i), p = x[0], q = x[1];
            x[0] = fmaf(p, c, -(q * s));
            x[1] = fmaf(q, c, p * s);
        }
    } else {
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            *reinterpret_cast<float4 *>(c + i) = __ldg(reinterpret_cast<const float4 *>(cs + i));
            *reinterpret_cast<float4 *>(s + i) = __ldg(reinterpret_cast<const float4 *>(cs + half + i));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = a.x[i], q = b.x[i];
            a.x[i] = fmaf(p, c[i], -(q * s[i]));
            b.x[i] = fmaf(q, c[i], p * s[i]);
        }
    }
}

// VEC: rope_dim and d are multiples of 16, so that sixteen components of a head are two pieces of one kind; otherwise a lane
// takes a pair at a time.
template <typename T, bool VEC> __global__ void __launch_bounds__(KA_WARPS * 32) kv_append_kernel(const AppendParams p, int parts)
{
    wait_for_previous_kernel();
    const AttnParams &a = p.a;
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * KA_WARPS + (threadIdx.x >> 5);
    const int index = (int)(w / parts), part = (int)(w % parts);
    const int32_t *offsets = p.path ? p.path_offsets : a.row_offsets;
    const int count = offsets[a.n_seq];
    const int bad_offsets = p.path ? GDN_ERR_PATH : GDN_ERR_TREE;
    if (w == 0 && count > a.total_rows && lane == 0) report_status(a.status_dev, bad_offsets);
    if (index >= count || index >= a.total_rows) return;
    const int b = warp_search(offsets, a.n_seq, index, lane);
    AttnSeq s;
    if (b < 0) {
        if (lane == 0) report_status(a.status_dev, bad_offsets);
        return;
    }
    const int t = index - offsets[b];
    if (!attn_seq(a, b, s, true)) return;
    if (t < 0 || (!p.path && t >= s.rows)) {
        if (lane == 0) report_status(a.status_dev, bad_offsets);
        return;
    }
    int row = s.row0 + t, depth = t;   // (the length of what is written counts into max_len with all rows of the call)
    if (p.path) {
        const int n = offsets[b + 1] - offsets[b];
        bool bad = t >= n || n > s.rows || offsets[b] < 0 || offsets[b + 1] > count;
        if (!bad)
            for (int i = lane; i < n; i += 32) {
                const int node = p.path[offsets[b] + i], up = i ? p.path[offsets[b] + i - 1] : -1;
                if (node < 0 || node >= s.rows) bad = true;
                else if (a.parent) bad |= a.parent[s.row0 + node] != up;
                else bad |= node <= up;   // (without parents only the order can be checked)
            }
        if (__any_sync(0xffffffffu, bad)) {
            if (lane == 0) report_status(a.status_dev, GDN_ERR_PATH);
            return;
        }
        row = s.row0 + p.path[index];
    } else if (a.parent) {
        depth = 0;
        bool bad = false;
        if (s.rows <= 64) {   // the parents in two registers per lane
            const int lo = lane < s.rows ? a.parent[s.row0 + lane] : -1, hi = lane + 32 < s.rows ? a.parent[s.row0 + lane + 32] : -1;
            int node = t;
            for (;;) {
                const int up = node < 32 ? __shfl_sync(0xffffffffu, lo, node) : __shfl_sync(0xffffffffu, hi, node - 32);
                bad = up < -1 || up >= node;
                if (bad || up < 0) break;
                node = up;
                ++depth;
            }
        } else {
            int node = t;
            for (;;) {
                const int up = a.parent[s.row0 + node];
                bad = up < -1 || up >= node;
                if (bad || up < 0) break;
                node = up;
                ++depth;
            }
        }
        if (bad) {
            if (lane == 0) report_status(a.status_dev, GDN_ERR_TREE);
            return;
        }
    }
    const long long slot = attn_token_offset(a, b, s.len + t, a.max_len);
    const float *cs = p.rope + (size_t)(s.len + depth) * p.rope_dim;
    const int heads_q = p.q_out ? a.h_q : 0, half = p.rope_dim / 2;
    const T *q = static_cast<const T *>(a.q) + (size_t)row * a.q_stride, *k = static_cast<const T *>(p.k) + (size_t)row * p.k_stride,
            *v = static_cast<const T *>(p.v) + (size_t)row * p.v_stride;
    T *q_out = static_cast<T *>(p.q_out) + (size_t)row * a.h_q * a.d, *k_out = static_cast<T *>(p.k_out) + slot,
      *v_out = static_cast<T *>(p.v_out) + slot;
    const int per = VEC ? a.d / 16 : a.d / 2, turned = VEC ? p.rope_dim / 16 : half;
    const int n_items = (heads_q + 2 * a.h_kv) * per;
    const bool stored = slot >= 0;   // (a page that is none: reported, nothing of this row goes to the cache)
#pragma unroll 4
    for (int item = part * 32 + lane; item < n_items; item += parts * 32) {
        int head = item / per;
        const int i = item % per;
        const T *src;
        T *dst;
        bool key = true;
        if (head < heads_q) {
            src = q + (size_t)head * a.d;
            dst = q_out + (size_t)head * a.d;
        } else {
            head -= heads_q;
            key = head < a.h_kv;
            if (!key) head -= a.h_kv;
            src = (key ? k : v) + (size_t)head * a.d;
            dst = (key ? k_out : v_out) + head * a.head_stride;
            if (!stored) continue;
        }
        const bool turn = key && i < turned;
        if constexpr (VEC) {
            const int first = turn && !p.interleaved ? 8 * i : 16 * i, second = turn && !p.interleaved ? first + half : first + 8;
            Piece<T> x, y;
            x.load(src + first);
            y.load(src + second);
            if (turn) rotate_pair(x, y, cs + 8 * i, half, p.interleaved);
            x.store(dst + first);
            y.store(dst + second);
        } else {
            const int first = turn && !p.interleaved ? i : 2 * i, second = turn && !p.interleaved ? i + half : 2 * i + 1;
            const float x = load_as_float(src + first), y = load_as_float(src + second);
            const float c = turn ? cs[i] : 1.f, sn = turn ? cs[half + i] : 0.f;
            store_from_float(dst + first, turn ? fmaf(x, c, -(y * sn)) : x);
            store_from_float(dst + second, turn ? fmaf(y, c, x * sn) : y);
        }
    }
}

}  // namespace

cudaError_t launch_kv_append(const AttnParams &a, bool bf16, const void *k, const void *v, long long k_stride, long long v_stride,
                             const float *rope, int rope_dim, bool interleaved, void *q_out, void *k_out, void *v_out,
                             const int32_t *path, const int32_t *path_offsets, cudaStream_t stream)
{
    const AppendParams p{a, k, v, k_stride, v_stride, rope, rope_dim, interleaved ? 1 : 0, q_out, k_out, v_out, path, path_offsets};
    const bool vec = a.d % 16 == 0 && rope_dim % 16 == 0;
    // a row over several warps while there are fewer than eight warps for each of about 150 SMs, each with two loads or more per lane
    const int items = ((q_out ? a.h_q : 0) + 2 * a.h_kv) * a.d / (vec ? 16 : 2);
    int parts = 1;
    while (parts < 16 && (long long)a.total_rows * parts < 1024 && items > 32 * parts) parts *= 2;
    const long long blocks = ((long long)a.total_rows * parts + KA_WARPS - 1) / KA_WARPS;
    const auto kernel = bf16 ? (vec ? kv_append_kernel<__nv_bfloat16, true> : kv_append_kernel<__nv_bfloat16, false>)
                             : (vec ? kv_append_kernel<float, true> : kv_append_kernel<float, false>);
    return launch_behind(kernel, dim3((unsigned)blocks), KA_WARPS * 32, 0, stream, p, parts);
}

}  // namespace gdn
