// Attention over a paged cache on CUDA cores: any head size, fp32 or bf16; and what every kernel of the family uses: the
// ancestors of large trees, the join of parts.
//
// For row i and the tokens t that it sees, with s_t = scale * q_i . k_t:
//     o_i = sum_t 2^(s'_t - m) v_t / sum_t 2^(s'_t - m),   s' = s * log2(e),  m = max_t s'_t,
// in one pass over the tokens: where a tile raises the maximum from m to m', what has been summed so far is multiplied
// by 2^(m - m').  A row that sees nothing has the sum 0 and the output 0.
#include "gdn_attn.cuh"

namespace gdn {

namespace {

constexpr int AG_THREADS = 128;
constexpr int AG_M = 16;       // rows of a unit: four per warp
constexpr int AG_TN = 32;      // tokens of a tile: one per lane
constexpr int AG_STAGES = 2;

template <typename T> __host__ __device__ constexpr int ag_pitch(int d) { return d * (int)sizeof(T) + 16; }   // the next row begins four banks on
template <typename T> constexpr size_t ag_smem(int d)
{
    return (size_t)AG_STAGES * 2 * AG_TN * ag_pitch<T>(d) + AG_M * d * sizeof(float) + 2 * AG_M * AG_TN * sizeof(float);
}

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

__device__ __forceinline__ float4 four(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ float4 four(const __nv_bfloat16 *p)
{
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                       __uint_as_float(u.y & 0xFFFF0000u));
}

// Four warps, each with four rows, or two or four of them with the same four where there are not enough: then each has a share of the
// components in the products with the keys and of the tokens in those with the values.  A lane has a token in the former and four
// components in the latter.  Bound by shared memory for many rows (a key's four components feed sixteen multiplications), by HBM for few.
// DD: the components where they are known beforehand (64, 128), else 0.
template <typename T, int DD> __global__ void __launch_bounds__(AG_THREADS, 3) attn_general_kernel(const AttnParams p)
{
    extern __shared__ __align__(16) unsigned char ag_smem_base[];
    __shared__ unsigned long long anc[AT_SMALL_ROWS];
    __shared__ int anc_up[AT_SMALL_ROWS];
    const int d = DD ? DD : p.d, pitch = ag_pitch<T>(d), stage_bytes = 2 * AG_TN * pitch;
    float *q_s = reinterpret_cast<float *>(ag_smem_base + AG_STAGES * stage_bytes);
    float *x_s = reinterpret_cast<float *>(ag_smem_base);   // at the end, over the tiles: [4 warps][4 rows][d], sums of warps that share rows
    float *w_s = q_s + AG_M * d;        // [4 warps][AG_TN][4]: weights
    float *s_s = w_s + AG_M * AG_TN;    // [4 warps][4][AG_TN]: scores over a warp's share of the components
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = (int)blockIdx.x;
    const AttnMaskKind kind = attn_mask_kind(p);
    const T *k_cache = static_cast<const T *>(p.k_cache), *v_cache = static_cast<const T *>(p.v_cache);
    wait_for_previous_kernel();

    AttnWalk walk;
    AttnSegment g;
    walk.begin(p, cta, AG_M, AG_TN);
    while (walk.next(p, cta, AG_M, AG_TN, g)) {
        if (p.row_offsets && kind == AT_WORDS64 && !attn_ancestors(p, g.s, anc, anc_up)) {
            if (tid == 0) report_status(p.status_dev, GDN_ERR_TREE);
            continue;
        }
        if (p.row_offsets && kind == AT_WORDS && !p.tree_ok[g.b]) continue;
        const int row_first = g.m_tile * AG_M, rows = min(AG_M, g.s.rows * p.group - row_first);
        for (int i = tid; i < rows * (d / 4); i += AG_THREADS) {
            const int r = i / (d / 4), c = i % (d / 4) * 4, u = row_first + r, node = u / p.group;
            *reinterpret_cast<float4 *>(q_s + r * d + c) = four(static_cast<const T *>(p.q) + (size_t)(g.s.row0 + node) * p.q_stride +
                                                                (size_t)(g.head * p.group + u % p.group) * d + c);
        }
        const int with = rows <= 4 ? 4 : rows <= 8 ? 2 : 1, part = warp % with, row_group = warp / with;   // warps with the same rows
        // the last token that any of these rows sees: rows come in an order in which ancestors are in front
        const int last_node = (row_first + rows - 1) / p.group, upto = p.row_offsets ? g.s.len + last_node + 1 : g.s.len;
        const int tile1 = min(g.tile1, max((upto + AG_TN - 1) / AG_TN, g.tile0));

        // the page of this lane's token of a tile: asked for one tile ahead of the tile that is on its way
        const int last_token = min(g.s.held, upto);
        auto page_of = [&](int tile) {
            const int t = tile * AG_TN + lane;
            return tile < tile1 && t < last_token
                       ? p.page_table[(size_t)g.b * p.max_pages + (p.page_shift >= 0 ? t >> p.page_shift : t / p.page_size)] : -1;
        };
        auto fetch = [&](int tile, int page) {   // rows warp * 8 ... + 7 of the keys and of the values
            if (tile < tile1) {
                const uint32_t base = smem_u32(ag_smem_base) + (tile % AG_STAGES) * stage_bytes;
                const int t = tile * AG_TN + lane;
                long long mine = -1;
                if (t < last_token) {
                    if (page < 0 || page >= p.n_pages) report_status(p.status_dev, GDN_ERR_PAGE);
                    else mine = page * p.page_stride + (p.page_shift >= 0 ? t & (p.page_size - 1) : t % p.page_size) * p.token_stride;
                }
                // 16-byte pieces of a row, and rows that an access of the warp covers
                constexpr int PIECES = DD ? DD * (int)sizeof(T) / 16 : 32, ROWS = 32 / PIECES;
                const int col = lane % PIECES;
                const char *k_from = reinterpret_cast<const char *>(k_cache + g.head * p.head_stride) + col * 16;
                const char *v_from = reinterpret_cast<const char *>(v_cache + g.head * p.head_stride) + col * 16;
                mine *= (long long)sizeof(T);
#pragma unroll
                for (int h = 0; h < 8 / ROWS; ++h) {
                    const int r = warp * 8 + h * ROWS + lane / PIECES;
                    const long long at = __shfl_sync(0xffffffffu, mine, r), from = at < 0 ? 0 : at;
                    if (DD || col * 16 < d * (int)sizeof(T)) {
                        cp_async_16(base + r * pitch + col * 16, k_from + from, at >= 0);
                        cp_async_16(base + (AG_TN + r) * pitch + col * 16, v_from + from, at >= 0);
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };

        // tokens that all rows of the unit see: in tiles of no others nothing is looked at token by token
        const int common = !p.row_offsets ? upto : kind == AT_CHAIN ? g.s.len + row_first / p.group + 1 : g.s.len;
        int node[4];
        float m[4], l[4], acc[4][4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            node[r] = (row_first + row_group * 4 + r) / p.group;
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[r][c] = 0.f;
        }
        int page = page_of(g.tile0 + 1);
        fetch(g.tile0, page_of(g.tile0));
        for (int tile = g.tile0; tile < tile1; ++tile) {
            fetch(tile + 1, page);
            page = page_of(tile + 2);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncthreads();
            const bool busy = row_group * 4 < rows, clean = (tile + 1) * AG_TN <= common;
            float sc[4] = {0.f, 0.f, 0.f, 0.f};
            if (busy) {
                const T *k_s = reinterpret_cast<const T *>(ag_smem_base + (tile % AG_STAGES) * stage_bytes + lane * pitch);
                const float *qw = q_s + row_group * 4 * d;
#pragma unroll 4
                for (int c = part * 4; c < d; c += with * 4) {
                    const float4 k4 = four(k_s + c);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float4 q4 = four(qw + r * d + c);
                        sc[r] = fmaf(q4.x, k4.x, fmaf(q4.y, k4.y, fmaf(q4.z, k4.z, fmaf(q4.w, k4.w, sc[r]))));
                    }
                }
                if (with > 1) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) s_s[(warp * 4 + r) * AG_TN + lane] = sc[r];
                }
            }
            if (with > 1) __syncthreads();
            if (busy) {
                if (with > 1) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        sc[r] = 0.f;
                        for (int o = 0; o < with; ++o) sc[r] += s_s[((row_group * with + o) * 4 + r) * AG_TN + lane];
                    }
                }
                const int t = tile * AG_TN + lane;
                float4 w;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool seen = clean || (row_group * 4 + r < rows && (t < g.s.len || (t < g.s.held && attn_sees(p, kind, anc, g.s.row0, node[r], t - g.s.len))));
                    const float x = seen ? sc[r] * p.scale_log2 : -INFINITY;
                    float top = x;
#pragma unroll
                    for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
                    top = fmaxf(top, m[r]);
                    const float ref = top == -INFINITY ? 0.f : top;
                    const float e = seen ? power_of_two(x - ref) : 0.f, fade = power_of_two(m[r] - ref);
                    m[r] = top;
                    l[r] = l[r] * fade + e;   // (of this lane's tokens)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[r][c] *= fade;
                    (&w.x)[r] = e;
                }
                reinterpret_cast<float4 *>(w_s)[warp * AG_TN + lane] = w;
                __syncwarp();
                if (lane * 4 < d) {
                    const T *v_s = reinterpret_cast<const T *>(ag_smem_base + (tile % AG_STAGES) * stage_bytes + AG_TN * pitch) + lane * 4;
                    auto add = [&](int j, auto all) {
                        const float4 e = reinterpret_cast<const float4 *>(w_s)[warp * AG_TN + j];
                        const float4 v4 = four(reinterpret_cast<const T *>(reinterpret_cast<const char *>(v_s) + j * pitch));
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float er = (&e.x)[r];
                            if (decltype(all)::value || er != 0.f) {   // (a value that a row does not see may be infinite or no number)
                                acc[r][0] = fmaf(er, v4.x, acc[r][0]);
                                acc[r][1] = fmaf(er, v4.y, acc[r][1]);
                                acc[r][2] = fmaf(er, v4.z, acc[r][2]);
                                acc[r][3] = fmaf(er, v4.w, acc[r][3]);
                            }
                        }
                    };
                    const int from = part * (AG_TN / with), to = from + AG_TN / with;
                    if (clean) {
#pragma unroll 8
                        for (int j = from; j < to; ++j) add(j, Yes{});
                    } else
                        for (int j = from; j < to; ++j) add(j, No{});
                }
            }
            __syncthreads();
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int off = 16; off; off >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], off);
        if (with > 1) {   // the warps' sums over their tokens
            if (lane * 4 < d)
#pragma unroll
                for (int r = 0; r < 4; ++r) *reinterpret_cast<float4 *>(x_s + (warp * 4 + r) * d + lane * 4) = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
            __syncthreads();
            if (part == 0 && lane * 4 < d)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    for (int o = 1; o < with; ++o) {
                        const float4 other = *reinterpret_cast<const float4 *>(x_s + ((warp + o) * 4 + r) * d + lane * 4);
                        acc[r][0] += other.x;
                        acc[r][1] += other.y;
                        acc[r][2] += other.z;
                        acc[r][3] += other.w;
                    }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = row_group * 4 + r;
            if (row >= rows || part != 0) continue;
            if (g.slot < 0) {
                if (lane * 4 < d) {
                    const int u = row_first + row;
                    T *o = static_cast<T *>(p.o) + ((size_t)(g.s.row0 + u / p.group) * p.h_q + g.head * p.group + u % p.group) * d + lane * 4;
                    const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
#pragma unroll
                    for (int c = 0; c < 4; ++c) store_from_float(o + c, acc[r][c] * inv);
                }
            } else {
                const size_t at = (size_t)g.slot * AG_M + row;
                if (lane * 4 < d) *reinterpret_cast<float4 *>(p.part_o + at * d + lane * 4) = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
                if (lane == 0) *reinterpret_cast<float2 *>(p.part_ml + at * 2) = make_float2(m[r], l[r]);
            }
        }
        __syncthreads();   // (the next unit's queries and ancestors)
    }
}

// Ancestors of the nodes of trees above AT_SMALL_ROWS nodes, as a bit per node of the tree: row i of `mask` holds the words up
// to that of node i itself.  A thread walks its node's root path; ids fall along it, so that every word is written once.
constexpr int AM_THREADS = 256;
__global__ void __launch_bounds__(AM_THREADS) attn_mask_kernel(const AttnParams p)
{
    extern __shared__ int am_parent[];
    wait_for_previous_kernel();
    const int b = (int)blockIdx.y, first = (int)blockIdx.x * AM_THREADS;
    AttnSeq s;
    const bool fits = attn_seq(p, b, s, false);
    if (!fits || (first > 0 && first >= s.rows)) return;   // (first = 0: an empty tree is one)
    bool bad = false;
    for (int i = threadIdx.x; i < s.rows; i += AM_THREADS) {
        const int parent = p.parent[s.row0 + i];
        am_parent[i] = parent;
        bad |= parent < -1 || parent >= i;
    }
    bad = __syncthreads_or(bad);
    if (first == 0 && threadIdx.x == 0) {
        p.tree_ok[b] = !bad;
        if (bad) report_status(p.status_dev, GDN_ERR_TREE);
    }
    const int i = first + (int)threadIdx.x;
    if (bad || i >= s.rows) return;
    int node = i;
    for (int w = i >> 5; w >= 0; --w) {
        uint32_t bits = 0;
        while (node >= 0 && node >> 5 == w) {
            bits |= 1u << (node & 31);
            node = am_parent[node];
        }
        p.mask[(size_t)(s.row0 + i) * p.mask_words + w] = bits;
    }
}

// The parts of a split unit, in the order of their tiles, to its rows: o = sum_p 2^(m_p - m) o_p / sum_p 2^(m_p - m) l_p.
// A thread has four components of a row; the threads of a CTA read neighbouring pieces of each part, which lie [M][d / 4] or, where a
// thread of the kernel in front has a row (columns_first), [d / 4][M].  A unit that one run held is left alone.
constexpr int AJ_THREADS = 128;
template <typename T> __global__ void __launch_bounds__(AJ_THREADS) attn_join_kernel(const AttnParams p, int M, int TN, int columns_first)
{
    // (lengths and trees are as the kernel in front found them, which began behind everything that writes them: what follows from them is
    // worked out while that one runs)
    const int units = p.h_kv * p.m_tiles, b = (int)blockIdx.x / units, head = (int)blockIdx.x % units / p.m_tiles, m_tile = (int)blockIdx.x % p.m_tiles;
    const int pieces = p.d / 4;
    // the first tile of this unit among those of all units, as AttnWalk counts them
    AttnSeq s;
    const bool fits = attn_seq(p, b, s, false);
    const AttnTotal sum = attn_total<true>(p, M, TN, b, false);
    // (no CTA ends before the kernel in front: what is behind this one must not overtake that)
    const int row_first = m_tile * M, rows = fits ? min(M, s.rows * p.group - row_first) : 0;
    if (rows <= 0) {
        wait_for_previous_kernel();
        return;
    }
    bool bad = false;
    if (p.row_offsets && p.parent) {
        if (p.max_rows > AT_SMALL_ROWS) bad = !p.tree_ok[b];
        else {
            if ((int)threadIdx.x < s.rows) {
                const int parent = p.parent[s.row0 + threadIdx.x];
                bad = parent < -1 || parent >= (int)threadIdx.x;
            }
            bad = __syncthreads_or(bad);
        }
    }
    const int tiles = attn_tiles(s, TN), m_tiles = (s.rows * p.group + M - 1) / M;
    const long long first = sum.before + (long long)(head * m_tiles + m_tile) * (tiles + sum.over) + sum.over, last = first + tiles - 1;
    const long long runs = sum.runs(p);
    const int c0 = sum.run_of(first, runs), c1 = sum.run_of(last, runs);
    wait_for_previous_kernel();
    if (bad || c0 == c1) return;

    auto slot = [&](int c) { return (size_t)(c == c0 ? 2 * c + 1 : 2 * c); };
    for (int piece = (int)blockIdx.y * AJ_THREADS + (int)threadIdx.x; piece < M * pieces; piece += (int)gridDim.y * AJ_THREADS) {
        const int row = columns_first ? piece % M : piece / pieces, column = columns_first ? piece / M : piece % pieces;
        if (row >= rows) continue;
        // eight parts at a time, their loads all on their way together
        float m = -INFINITY, acc[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f;
        for (int c = c0; c <= c1; c += 8) {
            float2 ml[8];
            float4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool there = c + k <= c1;
                ml[k] = there ? *reinterpret_cast<const float2 *>(p.part_ml + (slot(c + k) * M + row) * 2) : make_float2(-INFINITY, 0.f);
                v[k] = there ? *reinterpret_cast<const float4 *>(p.part_o + (slot(c + k) * M * pieces + piece) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            float top = m;
#pragma unroll
            for (int k = 0; k < 8; ++k) top = fmaxf(top, ml[k].x);
            const float ref = top == -INFINITY ? 0.f : top, fade = power_of_two(m - ref);
            m = top;
            l *= fade;
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] *= fade;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float f = power_of_two(ml[k].x - ref);
                l = fmaf(f, ml[k].y, l);
                acc[0] = fmaf(f, v[k].x, acc[0]);
                acc[1] = fmaf(f, v[k].y, acc[1]);
                acc[2] = fmaf(f, v[k].z, acc[2]);
                acc[3] = fmaf(f, v[k].w, acc[3]);
            }
        }
        const int u = row_first + row;
        T *o = static_cast<T *>(p.o) + ((size_t)(s.row0 + u / p.group) * p.h_q + head * p.group + u % p.group) * p.d + column * 4;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(o) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
        else *reinterpret_cast<uint2 *>(o) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
    }
}

}  // namespace

cudaError_t launch_attn_masks(const AttnParams &p, cudaStream_t stream)
{
    return launch_behind(attn_mask_kernel, dim3((unsigned)((p.max_rows + AM_THREADS - 1) / AM_THREADS), (unsigned)p.n_seq), AM_THREADS,
                         (size_t)p.max_rows * sizeof(int), stream, p);
}

cudaError_t launch_attn_join(const AttnParams &p, bool bf16, int M, int TN, bool columns_first, cudaStream_t stream)
{
    // CTAs of a unit: one per 128 pieces of four components while that are fewer than eight per SM, else as many as make up those
    const long long units = (long long)p.n_seq * p.h_kv * p.m_tiles, all = ((columns_first ? M : min(M, p.max_rows * p.group)) * (p.d / 4) + AJ_THREADS - 1) / AJ_THREADS;
    const long long per_unit = max(1LL, min(all, 8LL * AT_SMS / units));
    const dim3 grid((unsigned)units, (unsigned)per_unit);
    return launch_behind(bf16 ? attn_join_kernel<__nv_bfloat16> : attn_join_kernel<float>, grid, AJ_THREADS, 0, stream, p, M, TN, columns_first ? 1 : 0);
}

AttnTiling attn_general_tiling(bool bf16, int d)
{
    return {AG_M, AG_TN, (bf16 ? ag_smem<__nv_bfloat16>(d) : ag_smem<float>(d)) <= (74 << 10) ? 3 : 2, 2};
}

cudaError_t launch_attn_general(const AttnParams &p, bool bf16, int grid, cudaStream_t stream)
{
    // (bf16 with heads of 64 or 128 components has kernels of its own)
    static PerContext seen[4];
    using Kernel = void (*)(const AttnParams);
    static const Kernel kernels[4] = {attn_general_kernel<__nv_bfloat16, 0>, attn_general_kernel<float, 0>, attn_general_kernel<float, 64>,
                                      attn_general_kernel<float, 128>};
    const int which = bf16 ? 0 : p.d == 64 ? 2 : p.d == 128 ? 3 : 1;
    const Kernel kernel = kernels[which];
    int sms = 0;
    const cudaError_t e = device_sms(seen[which], reinterpret_cast<const void *>(kernel),
                                     bf16 ? ag_smem<__nv_bfloat16>(GDN_MAX_HEAD_DIM) : ag_smem<float>(GDN_MAX_HEAD_DIM), &sms);
    if (e != cudaSuccess) return e;
    return launch_behind(kernel, dim3((unsigned)grid), AG_THREADS, bf16 ? ag_smem<__nv_bfloat16>(p.d) : ag_smem<float>(p.d), stream, p);
}

}  // namespace gdn
