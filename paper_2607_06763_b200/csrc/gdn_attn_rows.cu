// Attention over a paged cache for units of at most 64 rows (one token, or a small tree, of the query heads that share a key/value
// head): bf16, heads of 64 or 128 components.  The formulas stand in gdn_attn_general.cu.
//
// Few rows: the keys and values decide, each read once, and what counts is to have enough of them on the way.  Three tiles of 64 tokens
// (32 KB each for 128 components) per CTA, two CTAs per SM: up to 128 KB in flight on an SM, where about 45 KB cover the latency
// at HBM's rate.  Sixteen rows of a unit are one operand of m16n8k16; a warp multiplies them with its share of the tile's tokens
// (WM warps for the rows, 4 / WM for the tokens), keeps maximum, denominator and sums of its share to itself, and the shares meet
// at the end of the unit: no exchange between warps inside the loop but the barrier that hands over the tiles.
// The weights go into the second product as bf16 (half a step off, as the outputs are); sums and statistics are fp32.
#include "gdn_attn.cuh"

namespace gdn {

namespace {

constexpr int AR_THREADS = 128;
constexpr int AR_TN = 64;
constexpr int AR_STAGES = 3;
template <int D> constexpr int ar_ctas() { return D == 128 ? 2 : 4; }
template <int D> __host__ __device__ constexpr int ar_stage_bytes() { return 2 * AR_TN * D * 2; }
template <int D> constexpr size_t ar_smem() { return (size_t)AR_STAGES * ar_stage_bytes<D>(); }

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Byte offset of 16-byte piece `c` of row `r` of a tile: eight rows of one column lie in eight different bank groups.
template <int D> __device__ __forceinline__ uint32_t ar_at(int r, int c) { return (uint32_t)(r * D * 2 + ((c ^ (r & 7)) << 4)); }

template <int D, int WM> __global__ void __launch_bounds__(AR_THREADS, ar_ctas<D>()) attn_rows_kernel(const AttnParams p)
{
    constexpr int M = 16 * WM, WN = 4 / WM, TW = AR_TN / WN, NB = TW / 8, KS = D / 16, PIECES = D / 8;
    extern __shared__ __align__(128) unsigned char ar_base[];
    __shared__ unsigned long long anc[AT_SMALL_ROWS];
    __shared__ int anc_up[AT_SMALL_ROWS];
    __shared__ long long off_s[4][AR_TN];
    __shared__ float ml_s[4][16][2];
    __shared__ int odd_s;   // some value of this call's rows is infinite or no number
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, wm = warp % WM, wn = warp / WM, cta = (int)blockIdx.x;
    const AttnMaskKind kind = attn_mask_kind(p);
    const uint32_t base = smem_u32(ar_base);
    const __nv_bfloat16 *k_cache = static_cast<const __nv_bfloat16 *>(p.k_cache), *v_cache = static_cast<const __nv_bfloat16 *>(p.v_cache);
    wait_for_previous_kernel();

    AttnWalk walk;
    AttnSegment g;
    walk.begin(p, cta, M, AR_TN);
    while (walk.next(p, cta, M, AR_TN, g)) {
        if (p.row_offsets && kind == AT_WORDS64 && !attn_ancestors(p, g.s, anc, anc_up)) {
            if (tid == 0) report_status(p.status_dev, GDN_ERR_TREE);
            continue;
        }
        if (p.row_offsets && kind == AT_WORDS && !p.tree_ok[g.b]) continue;
        const int row_first = g.m_tile * M, rows = min(M, g.s.rows * p.group - row_first);
        const int last_node = (row_first + rows - 1) / p.group, upto = p.row_offsets ? g.s.len + last_node + 1 : g.s.len;
        const int tile1 = min(g.tile1, max((upto + AR_TN - 1) / AR_TN, g.tile0));
        // tokens that all rows of the unit see: what lies behind them is hidden from some
        const int common = !p.row_offsets ? upto : kind == AT_CHAIN ? g.s.len + row_first / p.group + 1 : g.s.len;

        // queries, through the last stage's place, to registers
        {
            const uint32_t q_s = base + (AR_STAGES - 1) * ar_stage_bytes<D>();
            for (int i = tid; i < M * PIECES; i += AR_THREADS) {
                const int r = i / PIECES, c = i % PIECES, u = row_first + r;
                const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(p.q);
                if (r < rows) src += (size_t)(g.s.row0 + u / p.group) * p.q_stride + (size_t)(g.head * p.group + u % p.group) * D + c * 8;
                cp_async_16(q_s + ar_at<D>(r, c), src, r < rows);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        // places of the tokens: of the first three tiles at once, then of one tile per step, its page asked for a step ahead
        auto page_of = [&](int tile) {
            const int t = tile * AR_TN + tid;
            return tid < AR_TN && tile < tile1 && t < upto
                       ? p.page_table[(size_t)g.b * p.max_pages + (p.page_shift >= 0 ? t >> p.page_shift : t / p.page_size)] : -1;
        };
        auto put_place = [&](int tile, int page) {
            if (tid >= AR_TN || tile >= tile1) return;
            const int t = tile * AR_TN + tid;
            long long at = -1;
            if (t < upto) {
                if (page < 0 || page >= p.n_pages) report_status(p.status_dev, GDN_ERR_PAGE);
                else at = page * p.page_stride + (p.page_shift >= 0 ? t & (p.page_size - 1) : t % p.page_size) * p.token_stride;
            }
            off_s[tile & 3][tid] = at;
        };
        {
            int pages[3];
#pragma unroll
            for (int i = 0; i < 3; ++i) pages[i] = page_of(g.tile0 + i);
#pragma unroll
            for (int i = 0; i < 3; ++i) put_place(g.tile0 + i, pages[i]);
        }
        int page_ahead = page_of(g.tile0 + 3);
        if (tid == 0) odd_s = 0;
        const __nv_bfloat16 *k_head = k_cache + g.head * p.head_stride + (tid % PIECES) * 8, *v_head = v_cache + g.head * p.head_stride + (tid % PIECES) * 8;
        auto fetch = [&](int tile) {
            if (tile < tile1) {
                const uint32_t to = base + (tile % AR_STAGES) * ar_stage_bytes<D>();
#pragma unroll
                for (int j = 0; j < AR_TN * PIECES / AR_THREADS; ++j) {
                    const int r = tid / PIECES + j * (AR_THREADS / PIECES);
                    const long long at = off_s[tile & 3][r];
                    const long long from = at < 0 ? 0 : at;
                    cp_async_16(to + ar_at<D>(r, tid % PIECES), k_head + from, at >= 0);
                    cp_async_16(to + AR_TN * D * 2 + ar_at<D>(r, tid % PIECES), v_head + from, at >= 0);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        __syncthreads();
        // (tile numbers of a unit need not begin at 0: the stage of tile0 + 2 may be any, the queries' place is freed before it is filled)
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        uint32_t qf[KS][4];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            ldmatrix_x4(base + (AR_STAGES - 1) * ar_stage_bytes<D>() + ar_at<D>(wm * 16 + (lane & 15), ks * 2 + (lane >> 4)), qf[ks]);
        __syncthreads();
        fetch(g.tile0);
        fetch(g.tile0 + 1);

        float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;

        for (int tile = g.tile0; tile < tile1; ++tile) {
            asm volatile("cp.async.wait_group %0;" ::"n"(AR_STAGES - 2) : "memory");
            __syncthreads();
            fetch(tile + 2);
            put_place(tile + 3, page_ahead);
            page_ahead = page_of(tile + 4);
            const uint32_t k_s = base + (tile % AR_STAGES) * ar_stage_bytes<D>(), v_s = k_s + AR_TN * D * 2;
            const bool tail = (tile + 1) * AR_TN > common;   // has places that not every row sees
            if (tail && common < upto) {   // (0 times an infinite value is no number: the product gets a 0 there, the value is added at the end)
                for (int i = tid; i < AR_TN * PIECES; i += AR_THREADS) {
                    const int r = i / PIECES, t = tile * AR_TN + r;
                    if (t < common || t >= upto) continue;
                    uint4 *at = reinterpret_cast<uint4 *>(ar_base + (v_s - base) + ar_at<D>(r, i % PIECES));
                    uint4 u = *at;
                    bool odd = false;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t &x = (&u.x)[j];
                        if ((x & 0x7F80u) == 0x7F80u) { x &= 0xFFFF0000u; odd = true; }
                        if ((x & 0x7F800000u) == 0x7F800000u) { x &= 0xFFFFu; odd = true; }
                    }
                    if (odd) {
                        *at = u;
                        odd_s = 1;
                    }
                }
                __syncthreads();
            }
            float s[NB][4];
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int nb = 0; nb < NB; nb += 2) {
                    uint32_t kf[4];
                    ldmatrix_x4(k_s + ar_at<D>(wn * TW + nb * 8 + (lane & 7) + ((lane >> 4) << 3), ks * 2 + ((lane >> 3) & 1)), kf);
                    mma_bf16(s[nb], qf[ks], kf[0], kf[1]);
                    mma_bf16(s[nb + 1], qf[ks], kf[2], kf[3]);
                }
            const int token = tile * AR_TN + wn * TW + (lane & 3) * 2;
            float top[2] = {m[0], m[1]};
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[nb][j] *= p.scale_log2;
            if (tail) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int r = wm * 16 + (lane >> 2) + half * 8, node = (row_first + r) / p.group;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int t = token + nb * 8 + j;
                            const bool seen = t < g.s.len || (t < upto && r < rows && attn_sees(p, kind, anc, g.s.row0, node, t - g.s.len));
                            if (!seen) s[nb][half * 2 + j] = -INFINITY;
                        }
                }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                top[0] = fmaxf(top[0], fmaxf(s[nb][0], s[nb][1]));
                top[1] = fmaxf(top[1], fmaxf(s[nb][2], s[nb][3]));
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                top[half] = fmaxf(top[half], __shfl_xor_sync(0xffffffffu, top[half], 1));
                top[half] = fmaxf(top[half], __shfl_xor_sync(0xffffffffu, top[half], 2));
            }
            const float ref[2] = {top[0] == -INFINITY ? 0.f : top[0], top[1] == -INFINITY ? 0.f : top[1]};
            const float fade[2] = {power_of_two(m[0] - ref[0]), power_of_two(m[1] - ref[1])};
            m[0] = top[0];
            m[1] = top[1];
            l[0] *= fade[0];
            l[1] *= fade[1];
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                o[i][0] *= fade[0];
                o[i][1] *= fade[0];
                o[i][2] *= fade[1];
                o[i][3] *= fade[1];
            }
#pragma unroll
            for (int ks = 0; ks < NB / 2; ++ks) {
                uint32_t pf[4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float *x = s[2 * ks + i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = power_of_two(x[j] - ref[j >> 1]);
                    l[0] += x[0] + x[1];
                    l[1] += x[2] + x[3];
                    pf[2 * i] = pack_bf16(x[0], x[1]);
                    pf[2 * i + 1] = pack_bf16(x[2], x[3]);
                }
#pragma unroll
                for (int nb = 0; nb < D / 8; nb += 2) {
                    uint32_t vf[4];
                    ldmatrix_x4_trans(v_s + ar_at<D>(wn * TW + ks * 16 + (lane & 7) + ((lane >> 3) & 1) * 8, nb + (lane >> 4)), vf);
                    mma_bf16(o[nb], pf, vf[0], vf[1]);
                    mma_bf16(o[nb + 1], pf, vf[2], vf[3]);
                }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        // the warps' shares, through shared memory: [warp][16][D]
        float *x_s = reinterpret_cast<float *>(ar_base);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = (lane >> 2) + half * 8;
            float sum = l[half];
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            if ((lane & 3) == 0) {
                ml_s[warp][r][0] = m[half];
                ml_s[warp][r][1] = sum;
            }
            // (pieces of eight floats turn with the row, so that the eight rows of a store lie apart)
#pragma unroll
            for (int nb = 0; nb < D / 8; ++nb)
                *reinterpret_cast<float2 *>(x_s + (warp * 16 + r) * D + ((nb ^ (r & 7)) * 8) + (lane & 3) * 2) = make_float2(o[nb][half * 2], o[nb][half * 2 + 1]);
        }
        __syncthreads();
        const bool odd = odd_s != 0;
        for (int i = tid; i < rows * PIECES; i += AR_THREADS) {
            const int r = i / PIECES, c = i % PIECES, w0 = r / 16, in = r % 16;
            float top = -INFINITY, den = 0.f, x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < WN; ++k) top = fmaxf(top, ml_s[w0 + k * WM][in][0]);
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int k = 0; k < WN; ++k) {
                const int w = w0 + k * WM;
                const float f = power_of_two(ml_s[w][in][0] - ref);
                den = fmaf(f, ml_s[w][in][1], den);
                const float *src = x_s + (w * 16 + in) * D + (c ^ (in & 7)) * 8;
                const float4 a = *reinterpret_cast<const float4 *>(src), b = *reinterpret_cast<const float4 *>(src + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] = fmaf(f, (&a.x)[j], x[j]);
                    x[4 + j] = fmaf(f, (&b.x)[j], x[4 + j]);
                }
            }
            const int u = row_first + r, node = u / p.group;
            if (odd)
                for (int j = common - g.s.len; j <= node; ++j) {
                    const int t = g.s.len + j;
                    if (t < g.tile0 * AR_TN || t >= tile1 * AR_TN || !attn_sees(p, kind, anc, g.s.row0, node, j)) continue;
                    const long long at = attn_token_offset(p, g.b, t, upto);
                    if (at < 0) continue;
                    for (int e = 0; e < 8; ++e) {
                        const float v = __bfloat162float(v_cache[at + g.head * p.head_stride + c * 8 + e]);
                        if (!(fabsf(v) < INFINITY)) x[e] += v;
                    }
                }
            if (g.slot < 0) {
                const float inv = den == 0.f ? 0.f : 1.f / den;
                *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.o) + ((size_t)(g.s.row0 + node) * p.h_q + g.head * p.group + u % p.group) * D + c * 8) =
                    make_uint4(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv), pack_bf16(x[4] * inv, x[5] * inv),
                               pack_bf16(x[6] * inv, x[7] * inv));
            } else {
                const size_t at = (size_t)g.slot * M + r;
                float4 *to = reinterpret_cast<float4 *>(p.part_o + at * D + c * 8);
                to[0] = make_float4(x[0], x[1], x[2], x[3]);
                to[1] = make_float4(x[4], x[5], x[6], x[7]);
                if (c == 0) *reinterpret_cast<float2 *>(p.part_ml + at * 2) = make_float2(top, den);
            }
        }
        __syncthreads();   // (the next unit's queries, places and ancestors)
    }
}

}  // namespace

AttnTiling attn_rows_tiling(int rows, int d)
{
    return {rows <= 16 ? 16 : rows <= 32 ? 32 : 64, AR_TN, d == 128 ? ar_ctas<128>() : ar_ctas<64>(), 2};
}

cudaError_t launch_attn_rows(const AttnParams &p, int M, int grid, cudaStream_t stream)
{
    static PerContext seen[6];
    using Kernel = void (*)(const AttnParams);
    static const Kernel kernels[6] = {attn_rows_kernel<64, 1>, attn_rows_kernel<64, 2>, attn_rows_kernel<64, 4>,
                                      attn_rows_kernel<128, 1>, attn_rows_kernel<128, 2>, attn_rows_kernel<128, 4>};
    const int i = (p.d == 128 ? 3 : 0) + (M == 16 ? 0 : M == 32 ? 1 : 2);
    const size_t smem = p.d == 128 ? ar_smem<128>() : ar_smem<64>();
    int sms = 0;
    const cudaError_t e = device_sms(seen[i], reinterpret_cast<const void *>(kernels[i]), smem, &sms);
    if (e != cudaSuccess) return e;
    return launch_behind(kernels[i], dim3((unsigned)grid), AR_THREADS, smem, stream, p);
}

}  // namespace gdn
