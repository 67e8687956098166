// Attention over a paged cache for units of more than 64 rows (trees and prompt chunks of the query heads that share a key/value
// head): bf16, heads of 64 or 128 components, both products on the tensor cores with their sums in tensor memory.  The formulas stand
// in gdn_attn_general.cu.
//
// A unit has 256 rows, two streams of 128 that share every tile of 128 keys and values: at the tensor cores' rate a tile for one
// stream alone would ask L2 for 64 bytes per clock and SM, for two for half of that.  Per tile a stream goes through
//     S = Q K^T  ->  weights P of its rows (one thread each)  ->  O += P V
// and its next S stands behind its P V in the tensor cores' queue; while one stream forms weights the other multiplies.  P
// overwrites S in tensor memory (128 columns of S and D of O per stream).  Maxima that rise by less than 2^8 do not move the sums:
// weights up to 256 are as exact in bf16, and O is multiplied only where a row's maximum has risen by more.
//
// Roles: warps 0-3 and 4-7 the rows of the streams, warp 8 the tiles of keys and warp 9 those of values (cp.async, so that pages of any
// size and stride do, into the swizzled layout of the products' operands), warp 11 the queries, warp 10 the products.  Two stages of
// keys and of values, each with its own barriers.
// Every wait is bounded; one that expires raises a flag that ends the others.
#include "gdn_attn.cuh"

namespace gdn {

namespace {

constexpr int AS_THREADS = 384;
constexpr int AS_M = 256, AS_TN = 128, AS_STAGES = 2;
constexpr float AS_SLACK = 8.f;   // a maximum may rise by this many powers of two before the sums follow

template <int D> __host__ __device__ constexpr int as_tile_bytes() { return AS_TN * D * 2; }
template <int D> __host__ __device__ constexpr size_t as_smem() { return (size_t)as_tile_bytes<D>() * (2 + 2 * AS_STAGES) + 1024; }

struct SplitShared {
    unsigned long long anc[AT_SMALL_ROWS];
    int anc_up[AT_SMALL_ROWS];
    unsigned long long q_full, k_full[AS_STAGES], v_full[AS_STAGES], k_empty[AS_STAGES], v_empty[AS_STAGES], s_full[2], p_full[2], o_full[2];
    uint32_t tmem;
    int odd, dead;
};

// Byte offset of 16-byte piece c of row r of a [128][D] operand tile: [D / 64][128 rows][128 bytes], swizzled.
__device__ __forceinline__ uint32_t as_at(int r, int c) { return (uint32_t)((c >> 3) * (AS_TN * 128)) + sw128_row_offset(r, c & 7); }

// The same tile seen with its rows along the product's K (values): 64 components contiguous, blocks of 64 AS_TN * 128 bytes
// apart, eight rows 1024.
__device__ __forceinline__ uint64_t desc_rows_along_k(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)((AS_TN * 128) >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void umma_bf16_ts_into(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
#define GDN_TMEM_ST32(taddr, r)                                                                              \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "                                             \
                 "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"                                  \
                 "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"                         \
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),       \
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), \
                   "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),           \
                   "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])                        \
                 : "memory")
#define GDN_TMEM_ST16(taddr, r)                                                                              \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"    \
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),       \
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])              \
                 : "memory")

__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

// Bit j: row node `node` sees token t0 + j.
__device__ __forceinline__ uint32_t seen_word(const AttnParams &p, AttnMaskKind kind, const unsigned long long *anc, const AttnSeq &s, int node, int t0)
{
    if (!p.row_offsets) return low_bits(s.len - t0);
    if (kind == AT_CHAIN) return low_bits(s.len + node + 1 - t0);
    const int first = t0 - s.len;   // the node whose bit comes first, negative: that many committed tokens in front
    if (first <= -32) return ~0u;
    if (kind == AT_WORDS64) {
        const unsigned long long a = anc[node];
        return first >= 64 ? 0u : first >= 0 ? (uint32_t)(a >> first) : (uint32_t)(a << -first) | low_bits(-first);
    }
    const uint32_t *row = p.mask + (size_t)(s.row0 + node) * p.mask_words;   // (words behind the node's own are not written)
    const int last = node >> 5;
    if (first < 0) return row[0] << -first | low_bits(-first);
    const int w = first >> 5;
    const uint32_t lo = w <= last ? row[w] : 0u, hi = w + 1 <= last ? row[w + 1] : 0u;
    return __funnelshift_r(lo, hi, first & 31);
}

template <int D> __global__ void __launch_bounds__(AS_THREADS, 1) attn_sm100_kernel(const AttnParams p)
{
    constexpr int TILE = as_tile_bytes<D>(), KS = D / 16, PIECES = D / 8;
    extern __shared__ __align__(16) unsigned char as_raw[];
    __shared__ SplitShared sh;
    unsigned char *const data = as_raw + ((1024u - (smem_u32(as_raw) & 1023u)) & 1023u);   // swizzled tiles begin on 1024 bytes
    const uint32_t q_s = smem_u32(data), k_s = q_s + 2 * TILE, v_s = k_s + AS_STAGES * TILE;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = (int)blockIdx.x;
    const AttnMaskKind kind = attn_mask_kind(p);
    const __nv_bfloat16 *k_cache = static_cast<const __nv_bfloat16 *>(p.k_cache), *v_cache = static_cast<const __nv_bfloat16 *>(p.v_cache);

    if (tid == 0) {
        mbar_init(smem_u32(&sh.q_full), 32);
        for (int i = 0; i < AS_STAGES; ++i) {
            mbar_init(smem_u32(&sh.k_full[i]), 32);
            mbar_init(smem_u32(&sh.v_full[i]), 32);
            mbar_init(smem_u32(&sh.k_empty[i]), 1);
            mbar_init(smem_u32(&sh.v_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh.s_full[i]), 1);
            mbar_init(smem_u32(&sh.p_full[i]), 128);
            mbar_init(smem_u32(&sh.o_full[i]), 1);
        }
        sh.dead = 0;
    }
    wait_for_previous_kernel();
    if (warp == 10) tmem_alloc(smem_u32(&sh.tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;   // stream s: S (and P over it) at columns s * 256, O at s * 256 + 128
    volatile int *dead = &sh.dead;

    auto wait = [&](unsigned long long *bar, uint32_t parity) {   // by a whole warp; false: expired here or elsewhere
        const uint32_t at = smem_u32(bar);
        bool there = mbar_try_wait(at, parity);
        if (!there) {
            const long long t0 = clock64();
            while (!(there = mbar_try_wait(at, parity)) && !*dead)
                if (clock64() - t0 > 400000000LL) {
                    *dead = 1;
                    report_status(p.status_dev, GDN_ERR_TIMEOUT);
                }
        }
        return __all_sync(0xffffffffu, there) != 0;
    };

    // what has gone through the barriers before this unit: tiles, and tiles of the second stream; units
    uint32_t done = 0, done1 = 0, units = 0, units1 = 0;
    AttnWalk walk;
    AttnSegment g;
    walk.begin(p, cta, AS_M, AS_TN);
    while (walk.next(p, cta, AS_M, AS_TN, g)) {
        __syncthreads();   // the unit before is through
        if (*dead) break;
        if (p.row_offsets && kind == AT_WORDS64 && !attn_ancestors(p, g.s, sh.anc, sh.anc_up)) {
            if (tid == 0) report_status(p.status_dev, GDN_ERR_TREE);
            continue;
        }
        if (p.row_offsets && kind == AT_WORDS && !p.tree_ok[g.b]) continue;
        const int row_first = g.m_tile * AS_M, rows = min(AS_M, g.s.rows * p.group - row_first);
        const int last_node = (row_first + rows - 1) / p.group, upto = p.row_offsets ? g.s.len + last_node + 1 : g.s.len;
        const int tile1 = min(g.tile1, max((upto + AS_TN - 1) / AS_TN, g.tile0)), n_tiles = tile1 - g.tile0;
        const bool many = p.row_offsets && g.s.rows > 1;
        const int streams = rows > 128 ? 2 : 1;
        if (tid == 0) sh.odd = 0;
        __syncthreads();

        if (warp < 8) {   // ---- a row per thread
            const int stream = warp >> 2;
            if (stream < streams) {
                const int r = tid, u = row_first + r, node = u / p.group;
                const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_at = tmem + lanes + stream * 256, o_at = s_at + 128;
                const uint32_t seen_before = stream ? done1 : done;
                float m = -INFINITY, l = 0.f;   // m: of the raw scores, as the sums stand
                bool ok = true;
                for (int i = 0; i < n_tiles; ++i) {
                    const int tile = g.tile0 + i;
                    ok = wait(&sh.s_full[stream], (seen_before + i) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    // bit j of word c: this row sees token tile * AS_TN + 32 c + j
                    uint32_t see[4] = {~0u, ~0u, ~0u, ~0u};
                    bool tail = (tile + 1) * AS_TN > g.s.len || stream * 128 + 128 > rows;
                    if (tail) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) see[c] = r < rows ? seen_word(p, kind, sh.anc, g.s, node, tile * AS_TN + c * 32) : 0;
                        tail = __any_sync(0xffffffffu, (see[0] & see[1] & see[2] & see[3]) != ~0u);
                    }
                    float top = -INFINITY;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t x[32];
                        GDN_TMEM_LD32(s_at + c * 32, x);
                        tmem_wait_ld();
                        if (tail) {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (!(see[c] >> j & 1)) x[j] = 0xFF800000u;
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j) top = fmaxf(top, __uint_as_float(x[j]));
                    }
                    const bool first = i == 0;
                    const bool raise = first || (top - m) * p.scale_log2 > AS_SLACK || (m == -INFINITY && top > -INFINITY);
                    float fade = 1.f;
                    if (raise) {
                        const float m_new = fmaxf(m, top);
                        fade = first || m == -INFINITY ? 0.f : power_of_two((m - m_new) * p.scale_log2);
                        m = m_new;
                        l *= fade;
                    }
                    if (!first && __any_sync(0xffffffffu, raise)) {
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t x[32];
                            GDN_TMEM_LD32(o_at + c * 32, x);
                            tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[j] = __float_as_uint(__uint_as_float(x[j]) * fade);
                            GDN_TMEM_ST32(o_at + c * 32, x);
                        }
                    }
                    const float ref = m == -INFINITY ? 0.f : m * p.scale_log2;
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t x[32], w[16];
                        GDN_TMEM_LD32(s_at + c * 32, x);
                        tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            float e = power_of_two(fmaf(__uint_as_float(x[j]), p.scale_log2, -ref));
                            if (tail && !(see[c] >> j & 1)) e = 0.f;
                            sum[j & 3] += e;
                            x[j] = __float_as_uint(e);
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j) w[j] = pack_bf16(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1]));
                        GDN_TMEM_ST16(s_at + c * 16, w);
                    }
                    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(smem_u32(&sh.p_full[stream]));
                }
                if (ok && n_tiles > 0) ok = wait(&sh.o_full[stream], (stream ? units1 : units) & 1);
                tc_fence_after();
                if (ok) {
                    const bool odd = sh.odd != 0;
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(p.o) + ((size_t)(g.s.row0 + node) * p.h_q + g.head * p.group + u % p.group) * D;
                    const size_t part = (size_t)(g.slot < 0 ? 0 : g.slot) * AS_M + r;
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t x[32];
                        if (n_tiles > 0) {
                            GDN_TMEM_LD32(o_at + c * 32, x);
                            tmem_wait_ld();
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[j] = 0;
                        }
                        if (odd && r < rows)
                            for (int j = 0; j <= node; ++j) {
                                const int t = g.s.len + j;
                                if (t < g.tile0 * AS_TN || t >= tile1 * AS_TN || !attn_sees(p, kind, sh.anc, g.s.row0, node, j)) continue;
                                const long long at = attn_token_offset(p, g.b, t, upto);
                                if (at < 0) continue;
                                const __nv_bfloat16 *v = v_cache + at + g.head * p.head_stride + c * 32;
#pragma unroll
                                for (int e = 0; e < 32; ++e) {
                                    const float y = __bfloat162float(v[e]);
                                    if (!(fabsf(y) < INFINITY)) x[e] = __float_as_uint(__uint_as_float(x[e]) + y);
                                }
                            }
                        if (r >= rows) continue;
                        if (g.slot < 0) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                uint32_t w[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    w[k] = pack_bf16(__uint_as_float(x[8 * j + 2 * k]) * inv, __uint_as_float(x[8 * j + 2 * k + 1]) * inv);
                                *reinterpret_cast<uint4 *>(o + c * 32 + j * 8) = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                *reinterpret_cast<uint4 *>(p.part_o + part * D + c * 32 + j * 4) = make_uint4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                        }
                    }
                    if (r < rows && g.slot >= 0)
                        *reinterpret_cast<float2 *>(p.part_ml + part * 2) = make_float2(m == -INFINITY ? m : m * p.scale_log2, l);
                }
                tc_fence_before();
            }
        } else if (warp < 10) {   // ---- tiles, of keys or of values: 32 lanes, each with the places of four tokens
            const bool keys = warp == 8;
            constexpr int ROWS = 32 / PIECES;   // rows that one access of the warp covers
            const int col = lane % PIECES;
            const __nv_bfloat16 *from_head = (keys ? k_cache : v_cache) + g.head * p.head_stride + col * 8;
            const uint32_t to = keys ? k_s : v_s;
            unsigned long long *full = keys ? sh.k_full : sh.v_full, *empty = keys ? sh.k_empty : sh.v_empty;
            int page[4];
            auto ask = [&](int tile) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int t = tile * AS_TN + k * 32 + lane;
                    page[k] = tile < tile1 && t < upto
                                  ? p.page_table[(size_t)g.b * p.max_pages + (p.page_shift >= 0 ? t >> p.page_shift : t / p.page_size)] : -1;
                }
            };
            ask(g.tile0);
            for (int i = 0; i < n_tiles; ++i) {
                const uint32_t n = done + i;
                const int stage = n % AS_STAGES, tile = g.tile0 + i;
                long long place[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int t = tile * AS_TN + k * 32 + lane;
                    place[k] = -1;
                    if (t < upto) {
                        if (page[k] < 0 || page[k] >= p.n_pages) report_status(p.status_dev, GDN_ERR_PAGE);
                        else place[k] = page[k] * p.page_stride + (p.page_shift >= 0 ? t & (p.page_size - 1) : t % p.page_size) * p.token_stride;
                    }
                }
                ask(tile + 1);
                if (n >= AS_STAGES && !wait(&empty[stage], (n / AS_STAGES - 1) & 1)) break;
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll 8
                    for (int h = 0; h < 32 / ROWS; ++h) {
                        const int in = h * ROWS + lane / PIECES;
                        const long long at = __shfl_sync(0xffffffffu, place[k], in);
                        cp_async_16(to + stage * TILE + as_at(k * 32 + in, col), from_head + (at < 0 ? 0 : at), at >= 0);
                    }
                cp_async_wait_all();
                if (!keys && many && (tile + 1) * AS_TN > g.s.len)   // (an infinite value times a weight of 0 is no number: see the end of a unit)
                    for (int k = 0; k < AS_TN / ROWS; ++k) {
                        const int row = k * ROWS + lane / PIECES, t = tile * AS_TN + row;
                        if (t < g.s.len || t >= upto) continue;
                        uint4 *at = reinterpret_cast<uint4 *>(data + (v_s - q_s) + stage * TILE + as_at(row, col));   // (as this lane has copied it)
                        uint4 x = *at;
                        bool odd = false;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t &y = (&x.x)[e];
                            if ((y & 0x7F80u) == 0x7F80u) { y &= 0xFFFF0000u; odd = true; }
                            if ((y & 0x7F800000u) == 0x7F800000u) { y &= 0xFFFFu; odd = true; }
                        }
                        if (odd) {
                            *at = x;
                            sh.odd = 1;
                        }
                    }
                fence_proxy_async();
                mbar_arrive(smem_u32(&full[stage]));
            }
        } else if (warp == 11) {   // ---- queries of the streams
            if (n_tiles > 0) {
#pragma unroll 8
                for (int i = lane; i < streams * 128 * PIECES; i += 32) {
                    const int r = i / PIECES, c = i % PIECES, u = row_first + r;
                    const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(p.q);
                    if (r < rows) src += (size_t)(g.s.row0 + u / p.group) * p.q_stride + (size_t)(g.head * p.group + u % p.group) * D + c * 8;
                    cp_async_16(q_s + (r >> 7) * TILE + as_at(r & 127, c), src, r < rows);
                }
                cp_async_wait_all();
                fence_proxy_async();
                mbar_arrive(smem_u32(&sh.q_full));
            }
        } else if (n_tiles > 0) {   // ---- products
            constexpr uint32_t id_s = idesc_bf16(128, 128), id_o = idesc_bf16(128, D) | (1u << 16);
            bool ok = wait(&sh.q_full, units & 1);
            auto scores = [&](int s, int i) {
                const uint32_t k_at = k_s + ((done + i) % AS_STAGES) * TILE, q_at = q_s + s * TILE;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < KS; ++k)
                        umma_bf16(tmem + s * 256, smem_desc_sw128(q_at + (k >> 2) * (AS_TN * 128) + (k & 3) * 32),
                                  smem_desc_sw128(k_at + (k >> 2) * (AS_TN * 128) + (k & 3) * 32), id_s, k != 0);
                    umma_commit(smem_u32(&sh.s_full[s]));
                }
                __syncwarp();
            };
            ok = ok && wait(&sh.k_full[done % AS_STAGES], (done / AS_STAGES) & 1);
            tc_fence_after();
            if (ok) {
                for (int s = 0; s < streams; ++s) scores(s, 0);
                if (elect_one()) umma_commit(smem_u32(&sh.k_empty[done % AS_STAGES]));
                __syncwarp();
            }
            for (int i = 0; i < n_tiles && ok; ++i) {
                const uint32_t n = done + i, next = n + 1;
                const int stage = n % AS_STAGES;
                ok = wait(&sh.v_full[stage], (n / AS_STAGES) & 1);
                for (int s = 0; s < streams && ok; ++s) {
                    ok = wait(&sh.p_full[s], ((s ? done1 : done) + i) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < AS_TN / 16; ++k)
                            umma_bf16_ts_into(tmem + s * 256 + 128, tmem + s * 256 + k * 8, desc_rows_along_k(v_s + stage * TILE + k * 2048), id_o,
                                              i > 0 || k > 0);
                        if (i + 1 == n_tiles) umma_commit(smem_u32(&sh.o_full[s]));
                    }
                    __syncwarp();
                    if (i + 1 < n_tiles) {
                        if (s == 0) {
                            ok = wait(&sh.k_full[next % AS_STAGES], (next / AS_STAGES) & 1);
                            tc_fence_after();
                        }
                        if (ok) scores(s, i + 1);
                    }
                }
                if (ok && elect_one()) {
                    umma_commit(smem_u32(&sh.v_empty[stage]));
                    if (i + 1 < n_tiles) umma_commit(smem_u32(&sh.k_empty[next % AS_STAGES]));
                }
                __syncwarp();
            }
        }
        done += n_tiles;
        if (n_tiles > 0) ++units;
        if (streams == 2) {
            done1 += n_tiles;
            if (n_tiles > 0) ++units1;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (*dead) {   // products may still be on their way: behind them all comes this one's arrival
        if (warp == 10) {
            tc_fence_after();
            if (elect_one()) umma_commit(smem_u32(&sh.q_full));
            __syncwarp();
            const long long t0 = clock64();
            while (clock64() - t0 < 2000000) {}   // a millisecond, far longer than what can be in the queue takes
        }
        __syncthreads();
    }
    if (warp == 10) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

}  // namespace

AttnTiling attn_sm100_tiling() { return {AS_M, AS_TN, 1}; }

cudaError_t launch_attn_sm100(const AttnParams &p, int grid, cudaStream_t stream)
{
    static PerContext seen[2];
    const auto kernel = p.d == 128 ? attn_sm100_kernel<128> : attn_sm100_kernel<64>;
    const size_t smem = p.d == 128 ? as_smem<128>() : as_smem<64>();
    int sms = 0;
    const cudaError_t e = device_sms(seen[p.d == 128], reinterpret_cast<const void *>(kernel), smem, &sms);
    if (e != cudaSuccess) return e;
    return launch_behind(kernel, dim3((unsigned)grid), AS_THREADS, smem, stream, p);
}

}  // namespace gdn
