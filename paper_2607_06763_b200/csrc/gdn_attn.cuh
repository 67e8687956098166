// What the attention kernels over a paged cache have in common: their arguments, how the work is cut up and handed out, which
// cached token a row may see, and the places in the workspace.
//
// A unit is (sequence, key/value head, tile of M rows); row r of a unit is node r / G of the sequence's rows with query head
// head * G + r % G (G = h_q / h_kv), so that the G query heads that share a key/value head share its tiles.  The tokens of a
// unit come in tiles of TN.  Where a call has more than one tile per unit, the tiles of all units, one behind the other,
// are cut into as many equal runs as there are CTAs: a batch of lengths from one to many thousands keeps every SM busy to the
// end, whatever the lengths, which only the device knows.  A run that holds a whole unit writes its rows; the others leave
// their unnormalised sums with maximum and denominator in the workspace, where the join kernel finds them by the same
// arithmetic.  A CTA has at most two such parts: the first unit of its run, begun by another CTA, and the last.
#pragma once

#include "gdn_internal.cuh"
#include "gdn_path.cuh"
#include "gdn_tc.cuh"

namespace gdn {

constexpr int AT_SMALL_ROWS = 64;   // trees up to this size: every CTA derives the ancestors itself (one 64-bit word per node)

struct AttnParams {
    int n_seq, h_q, h_kv, group, d, total_rows, max_rows, n_pages, page_size, page_shift, max_pages, max_len;
    float scale_log2;                                // scale * log2(e): scores in units of a power of two
    long long page_stride, token_stride, head_stride, q_stride;   // in elements
    const void *q, *k_cache, *v_cache;
    const int32_t *page_table, *seq_lens, *row_offsets, *parent;  // row_offsets null: one row per sequence, all of its tokens seen
    void *o;
    int32_t *status_dev;
    int split;                                       // 0: CTA = unit
    int m_tiles;                                     // tiles of M rows that the longest sequence has
    // workspace: ancestors of trees above AT_SMALL_ROWS nodes, then the parts of split units
    uint32_t *mask;                                  // [total_rows][mask_words]
    int mask_words;
    int32_t *tree_ok;                                // [n_seq]
    float *part_o, *part_ml;                         // [2 * CTAs][M * d], [2 * CTAs][M][2]: sums; maximum, denominator
    int n_ctas, over;                                // runs; tiles that a unit counts for beyond its own
};

struct AttnLayout {
    size_t mask, tree_ok, part_o, part_ml, total;
};

#ifdef __CUDACC__
// 2^x to 2^-22 of itself (0 for -inf).
__device__ __forceinline__ float power_of_two(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct AttnSeq {
    int len, rows, row0, held;   // committed tokens; rows of the call, the first of them; tokens that any row sees
};

// Lengths of sequence b; false where they are not possible (reported by the caller that is asked to).
__device__ __forceinline__ bool attn_seq(const AttnParams &p, int b, AttnSeq &s, bool report)
{
    s.len = p.seq_lens[b];
    if (p.row_offsets) {
        const int r0 = p.row_offsets[b], r1 = p.row_offsets[b + 1];
        s.row0 = r0;
        s.rows = r1 - r0;
        if (r0 < 0 || r1 > p.total_rows || r1 < r0 || s.rows > p.max_rows) {
            if (report) report_status(p.status_dev, GDN_ERR_TREE);
            return false;
        }
        if (s.len < 0 || s.len > p.max_len - s.rows) {
            if (report) report_status(p.status_dev, GDN_ERR_PAGE);
            return false;
        }
        s.held = s.len + s.rows;
    } else {
        s.row0 = b;
        s.rows = 1;
        s.held = s.len;
        if (s.len < 0 || s.len > p.max_len) {
            if (report) report_status(p.status_dev, GDN_ERR_PAGE);
            return false;
        }
    }
    return true;
}

struct AttnSegment {
    AttnSeq s;
    int b, head, m_tile;
    int tile0, tile1, tiles;   // tiles [tile0, tile1) of the unit's `tiles`
    int slot;                  // place of the part in the workspace, -1: the whole unit
};

__device__ __forceinline__ int attn_tiles(const AttnSeq &s, int TN) { return s.held > TN ? (s.held + TN - 1) / TN : 1; }

// Units of sequence b, each of attn_tiles(s, TN) tiles; 0 where its lengths are not possible.
__device__ __forceinline__ int attn_units(const AttnParams &p, int b, int M, AttnSeq &s, bool report)
{
    return attn_seq(p, b, s, report) ? p.h_kv * ((s.rows * p.group + M - 1) / M) : 0;
}

// a * b / c, by a 32-bit division wherever the product fits (a 64-bit one takes some hundred instructions).
__device__ __forceinline__ long long times_over(long long a, long long b, long long c)
{
    const unsigned long long ab = (unsigned long long)a * (unsigned long long)b;
    return ((ab | (unsigned long long)c) >> 32) == 0 ? (long long)((uint32_t)ab / (uint32_t)c) : (long long)(ab / (unsigned long long)c);
}

// Sum over the lanes up to and including this one.
__device__ __forceinline__ long long warp_scan(long long x, int lane)
{
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += up;
    }
    return x;
}

// Sum over the lanes of numbers below 2^50, by two reductions of 32 bits.
__device__ __forceinline__ long long warp_sum(long long x)
{
    const uint32_t lo = (uint32_t)x & 0xFFFFFFu, hi = (uint32_t)(x >> 24);
    return ((long long)__reduce_add_sync(0xffffffffu, hi) << 24) + __reduce_add_sync(0xffffffffu, lo);
}

// What all runs together hold, and what of it lies in the sequences of this lane and in front of sequence `before_b`, by a whole warp.
struct AttnTotal {
    long long total, mine, before;
    int over;        // tiles that a unit counts for beyond its own
    long long per;   // small calls: tiles of a run (as many as the longest would have if all were alike, so that fewer runs lie across two units); else 0
    __device__ __forceinline__ long long runs(const AttnParams &p) const
    {
        return per ? times_over(total + per - 1, 1, per) : total < p.n_ctas ? total : p.n_ctas;
    }
    __device__ __forceinline__ long long begin(long long run, long long runs) const { return per ? min(run * per, total) : times_over(total, run, runs); }
    // of a place of the total, the last run that begins at it or in front of it
    __device__ __forceinline__ int run_of(long long place, long long runs) const
    {
        return (int)(per ? times_over(place, 1, per) : times_over((place + 1) * runs - 1, 1, total));
    }
};
template <bool BEFORE> __device__ __forceinline__ AttnTotal attn_total(const AttnParams &p, int M, int TN, int before_b, bool report)
{
    const int lane = threadIdx.x & 31, per = (p.n_seq + 31) / 32, b0 = min(lane * per, p.n_seq), b1 = min(b0 + per, p.n_seq);
    long long tiles = 0, units = 0, tiles_before = 0, units_before = 0;
    for (int i = b0; i < b1; ++i) {
        AttnSeq s;
        const int n = attn_units(p, i, M, s, report);
        const long long t = n ? (long long)n * attn_tiles(s, TN) : 0;
        tiles += t;
        units += n;
        if (i < before_b) {
            tiles_before += t;
            units_before += n;
        }
    }
    const long long all_tiles = warp_sum(tiles), all_units = __reduce_add_sync(0xffffffffu, (uint32_t)units);
    AttnTotal r;
    r.over = all_tiles >= 4ll * p.n_ctas ? p.over : 0;   // (p.over > 0)
    r.total = all_tiles + all_units * r.over;
    r.per = r.over ? 0 : times_over(all_tiles + p.n_ctas - 1, 1, p.n_ctas);
    r.mine = tiles + units * r.over;
    r.before = BEFORE ? warp_sum(tiles_before + units_before * r.over) : 0;
    return r;
}

// The run of one CTA, walked by every warp on its own (the same values in all of them; no exchange between warps).
struct AttnWalk {
    long long at, end;   // the run, counted over all units
    long long seq_at;    // where sequence b begins
    int b, over;
    AttnSeq s;

    __device__ __forceinline__ void begin(const AttnParams &p, int cta, int M, int TN)
    {
        if (!p.split) {   // CTA = unit, the last rows (the most tokens) first
            at = 0;
            end = 1;
            return;
        }
        const int lane = threadIdx.x & 31;
        const int per = (p.n_seq + 31) / 32, b0 = min(lane * per, p.n_seq), b1 = min(b0 + per, p.n_seq);
        const AttnTotal sum = attn_total<false>(p, M, TN, 0, cta == 0 && threadIdx.x < 32);
        const long long mine = sum.mine, upto = warp_scan(mine, lane);
        over = sum.over;
        const long long runs = sum.runs(p);
        at = end = 0;
        if (cta >= runs) return;
        at = sum.begin(cta, runs);
        end = sum.begin(cta + 1, runs);
        // the lane whose sequences hold tile `at` looks for it among them
        const unsigned holds = __ballot_sync(0xffffffffu, upto > at);
        const int owner = __ffs(holds) - 1;
        int found = 0;
        long long begins = upto - mine;
        if (lane == owner)
            for (int i = b0; i < b1; ++i) {
                AttnSeq t;
                const int n = attn_units(p, i, M, t, false);
                const long long w = n ? (long long)n * (attn_tiles(t, TN) + over) : 0;
                if (begins + w > at) {
                    found = i;
                    break;
                }
                begins += w;
            }
        b = __shfl_sync(0xffffffffu, found, owner);
        seq_at = __shfl_sync(0xffffffffu, begins, owner);
    }

    __device__ __forceinline__ bool next(const AttnParams &p, int cta, int M, int TN, AttnSegment &g)
    {
        if (at >= end) return false;
        if (!p.split) {
            at = end;
            const int per_seq = p.h_kv * p.m_tiles;
            g.b = cta / per_seq;
            g.m_tile = p.m_tiles - 1 - cta % per_seq / p.h_kv;
            g.head = cta % p.h_kv;
            g.tile0 = 0;
            g.slot = -1;
            if (!attn_seq(p, g.b, g.s, g.head == 0 && g.m_tile == 0) || g.m_tile * M >= g.s.rows * p.group) return false;
            g.tile1 = g.tiles = attn_tiles(g.s, TN);
            return true;
        }
        do {   // (what a unit counts for beyond its tiles is no work)
            if (at >= end) return false;
            for (;;) {   // place `at` of the total belongs to some sequence
                if (b >= p.n_seq) return false;   // (lengths that changed meanwhile)
                const int n = attn_units(p, b, M, s, false);
                const long long w = n ? (long long)n * (attn_tiles(s, TN) + over) : 0;
                if (at < seq_at + w) break;
                seq_at += w;
                ++b;
            }
            g.s = s;
            g.b = b;
            g.tiles = attn_tiles(s, TN);
            const int per = g.tiles + over, unit = (int)times_over(at - seq_at, 1, per), m_tiles = (s.rows * p.group + M - 1) / M;
            g.head = unit / m_tiles;
            g.m_tile = unit % m_tiles;
            const int from = (int)((at - seq_at) - (long long)unit * per);
            const long long left = end - at;
            const int to = left < per - from ? from + (int)left : per;
            g.tile0 = max(from - over, 0);
            g.tile1 = max(to - over, 0);
            at += to - from;
        } while (g.tile0 == g.tile1);
        g.slot = g.tile0 == 0 ? (g.tile1 == g.tiles ? -1 : 2 * cta + 1) : 2 * cta;
        return true;
    }
};

// Where token t of sequence b lies in the cache, in elements from its base for head 0; -1 where the page table says nothing
// possible (reported) or t is behind the last token.
__device__ __forceinline__ long long attn_token_offset(const AttnParams &p, int b, int t, int held)
{
    if (t >= held) return -1;
    const int entry = p.page_shift >= 0 ? t >> p.page_shift : t / p.page_size;
    const int page = p.page_table[(size_t)b * p.max_pages + entry];
    if (page < 0 || page >= p.n_pages) {
        report_status(p.status_dev, GDN_ERR_PAGE);
        return -1;
    }
    return page * p.page_stride + (t - entry * p.page_size) * p.token_stride;
}

// Ancestors of the nodes of a tree of at most 64 nodes, the node itself among them, for all threads of the CTA, by its first warp
// (two nodes per lane); a and up are [64] each.  False where the tree is none, for all threads alike: the verdict comes with the barrier, for a
// flag in shared memory could be that of the next unit's tree before the last thread has read it.  Doubling: after k rounds a node knows
// its next 2^k ancestors.
__device__ __forceinline__ bool attn_ancestors(const AttnParams &p, const AttnSeq &s, unsigned long long *a, int *up)
{
    const int lane = threadIdx.x;
    bool bad = false;
    if (lane < 32) {
        int next[2];
        unsigned long long seen[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = lane + 32 * h;
            next[h] = i < s.rows ? p.parent[s.row0 + i] : -1;
            bad |= next[h] < -1 || next[h] >= i;
        }
        bad = __any_sync(0xffffffffu, bad);
        for (int step = 1; !bad && step < 2 * s.rows; step <<= 1) {   // (the last round only writes)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = lane + 32 * h;
                if (step == 1) seen[h] = 1ull << i;
                a[i] = seen[h];
                up[i] = next[h];
            }
            __syncwarp();
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (next[h] >= 0) {
                    seen[h] |= a[next[h]];
                    next[h] = up[next[h]];
                }
            __syncwarp();
        }
    }
    return !__syncthreads_or(bad);
}

// Whether row node i sees node j of its sequence's rows (i, j < rows).
enum AttnMaskKind { AT_CHAIN, AT_WORDS64, AT_WORDS };
__device__ __forceinline__ bool attn_sees(const AttnParams &p, AttnMaskKind kind, const unsigned long long *a, int row0, int i, int j)
{
    if (j > i) return false;
    if (kind == AT_CHAIN) return true;
    if (kind == AT_WORDS64) return a[i] >> j & 1;
    return p.mask[(size_t)(row0 + i) * p.mask_words + (j >> 5)] >> (j & 31) & 1;
}
__device__ __forceinline__ AttnMaskKind attn_mask_kind(const AttnParams &p)
{
    return !p.parent ? AT_CHAIN : p.max_rows <= AT_SMALL_ROWS ? AT_WORDS64 : AT_WORDS;
}
#endif

constexpr int AT_SMS = 148;
struct AttnTiling {
    int M, TN, ctas, over;   // rows and tokens of a tile, CTAs that an SM holds, tiles that take as long as what a unit takes beside its own
};
AttnTiling attn_general_tiling(bool bf16, int d);
// `bf16`: the type of rows, cache and outputs; otherwise fp32.
cudaError_t launch_attn_general(const AttnParams &p, bool bf16, int grid, cudaStream_t stream);
// bf16, d = 64 or 128, tiles of 16, 32 or 64 rows.
AttnTiling attn_rows_tiling(int rows, int d);
cudaError_t launch_attn_rows(const AttnParams &p, int M, int grid, cudaStream_t stream);
// bf16, d = 64 or 128, scale > 0, tiles of 256 rows.
AttnTiling attn_sm100_tiling();
cudaError_t launch_attn_sm100(const AttnParams &p, int grid, cudaStream_t stream);
cudaError_t launch_attn_masks(const AttnParams &p, cudaStream_t stream);
// columns_first: parts lie [d / 4][M][4], not [M][d].
cudaError_t launch_attn_join(const AttnParams &p, bool bf16, int M, int TN, bool columns_first, cudaStream_t stream);

cudaError_t launch_kv_append(const AttnParams &a, bool bf16, const void *k, const void *v, long long k_stride, long long v_stride,
                             const float *rope, int rope_dim, bool interleaved, void *q_out, void *k_out, void *v_out,
                             const int32_t *path, const int32_t *path_offsets, cudaStream_t stream);

// A launch that may become resident under the tail of the kernel in front of it, where it waits (wait_for_previous_kernel).
template <typename... KernelArgs, typename... Args>
cudaError_t launch_behind(void (*kernel)(KernelArgs...), dim3 grid, int threads, size_t smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace gdn
