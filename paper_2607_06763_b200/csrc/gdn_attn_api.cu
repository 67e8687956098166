// C-ABI entry points of the operators over a paged key/value cache and of the sampler: argument checks, the choice of a
// kernel, the places in the workspace.  See include/gdn_tree.h for the contract of every function.
#include "gdn_attn.cuh"
#include "gdn_sample.cuh"

using namespace gdn;

namespace {

inline bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int check_attn_shape(const gdn_attn_shape_t *s)
{
    if (!s) return GDN_ERR_NULL;
    if (s->dtype != GDN_F32 && s->dtype != GDN_BF16) return GDN_ERR_DTYPE;
    if (s->n_seq < 0 || s->h_kv < 1 || s->h_q < 1 || s->h_q % s->h_kv != 0) return GDN_ERR_SHAPE;
    if (s->d < 8 || s->d > GDN_MAX_HEAD_DIM || s->d % 8 != 0) return GDN_ERR_SHAPE;
    if (s->total_rows < 0 || s->max_rows < 1 || s->n_pages < 1 || s->page_size < 1 || s->max_pages < 1 || s->max_len < 1)
        return GDN_ERR_SHAPE;
    if (s->max_len > (long long)s->max_pages * s->page_size || s->max_len > (1 << 30)) return GDN_ERR_SHAPE;
    if (!(s->scale == s->scale)) return GDN_ERR_SHAPE;   // NaN
    const int piece = s->dtype == GDN_BF16 ? 8 : 4;      // elements of 16 bytes
    if (s->page_stride < 0 || s->token_stride < 0 || s->head_stride < 0 || s->page_stride % piece || s->token_stride % piece ||
        s->head_stride % piece)
        return GDN_ERR_SHAPE;
    const long long row = (long long)s->h_q * s->d, kv_row = (long long)s->h_kv * s->d;
    if (row > (1 << 30) || s->q_stride < row || s->k_stride < kv_row || s->v_stride < kv_row || s->q_stride % piece ||
        s->k_stride % piece || s->v_stride % piece)
        return GDN_ERR_SHAPE;
    if ((long long)s->max_rows * (s->h_q / s->h_kv) > (1 << 30)) return GDN_ERR_SHAPE;
    return GDN_OK;
}

struct Choice {
    AttnTiling tiling;
    int m_tiles, grid;
    bool split;
    enum { GENERAL, ROWS, SM100 } kernel;
    AttnLayout layout;
};

// Grid of a kernel with the given tiles, and whether units are split; false: more units than a grid has CTAs.
bool place(const gdn_attn_shape_t &s, const AttnTiling &t, Choice &c)
{
    const long long rows = (long long)s.max_rows * (s.h_q / s.h_kv);
    c.tiling = t;
    c.m_tiles = (int)((rows + t.M - 1) / t.M);
    const long long units = (long long)s.n_seq * s.h_kv * c.m_tiles, tiles = ((long long)s.max_len + t.TN - 1) / t.TN;
    if (units > 0x7fffffffLL) return false;
    const long long resident = (long long)t.ctas * AT_SMS;
    // a chunk of a prompt with more units than two for every CTA goes without: its units see ever more tokens, and the longest begin first
    c.split = tiles > 1 && !(c.m_tiles > 1 && units >= 2 * resident);
    c.grid = (int)(!c.split ? units : units * tiles < resident ? units * tiles : resident);
    return true;
}

// The kernel for a shape, its grid, and the places in the workspace.
bool choose(const gdn_attn_shape_t &s, Choice &c)
{
    const long long rows = (long long)s.max_rows * (s.h_q / s.h_kv);
    // up to 64 rows per key/value head the keys and values decide, and one tile of rows reads them once; above, the products do.
    // (The kernel of the latter takes maxima of unscaled scores: a scale that turns or hides their order is the other's.)
    c.kernel = !(s.dtype == GDN_BF16 && (s.d == 64 || s.d == 128)) ? Choice::GENERAL : rows <= 64 || !(s.scale > 0.f) ? Choice::ROWS : Choice::SM100;
    const AttnTiling by_rows = attn_rows_tiling(rows < 64 ? (int)rows : 64, s.d);
    Choice other;   // (one workspace serves all scales)
    if (!place(s, c.kernel == Choice::GENERAL ? attn_general_tiling(s.dtype == GDN_BF16, s.d) : c.kernel == Choice::ROWS ? by_rows : attn_sm100_tiling(), c) ||
        !place(s, by_rows, other))
        return false;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align256(off + bytes);
        return at;
    };
    // (a call without parents needs no masks; the size is the same, so that one workspace serves all calls of a shape)
    const bool masks = s.max_rows > AT_SMALL_ROWS && s.max_rows <= GDN_MAX_TREE_NODES;
    c.layout.mask = take(masks ? sizeof(uint32_t) * (size_t)s.total_rows * ((s.max_rows + 31) / 32) : 0);
    c.layout.tree_ok = take(masks ? sizeof(int32_t) * (size_t)s.n_seq : 0);
    auto parts = [](const Choice &x) { return x.split ? 2 * (size_t)x.grid * x.tiling.M : 0; };
    size_t most = parts(c);
    if (c.kernel != Choice::GENERAL && rows > 64) {
        Choice tall;
        if (!place(s, attn_sm100_tiling(), tall)) return false;
        most = parts(tall) > parts(other) ? parts(tall) : parts(other);
    }
    c.layout.part_o = take(most * s.d * sizeof(float));
    c.layout.part_ml = take(most * 2 * sizeof(float));
    c.layout.total = off ? off : 256;
    return true;
}

AttnParams attn_params(const gdn_attn_shape_t &s, const void *q, const void *k_cache, const void *v_cache, const int32_t *page_table,
                       const int32_t *seq_lens, const int32_t *row_offsets, const int32_t *parent, void *o, int32_t *status_dev)
{
    AttnParams p{};
    p.n_seq = s.n_seq; p.h_q = s.h_q; p.h_kv = s.h_kv; p.group = s.h_q / s.h_kv; p.d = s.d;
    p.total_rows = s.total_rows; p.max_rows = s.max_rows; p.n_pages = s.n_pages; p.page_size = s.page_size;
    p.page_shift = -1;
    for (int i = 0; i < 31; ++i)
        if (1 << i == s.page_size) p.page_shift = i;
    p.max_pages = s.max_pages; p.max_len = s.max_len;
    p.scale_log2 = s.scale * 1.44269504088896340736f;
    p.page_stride = s.page_stride; p.token_stride = s.token_stride; p.head_stride = s.head_stride; p.q_stride = s.q_stride;
    p.q = q; p.k_cache = k_cache; p.v_cache = v_cache;
    p.page_table = page_table; p.seq_lens = seq_lens; p.row_offsets = row_offsets; p.parent = parent;
    p.o = o;
    p.status_dev = status_dev;
    return p;
}

int attention(const gdn_attn_shape_t *shape, const void *q, const void *k_cache, const void *v_cache, const int32_t *page_table,
              const int32_t *seq_lens, bool tree, const int32_t *parent, const int32_t *row_offsets, void *o, void *workspace,
              size_t workspace_bytes, int32_t *status_dev, void *cuda_stream)
{
    const int rc = check_attn_shape(shape);
    if (rc != GDN_OK) return rc;
    const gdn_attn_shape_t &s = *shape;
    if (!tree && (s.max_rows != 1 || s.total_rows != s.n_seq)) return GDN_ERR_SHAPE;
    if (parent && s.max_rows > GDN_MAX_TREE_NODES) return GDN_ERR_SHAPE;
    if (s.n_seq == 0 || s.total_rows == 0) return GDN_OK;
    if (!q || !k_cache || !v_cache || !page_table || !seq_lens || (tree && !row_offsets) || !o || !status_dev) return GDN_ERR_NULL;
    if (!workspace) return GDN_ERR_WORKSPACE;
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(o, 16) || !aligned(workspace, 256) ||
        !aligned(page_table, 4) || !aligned(seq_lens, 4) || !aligned(row_offsets, 4) || !aligned(parent, 4) || !aligned(status_dev, 4))
        return GDN_ERR_ALIGN;
    Choice c;
    if (!choose(s, c)) return GDN_ERR_UNSUPPORTED;
    if (parent && s.n_seq > 65535 && s.max_rows > AT_SMALL_ROWS) return GDN_ERR_UNSUPPORTED;
    if (workspace_bytes < c.layout.total) return GDN_ERR_WORKSPACE;
    AttnParams p = attn_params(s, q, k_cache, v_cache, page_table, seq_lens, row_offsets, parent, o, status_dev);
    char *w = static_cast<char *>(workspace);
    p.split = c.split;
    p.m_tiles = c.m_tiles;
    p.mask = reinterpret_cast<uint32_t *>(w + c.layout.mask);
    p.mask_words = (s.max_rows + 31) / 32;
    p.tree_ok = reinterpret_cast<int32_t *>(w + c.layout.tree_ok);
    p.part_o = reinterpret_cast<float *>(w + c.layout.part_o);
    p.part_ml = reinterpret_cast<float *>(w + c.layout.part_ml);
    p.n_ctas = c.grid;
    p.over = c.tiling.over;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool bf16 = s.dtype == GDN_BF16;
    if (parent && s.max_rows > AT_SMALL_ROWS && launch_attn_masks(p, stream) != cudaSuccess) return GDN_ERR_CUDA;
    const cudaError_t e = c.kernel == Choice::GENERAL ? launch_attn_general(p, bf16, c.grid, stream)
                          : c.kernel == Choice::ROWS  ? launch_attn_rows(p, c.tiling.M, c.grid, stream)
                                                      : launch_attn_sm100(p, c.grid, stream);
    if (e != cudaSuccess) return GDN_ERR_CUDA;
    if (c.split && launch_attn_join(p, bf16, c.tiling.M, c.tiling.TN, c.kernel == Choice::SM100, stream) != cudaSuccess) return GDN_ERR_CUDA;
    return GDN_OK;
}

// Rows into the cache: all of a call's (path null), or those of accepted paths.
int write_rows(const gdn_attn_shape_t *shape, const void *q, const void *k, const void *v, const float *rope, int32_t rope_len,
               int32_t rope_dim, int32_t interleaved, const int32_t *parent, const int32_t *row_offsets, bool accepted,
               const int32_t *path, const int32_t *path_offsets, const int32_t *seq_lens, const int32_t *page_table, void *q_out,
               void *k_cache, void *v_cache, int32_t *status_dev, void *cuda_stream)
{
    const int rc = check_attn_shape(shape);
    if (rc != GDN_OK) return rc;
    const gdn_attn_shape_t &s = *shape;
    if (rope_dim < 0 || rope_dim > s.d || rope_dim % 2 != 0) return GDN_ERR_SHAPE;
    if (rope_dim > 0 && rope_len < s.max_len) return GDN_ERR_SHAPE;
    if (s.n_seq == 0 || s.total_rows == 0) return GDN_OK;
    if (!k || !v || !row_offsets || !seq_lens || !page_table || !k_cache || !v_cache || !status_dev || (rope_dim > 0 && !rope))
        return GDN_ERR_NULL;
    if ((q == nullptr) != (q_out == nullptr) || (accepted && (!path || !path_offsets))) return GDN_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(rope, 16) || !aligned(q_out, 16) || !aligned(k_cache, 16) ||
        !aligned(v_cache, 16) || !aligned(parent, 4) || !aligned(row_offsets, 4) || !aligned(path, 4) || !aligned(path_offsets, 4) ||
        !aligned(seq_lens, 4) || !aligned(page_table, 4) || !aligned(status_dev, 4))
        return GDN_ERR_ALIGN;
    if (q && q == q_out && s.q_stride != (long long)s.h_q * s.d) return GDN_ERR_SHAPE;   // rows would move onto one another
    const AttnParams p = attn_params(s, q, k_cache, v_cache, page_table, seq_lens, row_offsets, parent, nullptr, status_dev);
    return launch_kv_append(p, s.dtype == GDN_BF16, k, v, s.k_stride, s.v_stride, rope, rope_dim, interleaved != 0, q_out, k_cache,
                            v_cache, path, path_offsets, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess
               ? GDN_OK : GDN_ERR_CUDA;
}

}  // namespace

extern "C" size_t gdn_attn_workspace_bytes(const gdn_attn_shape_t *shape)
{
    Choice c;
    return check_attn_shape(shape) == GDN_OK && choose(*shape, c) ? c.layout.total : 0;
}

extern "C" int gdn_attn_decode(const gdn_attn_shape_t *shape, const void *q, const void *k_cache, const void *v_cache,
                               const int32_t *page_table, const int32_t *seq_lens, void *o, void *workspace, size_t workspace_bytes,
                               int32_t *status_dev, void *cuda_stream)
{
    return attention(shape, q, k_cache, v_cache, page_table, seq_lens, false, nullptr, nullptr, o, workspace, workspace_bytes,
                     status_dev, cuda_stream);
}

extern "C" int gdn_attn_tree_verify(const gdn_attn_shape_t *shape, const void *q, const void *k_cache, const void *v_cache,
                                    const int32_t *page_table, const int32_t *seq_lens, const int32_t *parent,
                                    const int32_t *row_offsets, void *o, void *workspace, size_t workspace_bytes, int32_t *status_dev,
                                    void *cuda_stream)
{
    return attention(shape, q, k_cache, v_cache, page_table, seq_lens, true, parent, row_offsets, o, workspace, workspace_bytes,
                     status_dev, cuda_stream);
}

extern "C" int gdn_kv_append(const gdn_attn_shape_t *shape, const void *q, const void *k, const void *v, const float *rope,
                             int32_t rope_len, int32_t rope_dim, int32_t interleaved, const int32_t *parent,
                             const int32_t *row_offsets, const int32_t *seq_lens, const int32_t *page_table, void *q_out, void *k_cache,
                             void *v_cache, int32_t *status_dev, void *cuda_stream)
{
    return write_rows(shape, q, k, v, rope, rope_len, rope_dim, interleaved, parent, row_offsets, false, nullptr, nullptr, seq_lens,
                      page_table, q_out, k_cache, v_cache, status_dev, cuda_stream);
}

extern "C" int gdn_kv_commit(const gdn_attn_shape_t *shape, const void *k, const void *v, const float *rope, int32_t rope_len,
                             int32_t rope_dim, int32_t interleaved, const int32_t *parent, const int32_t *row_offsets,
                             const int32_t *path, const int32_t *path_offsets, const int32_t *seq_lens, const int32_t *page_table,
                             void *k_cache, void *v_cache, int32_t *status_dev, void *cuda_stream)
{
    return write_rows(shape, nullptr, k, v, rope, rope_len, rope_dim, interleaved, parent, row_offsets, true, path, path_offsets,
                      seq_lens, page_table, nullptr, k_cache, v_cache, status_dev, cuda_stream);
}

extern "C" int gdn_sample(const gdn_sample_shape_t *shape, const void *logits, const float *temperature, const int32_t *top_k,
                          const float *top_p, const float *min_p, const float *uniform, int32_t *token, float *prob, int32_t *status_dev,
                          void *cuda_stream)
{
    if (!shape) return GDN_ERR_NULL;
    const gdn_sample_shape_t &s = *shape;
    if (s.dtype != GDN_F32 && s.dtype != GDN_BF16) return GDN_ERR_DTYPE;
    if (s.n_rows < 0 || s.vocab < 1 || s.vocab > GDN_MAX_VOCAB || s.row_stride < s.vocab) return GDN_ERR_SHAPE;
    if (s.n_rows == 0) return GDN_OK;
    if (!logits || !uniform || !token || !status_dev) return GDN_ERR_NULL;
    if (!aligned(logits, s.dtype == GDN_BF16 ? 2 : 4) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) ||
        !aligned(min_p, 4) || !aligned(uniform, 4) || !aligned(token, 4) || !aligned(prob, 4) || !aligned(status_dev, 4))
        return GDN_ERR_ALIGN;
    const SampleParams p{s.n_rows, s.vocab, s.row_stride, logits, temperature, top_k, top_p, min_p, uniform, token, prob};
    return launch_sample(p, s.dtype == GDN_BF16, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? GDN_OK : GDN_ERR_CUDA;
}
