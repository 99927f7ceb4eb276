// C-ABI entry points of the recurrent layers' operators and of the cache's pages: argument checks and dispatch.
#include "layers.cuh"
#include "cache_pages.cuh"

namespace {

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline uintptr_t size_of(int32_t dt) { return dt == GDN_BF16 ? 2 : 4; }

int32_t done(cudaError_t e, int launches)
{
    if (e == cudaErrorNotSupported) return GDN_ERR_UNSUPPORTED;
    if (e != cudaSuccess) return GDN_ERR_CUDA;
    gdn::set_launch_count(launches);
    return GDN_OK;
}

// Rows of a packed batch, and pages that a call ranks: the kernels add up to a block's rows, or a CTA's threads and a share's rounding, to their numbers in 32 bits.
constexpr int64_t kMostRows = 0x7fffffffLL - 63;
constexpr int32_t kMostPages = 1 << 30;

// What the two layers have in common.  `step`: one token per request, states in and out.
int32_t check_layer(int32_t channels, int32_t io_dtype, int32_t num_seqs, int64_t total, int32_t num_init, int32_t num_out, const int32_t* cu,
                    const int32_t* init_slots, const int32_t* out_slots, const int32_t* status_word, const void* state_in, const void* state_out, bool step)
{
    if (channels <= 0 || num_seqs < 0 || (io_dtype != GDN_F32 && io_dtype != GDN_BF16)) return GDN_ERR_INVALID_ARG;
    if (!step && (total < 0 || total > kMostRows || !cu || !aligned(cu, 4))) return GDN_ERR_INVALID_ARG;
    if (step && (!state_in || !state_out)) return GDN_ERR_INVALID_ARG;
    if (!aligned(init_slots, 4) || !aligned(out_slots, 4) || !aligned(status_word, 4) || !aligned(state_in, 16) || !aligned(state_out, 16))
        return GDN_ERR_INVALID_ARG;
    if (num_init < 0 || num_out < 0) return GDN_ERR_INVALID_ARG;
    // without a list, request n has slot n: the pools have to hold that many
    if (!init_slots && state_in && num_init < num_seqs) return GDN_ERR_INVALID_ARG;
    if ((step ? !init_slots : !out_slots) && state_out && num_out < num_seqs) return GDN_ERR_INVALID_ARG;
    return GDN_OK;
}

// a [rows, channels] argument in the io dtype (without rows it may be NULL)
struct Rows {
    int64_t rows;
    uintptr_t esz;
    bool operator()(const void* p, int64_t stride, int64_t least) const
    {
        return (p || rows == 0) && aligned(p, esz) && stride >= least && stride <= (1LL << 40);
    }
};

// Whether `out` begins where an input does but its rows lie elsewhere: one row's result would replace another row's input.
inline bool crosses(const void* out, int64_t out_stride, const void* in, int64_t stride, int64_t rows)
{
    return rows > 1 && out && out == in && out_stride != stride;
}

int32_t conv(const gdn_conv_desc* d, const void* x, const void* weight, const void* bias, const int32_t* cu, const void* state_in, void* out,
             void* state_out, bool step)
{
    gdn::set_launch_count(0);
    if (!d) return GDN_ERR_INVALID_ARG;
    const int32_t rc = check_layer(d->channels, d->io_dtype, d->num_seqs, d->total_tokens, d->num_init_states, d->num_out_states, cu, d->init_slots,
                                   d->out_slots, d->status_word, state_in, state_out, step);
    if (rc != GDN_OK) return rc;
    const uintptr_t e = size_of(d->io_dtype);
    if (!weight || !aligned(weight, e) || !aligned(bias, e) || (d->silu != 0 && d->silu != 1)) return GDN_ERR_INVALID_ARG;
    const Rows rows_ok{step ? d->num_seqs : d->total_tokens, e};
    if (!rows_ok(x, d->x_stride, d->channels) || !rows_ok(out, d->out_stride, d->channels)) return GDN_ERR_INVALID_ARG;
    if (!step && out == x && x) return GDN_ERR_INVALID_ARG;
    if (crosses(out, d->out_stride, x, d->x_stride, rows_ok.rows)) return GDN_ERR_INVALID_ARG;
    if (d->width < 2 || d->width > 4) return GDN_ERR_UNSUPPORTED;
    if (d->num_seqs == 0) return GDN_OK;
    gdn::ConvArgs a = {};
    a.x = x; a.weight = weight; a.bias = bias; a.init_state = state_in; a.out = out; a.out_state = state_out; a.cu = cu;
    a.init_slots = d->init_slots; a.out_slots = d->out_slots; a.status_word = d->status_word;
    a.x_stride = d->x_stride; a.out_stride = d->out_stride; a.total_tokens = d->total_tokens;
    a.channels = d->channels; a.num_seqs = d->num_seqs; a.num_init = d->num_init_states; a.num_out = d->num_out_states; a.silu = d->silu;
    return done(gdn::launch_conv(a, d->io_dtype, d->width, step, (cudaStream_t)d->stream), 1);
}

int32_t scan(const gdn_scan_desc* d, const void* x, const void* dt, const float* a, const void* b, const void* c, const float* skip, const void* z,
             const float* dt_bias, const int32_t* cu, const float* state_in, void* out, float* state_out, bool step)
{
    gdn::set_launch_count(0);
    if (!d) return GDN_ERR_INVALID_ARG;
    const int32_t rc = check_layer(d->channels, d->io_dtype, d->num_seqs, d->total_tokens, d->num_init_states, d->num_out_states, cu, d->init_slots,
                                   d->out_slots, d->status_word, state_in, state_out, step);
    if (rc != GDN_OK) return rc;
    const uintptr_t e = size_of(d->io_dtype);
    if (d->groups <= 0 || d->channels % d->groups != 0 || (d->softplus != 0 && d->softplus != 1) || d->states <= 0) return GDN_ERR_INVALID_ARG;
    const int64_t bc = (int64_t)d->groups * d->states;
    if (!a || !aligned(a, 16) || !aligned(skip, 4) || !aligned(dt_bias, 4)) return GDN_ERR_INVALID_ARG;
    const Rows rows_ok{step ? d->num_seqs : d->total_tokens, e};
    if (!rows_ok(x, d->x_stride, d->channels) || !rows_ok(dt, d->dt_stride, d->channels) || !rows_ok(out, d->out_stride, d->channels) ||
        !rows_ok(b, d->b_stride, bc) || !rows_ok(c, d->c_stride, bc) || (z && !rows_ok(z, d->z_stride, d->channels)))
        return GDN_ERR_INVALID_ARG;
    if (crosses(out, d->out_stride, x, d->x_stride, rows_ok.rows) || crosses(out, d->out_stride, dt, d->dt_stride, rows_ok.rows) ||
        crosses(out, d->out_stride, z, d->z_stride, rows_ok.rows))
        return GDN_ERR_INVALID_ARG;
    if (d->states != 8 && d->states != 16 && d->states != 32 && d->states != 64) return GDN_ERR_UNSUPPORTED;
    if (d->num_seqs == 0) return GDN_OK;
    gdn::ScanArgs s = {};
    s.x = x; s.dt = dt; s.b = b; s.c = c; s.z = z; s.a = a; s.d = skip; s.dt_bias = dt_bias; s.init_state = state_in; s.out = out;
    s.out_state = state_out; s.cu = cu; s.init_slots = d->init_slots; s.out_slots = d->out_slots; s.status_word = d->status_word;
    s.x_stride = d->x_stride; s.dt_stride = d->dt_stride; s.b_stride = d->b_stride; s.c_stride = d->c_stride; s.z_stride = d->z_stride;
    s.out_stride = d->out_stride; s.total_tokens = d->total_tokens; s.channels = d->channels; s.groups = d->groups; s.num_seqs = d->num_seqs;
    s.num_init = d->num_init_states; s.num_out = d->num_out_states; s.softplus = d->softplus;
    cudaStream_t stream = (cudaStream_t)d->stream;
    return done(step ? gdn::launch_scan_step(s, d->io_dtype, d->states, stream) : gdn::launch_scan(s, d->io_dtype, d->states, stream), 1);
}

// `pools`: the call moves pages; `count`: rows or pairs that it names; `tables`: it reads or writes the tables
int32_t check_cache(const gdn_cache_desc* d, bool pools, int64_t count, bool tables)
{
    gdn::set_launch_count(0);
    if (!d || d->num_pages <= 0 || count < 0 || count > 0x7fffffffLL || !aligned(d->status_word, 4)) return GDN_ERR_INVALID_ARG;
    if (pools) {
        if (d->num_pools < 0 || (d->num_pools > 0 && !d->pools)) return GDN_ERR_INVALID_ARG;
        for (int32_t i = 0; i < d->num_pools; ++i) {
            const gdn_pool& p = d->pools[i];
            if (!p.base || !aligned(p.base, 16) || p.page_bytes <= 0 || p.page_bytes % 16 != 0) return GDN_ERR_INVALID_ARG;
            if (p.page_bytes > (1LL << 32)) return GDN_ERR_UNSUPPORTED;
        }
    }
    if (tables) {
        if (d->num_rows <= 0 || d->row_pages <= 0) return GDN_ERR_INVALID_ARG;
        if ((int64_t)d->num_rows * d->row_pages > 0x7fffffffLL || count * d->row_pages > 0x7fffffffLL) return GDN_ERR_UNSUPPORTED;
    }
    return GDN_OK;
}

int32_t check_workspace(const gdn_cache_desc* d, int32_t count)
{
    if (!d->workspace || d->workspace_bytes < gdn_cache_workspace_size(d, count)) return GDN_ERR_WORKSPACE;
    return aligned(d->workspace, 256) ? GDN_OK : GDN_ERR_INVALID_ARG;
}

inline bool ints(const void* p) { return p && aligned(p, 4); }

}  // namespace

extern "C" {

int32_t gdn_short_conv(const gdn_conv_desc* desc, const void* x, const void* weight, const void* bias, const int32_t* cu_tail_lens,
                       const void* init_state, void* out, void* out_state)
{
    return conv(desc, x, weight, bias, cu_tail_lens, init_state, out, out_state, false);
}

int32_t gdn_short_conv_step(const gdn_conv_desc* desc, const void* x, const void* weight, const void* bias, const void* state_in, void* out,
                            void* state_out)
{
    return conv(desc, x, weight, bias, nullptr, state_in, out, state_out, true);
}

int32_t gdn_selective_scan(const gdn_scan_desc* desc, const void* x, const void* dt, const float* a, const void* b, const void* c, const float* d,
                           const void* z, const float* dt_bias, const int32_t* cu_tail_lens, const float* init_state, void* out, float* out_state)
{
    return scan(desc, x, dt, a, b, c, d, z, dt_bias, cu_tail_lens, init_state, out, out_state, false);
}

int32_t gdn_selective_scan_step(const gdn_scan_desc* desc, const void* x, const void* dt, const float* a, const void* b, const void* c,
                                const float* d, const void* z, const float* dt_bias, const float* state_in, void* out, float* state_out)
{
    return scan(desc, x, dt, a, b, c, d, z, dt_bias, nullptr, state_in, out, state_out, true);
}

size_t gdn_cache_workspace_size(const gdn_cache_desc* d, int32_t count)
{
    if (!d || d->num_pages <= 0 || count < 0) return 0;
    // five numbers per fork; three per page and the header of a compaction
    const size_t n = count > 0 ? 20 * (size_t)count : 256 + 12 * (size_t)d->num_pages;
    return (n + 255) & ~(size_t)255;
}

int32_t gdn_cache_copy(const gdn_cache_desc* d, const int32_t* src, const int32_t* dst, int32_t count)
{
    const int32_t rc = check_cache(d, true, count, false);
    if (rc != GDN_OK) return rc;
    if (count == 0 || d->num_pools == 0) return GDN_OK;
    if (!ints(src) || !ints(dst)) return GDN_ERR_INVALID_ARG;
    return done(gdn::launch_cache_copy(d, src, dst, count), gdn::pool_launches(d));
}

int32_t gdn_cache_fork(const gdn_cache_desc* d, int32_t* refcounts, int32_t* tables, const int32_t* parents, const int32_t* children,
                       const int32_t* tokens, int32_t count)
{
    int32_t rc = check_cache(d, true, count, true);
    if (rc != GDN_OK) return rc;
    if (d->page_tokens <= 0) return GDN_ERR_INVALID_ARG;
    if (d->num_pages > kMostPages || d->num_rows > GDN_CACHE_MAX_ROWS || count > GDN_CACHE_MAX_FORKS) return GDN_ERR_UNSUPPORTED;
    if (count == 0) return GDN_OK;
    if (!ints(refcounts) || !ints(tables) || !ints(parents) || !ints(children) || !ints(tokens)) return GDN_ERR_INVALID_ARG;
    if ((rc = check_workspace(d, count)) != GDN_OK) return rc;
    return done(gdn::launch_cache_fork(d, refcounts, tables, parents, children, tokens, count), gdn::fork_launches(d));
}

int32_t gdn_cache_free(const gdn_cache_desc* d, int32_t* refcounts, int32_t* tables, const int32_t* rows, int32_t count)
{
    const int32_t rc = check_cache(d, false, count, true);
    if (rc != GDN_OK) return rc;
    if (count == 0) return GDN_OK;
    if (!ints(refcounts) || !ints(tables) || !ints(rows)) return GDN_ERR_INVALID_ARG;
    return done(gdn::launch_cache_free(d, refcounts, tables, rows, count), 1);
}

int32_t gdn_cache_compact(const gdn_cache_desc* d, const int32_t* refcounts, const int32_t* tables, int32_t* out_refcounts, int32_t* out_tables,
                          int32_t* page_map, int32_t* live)
{
    int32_t rc = check_cache(d, true, 0, true);
    if (rc != GDN_OK) return rc;
    if (d->num_pages > kMostPages) return GDN_ERR_UNSUPPORTED;
    if (!ints(refcounts) || !ints(tables) || !ints(out_refcounts) || !ints(out_tables) || !ints(page_map) || !ints(live)) return GDN_ERR_INVALID_ARG;
    if ((rc = check_workspace(d, 0)) != GDN_OK) return rc;
    return done(gdn::launch_cache_compact(d, refcounts, tables, out_refcounts, out_tables, page_map, live), 1 + gdn::pool_launches(d));
}

}  // extern "C"
