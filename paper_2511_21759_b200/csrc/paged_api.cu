// C entries of the paged K/V cache: argument checks, the handle and its workspace.
#include <math.h>

#include <new>

#include "paged.cuh"

using namespace odb;

struct odb_paged {
    odb_paged_config cfg;
    int device, sms, page_shift;
    __nv_bfloat16* kv;
    int* status;
    unsigned int* arrivals;
    PagedShared* shared;
    float *part_o, *part_ml;
    int pool_rows, layer_rows;      // rows of head_dim values: of the whole pool, of the K or the V of a layer
    PagedMaps maps;
};

namespace {

constexpr size_t kStatusBytes = 256;
constexpr size_t kArrivalBytes = (kPagedMaxCtas * sizeof(unsigned int) + 255) / 256 * 256;
constexpr size_t kSharedBytes = (kPagedMaxCtas * sizeof(PagedShared) + 255) / 256 * 256;

int32_t check_config(const odb_paged_config* c) {
    if (!c) return ODB_ERR_ARG;
    if (c->n_layers < 1 || c->n_heads < 1 || c->n_kv_heads < 1 || c->n_pages < 1) return ODB_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128) return ODB_ERR_SHAPE;
    if (c->n_heads % c->n_kv_heads || c->n_heads > 1024) return ODB_ERR_SHAPE;
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return ODB_ERR_SHAPE;
    // slots and rows of the pool are 32-bit numbers
    const double slots = static_cast<double>(c->n_pages) * c->page_size, rows = slots * c->n_kv_heads * 2 * c->n_layers;
    if (slots >= 2147483648.0 || rows >= 2147483648.0 - 65536) return ODB_ERR_SHAPE;
    return ODB_OK;
}

int32_t check_call(const odb_paged* h, int32_t layer) {
    if (!h) return ODB_ERR_ARG;
    if (layer < 0 || layer >= h->cfg.n_layers) return ODB_ERR_ARG;
    int dev = -1;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    return dev == h->device ? ODB_OK : ODB_ERR_STATE;
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Rows of `width` elements of bf16, `stride` apart.
struct Rows {
    const void* at;
    int64_t stride, width;
};
// Whether n rows of each have a byte in common (rows of one tensor's slices lie between one another without that).  A row at `from` bytes
// behind b's first meets row k of b where from - (b's width) < k * (b's stride) < from + (a's width).
bool overlap(const Rows& a, const Rows& b, int32_t n) {
    typedef __int128 wide;                                  // strides are the caller's numbers
    const wide sa = 2 * static_cast<wide>(a.stride), sb = 2 * static_cast<wide>(b.stride), wa = 2 * a.width, wb = 2 * b.width, last = n - 1;
    const wide from = static_cast<wide>(reinterpret_cast<uintptr_t>(a.at)) - static_cast<wide>(reinterpret_cast<uintptr_t>(b.at));
    auto meets = [&](wide d, wide lo, wide hi) {            // some row k of b with lo <= k <= hi
        const wide x = d + wa - 1;
        wide k = x >= 0 ? x / sb : -((sb - 1 - x) / sb);    // the largest k with k * sb <= x
        if (k > hi) k = hi;
        return k >= lo && k * sb > d - wb;
    };
    if (from + last * sa + wa <= 0 || from >= last * sb + wb) return false;
    if (sa == sb) return meets(from, -last, last);
    for (int32_t i = 0; i < n; ++i)
        if (meets(from + i * sa, 0, last)) return true;
    return false;
}

int32_t enqueued(cudaError_t e) { return e == cudaSuccess ? ODB_OK : record_cuda_error(e); }

}  // namespace

extern "C" {

size_t odb_paged_kv_bytes(const odb_paged_config* c) {
    if (check_config(c) != ODB_OK) return 0;
    return static_cast<size_t>(c->n_layers) * 2 * c->n_pages * c->n_kv_heads * c->page_size * c->head_dim * 2;
}

size_t odb_paged_workspace_bytes(const odb_paged_config* c) {
    if (check_config(c) != ODB_OK) return 0;
    return kStatusBytes + kArrivalBytes + kSharedBytes + paged_part_bytes(c->head_dim);
}

int32_t odb_paged_create(const odb_paged_config* cfg, void* kv, size_t kv_bytes, void* workspace, size_t ws_bytes, void* stream,
                         odb_paged** out) {
    const int32_t rc = check_config(cfg);
    if (rc != ODB_OK) return rc;
    if (!kv || !workspace || !out || !aligned(kv, 256) || !aligned(workspace, 256)) return ODB_ERR_ARG;
    if (kv_bytes < odb_paged_kv_bytes(cfg) || ws_bytes < odb_paged_workspace_bytes(cfg)) return ODB_ERR_WORKSPACE;
    odb_paged* h = new (std::nothrow) odb_paged();
    if (!h) return ODB_ERR_ARG;
    h->cfg = *cfg;
    h->kv = static_cast<__nv_bfloat16*>(kv);
    for (h->page_shift = 0; (1 << h->page_shift) < cfg->page_size;) ++h->page_shift;
    h->layer_rows = cfg->n_pages * cfg->n_kv_heads * cfg->page_size;
    h->pool_rows = h->layer_rows * 2 * cfg->n_layers;
    char* ws = static_cast<char*>(workspace);
    h->status = reinterpret_cast<int*>(ws);
    h->arrivals = reinterpret_cast<unsigned int*>(ws + kStatusBytes);
    h->part_o = reinterpret_cast<float*>(ws + kStatusBytes + kArrivalBytes + kSharedBytes);
    h->shared = reinterpret_cast<PagedShared*>(ws + kStatusBytes + kArrivalBytes);
    h->part_ml = h->part_o + paged_part_bytes(cfg->head_dim) / sizeof(float) / (cfg->head_dim + 2) * cfg->head_dim;
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, h->device);
    if (e == cudaSuccess && h->sms > 148) h->sms = 148;         // what the workspace has parts for
    if (e == cudaSuccess) e = make_pool_tmap(&h->maps.rows, kv, h->pool_rows, cfg->head_dim, cfg->page_size < 64 ? cfg->page_size : 64, cfg->head_dim / 64);
    if (e == cudaSuccess) e = make_pool_tmap(&h->maps.atoms, kv, h->pool_rows, cfg->head_dim, cfg->page_size < 64 ? cfg->page_size : 64, 1);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (e == cudaSuccess) e = cudaMemsetAsync(ws, 0, kStatusBytes + kArrivalBytes, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) {
        delete h;
        return record_cuda_error(e);
    }
    *out = h;
    return ODB_OK;
}

int32_t odb_paged_destroy(odb_paged* h) {
    delete h;
    return ODB_OK;
}

int32_t odb_paged_status(odb_paged* h, void* stream) {
    if (!h) return ODB_ERR_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int word = 0;
    cudaError_t e = cudaMemcpyAsync(&word, h->status, sizeof(int), cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, sizeof(int), st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    return e == cudaSuccess ? word : record_cuda_error(e);
}

int32_t odb_paged_layout(odb_paged* h, const odb_paged_batch* b, void* stream) {
    const int32_t rc = check_call(h, 0);
    if (rc != ODB_OK) return rc;
    if (!b || b->n_seqs < 0 || b->max_rows < 0 || b->table_stride < 1) return ODB_ERR_ARG;
    if (b->n_seqs > kPagedMaxSeqs || (static_cast<long long>(b->table_stride) << h->page_shift) >= kPagedUnlimited) return ODB_ERR_SHAPE;
    if (!b->row_start || (b->n_seqs && (!b->len_before || !b->len_after || !b->first || !b->count || !b->table || !b->free_pages)) ||
        (b->max_rows && (!b->row_seq || !b->row_pos || !b->row_slot)))
        return ODB_ERR_ARG;
    PagedLayoutArgs a{b->len_before, b->len_after, b->first, b->count, b->table, b->free_pages, b->row_start, b->row_seq, b->row_pos,
                      b->row_slot, b->n_seqs, b->max_rows, h->page_shift, h->cfg.n_pages, b->table_stride, h->status};
    return enqueued(launch_paged_layout(a, static_cast<cudaStream_t>(stream)));
}

int32_t odb_rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double original_len, double beta_slow,
                             double beta_fast, uint64_t* turns_host, float* magnitude) {
    if (!turns_host || !magnitude) return ODB_ERR_ARG;
    if (rot_dim < 0 || rot_dim > 128 || rot_dim % 8) return ODB_ERR_SHAPE;
    if (!(theta >= 1.0) || !isfinite(theta)) return ODB_ERR_ARG;
    if (scaling < ODB_ROPE_PLAIN || scaling > ODB_ROPE_YARN) return ODB_ERR_ARG;
    if (scaling != ODB_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return ODB_ERR_ARG;
    if (scaling == ODB_ROPE_YARN && (!(original_len >= 1.0) || !isfinite(original_len) || !(beta_fast > beta_slow) || !(beta_slow >= 0.0) || !isfinite(beta_fast)))
        return ODB_ERR_ARG;
    const double pi = 3.14159265358979323846;
    if (scaling == ODB_ROPE_NTK && rot_dim > 2) theta *= pow(factor, static_cast<double>(rot_dim) / (rot_dim - 2));
    *magnitude = 1.0f;
    if (scaling == ODB_ROPE_YARN) *magnitude = static_cast<float>(0.1 * log(factor) + 1.0);
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(theta, -2.0 * i / rot_dim);             // radians per position
        if (scaling == ODB_ROPE_LINEAR) f /= factor;
        if (scaling == ODB_ROPE_YARN) {
            double keep = (original_len * f / (2 * pi) - beta_slow) / (beta_fast - beta_slow);
            keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
            f *= keep + (1 - keep) / factor;
        }
        turns_host[i] = static_cast<uint64_t>(llrint(f / (2 * pi) * 0x1p62)) << 2;   // below 1 / (2 pi): no overflow
    }
    return ODB_OK;
}

int32_t odb_paged_norm_rope_store(odb_paged* h, int32_t layer, const odb_paged_batch* b, const odb_paged_rows* r, const odb_rope* rope,
                                  float eps, void* stream) {
    const int32_t rc = check_call(h, layer);
    if (rc != ODB_OK) return rc;
    if (!b || !r || !rope || b->max_rows < 0) return ODB_ERR_ARG;
    const odb_paged_config& c = h->cfg;
    if (rope->rot_dim < 0 || rope->rot_dim > c.head_dim || rope->rot_dim % 8) return ODB_ERR_SHAPE;
    if (b->max_rows == 0) return ODB_OK;
    if (!r->q || !r->k || !r->v || !r->q_out || !b->row_pos || !b->row_slot || (rope->rot_dim && !rope->turns)) return ODB_ERR_ARG;
    if (!(eps >= 0.f) || !isfinite(eps) || !isfinite(rope->magnitude)) return ODB_ERR_ARG;
    const int64_t qw = static_cast<int64_t>(c.n_heads) * c.head_dim, kw = static_cast<int64_t>(c.n_kv_heads) * c.head_dim;
    if (r->q_stride < qw || r->out_stride < qw || r->k_stride < kw || r->v_stride < kw) return ODB_ERR_ARG;
    if (!aligned(r->q, 8) || !aligned(r->k, 8) || !aligned(r->v, 8) || !aligned(r->q_out, 8) || !aligned(r->q_gain, 16) || !aligned(r->k_gain, 16) ||
        !aligned(rope->turns, 16) || ((r->q_stride | r->k_stride | r->v_stride | r->out_stride) & 3))
        return ODB_ERR_ARG;
    // other blocks read their rows after the first have written
    const Rows out{r->q_out, r->out_stride, qw};
    if (((r->q_out != r->q || r->out_stride != r->q_stride) && overlap(out, {r->q, r->q_stride, qw}, b->max_rows)) ||
        overlap(out, {r->k, r->k_stride, kw}, b->max_rows) || overlap(out, {r->v, r->v_stride, kw}, b->max_rows))
        return ODB_ERR_ARG;
    if (static_cast<double>(b->max_rows) * (c.n_heads + 2 * c.n_kv_heads) >= 2147483648.0) return ODB_ERR_SHAPE;
    PagedStoreArgs a{};
    a.q = static_cast<const __nv_bfloat16*>(r->q);
    a.k = static_cast<const __nv_bfloat16*>(r->k);
    a.v = static_cast<const __nv_bfloat16*>(r->v);
    a.q_out = static_cast<__nv_bfloat16*>(r->q_out);
    a.q_stride = r->q_stride; a.k_stride = r->k_stride; a.v_stride = r->v_stride; a.out_stride = r->out_stride;
    a.q_gain = r->q_gain; a.k_gain = r->k_gain; a.eps = eps;
    a.turns = reinterpret_cast<const unsigned long long*>(rope->turns);
    a.magnitude = rope->magnitude;
    a.row_pos = b->row_pos; a.row_slot = b->row_slot;
    a.k_pool = h->kv + static_cast<size_t>(2 * layer) * h->layer_rows * c.head_dim;
    a.v_pool = a.k_pool + static_cast<size_t>(h->layer_rows) * c.head_dim;
    a.rows = b->max_rows; a.H = c.n_heads; a.KV = c.n_kv_heads; a.HD = c.head_dim;
    a.rot = rope->rot_dim; a.interleaved = rope->interleaved != 0; a.page_shift = h->page_shift; a.n_pages = c.n_pages;
    return enqueued(launch_paged_store(a, static_cast<cudaStream_t>(stream)));
}

int32_t odb_paged_attention(odb_paged* h, int32_t layer, const odb_paged_batch* b, const void* q, int64_t q_stride, void* out,
                            int64_t out_stride, float* lse, float scale, int32_t left, int32_t right, int32_t sinks, void* stream) {
    const int32_t rc = check_call(h, layer);
    if (rc != ODB_OK) return rc;
    if (!b || b->n_seqs < 0 || b->max_rows < 0 || b->max_new < 0 || b->table_stride < 1) return ODB_ERR_ARG;
    if (left < -1 || right < -1 || sinks < 0 || !isfinite(scale)) return ODB_ERR_ARG;
    const odb_paged_config& c = h->cfg;
    const long long longest = static_cast<long long>(b->table_stride) << h->page_shift;
    if (b->n_seqs > kPagedMaxSeqs || longest >= kPagedUnlimited) return ODB_ERR_SHAPE;
    if (b->n_seqs == 0 || b->max_rows == 0) return ODB_OK;
    if (!q || !out || !b->len_after || !b->first || !b->row_start || !b->table) return ODB_ERR_ARG;
    const int64_t qw = static_cast<int64_t>(c.n_heads) * c.head_dim;
    if (q_stride < qw || out_stride < qw || ((q_stride | out_stride) & 7) || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4)) return ODB_ERR_ARG;
    if (overlap({out, out_stride, qw}, {q, q_stride, qw}, b->max_rows)) return ODB_ERR_ARG;   // some CTAs read Q after others have written
    const int G = c.n_heads / c.n_kv_heads;
    if (static_cast<double>(b->max_rows) * c.n_heads >= 2147483648.0 - 65536) return ODB_ERR_SHAPE;   // packed rows are 32-bit numbers
    const int q_tiles = paged_attention_kernel_of(b->n_seqs, b->max_rows, b->max_new, G, c.n_kv_heads, longest, out_stride);
    if (q_tiles < 0) return ODB_ERR_SHAPE;
    PagedAttnArgs a{};
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.out = static_cast<__nv_bfloat16*>(out);
    a.lse = lse;
    a.q_stride = q_stride; a.out_stride = out_stride;
    a.table = b->table; a.len = b->len_after; a.first = b->first; a.row_start = b->row_start;
    a.n_seqs = b->n_seqs; a.max_rows = b->max_rows; a.H = c.n_heads; a.KV = c.n_kv_heads; a.G = G;
    a.page_shift = h->page_shift; a.n_pages = c.n_pages; a.table_stride = b->table_stride;
    a.pool = reinterpret_cast<const unsigned short*>(h->kv);
    a.k_row0 = 2 * layer * h->layer_rows; a.v_row0 = a.k_row0 + h->layer_rows; a.pool_rows = h->pool_rows;
    a.left = left < 0 || left > kPagedUnlimited ? kPagedUnlimited : left;
    a.right = right < 0 || right > kPagedUnlimited ? kPagedUnlimited : right;
    a.sinks = sinks > kPagedUnlimited ? kPagedUnlimited : sinks;
    a.scale_log2 = (scale != 0.f ? scale : 1.0f / sqrtf(static_cast<float>(c.head_dim))) * 1.4426950408889634f;
    a.status = h->status; a.arrivals = h->arrivals; a.part_o = h->part_o; a.part_ml = h->part_ml;
    a.shared = h->shared;
    return enqueued(launch_paged_attention(a, h->maps, c.head_dim, q_tiles, h->sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
