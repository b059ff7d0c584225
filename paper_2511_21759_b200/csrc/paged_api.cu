// C entries of the paged K/V cache: argument checks, the handle and its workspace.
#include <math.h>

#include <new>

#include "paged.cuh"

using namespace odb;

struct odb_paged {
    odb_paged_config cfg;
    int device, sms, page_shift;
    void* kv;
    float* scales;                  // null: the pool is bf16
    int* status;
    unsigned int* arrivals;
    PagedShared* shared;
    float *part_o, *part_ml;
    int pool_rows, layer_rows;      // rows of head_dim values: of the whole pool, of the K or the V of a layer
    PagedMaps maps;                 // pools of 8 bits: rows alone
    __nv_bfloat16* layer;           // pools of 8 bits: room for a layer's K and V in bf16, null: there is none
    PagedMaps layer_maps;
    int value_bytes() const { return scales ? 1 : 2; }
    // the layer's K, and V behind it
    char* k_of(int layer) const { return static_cast<char*>(kv) + static_cast<size_t>(2 * layer) * layer_rows * cfg.head_dim * value_bytes(); }
    char* v_of(int layer) const { return k_of(layer) + static_cast<size_t>(layer_rows) * cfg.head_dim * value_bytes(); }
    float* k_scales_of(int layer) const { return scales ? scales + static_cast<size_t>(2 * layer) * (layer_rows / kPagedBlock) : nullptr; }
    float* v_scales_of(int layer) const { return scales ? k_scales_of(layer) + layer_rows / kPagedBlock : nullptr; }
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

size_t pool_values(const odb_paged_config* c) {
    return static_cast<size_t>(c->n_layers) * 2 * c->n_pages * c->n_kv_heads * c->page_size * c->head_dim;
}

// a handle over a pool of bf16, or of codes with scales
int32_t create(const odb_paged_config* cfg, void* kv, size_t kv_bytes, float* scales, void* workspace, size_t ws_bytes, cudaStream_t st, odb_paged** out) {
    if (!kv || !workspace || !out || !aligned(kv, 256) || !aligned(workspace, 256)) return ODB_ERR_ARG;
    if (kv_bytes < pool_values(cfg) * (scales ? 1 : 2) || ws_bytes < odb_paged_workspace_bytes(cfg)) return ODB_ERR_WORKSPACE;
    odb_paged* h = new (std::nothrow) odb_paged();
    if (!h) return ODB_ERR_ARG;
    h->cfg = *cfg;
    h->kv = kv;
    h->scales = scales;
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
    const int box_rows = cfg->page_size < 64 ? cfg->page_size : 64;
    if (scales) {
        if (e == cudaSuccess) e = make_pool_e4m3_tmap(&h->maps.rows, kv, h->pool_rows, cfg->head_dim, box_rows);
        if (ws_bytes >= odb_paged_workspace_bytes(cfg) + odb_paged_e4m3_layer_bytes(cfg)) {
            h->layer = reinterpret_cast<__nv_bfloat16*>(ws + odb_paged_workspace_bytes(cfg));
            if (e == cudaSuccess) e = make_pool_tmap(&h->layer_maps.rows, h->layer, 2ull * h->layer_rows, cfg->head_dim, box_rows, cfg->head_dim / 64);
            if (e == cudaSuccess) e = make_pool_tmap(&h->layer_maps.atoms, h->layer, 2ull * h->layer_rows, cfg->head_dim, box_rows, 1);
        }
    } else {
        if (e == cudaSuccess) e = make_pool_tmap(&h->maps.rows, kv, h->pool_rows, cfg->head_dim, box_rows, cfg->head_dim / 64);
        if (e == cudaSuccess) e = make_pool_tmap(&h->maps.atoms, kv, h->pool_rows, cfg->head_dim, box_rows, 1);
    }
    if (e == cudaSuccess) e = cudaMemsetAsync(ws, 0, kStatusBytes + kArrivalBytes, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) {
        delete h;
        return record_cuda_error(e);
    }
    *out = h;
    return ODB_OK;
}

int32_t enqueued(cudaError_t e) { return e == cudaSuccess ? ODB_OK : record_cuda_error(e); }

}  // namespace

extern "C" {

size_t odb_paged_kv_bytes(const odb_paged_config* c) {
    if (check_config(c) != ODB_OK) return 0;
    return pool_values(c) * 2;
}

size_t odb_paged_workspace_bytes(const odb_paged_config* c) {
    if (check_config(c) != ODB_OK) return 0;
    return kStatusBytes + kArrivalBytes + kSharedBytes + paged_part_bytes(c->head_dim);
}

int32_t odb_paged_create(const odb_paged_config* cfg, void* kv, size_t kv_bytes, void* workspace, size_t ws_bytes, void* stream,
                         odb_paged** out) {
    const int32_t rc = check_config(cfg);
    return rc != ODB_OK ? rc : create(cfg, kv, kv_bytes, nullptr, workspace, ws_bytes, static_cast<cudaStream_t>(stream), out);
}

size_t odb_paged_e4m3_kv_bytes(const odb_paged_config* c) { return check_config(c) != ODB_OK ? 0 : pool_values(c); }

size_t odb_paged_e4m3_scale_bytes(const odb_paged_config* c) {
    return check_config(c) != ODB_OK ? 0 : pool_values(c) / c->head_dim / kPagedBlock * sizeof(float);
}

size_t odb_paged_e4m3_layer_bytes(const odb_paged_config* c) {
    return check_config(c) != ODB_OK ? 0 : pool_values(c) / c->n_layers * sizeof(__nv_bfloat16);
}

int32_t odb_paged_create_e4m3(const odb_paged_config* cfg, void* kv, size_t kv_bytes, void* scales, size_t scale_bytes, void* workspace,
                              size_t ws_bytes, void* stream, odb_paged** out) {
    const int32_t rc = check_config(cfg);
    if (rc != ODB_OK) return rc;
    if (!scales || !aligned(scales, 256)) return ODB_ERR_ARG;
    if (scale_bytes < odb_paged_e4m3_scale_bytes(cfg)) return ODB_ERR_WORKSPACE;
    return create(cfg, kv, kv_bytes, static_cast<float*>(scales), workspace, ws_bytes, static_cast<cudaStream_t>(stream), out);
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
                      b->row_slot, b->n_seqs, b->max_rows, h->page_shift, h->cfg.n_pages, b->table_stride, h->status,
                      h->scales, 2 * h->cfg.n_layers, h->cfg.n_kv_heads * (h->cfg.page_size / kPagedBlock)};
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
    if (h->scales && (!b->row_seq || !b->len_after || b->n_seqs < 1)) return ODB_ERR_ARG;
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
    a.rows = b->max_rows; a.H = c.n_heads; a.KV = c.n_kv_heads; a.HD = c.head_dim;
    a.rot = rope->rot_dim; a.interleaved = rope->interleaved != 0; a.page_shift = h->page_shift; a.n_pages = c.n_pages;
    if (h->scales) {
        PagedE4m3StoreArgs p{};
        p.rows = a;
        p.rows.KV = 0;
        p.row_seq = b->row_seq; p.len = b->len_after;
        p.k_pool = reinterpret_cast<unsigned char*>(h->k_of(layer)); p.v_pool = reinterpret_cast<unsigned char*>(h->v_of(layer));
        p.k_scales = h->k_scales_of(layer); p.v_scales = h->v_scales_of(layer);
        p.KV = c.n_kv_heads; p.n_seqs = b->n_seqs;
        // Maps of 16 rows at once where requests have eight and more on average (256 requests of 8 rows, 32 + 8 heads: 10.0 us, 12.8 with a row
        // at a time; of 32 rows 5.7 and 11.8; 48 requests of 4 rows 6.4 and 6.3, of one 17.7 and 4.2: the blocks of a window follow one another).
        p.window = b->max_rows / b->n_seqs >= kPagedBlock / 2 ? kPagedBlock : 1;
        const int windows = (b->max_rows + p.window - 1) / p.window;
        // Heads of a unit: as many, up to 8, as leave a wave of some 1000 (256 tokens: 11.3 us with one, 7.2 with four, 9.1 with eight; 16384 rows
        // of prompts 84 with one, 62 with eight; 48 tokens 4.1 with one, 6.4 with eight).
        p.heads = 1;
        while (p.heads < 8 && p.heads < c.n_kv_heads && static_cast<long long>(windows) * 2 * c.n_kv_heads / (2 * p.heads) >= 1000) p.heads *= 2;
        return enqueued(launch_paged_e4m3_store(p, static_cast<cudaStream_t>(stream)));
    }
    a.k_pool = reinterpret_cast<__nv_bfloat16*>(h->k_of(layer)); a.v_pool = reinterpret_cast<__nv_bfloat16*>(h->v_of(layer));
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
    const int kernel = h->scales ? paged_e4m3_attention_kernel_of(b->n_seqs, b->max_rows, b->max_new, G, c.n_kv_heads, longest, out_stride, h->layer != nullptr)
                                 : paged_attention_kernel_of(b->n_seqs, b->max_rows, b->max_new, G, c.n_kv_heads, longest, out_stride);
    if (kernel < 0) return ODB_ERR_SHAPE;
    PagedAttnArgs a{};
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.out = static_cast<__nv_bfloat16*>(out);
    a.lse = lse;
    a.q_stride = q_stride; a.out_stride = out_stride;
    a.table = b->table; a.len = b->len_after; a.first = b->first; a.row_start = b->row_start;
    a.n_seqs = b->n_seqs; a.max_rows = b->max_rows; a.H = c.n_heads; a.KV = c.n_kv_heads; a.G = G;
    a.page_shift = h->page_shift; a.n_pages = c.n_pages; a.table_stride = b->table_stride;
    a.pool = static_cast<const unsigned short*>(h->kv);
    a.scales = h->scales;
    a.k_row0 = 2 * layer * h->layer_rows; a.v_row0 = a.k_row0 + h->layer_rows; a.pool_rows = h->pool_rows;
    a.left = left < 0 || left > kPagedUnlimited ? kPagedUnlimited : left;
    a.right = right < 0 || right > kPagedUnlimited ? kPagedUnlimited : right;
    a.sinks = sinks > kPagedUnlimited ? kPagedUnlimited : sinks;
    a.scale_log2 = (scale != 0.f ? scale : 1.0f / sqrtf(static_cast<float>(c.head_dim))) * 1.4426950408889634f;
    a.status = h->status; a.arrivals = h->arrivals; a.part_o = h->part_o; a.part_ml = h->part_ml;
    a.shared = h->shared;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!h->scales) return enqueued(launch_paged_attention(a, h->maps, c.head_dim, kernel, h->sms, st));
    if (kernel != 2) return enqueued(launch_paged_e4m3_attention(a, h->maps.rows, c.head_dim, kernel, h->sms, st));
    a.by_rows = PagedDiv::by(1);                            // of no use to the copy, but read
    a.by_group = a.by_rows;
    const cudaError_t e = launch_paged_expand(a, h->layer, h->layer_rows, c.head_dim, st);
    if (e != cudaSuccess) return record_cuda_error(e);
    a.pool = reinterpret_cast<const unsigned short*>(h->layer);
    a.scales = nullptr;
    a.k_row0 = 0; a.v_row0 = h->layer_rows; a.pool_rows = 2 * h->layer_rows;
    return enqueued(launch_paged_attention(a, h->layer_maps, c.head_dim, kernel, h->sms, st));
}

int32_t odb_paged_load(odb_paged* h, int32_t layer, const odb_paged_batch* b, void* k, int64_t k_stride, void* v, int64_t v_stride, void* stream) {
    const int32_t rc = check_call(h, layer);
    if (rc != ODB_OK) return rc;
    if (!b || b->max_rows < 0) return ODB_ERR_ARG;
    if (b->max_rows == 0) return ODB_OK;
    const odb_paged_config& c = h->cfg;
    const int64_t width = static_cast<int64_t>(c.n_kv_heads) * c.head_dim;
    if (!k || !v || !b->row_slot || k_stride < width || v_stride < width || ((k_stride | v_stride) & 7) || !aligned(k, 16) || !aligned(v, 16)) return ODB_ERR_ARG;
    if (overlap({k, k_stride, width}, {v, v_stride, width}, b->max_rows)) return ODB_ERR_ARG;
    if (static_cast<double>(b->max_rows) * c.n_kv_heads >= 1073741824.0) return ODB_ERR_SHAPE;   // blocks' rows are 32-bit numbers
    PagedLoadArgs a{};
    a.k_pool = reinterpret_cast<const unsigned char*>(h->k_of(layer)); a.v_pool = reinterpret_cast<const unsigned char*>(h->v_of(layer));
    a.k_scales = h->k_scales_of(layer); a.v_scales = h->v_scales_of(layer);
    a.row_slot = b->row_slot;
    a.k_out = static_cast<__nv_bfloat16*>(k); a.v_out = static_cast<__nv_bfloat16*>(v);
    a.k_stride = k_stride; a.v_stride = v_stride;
    a.rows = b->max_rows; a.KV = c.n_kv_heads; a.HD = c.head_dim; a.page_shift = h->page_shift; a.n_pages = c.n_pages;
    return enqueued(launch_paged_load(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
