// C-ABI layer of the token operators (include/cbconv.h): arguments are checked here, once and on the host, so that the kernels'
// indexing holds whatever the device arrays contain.
#include <atomic>
#include <cmath>

#include "cb_kernels.h"
#include "cb_tokens.h"

namespace cb {

int device_units()
{
    static std::atomic<int> units[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    int n = units[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) n = 256;
        units[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

namespace {
size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
}

ScratchPlan scratch_plan(const Cache& c, int q_heads)
{
    const size_t pairs = (size_t)c.seqs * c.heads;
    const int dp = c.dim <= 64 ? 64 : (c.dim <= 128 ? 128 : 256);
    ScratchPlan p;
    p.parts = p.moves = p.pages = align256(COUNTER_BYTES);
    p.sums = p.parts + (q_heads ? align256((size_t)2 * MAX_GROUPS * ATTEND_ROWS * (dp + 2) * 4) : 0);
    p.scores = p.sums + (c.weight ? align256((size_t)c.seqs * q_heads * 8) : 0);
    const size_t attend = p.scores + (c.weight ? align256((size_t)c.seqs * q_heads * c.capacity * 4) : 0);
    const size_t evict = p.moves + (c.weight ? align256(pairs * (1 + 2 * (size_t)c.capacity) * 4) : 0);
    const size_t choose = p.pages + (c.bounds ? align256(pairs * (size_t)rank_pitch(c) * 4) : 0);
    p.total = attend > evict ? attend : evict;
    p.total = p.total > choose ? p.total : choose;
    return p;
}

namespace {

// The cache as the launchers take it; scratch: whether the call needs one with room for q_heads query heads.
int check_cache(const cb_cache* d, bool scratch, int q_heads, Cache* c)
{
    if (!d || d->reserved != 0) return CB_EINVAL;
    if (d->n_seq < 1 || d->n_seq > 65535 || d->n_kv_heads < 1 || d->n_kv_heads > 1024) return CB_EINVAL;
    if (d->head_dim < 8 || d->head_dim > 256 || d->head_dim % 8) return CB_EINVAL;
    if (d->page_tokens < 16 || d->page_tokens > 1024 || (d->page_tokens & (d->page_tokens - 1))) return CB_EINVAL;
    if (d->max_pages < 1 || d->n_pages < 1 || (long)d->max_pages * d->page_tokens > (1L << 30)) return CB_EINVAL;
    const bool bytes = d->dtype == CB_E4M3;
    if (d->dtype != CB_F32 && d->dtype != CB_BF16 && !bytes) return CB_EINVAL;
    if (bytes && (d->head_dim % 16 || (d->values_dtype != CB_F32 && d->values_dtype != CB_BF16))) return CB_EINVAL;
    if (d->reserved2 != 0) return CB_EINVAL;
    c->seqs = d->n_seq; c->heads = d->n_kv_heads; c->dim = d->head_dim;
    c->page_shift = __builtin_ctz((unsigned)d->page_tokens);
    c->max_pages = d->max_pages; c->n_pages = d->n_pages;
    c->capacity = d->max_pages * d->page_tokens;
    c->e4m3 = bytes;
    c->bf16 = (bytes ? d->values_dtype : d->dtype) == CB_BF16;
    c->k_scale = bytes ? d->k_scale_dev : nullptr; c->v_scale = bytes ? d->v_scale_dev : nullptr;
    c->bounds = d->bounds_dev;
    c->k = d->k_pages_dev; c->v = d->v_pages_dev;
    c->table = d->table_dev; c->lengths = d->lengths_dev;
    c->weight = d->weight_dev; c->time = d->time_dev;
    c->scratch = static_cast<char*>(d->scratch_dev);
    if (!scratch) return CB_OK;
    if (!c->k || !c->v || ((uintptr_t)c->k & 15) || ((uintptr_t)c->v & 15) || !c->table || !c->lengths) return CB_EINVAL;
    if (((uintptr_t)c->weight & 15) || ((uintptr_t)c->time & 15) || ((uintptr_t)c->bounds & 15)) return CB_EINVAL;
    if (bytes && (!c->k_scale || !c->v_scale || ((uintptr_t)c->k_scale & 3) || ((uintptr_t)c->v_scale & 3))) return CB_EINVAL;
    if (!c->scratch || ((uintptr_t)c->scratch & 255)) return CB_EINVAL;
    if (d->scratch_bytes < scratch_plan(*c, q_heads).total) return CB_ENOMEM;
    return CB_OK;
}

int check_rotary(const cb_rotary_desc& d)
{
    if (d.head_dim < 8 || d.head_dim > 256 || d.head_dim % 8 || d.n_axes < 1 || d.n_axes > CB_ROTARY_MAX_AXES || d.reserved != 0) return CB_EINVAL;
    if (d.layout != CB_PAIRS_HALVES && d.layout != CB_PAIRS_ADJACENT) return CB_EINVAL;
    if (d.ladder != CB_LADDER_SHARED && d.ladder != CB_LADDER_PER_AXIS) return CB_EINVAL;
    if (!(d.base > 0.0f) || std::isinf(d.base)) return CB_EINVAL;
    int n = 0;
    for (int a = 0; a < CB_ROTARY_MAX_AXES; ++a) {
        if (d.pairs[a] < 0 || d.pairs[a] > d.head_dim / 2 || (a >= d.n_axes && d.pairs[a] != 0)) return CB_EINVAL;
        n += d.pairs[a];
    }
    return n >= 1 && n <= d.head_dim / 2 ? CB_OK : CB_EINVAL;
}

// The type of what comes and goes.
int values_dtype(const cb_cache& d) { return d.dtype == CB_E4M3 ? d.values_dtype : d.dtype; }

int check_heads(const cb_heads* h, int dtype, Heads* to, bool empty)
{
    if (!h || h->reserved != 0 || h->heads < 1 || h->heads > 65536) return CB_EINVAL;
    if (!empty && (!h->data_dev || (uintptr_t)h->data_dev % (dtype == CB_BF16 ? 2 : 4))) return CB_EINVAL;
    to->data = h->data_dev; to->token = (long)h->token_stride; to->head = (long)h->head_stride; to->heads = h->heads;
    return CB_OK;
}

// What attention checks whichever slots it reads.
int check_attend(const cb_cache* cache, const cb_attend_params* params, const cb_heads* q, const cb_heads* out, Cache* c, AttendJob* j)
{
    if (!params || !q || !out || params->reserved != 0) return CB_EINVAL;
    if (!std::isfinite(params->scale) || !std::isfinite(params->softcap) || params->softcap < 0.0f) return CB_EINVAL;
    if (!(params->decay >= 0.0f && params->decay <= 1.0f) || (params->accumulate != 0 && params->accumulate != 1)) return CB_EINVAL;
    int rc = check_cache(cache, false, 0, c);
    if (rc == CB_OK) rc = check_heads(q, values_dtype(*cache), &j->q, false);
    if (rc == CB_OK) rc = check_heads(out, values_dtype(*cache), &j->out, false);
    if (rc != CB_OK) return rc;
    if (q->heads != out->heads || q->heads % c->heads) return CB_EINVAL;
    j->scale = params->scale; j->softcap = params->softcap; j->decay = params->decay;
    j->accumulate = params->accumulate;
    return CB_OK;
}

// Tokens whose heads are normed and turned; w: the weights' type.
int check_norm(const cb_rotary* rotary, int dtype, int64_t n_tokens, const int32_t* positions, float eps, int w, NormJob* n)
{
    if (!rotary) return CB_EINVAL;
    const int rc = check_rotary(rotary->desc);
    if (rc != CB_OK) return rc;
    if ((dtype != CB_F32 && dtype != CB_BF16) || (w != CB_F32 && w != CB_BF16) || n_tokens < 0 || n_tokens >= (1LL << 31)) return CB_EINVAL;
    if (!(eps >= 0.0f) || std::isinf(eps) || (!positions && n_tokens)) return CB_EINVAL;
    n->eps = eps;
    n->weight_bf16 = w == CB_BF16;
    return CB_OK;
}

bool aligned_to(const void* p, int dtype) { return (uintptr_t)p % (dtype == CB_BF16 ? 2 : 4) == 0; }

void set_rotary(const cb_rotary* r, RotaryJob* j)
{
    j->axes = r->desc.n_axes;
    j->pos_axes = r->desc.n_axes;
    j->adjacent = r->desc.layout == CB_PAIRS_ADJACENT;
    j->dim = r->desc.head_dim;
    int n = 0;
    for (int a = 0; a < CB_ROTARY_MAX_AXES; ++a) j->end[a] = n += r->desc.pairs[a];
    j->pairs = n;
    for (int i = 0; i < n; ++i) j->turns[i] = r->turns[i];
}

}  // namespace

}  // namespace cb

#define CB_CHECKED(expr) do { const int rc_ = (expr); if (rc_ != CB_OK) return rc_; } while (0)
#define CB_LAUNCHED(expr) do { const hipError_t e_ = (expr); if (e_ != hipSuccess) return cb::note_hip_error(e_); } while (0)

extern "C" {

int cb_rotary_init(const cb_rotary_desc* desc, cb_rotary* rotary)
{
    if (!desc || !rotary) return CB_EINVAL;
    CB_CHECKED(cb::check_rotary(*desc));
    const cb_rotary_desc d = *desc;
    int n = 0, at = 0;
    for (int a = 0; a < d.n_axes; ++a) n += d.pairs[a];
    for (int i = 0; i < CB_ROTARY_MAX_PAIRS; ++i) rotary->turns[i] = 0.0;
    for (int a = 0; a < d.n_axes; ++a)
        for (int i = 0; i < d.pairs[a]; ++i, ++at) {
            const double step = d.ladder == CB_LADDER_SHARED ? (double)at / n : (double)i / d.pairs[a];
            rotary->turns[at] = std::pow((double)d.base, -step) / 6.283185307179586476925286766559;
        }
    rotary->desc = d;
    return CB_OK;
}

int cb_rotate(const cb_rotary* rotary, int32_t dtype, int64_t n_tokens, const int32_t* positions_dev, const cb_heads* q,
              const cb_heads* q_out, const cb_heads* k, const cb_heads* k_out, int32_t inverse, void* hip_stream)
{
    if (!rotary || !q || !q_out || (k == nullptr) != (k_out == nullptr)) return CB_EINVAL;
    CB_CHECKED(cb::check_rotary(rotary->desc));
    if ((dtype != CB_F32 && dtype != CB_BF16) || n_tokens < 0 || n_tokens >= (1LL << 31) || (inverse != 0 && inverse != 1)) return CB_EINVAL;
    const bool empty = n_tokens == 0;
    if (!positions_dev && !empty) return CB_EINVAL;
    cb::RotaryJob j = {};
    cb::set_rotary(rotary, &j);
    j.bf16 = dtype == CB_BF16;
    j.inverse = inverse;
    j.tokens = (long)n_tokens;
    j.positions = positions_dev;
    CB_CHECKED(cb::check_heads(q, dtype, &j.q, empty));
    CB_CHECKED(cb::check_heads(q_out, dtype, &j.q_out, empty));
    if (q->heads != q_out->heads) return CB_EINVAL;
    if (k) {
        CB_CHECKED(cb::check_heads(k, dtype, &j.k, empty));
        CB_CHECKED(cb::check_heads(k_out, dtype, &j.k_out, empty));
        if (k->heads != k_out->heads) return CB_EINVAL;
    }
    CB_LAUNCHED(cb::launch_rotate(j, (hipStream_t)hip_stream));
    return CB_OK;
}

int cb_norm_rotate(const cb_rotary* rotary, int32_t dtype, int64_t n_tokens, const int32_t* positions_dev, float eps, int32_t weight_dtype,
                   const cb_heads* q, const void* q_weight_dev, const cb_heads* q_out, const cb_heads* k, const void* k_weight_dev,
                   const cb_heads* k_out, void* hip_stream)
{
    cb::NormJob n = {};
    CB_CHECKED(cb::check_norm(rotary, dtype, n_tokens, positions_dev, eps, weight_dtype, &n));
    if (!q || !q_out || (k == nullptr) != (k_out == nullptr) || (k == nullptr) != (k_weight_dev == nullptr)) return CB_EINVAL;
    if (!q_weight_dev || !cb::aligned_to(q_weight_dev, weight_dtype) || !cb::aligned_to(k_weight_dev, weight_dtype)) return CB_EINVAL;
    const bool empty = n_tokens == 0;
    cb::RotaryJob& j = n.r;
    cb::set_rotary(rotary, &j);
    j.bf16 = dtype == CB_BF16;
    j.tokens = (long)n_tokens;
    j.positions = positions_dev;
    n.q_weight = q_weight_dev;
    n.k_weight = k_weight_dev;
    CB_CHECKED(cb::check_heads(q, dtype, &j.q, empty));
    CB_CHECKED(cb::check_heads(q_out, dtype, &j.q_out, empty));
    if (q->heads != q_out->heads) return CB_EINVAL;
    if (k) {
        CB_CHECKED(cb::check_heads(k, dtype, &j.k, empty));
        CB_CHECKED(cb::check_heads(k_out, dtype, &j.k_out, empty));
        if (k->heads != k_out->heads) return CB_EINVAL;
    }
    CB_LAUNCHED(cb::launch_norm_rotate(n, (hipStream_t)hip_stream));
    return CB_OK;
}

int cb_norm_rotate_back_scratch_bytes(const cb_rotary* rotary, size_t* bytes)
{
    if (!rotary || !bytes) return CB_EINVAL;
    CB_CHECKED(cb::check_rotary(rotary->desc));
    *bytes = (size_t)cb::NORM_GROUPS * 2 * rotary->desc.head_dim * sizeof(float);
    return CB_OK;
}

int cb_norm_rotate_back(const cb_rotary* rotary, int32_t dtype, int64_t n_tokens, const int32_t* positions_dev, float eps, int32_t weight_dtype,
                        const cb_norm_back* q, const cb_norm_back* k, void* scratch_dev, size_t scratch_bytes, void* hip_stream)
{
    cb::NormJob n = {};
    CB_CHECKED(cb::check_norm(rotary, dtype, n_tokens, positions_dev, eps, weight_dtype, &n));
    if (!q && !k) return CB_EINVAL;
    const bool empty = n_tokens == 0;
    cb::RotaryJob& j = n.r;
    cb::set_rotary(rotary, &j);
    j.bf16 = dtype == CB_BF16;
    j.inverse = 1;
    j.tokens = (long)n_tokens;
    j.positions = positions_dev;
    for (int i = 0; i < 2; ++i) {
        const bool is_q = i == 0;
        const cb_norm_back* b = is_q ? q : k;
        if (!b) continue;
        cb::Heads &x = is_q ? j.q : j.k, &to = is_q ? j.q_out : j.k_out, &grad = is_q ? n.q_grad : n.k_grad;
        CB_CHECKED(cb::check_heads(&b->x, dtype, &x, empty));
        CB_CHECKED(cb::check_heads(&b->out_grad, dtype, &grad, empty));
        if (b->x_grad.data_dev) {
            CB_CHECKED(cb::check_heads(&b->x_grad, dtype, &to, empty));
            if (b->x_grad.heads != b->x.heads) return CB_EINVAL;
        }
        if (b->out_grad.heads != b->x.heads) return CB_EINVAL;
        if (!b->weight_dev || !cb::aligned_to(b->weight_dev, weight_dtype) || !cb::aligned_to(b->weight_grad_dev, weight_dtype)) return CB_EINVAL;
        (is_q ? n.q_weight : n.k_weight) = b->weight_dev;
        (is_q ? n.q_weight_grad : n.k_weight_grad) = b->weight_grad_dev;
    }
    if (n.q_weight_grad || n.k_weight_grad) {
        size_t need = 0;
        CB_CHECKED(cb_norm_rotate_back_scratch_bytes(rotary, &need));
        if (!scratch_dev || ((uintptr_t)scratch_dev & 15)) return CB_EINVAL;
        if (scratch_bytes < need) return CB_ENOMEM;
        n.sums = static_cast<float*>(scratch_dev);
    }
    CB_LAUNCHED(cb::launch_norm_rotate_back(n, (hipStream_t)hip_stream));
    return CB_OK;
}

int cb_cache_scratch_bytes(const cb_cache* cache, int32_t n_q_heads, size_t* bytes)
{
    cb::Cache c = {};
    if (!bytes) return CB_EINVAL;
    CB_CHECKED(cb::check_cache(cache, false, 0, &c));
    if (n_q_heads < 0 || n_q_heads > 65536 || n_q_heads % c.heads) return CB_EINVAL;
    *bytes = cb::scratch_plan(c, n_q_heads).total;
    return CB_OK;
}

int cb_cache_append(const cb_cache* cache, const cb_rotary* rotary, int32_t n_tokens, const int32_t* positions_dev,
                    const int32_t* offsets_dev, const int32_t* start_dev, const cb_heads* k, const cb_heads* v,
                    const cb_heads* q, const cb_heads* q_out, void* hip_stream)
{
    cb::Cache c = {};
    CB_CHECKED(cb::check_cache(cache, true, 0, &c));
    const int dtype = cb::values_dtype(*cache);
    if (n_tokens < 0 || n_tokens > cb::MOST_TOKENS || (!offsets_dev && n_tokens != c.seqs)) return CB_EINVAL;
    const bool empty = n_tokens == 0;
    if (q && (!rotary || !q_out)) return CB_EINVAL;
    if (!q && q_out) return CB_EINVAL;
    cb::RotaryJob j = {};
    j.dim = c.dim;
    j.pos_axes = 1;
    if (rotary) {
        CB_CHECKED(cb::check_rotary(rotary->desc));
        if (rotary->desc.head_dim != c.dim || (!positions_dev && !empty)) return CB_EINVAL;
        cb::set_rotary(rotary, &j);
    }
    j.bf16 = c.bf16;
    j.tokens = n_tokens;
    j.positions = positions_dev;
    j.offsets = offsets_dev;
    j.start = start_dev ? start_dev : c.lengths;
    CB_CHECKED(cb::check_heads(k, dtype, &j.k, empty));
    CB_CHECKED(cb::check_heads(v, dtype, &j.v, empty));
    if (k->heads != c.heads || v->heads != c.heads) return CB_EINVAL;
    if (q) {
        CB_CHECKED(cb::check_heads(q, dtype, &j.q, empty));
        CB_CHECKED(cb::check_heads(q_out, dtype, &j.q_out, empty));
        if (q->heads != q_out->heads) return CB_EINVAL;
    }
    CB_LAUNCHED(cb::launch_append(j, c, (hipStream_t)hip_stream));
    return CB_OK;
}

int cb_cache_attend(const cb_cache* cache, const cb_attend_params* params, const cb_heads* q, const cb_heads* out, float* lse_dev,
                    void* hip_stream)
{
    cb::Cache c = {};
    cb::AttendJob j = {};
    CB_CHECKED(cb::check_attend(cache, params, q, out, &c, &j));
    if (params->accumulate && !c.weight) return CB_EINVAL;
    CB_CHECKED(cb::check_cache(cache, true, q->heads, &c));
    if (!cb::attend_fits(c, q->heads)) return CB_EINVAL;
    j.lse = lse_dev;
    CB_LAUNCHED(cb::launch_attend(j, c, (hipStream_t)hip_stream));
    return CB_OK;
}

int cb_cache_attend_chosen(const cb_cache* cache, const cb_attend_params* params, const cb_heads* q, const cb_heads* out, float* lse_dev,
                           const int32_t* chosen_dev, const int32_t* count_dev, int32_t budget, void* hip_stream)
{
    cb::Cache c = {};
    cb::AttendJob j = {};
    CB_CHECKED(cb::check_attend(cache, params, q, out, &c, &j));
    if (params->accumulate || !chosen_dev || !count_dev || budget < 1 || budget > cb::MOST_CHOSEN) return CB_EINVAL;
    CB_CHECKED(cb::check_cache(cache, true, q->heads, &c));
    if (!cb::attend_fits(c, q->heads)) return CB_EINVAL;
    j.lse = lse_dev;
    j.chosen = chosen_dev;
    j.count = count_dev;
    j.budget = budget;
    CB_LAUNCHED(cb::launch_attend(j, c, (hipStream_t)hip_stream));
    return CB_OK;
}

int cb_cache_bound(const cb_cache* cache, const int32_t* since_dev, void* hip_stream)
{
    cb::Cache c = {};
    CB_CHECKED(cb::check_cache(cache, true, 0, &c));
    if (!c.bounds || !cb::choose_fits(c)) return CB_EINVAL;
    CB_LAUNCHED(cb::launch_bound(since_dev, c, (hipStream_t)hip_stream));
    return CB_OK;
}

int cb_cache_choose(const cb_cache* cache, const cb_choose_params* params, const cb_heads* q, int32_t* chosen_dev, int32_t* count_dev,
                    void* hip_stream)
{
    if (!params || !q || params->reserved != 0 || !chosen_dev || !count_dev) return CB_EINVAL;
    if (params->budget < 1 || params->budget > cb::MOST_CHOSEN || params->first < 0 || params->recent < 0 || (long)params->first + params->recent > params->budget) return CB_EINVAL;
    cb::Cache c = {};
    CB_CHECKED(cb::check_cache(cache, true, 0, &c));
    cb::ChooseJob j = {};
    CB_CHECKED(cb::check_heads(q, cb::values_dtype(*cache), &j.q, false));
    if (!c.bounds || q->heads % c.heads || !cb::choose_fits(c)) return CB_EINVAL;
    j.budget = params->budget; j.first = params->first; j.recent = params->recent;
    j.chosen = chosen_dev; j.count = count_dev;
    CB_LAUNCHED(cb::launch_choose(j, c, (hipStream_t)hip_stream));
    return CB_OK;
}

int cb_cache_evict(const cb_cache* cache, const cb_evict_params* params, void* hip_stream)
{
    if (!params) return CB_EINVAL;
    cb::Cache c = {};
    CB_CHECKED(cb::check_cache(cache, true, 0, &c));
    if (c.e4m3 || !c.weight || !c.time || params->budget < 1 || params->budget > c.capacity || params->window < 0) return CB_EINVAL;
    cb::EvictJob j;
    j.budget = params->budget; j.window = params->window;
    j.weight_in = params->weight_in_dev ? params->weight_in_dev : c.weight;
    j.time_in = params->time_in_dev ? params->time_in_dev : c.time;
    if (((uintptr_t)j.weight_in & 15) || ((uintptr_t)j.time_in & 15)) return CB_EINVAL;
    j.lengths_in = params->lengths_in_dev ? params->lengths_in_dev : c.lengths;
    CB_LAUNCHED(cb::launch_evict(j, c, (hipStream_t)hip_stream));
    return CB_OK;
}

}  // extern "C"
