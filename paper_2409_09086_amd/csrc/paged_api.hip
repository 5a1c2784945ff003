// Host side of the rotary and paged-cache entry points declared in include/infmllm.h: argument checks, workspace carving and
// launches.  No device memory is allocated here and nothing synchronises.
#include "../../include/infmllm.h"

#include <algorithm>
#include <climits>
#include <cmath>
#include <new>

#include "errors.h"
#include "launch.h"
#include "paged.h"

using namespace infmllm;

namespace {

constexpr size_t ALIGN = 256;
size_t up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }

// Launches go to the device that was current at attach, whichever is now.
struct OnDevice {
    int before = -1;
    hipError_t err;
    explicit OnDevice(int dev)
    {
        int now = -1;
        err = hipGetDevice(&now);
        if (err == hipSuccess && now != dev) {
            err = hipSetDevice(dev);
            if (err == hipSuccess) before = now;
        }
    }
    ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};

// Rows of a token tensor: `heads` heads of d elements per token.
int check_rows(const char* who, const char* name, const void* p, int64_t stride, int heads, int d, int elt)
{
    if (!p) return fail(INFMLLM_EINVAL, "%s: %s must not be null", who, name);
    if ((uintptr_t)p % 16) return fail(INFMLLM_EINVAL, "%s: %s must be aligned to 16 bytes", who, name);
    if (stride < (int64_t)heads * d || stride > (1ll << 40) || stride % (16 / elt))
        return fail(INFMLLM_EINVAL, "%s: the stride of %s must be a multiple of 16 bytes and at least a token's heads (got %lld elements)",
                    who, name, (long long)stride);
    return INFMLLM_OK;
}

// A weight vector (or null), read sixteen bytes at a time.
int check_weight(const char* who, const char* name, const void* p)
{
    if ((uintptr_t)p % 16) return fail(INFMLLM_EINVAL, "%s: %s must be aligned to 16 bytes", who, name);
    return INFMLLM_OK;
}

int check_batch(const char* who, const infmllm_batch_t* b)
{
    if (!b) return fail(INFMLLM_EINVAL, "%s: batch is null", who);
    if (b->seqs < 1 || b->seqs > 65536) return fail(INFMLLM_EINVAL, "%s: seqs must lie in 1..65536 (got %d)", who, b->seqs);
    if (b->tokens < 0 || b->tokens > (1 << 24)) return fail(INFMLLM_EINVAL, "%s: tokens must lie in 0..2^24 (got %d)", who, b->tokens);
    if (b->max_new < 0 || b->max_len < 0) return fail(INFMLLM_EINVAL, "%s: max_new and max_len must not be negative", who);
    if (b->pages_per_seq < 1 || b->pages_per_seq > (1 << 26))
        return fail(INFMLLM_EINVAL, "%s: pages_per_seq must lie in 1..2^26 (got %d)", who, b->pages_per_seq);
    if (!b->starts || !b->lens || !b->table) return fail(INFMLLM_EINVAL, "%s: starts, lens and table must not be null", who);
    if (((uintptr_t)b->starts | (uintptr_t)b->lens | (uintptr_t)b->table) % 4)
        return fail(INFMLLM_EINVAL, "%s: starts, lens and table must be aligned to 4 bytes", who);
    return INFMLLM_OK;
}

bool whole(double v) { return v == std::floor(v); }
bool normal_float(double v) { return std::isnormal((float)v); }
constexpr double LOG2E = 1.4426950408889634;

// Whether the kernel for few rows (32 a unit) is the faster one for bf16 queries, by what the two should take, in us.  It reads the keys once
// for every 32 rows; where there are no more units than teams those of one head run beside each other and find them in the L2, otherwise they
// come from behind it, at 6 TB/s.  The kernel for chunks takes some 40 us for a grid that its units do not fill (pieces and
// their merge), else 14 and its tiles of 256 rows by 64 keys.  Measured, us, few rows / chunks, heads of 128 in groups of 4, rows of a
// sequence: 1 x 8000 keys, 8 kv-heads, 64 rows 24.1 / 44.6, 256 27.4 / 46.5; 4 x 4000, 8, 256 37.6 / 44.4; 16 x 4000, 8, 32 55.8 / 66.3,
// 64 56.7 / 67.4, 96 123.0 / 69.3; 16 x 4000, 2, 256 38.0 / 43.8; 32 x 2000, 8, 32 52.6 / 56.4, 64 90.4 / 57.5; 32 x 2000, 2, 128 25.0 / 38.4,
// 256 44.2 / 41.3; of 64: 16 x 4000, 8, 64 27.9 / 47.0, 96 61.8 / 49.1; 4 x 4000, 8, 256 27.1 / 32.4.
template <typename T>
bool few_rows_pay(const PagedArgs<T>& a, int d, int max_new, int max_len)
{
    const double rows = (double)std::min(max_new, a.tokens) * a.G, keys = std::min((double)max_len, (double)a.pages_per_seq * (1 << a.page_shift));
    if (rows <= 32) return true;
    const double seqs = std::min(a.seqs, a.tokens), all = (double)a.tokens * a.G;
    auto units = [&](int block) { return a.Hkv * std::min(seqs * std::ceil(rows / block), all / block + seqs); };
    const double memory = seqs * a.Hkv * keys * 4 * d / 5.3e6, few = units(32) * keys;
    const double t_few = units(32) <= PAGED_CUS ? (d == 128 ? 12 : 10) + std::max(memory, few / (d == 128 ? 43e3 : 60e3)) : 14 + few * 4 * d / 6e6;
    const double tiles = units(256) * keys / 64 / PAGED_CUS;
    const double t_many = std::max(d == 128 ? 40.0 : 28.0, (d == 128 ? 14 : 10) + std::max(memory, tiles * (d == 128 ? 1.75 : 1.0)));
    return t_few < t_many;
}

}  // namespace

struct infmllm_rotary {
    int d, dtype, max_positions;
    int dims, layout = 0;
    double eps = 1e-6;
    RotaryFrequencies f{10000.0, 1.0, 0.0, 1.0, 32.0, 1.0};
    bool attached = false;
    int dev = 0;
    hipStream_t st = nullptr;
    float* tab = nullptr;

    int turned() const { return f.base > 0.0 ? dims : 0; }
    size_t bytes() const { return up((size_t)max_positions * (turned() / 2) * sizeof(float2)); }
    template <typename T> void fill(RotaryArgs<T>& a) const
    {
        a.table_cs = (const float2*)tab;
        a.dims = turned(); a.half = layout == 0; a.max_positions = max_positions;
        a.eps = (float)eps;
    }
};

struct infmllm_paged {
    int pages, page_size, page_shift, Hq, Hkv, d, dtype, window = 0, kernel = 0;
    double scale;
    bool attached = false;
    int dev = 0;
    hipStream_t st = nullptr;

    int elt() const { return dtype == INFMLLM_BF16 ? 2 : 4; }
    PagedScratch sc{nullptr, nullptr};
    size_t part_bytes() const { return up(std::max(paged_rows_scratch(d, elt()), dtype == INFMLLM_BF16 ? paged_mixed_scratch(d) : 0)); }
    size_t bytes() const { return up(2 * PAGED_TEAMS * sizeof(int)) + part_bytes(); }
};

extern "C" {

// ---- rotary

int infmllm_rotary_create(int head_dim, int dtype, int max_positions, infmllm_rotary_t** out)
{
    if (!out) return fail(INFMLLM_EINVAL, "rotary_create: out is null");
    *out = nullptr;
    if (head_dim != 64 && head_dim != 128)
        return fail(INFMLLM_EINVAL, "rotary_create: head_dim must be 64 or 128 (got %d)", head_dim);
    if (dtype != INFMLLM_BF16 && dtype != INFMLLM_FP32) return fail(INFMLLM_EINVAL, "rotary_create: unknown dtype %d", dtype);
    if (max_positions < 1 || max_positions > (1 << 24))
        return fail(INFMLLM_EINVAL, "rotary_create: max_positions must lie in 1..2^24 (got %d)", max_positions);
    infmllm_rotary* r = new (std::nothrow) infmllm_rotary();
    if (!r) return fail(INFMLLM_ENOMEM, "rotary_create: out of host memory");
    r->d = r->dims = head_dim; r->dtype = dtype; r->max_positions = max_positions;
    *out = r;
    return INFMLLM_OK;
}

int infmllm_rotary_set_param(infmllm_rotary_t* r, int which, double value)
{
    if (!r) return fail(INFMLLM_EINVAL, "rotary_set_param: object is null");
    if (r->attached) return fail(INFMLLM_ESTATE, "rotary_set_param: parameters are fixed once the object is attached");
    if (!std::isfinite(value)) return fail(INFMLLM_EINVAL, "rotary_set_param: value is not finite");
    switch (which) {
        case INFMLLM_ROTARY_BASE:
            if (value != 0 && !(value > 1)) return fail(INFMLLM_EINVAL, "rotary_set_param: base must be 0 (off) or > 1");
            r->f.base = value;
            return INFMLLM_OK;
        case INFMLLM_ROTARY_DIMS:
            if (!whole(value) || value < 16 || value > r->d || (int)value % 16)
                return fail(INFMLLM_EINVAL, "rotary_set_param: dims must be a multiple of 16 in 16..head_dim");
            r->dims = (int)value;
            return INFMLLM_OK;
        case INFMLLM_ROTARY_LAYOUT:
            if (value != 0 && value != 1) return fail(INFMLLM_EINVAL, "rotary_set_param: layout must be 0 or 1");
            r->layout = (int)value;
            return INFMLLM_OK;
        case INFMLLM_ROTARY_FACTOR:
            if (value < 1) return fail(INFMLLM_EINVAL, "rotary_set_param: factor must be >= 1");
            r->f.factor = value;
            return INFMLLM_OK;
        case INFMLLM_ROTARY_TRAINED:
            if (value < 0) return fail(INFMLLM_EINVAL, "rotary_set_param: trained must be >= 0");
            r->f.trained = value;
            return INFMLLM_OK;
        case INFMLLM_ROTARY_LOW:
            if (value < 0) return fail(INFMLLM_EINVAL, "rotary_set_param: low must be >= 0");
            r->f.low = value;
            return INFMLLM_OK;
        case INFMLLM_ROTARY_HIGH:
            if (value <= 0) return fail(INFMLLM_EINVAL, "rotary_set_param: high must be > 0");
            r->f.high = value;
            return INFMLLM_OK;
        case INFMLLM_ROTARY_MAGNITUDE:
            if (value <= 0 || !normal_float(value)) return fail(INFMLLM_EINVAL, "rotary_set_param: magnitude must be > 0 and a normal float");
            r->f.magnitude = value;
            return INFMLLM_OK;
        case INFMLLM_ROTARY_EPS:
            if (value < 0 || (value > 0 && !normal_float(value))) return fail(INFMLLM_EINVAL, "rotary_set_param: eps must be 0 or a normal float > 0");
            r->eps = value;
            return INFMLLM_OK;
        default:
            return fail(INFMLLM_EINVAL, "rotary_set_param: unknown parameter %d", which);
    }
}

size_t infmllm_rotary_workspace_bytes(const infmllm_rotary_t* r) { return r ? r->bytes() : 0; }

int infmllm_rotary_attach(infmllm_rotary_t* r, void* ws, size_t bytes, void* hip_stream)
{
    if (!r) return fail(INFMLLM_EINVAL, "rotary_attach: object is null");
    if (r->attached) return fail(INFMLLM_ESTATE, "rotary_attach: the object is already attached");
    const size_t need = r->bytes();
    if (!ws && need) return fail(INFMLLM_EINVAL, "rotary_attach: workspace is null");
    if ((uintptr_t)ws % ALIGN) return fail(INFMLLM_EINVAL, "rotary_attach: workspace must be 256-byte aligned");
    if (bytes < need) return fail(INFMLLM_ENOMEM, "rotary_attach: workspace has %zu bytes, %zu needed", bytes, need);
    if (r->f.trained > 0 && r->f.low >= r->f.high) return fail(INFMLLM_EINVAL, "rotary_attach: low must lie below high");
    hipError_t e = hipGetDevice(&r->dev);
    if (e != hipSuccess) return fail_hip(e, "rotary_attach: hipGetDevice");
    if (need && (e = launch_rotary_table((float*)ws, r->turned() / 2, r->max_positions, r->f, (hipStream_t)hip_stream)) != hipSuccess)
        return fail_hip(e, "rotary_attach: position table");
    r->tab = (float*)ws;
    r->st = (hipStream_t)hip_stream;
    r->attached = true;
    return INFMLLM_OK;
}

int infmllm_rotary_apply(infmllm_rotary_t* r, const int32_t* positions, int tokens, int heads, int kv_heads, const void* q,
                         int64_t q_stride, const void* k, int64_t k_stride, const void* q_weight, const void* k_weight,
                         void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride)
{
    const char* who = "rotary_apply";
    if (!r) return fail(INFMLLM_EINVAL, "%s: object is null", who);
    if (!r->attached) return fail(INFMLLM_ESTATE, "%s: the object has no workspace attached", who);
    if (tokens < 0 || tokens > (1 << 24)) return fail(INFMLLM_EINVAL, "%s: tokens must lie in 0..2^24 (got %d)", who, tokens);
    if (tokens == 0) return INFMLLM_OK;
    if (heads < 0 || kv_heads < 0 || heads > 16384 || kv_heads > 16384 || heads + kv_heads == 0)
        return fail(INFMLLM_EINVAL, "%s: heads and kv_heads must lie in 0..16384, not both 0 (got %d, %d)", who, heads, kv_heads);
    if (!positions || (uintptr_t)positions % 4) return fail(INFMLLM_EINVAL, "%s: positions must not be null and be aligned to 4 bytes", who);
    const int elt = r->dtype == INFMLLM_BF16 ? 2 : 4;
    int rc;
    if (heads && ((rc = check_rows(who, "q", q, q_stride, heads, r->d, elt)) || (rc = check_rows(who, "q_out", q_out, q_out_stride, heads, r->d, elt)) ||
                  (rc = check_weight(who, "q_weight", q_weight))))
        return rc;
    if (kv_heads && ((rc = check_rows(who, "k", k, k_stride, kv_heads, r->d, elt)) ||
                     (rc = check_rows(who, "k_out", k_out, k_out_stride, kv_heads, r->d, elt)) || (rc = check_weight(who, "k_weight", k_weight))))
        return rc;
    OnDevice on(r->dev);
    if (on.err != hipSuccess) return fail_hip(on.err, who);
    auto go = [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        RotaryArgs<T> a{};
        a.q = (const T*)q; a.k = (const T*)k; a.q_out = (T*)q_out; a.k_out = (T*)k_out;
        a.q_weight = (const T*)q_weight; a.k_weight = (const T*)k_weight;
        a.q_stride = q_stride; a.k_stride = k_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
        a.positions = positions;
        a.tokens = tokens; a.heads = heads; a.kv_heads = kv_heads;
        r->fill(a);
        return launch_rotary<T>(a, r->d, false, r->st);
    };
    const hipError_t e = elt == 2 ? go((uint16_t*)nullptr) : go((float*)nullptr);
    return e == hipSuccess ? INFMLLM_OK : fail_hip(e, who);
}

void infmllm_rotary_destroy(infmllm_rotary_t* r) { delete r; }

// ---- paged caches

int infmllm_paged_create(int pages, int page_size, int heads, int kv_heads, int head_dim, int dtype, infmllm_paged_t** out)
{
    if (!out) return fail(INFMLLM_EINVAL, "paged_create: out is null");
    *out = nullptr;
    if (pages < 1 || pages > (1 << 30)) return fail(INFMLLM_EINVAL, "paged_create: pages must lie in 1..2^30 (got %d)", pages);
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)))
        return fail(INFMLLM_EINVAL, "paged_create: page_size must be a power of two in 16..1024 (got %d)", page_size);
    if (heads <= 0 || kv_heads <= 0 || heads % kv_heads != 0 || heads > 16384)
        return fail(INFMLLM_EINVAL, "paged_create: kv_heads must divide heads, at most 16384 (got %d, %d)", heads, kv_heads);
    if (heads / kv_heads > 4096) return fail(INFMLLM_EINVAL, "paged_create: at most 4096 heads share a kv-head (got %d)", heads / kv_heads);
    if (head_dim != 64 && head_dim != 128)
        return fail(INFMLLM_EINVAL, "paged_create: head_dim must be 64 or 128 (got %d)", head_dim);
    if (dtype != INFMLLM_BF16 && dtype != INFMLLM_FP32) return fail(INFMLLM_EINVAL, "paged_create: unknown dtype %d", dtype);
    if ((int64_t)kv_heads * page_size * head_dim * 4 > INT_MAX)
        return fail(INFMLLM_EINVAL, "paged_create: a page of %d rows of %d heads is too large", page_size, kv_heads);
    infmllm_paged* p = new (std::nothrow) infmllm_paged();
    if (!p) return fail(INFMLLM_ENOMEM, "paged_create: out of host memory");
    p->pages = pages; p->page_size = page_size; p->page_shift = __builtin_ctz((unsigned)page_size);
    p->Hq = heads; p->Hkv = kv_heads; p->d = head_dim; p->dtype = dtype;
    p->scale = 1.0 / std::sqrt((double)head_dim);
    *out = p;
    return INFMLLM_OK;
}

int infmllm_paged_set_param(infmllm_paged_t* p, int which, double value)
{
    if (!p) return fail(INFMLLM_EINVAL, "paged_set_param: object is null");
    if (p->attached) return fail(INFMLLM_ESTATE, "paged_set_param: parameters are fixed once the object is attached");
    if (!std::isfinite(value)) return fail(INFMLLM_EINVAL, "paged_set_param: value is not finite");
    switch (which) {
        case INFMLLM_PAGED_SCALE:
            if (value <= 0 || !normal_float(value * LOG2E))
                return fail(INFMLLM_EINVAL, "paged_set_param: scale must be > 0, its product with log2(e) a normal float");
            p->scale = value;
            return INFMLLM_OK;
        case INFMLLM_PAGED_WINDOW:
            if (value < 0 || value > (double)(1 << 30) || !whole(value))
                return fail(INFMLLM_EINVAL, "paged_set_param: window must be an integer in 0..2^30");
            p->window = (int)value;
            return INFMLLM_OK;
        case INFMLLM_PAGED_KERNEL:
            if (value != 0 && value != 1 && value != 2 && value != 3) return fail(INFMLLM_EINVAL, "paged_set_param: kernel must be 0, 1, 2 or 3");
            p->kernel = (int)value;
            return INFMLLM_OK;
        default:
            return fail(INFMLLM_EINVAL, "paged_set_param: unknown parameter %d", which);
    }
}

size_t infmllm_paged_workspace_bytes(const infmllm_paged_t* p) { return p ? p->bytes() : 0; }

int infmllm_paged_attach(infmllm_paged_t* p, void* ws, size_t bytes, void* hip_stream)
{
    if (!p) return fail(INFMLLM_EINVAL, "paged_attach: object is null");
    if (p->attached) return fail(INFMLLM_ESTATE, "paged_attach: the object is already attached");
    if (!ws) return fail(INFMLLM_EINVAL, "paged_attach: workspace is null");
    if ((uintptr_t)ws % ALIGN) return fail(INFMLLM_EINVAL, "paged_attach: workspace must be 256-byte aligned");
    if (bytes < p->bytes()) return fail(INFMLLM_ENOMEM, "paged_attach: workspace has %zu bytes, %zu needed", bytes, p->bytes());
    hipError_t e = hipGetDevice(&p->dev);
    if (e != hipSuccess) return fail_hip(e, "paged_attach: hipGetDevice");
    const size_t tickets = p->bytes() - p->part_bytes();
    if ((e = launch_zero(ws, tickets, (hipStream_t)hip_stream)) != hipSuccess) return fail_hip(e, "paged_attach: clearing the workspace");
    p->sc = PagedScratch{(float*)((char*)ws + tickets), (int*)ws};
    p->st = (hipStream_t)hip_stream;
    p->attached = true;
    return INFMLLM_OK;
}

int infmllm_paged_append(infmllm_paged_t* p, infmllm_rotary_t* rotary, const infmllm_batch_t* batch, const void* k, int64_t k_stride,
                         const void* v, int64_t v_stride, const void* k_weight, const void* q, int64_t q_stride, const void* q_weight,
                         void* q_out, int64_t q_out_stride, void* K, void* V)
{
    const char* who = "paged_append";
    if (!p) return fail(INFMLLM_EINVAL, "%s: object is null", who);
    if (!p->attached) return fail(INFMLLM_ESTATE, "%s: the object has no workspace attached", who);
    int rc;
    if ((rc = check_batch(who, batch))) return rc;
    if (batch->tokens == 0) return INFMLLM_OK;
    if (rotary) {
        if (!rotary->attached) return fail(INFMLLM_ESTATE, "%s: the rotary object has no workspace attached", who);
        if (rotary->d != p->d || rotary->dtype != p->dtype || rotary->dev != p->dev)
            return fail(INFMLLM_EINVAL, "%s: the rotary object is for another head_dim, dtype or device", who);
        if (rotary->turned() && batch->max_len > rotary->max_positions)
            return fail(INFMLLM_ECAPACITY, "%s: max_len %d exceeds the rotary object's %d positions", who, batch->max_len, rotary->max_positions);
    } else if (q || k_weight || q_weight) {
        return fail(INFMLLM_EINVAL, "%s: queries and norm weights need a rotary object", who);
    }
    if (q_weight && !q) return fail(INFMLLM_EINVAL, "%s: q_weight without q", who);
    const int elt = p->elt();
    if ((rc = check_rows(who, "k", k, k_stride, p->Hkv, p->d, elt)) || (rc = check_rows(who, "v", v, v_stride, p->Hkv, p->d, elt)) ||
        (rc = check_weight(who, "k_weight", k_weight)) || (rc = check_weight(who, "q_weight", q_weight)))
        return rc;
    if (q && ((rc = check_rows(who, "q", q, q_stride, p->Hq, p->d, elt)) || (rc = check_rows(who, "q_out", q_out, q_out_stride, p->Hq, p->d, elt))))
        return rc;
    if (!K || !V || ((uintptr_t)K | (uintptr_t)V) % 16) return fail(INFMLLM_EINVAL, "%s: K and V must not be null and be aligned to 16 bytes", who);
    OnDevice on(p->dev);
    if (on.err != hipSuccess) return fail_hip(on.err, who);
    auto go = [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        RotaryArgs<T> a{};
        a.q = (const T*)q; a.k = (const T*)k; a.v = (const T*)v; a.q_out = (T*)q_out;
        a.q_weight = (const T*)q_weight; a.k_weight = (const T*)k_weight;
        a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
        a.tokens = batch->tokens; a.heads = q ? p->Hq : 0; a.kv_heads = p->Hkv;
        if (rotary) rotary->fill(a);
        a.starts = batch->starts; a.lens = batch->lens; a.table = batch->table;
        a.K = (T*)K; a.V = (T*)V;
        a.seqs = batch->seqs; a.pages_per_seq = batch->pages_per_seq; a.pages = p->pages; a.page_shift = p->page_shift;
        return launch_rotary<T>(a, p->d, true, p->st);
    };
    const hipError_t e = elt == 2 ? go((uint16_t*)nullptr) : go((float*)nullptr);
    return e == hipSuccess ? INFMLLM_OK : fail_hip(e, who);
}

int infmllm_paged_attend(infmllm_paged_t* p, const infmllm_batch_t* batch, const void* q, int64_t q_stride, const void* K, const void* V,
                         void* out, float* lse)
{
    const char* who = "paged_attend";
    if (!p) return fail(INFMLLM_EINVAL, "%s: object is null", who);
    if (!p->attached) return fail(INFMLLM_ESTATE, "%s: the object has no workspace attached", who);
    int rc;
    if ((rc = check_batch(who, batch))) return rc;
    if (batch->tokens == 0) return INFMLLM_OK;
    const int elt = p->elt();
    if ((rc = check_rows(who, "q", q, q_stride, p->Hq, p->d, elt)) || (rc = check_rows(who, "out", out, (int64_t)p->Hq * p->d, p->Hq, p->d, elt)))
        return rc;
    if (!K || !V || ((uintptr_t)K | (uintptr_t)V) % 16) return fail(INFMLLM_EINVAL, "%s: K and V must not be null and be aligned to 16 bytes", who);
    if ((int64_t)batch->tokens * (p->Hq / p->Hkv) > (1 << 30))
        return fail(INFMLLM_EINVAL, "%s: tokens * heads / kv_heads must not exceed 2^30", who);
    if ((uintptr_t)lse % 4) return fail(INFMLLM_EINVAL, "%s: lse must be aligned to 4 bytes", who);
    OnDevice on(p->dev);
    if (on.err != hipSuccess) return fail_hip(on.err, who);
    auto go = [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        PagedArgs<T> a{};
        a.q = (const T*)q; a.K = (const T*)K; a.V = (const T*)V; a.out = (T*)out; a.lse = lse;
        a.starts = batch->starts; a.lens = batch->lens; a.table = batch->table;
        a.q_stride = q_stride;
        a.seqs = batch->seqs; a.tokens = batch->tokens; a.pages_per_seq = batch->pages_per_seq; a.pages = p->pages; a.page_shift = p->page_shift;
        a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = p->Hq / p->Hkv; a.window = p->window;
        a.inv_g = (uint32_t)((1ull << 32) / (unsigned)a.G + 1);
        a.c = (float)(p->scale * LOG2E);
        if constexpr (sizeof(T) == 2) {
            // Rows of sequences that run on their own beside chunks: a block of that kernel's.  Measured, us, 16 / 64, 32 heads of 128 on 2, 512 tokens beside
            // 31 decoded ones 60.3 / 60.1, 2 x 256 beside 100 53.4 / 54.1, 1024 beside 16 109 / 110; on 1, whose decoded tokens are 32 rows each, 63.4 /
            // 59.9, 58.1 / 53.4, 106 / 104.
            const int few = 16;
            int kernel = p->kernel;
            if (kernel == 0) {
                const bool alike = a.seqs == 1 || (int64_t)std::min(batch->max_new, a.tokens) * a.seqs == a.tokens;
                kernel = few_rows_pay(a, p->d, batch->max_new, batch->max_len) ? 1 : alike ? 2 : 3;
            }
            if (kernel == 2) return launch_paged_fwd(a, p->sc, p->d, p->st);
            if (kernel == 3) return launch_paged_mixed(a, p->sc, p->d, few, p->st);
        }
        return launch_paged_rows<T>(a, p->sc, p->d, batch->max_new, batch->max_len, p->st);
    };
    const hipError_t e = elt == 2 ? go((uint16_t*)nullptr) : go((float*)nullptr);
    return e == hipSuccess ? INFMLLM_OK : fail_hip(e, who);
}

void infmllm_paged_destroy(infmllm_paged_t* p) { delete p; }

}  // extern "C"
