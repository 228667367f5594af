// C ABI of the operators at a language model's ends: argument validation, scratch ownership and
// the choice of the operator's launches.  See include/deft_ends.h for the contract.
#include <cmath>
#include <cstring>
#include <new>

#include "ends.h"

using namespace deft;

namespace {

constexpr int32_t kMaxRows = 1 << 20;
constexpr int32_t kMaxVocab = 1 << 21;
constexpr int32_t kMaxHidden = 16384;
constexpr int32_t kMaxTopK = 1024;
constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr uint32_t kAll = DEFT_ENDS_EMBED | DEFT_ENDS_EMBED_GRAD | DEFT_ENDS_HEAD_LOSS | DEFT_ENDS_HEAD_GRAD | DEFT_ENDS_DISTILL;

struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev)
    {
        if (hipGetDevice(&prev) != hipSuccess) return;
        ok = (prev == dev) || hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard()
    {
        if (ok && prev >= 0) (void)hipSetDevice(prev);
    }
};

}  // namespace

struct deft_ends {
    deft_ends_config_t cfg{};
    int compute_units = 0;
    int64_t scratch_bytes = 0;
    EmbedPlan embed{};
    void *embed_scratch = nullptr;
    HeadPlan head{};
    void *head_scratch = nullptr;
};

namespace {

void free_handle(deft_ends *h)
{
    if (!h) return;
    DeviceGuard g(h->cfg.device);
    if (h->embed_scratch) (void)hipFree(h->embed_scratch);
    if (h->head_scratch) (void)hipFree(h->head_scratch);
    delete h;
}

deft_status_t alloc(void **p, int64_t bytes, int64_t *total)
{
    *p = nullptr;
    if (bytes <= 0) return DEFT_OK;
    const hipError_t e = hipMalloc(p, (size_t)bytes);
    if (e == hipSuccess) {
        *total += bytes;
        return DEFT_OK;
    }
    (void)hipGetLastError();
    *p = nullptr;
    return e == hipErrorOutOfMemory ? DEFT_ERR_OOM : DEFT_ERR_DEVICE;
}

deft_status_t done(hipError_t e)
{
    if (e == hipSuccess) return DEFT_OK;
    (void)hipGetLastError();
    return DEFT_ERR_DEVICE;
}

int64_t element(const deft_ends *h) { return h->cfg.dtype == DEFT_F32 ? 4 : 2; }

// rows of `width` elements, `stride` apart, at an address that its elements can have
bool rows_ok(const deft_ends *h, const void *p, int64_t width, int64_t stride)
{
    return p && stride >= width && stride <= kMaxStride && ((uintptr_t)p % (uintptr_t)element(h)) == 0;
}

bool words_ok(const void *p) { return p && ((uintptr_t)p & 3) == 0; }
bool words_or_null(const void *p) { return ((uintptr_t)p & 3) == 0; }

// What every call checks first: the handle serves the operator, and the sizes are within its limits.
deft_status_t sizes_ok(const deft_ends *h, uint32_t op, int32_t rows, int32_t vocab, int32_t hidden)
{
    if (rows < 0 || vocab < 1 || hidden < 1) return DEFT_ERR_INVALID_ARG;
    if (!(h->cfg.operators & op)) return DEFT_ERR_LIMIT;
    if (rows > h->cfg.max_rows || vocab > h->cfg.max_vocab) return DEFT_ERR_LIMIT;
    if (op != DEFT_ENDS_DISTILL && hidden > h->cfg.max_hidden) return DEFT_ERR_LIMIT;
    return DEFT_OK;
}

}  // namespace

extern "C" deft_status_t deft_ends_create(const deft_ends_config_t *cfg, deft_ends_t **out)
{
    if (out) *out = nullptr;
    if (!cfg || !out) return DEFT_ERR_INVALID_ARG;
    const bool table = (cfg->operators & ~DEFT_ENDS_DISTILL) != 0, distill = (cfg->operators & DEFT_ENDS_DISTILL) != 0;
    if (cfg->device < 0 || cfg->dtype < DEFT_F32 || cfg->dtype > DEFT_BF16 || cfg->operators == 0 ||
        (cfg->operators & ~kAll) != 0 || cfg->max_rows < 1 || cfg->max_vocab < 1 || cfg->max_hidden < (table ? 1 : 0) ||
        cfg->max_top_k < (distill ? 1 : 0))
        return DEFT_ERR_INVALID_ARG;
    if (cfg->max_rows > kMaxRows || cfg->max_vocab > kMaxVocab || cfg->max_hidden > kMaxHidden || cfg->max_top_k > kMaxTopK)
        return DEFT_ERR_LIMIT;

    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess) {
        (void)hipGetLastError();
        return DEFT_ERR_DEVICE;
    }
    if (cfg->device >= ndev) return DEFT_ERR_INVALID_ARG;
    hipDeviceProp_t prop;
    if (hipGetDeviceProperties(&prop, cfg->device) != hipSuccess) {
        (void)hipGetLastError();
        return DEFT_ERR_DEVICE;
    }
    if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0) return DEFT_ERR_DEVICE;
    DeviceGuard g(cfg->device);
    if (!g.ok) return DEFT_ERR_DEVICE;

    deft_ends *h = new (std::nothrow) deft_ends;
    if (!h) return DEFT_ERR_OOM;
    h->cfg = *cfg;
    h->compute_units = prop.multiProcessorCount;
    deft_status_t st = DEFT_OK;
    if (cfg->operators & DEFT_ENDS_EMBED_GRAD) {
        embed_grad_plan(cfg->max_rows, cfg->max_vocab, cfg->max_hidden, &h->embed);
        st = alloc(&h->embed_scratch, h->embed.scratch_bytes, &h->scratch_bytes);
    }
    if (st == DEFT_OK && (cfg->operators & (DEFT_ENDS_HEAD_LOSS | DEFT_ENDS_HEAD_GRAD))) {
        head_plan(cfg->dtype, cfg->max_rows, cfg->max_vocab, cfg->max_hidden, (cfg->operators & DEFT_ENDS_HEAD_GRAD) != 0,
                  h->compute_units, &h->head);
        st = alloc(&h->head_scratch, h->head.scratch_bytes, &h->scratch_bytes);
        if (st == DEFT_OK) st = done(head_prepare());
    }
    if (st != DEFT_OK) {
        free_handle(h);
        return st;
    }
    *out = h;
    return DEFT_OK;
}

extern "C" void deft_ends_destroy(deft_ends_t *h) { free_handle(h); }

extern "C" deft_status_t deft_ends_get_info(const deft_ends_t *h, deft_ends_info_t *info)
{
    if (!h || !info) return DEFT_ERR_INVALID_ARG;
    info->scratch_bytes = h->scratch_bytes;
    info->vocab_piece = (h->cfg.operators & DEFT_ENDS_HEAD_GRAD) ? h->head.piece : 0;
    info->compute_units = h->compute_units;
    return DEFT_OK;
}

extern "C" deft_status_t deft_embed(deft_ends_t *h, const deft_embed_t *e)
{
    if (!h || !e) return DEFT_ERR_INVALID_ARG;
    const deft_status_t s = sizes_ok(h, DEFT_ENDS_EMBED, e->n_rows, e->vocab, e->hidden);
    if (s != DEFT_OK) return s;
    if (e->n_rows == 0) return DEFT_OK;
    if (!words_ok(e->tokens) || !words_or_null(e->status) || !rows_ok(h, e->table, e->hidden, e->table_stride) ||
        !rows_ok(h, e->out, e->hidden, e->out_stride))
        return DEFT_ERR_INVALID_ARG;
    DeviceGuard g(h->cfg.device);
    if (!g.ok) return DEFT_ERR_DEVICE;
    return done(embed_launch(h->cfg.dtype, *e, static_cast<hipStream_t>(e->stream)));
}

extern "C" deft_status_t deft_embed_grad(deft_ends_t *h, const deft_embed_grad_t *e)
{
    if (!h || !e) return DEFT_ERR_INVALID_ARG;
    const deft_status_t s = sizes_ok(h, DEFT_ENDS_EMBED_GRAD, e->n_rows, e->vocab, e->hidden);
    if (s != DEFT_OK) return s;
    if ((e->accumulate & ~1) != 0 || !rows_ok(h, e->grad_table, e->hidden, e->grad_table_stride) ||
        (e->n_rows > 0 && (!words_ok(e->tokens) || !rows_ok(h, e->grad_out, e->hidden, e->grad_out_stride))))
        return DEFT_ERR_INVALID_ARG;
    if (e->n_rows == 0 && e->accumulate) return DEFT_OK;
    DeviceGuard g(h->cfg.device);
    if (!g.ok) return DEFT_ERR_DEVICE;
    return done(embed_grad_launch(h->embed, h->cfg.dtype, *e, h->embed_scratch, h->compute_units,
                                  static_cast<hipStream_t>(e->stream)));
}

extern "C" deft_status_t deft_head_loss(deft_ends_t *h, const deft_head_loss_t *a)
{
    if (!h || !a) return DEFT_ERR_INVALID_ARG;
    const deft_status_t s = sizes_ok(h, DEFT_ENDS_HEAD_LOSS, a->n_rows, a->vocab, a->hidden);
    if (s != DEFT_OK) return s;
    if (a->n_rows == 0) return DEFT_OK;
    if (!words_ok(a->labels) || !words_ok(a->loss) || !words_ok(a->lse) || !words_or_null(a->status) ||
        !rows_ok(h, a->hidden_states, a->hidden, a->hidden_stride) || !rows_ok(h, a->weight, a->hidden, a->weight_stride))
        return DEFT_ERR_INVALID_ARG;
    DeviceGuard g(h->cfg.device);
    if (!g.ok) return DEFT_ERR_DEVICE;
    return done(head_loss_launch(h->head, h->cfg.dtype, *a, h->head_scratch, h->compute_units,
                                 static_cast<hipStream_t>(a->stream)));
}

extern "C" deft_status_t deft_head_grad(deft_ends_t *h, const deft_head_grad_t *a)
{
    if (!h || !a) return DEFT_ERR_INVALID_ARG;
    const deft_status_t s = sizes_ok(h, DEFT_ENDS_HEAD_GRAD, a->n_rows, a->vocab, a->hidden);
    if (s != DEFT_OK) return s;
    if ((a->accumulate & ~1) != 0 || a->n_piece_events < 0 || (a->n_piece_events > 0 && !a->piece_events) ||
        (!a->grad_hidden && !a->grad_weight && a->n_rows > 0))
        return DEFT_ERR_INVALID_ARG;
    if (a->n_rows > 0 &&
        (!words_ok(a->labels) || !words_ok(a->lse) || !words_ok(a->row_grad) ||
         !rows_ok(h, a->hidden_states, a->hidden, a->hidden_stride) || !rows_ok(h, a->weight, a->hidden, a->weight_stride) ||
         (a->grad_hidden && !rows_ok(h, a->grad_hidden, a->hidden, a->grad_hidden_stride))))
        return DEFT_ERR_INVALID_ARG;
    if (a->grad_weight && !rows_ok(h, a->grad_weight, a->hidden, a->grad_weight_stride)) return DEFT_ERR_INVALID_ARG;
    DeviceGuard g(h->cfg.device);
    if (!g.ok) return DEFT_ERR_DEVICE;
    return done(head_grad_launch(h->head, h->cfg.dtype, *a, h->head_scratch, h->compute_units,
                                 static_cast<hipStream_t>(a->stream)));
}

extern "C" deft_status_t deft_distill(deft_ends_t *h, const deft_distill_t *a)
{
    if (!h || !a) return DEFT_ERR_INVALID_ARG;
    if (a->top_k < 1 || !(a->temperature > 0.0f) || !std::isfinite(a->temperature)) return DEFT_ERR_INVALID_ARG;
    const deft_status_t s = sizes_ok(h, DEFT_ENDS_DISTILL, a->n_rows, a->vocab, 1);
    if (s != DEFT_OK) return s;
    if (a->top_k > h->cfg.max_top_k) return DEFT_ERR_LIMIT;
    if (a->n_rows == 0) return DEFT_OK;
    if (!rows_ok(h, a->logits, a->vocab, a->logits_stride) || !words_ok(a->teacher_index) || !words_ok(a->teacher_logit) ||
        !words_ok(a->loss) || !words_or_null(a->status))
        return DEFT_ERR_INVALID_ARG;
    if (a->grad_logits &&
        (!words_ok(a->row_grad) || !rows_ok(h, a->grad_logits, a->vocab, a->grad_stride) ||
         (a->grad_logits == a->logits && a->grad_stride != a->logits_stride)))
        return DEFT_ERR_INVALID_ARG;
    DeviceGuard g(h->cfg.device);
    if (!g.ok) return DEFT_ERR_DEVICE;
    return done(distill_launch(h->cfg.dtype, *a, h->compute_units, static_cast<hipStream_t>(a->stream)));
}
