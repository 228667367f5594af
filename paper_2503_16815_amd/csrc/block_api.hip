// C ABI of the operators of a layer's feed-forward block: argument validation, scratch ownership and
// the choice of the operator's launches.  See include/deft_block.h for the contract.
#include <cstring>
#include <new>

#include "block.h"

using namespace deft;

namespace {

constexpr int32_t kMaxRows = 1 << 20;
constexpr int32_t kMaxHidden = 16384;
constexpr int32_t kMaxInner = 65536;
constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr uint32_t kFfn = DEFT_BLOCK_FFN | DEFT_BLOCK_FFN_GRAD;
constexpr uint32_t kAll = kFfn | DEFT_BLOCK_CHECKPOINT | DEFT_BLOCK_RESTORE;

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

struct deft_block {
    deft_block_config_t cfg{};
    int compute_units = 0;
    FfnPlan ffn{};
    void *scratch = nullptr;
};

namespace {

void free_handle(deft_block *h)
{
    if (!h) return;
    DeviceGuard g(h->cfg.device);
    if (h->scratch) (void)hipFree(h->scratch);
    delete h;
}

deft_status_t done(hipError_t e)
{
    if (e == hipSuccess) return DEFT_OK;
    (void)hipGetLastError();
    return DEFT_ERR_DEVICE;
}

// rows of `width` elements, `stride` apart, at an address that its elements can have
bool rows_ok(const deft_block *h, const void *p, int64_t width, int64_t stride)
{
    return p && stride >= width && stride <= kMaxStride && ((uintptr_t)p % (h->cfg.dtype == DEFT_F32 ? 4 : 2)) == 0;
}

bool checkpoint_ok(const deft_checkpoint_t &c, int64_t width)
{
    return c.codes && c.codes_stride >= width && c.codes_stride <= kMaxStride && c.scales && ((uintptr_t)c.scales & 1) == 0 &&
           c.scales_stride >= (width + kGroup - 1) / kGroup && c.scales_stride <= kMaxStride;
}

bool saved_ok(const deft_block *h, const deft_saved_t &s, int64_t inner)
{
    const auto one = [&](const deft_checkpoint_t &c) {
        if (s.kind == DEFT_SAVE_FULL && h->cfg.dtype == DEFT_F32) return rows_ok(h, c.codes, inner, c.codes_stride);
        return checkpoint_ok(c, inner) && (s.kind == DEFT_SAVE_PACKED || ((uintptr_t)c.codes & 1) == 0);
    };
    if (s.kind == DEFT_SAVE_FULL || s.kind == DEFT_SAVE_PACKED) return one(s.gate) && one(s.up);
    return s.kind == DEFT_SAVE_NONE;
}

deft_status_t ffn_sizes_ok(const deft_block *h, uint32_t op, int32_t rows, int32_t hidden, int32_t inner, int32_t activation)
{
    if (rows < 0 || hidden < 1 || inner < 1 || activation < DEFT_SILU || activation > DEFT_RELU) return DEFT_ERR_INVALID_ARG;
    if (!(h->cfg.operators & op)) return DEFT_ERR_LIMIT;
    if (rows > h->cfg.max_rows || hidden > h->cfg.max_hidden || inner > h->cfg.max_inner) return DEFT_ERR_LIMIT;
    return DEFT_OK;
}

deft_status_t checkpoint_sizes_ok(const deft_block *h, uint32_t op, int32_t rows, int32_t width)
{
    if (rows < 0 || width < 1) return DEFT_ERR_INVALID_ARG;
    if (!(h->cfg.operators & op)) return DEFT_ERR_LIMIT;
    if (rows > h->cfg.max_rows || (width > h->cfg.max_hidden && width > h->cfg.max_inner)) return DEFT_ERR_LIMIT;
    return DEFT_OK;
}

}  // namespace

extern "C" deft_status_t deft_block_create(const deft_block_config_t *cfg, deft_block_t **out)
{
    if (out) *out = nullptr;
    if (!cfg || !out) return DEFT_ERR_INVALID_ARG;
    const bool ffn = (cfg->operators & kFfn) != 0;
    if (cfg->device < 0 || cfg->dtype < DEFT_F32 || cfg->dtype > DEFT_BF16 || cfg->operators == 0 || (cfg->operators & ~kAll) != 0 ||
        cfg->max_rows < 1 || cfg->max_hidden < 1 || cfg->max_inner < (ffn ? 1 : 0))
        return DEFT_ERR_INVALID_ARG;
    if (cfg->max_rows > kMaxRows || cfg->max_hidden > kMaxHidden || cfg->max_inner > kMaxInner) return DEFT_ERR_LIMIT;

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

    deft_block *h = new (std::nothrow) deft_block;
    if (!h) return DEFT_ERR_OOM;
    h->cfg = *cfg;
    h->compute_units = prop.multiProcessorCount;
    deft_status_t st = DEFT_OK;
    if (ffn) {
        ffn_plan(cfg->dtype, cfg->max_rows, cfg->max_hidden, cfg->max_inner, (cfg->operators & DEFT_BLOCK_FFN_GRAD) != 0, h->compute_units, &h->ffn);
        const hipError_t e = hipMalloc(&h->scratch, (size_t)h->ffn.scratch_bytes);
        if (e != hipSuccess) {
            (void)hipGetLastError();
            h->scratch = nullptr;
            st = e == hipErrorOutOfMemory ? DEFT_ERR_OOM : DEFT_ERR_DEVICE;
        }
        if (st == DEFT_OK) st = done(ffn_prepare());
    }
    if (st != DEFT_OK) {
        free_handle(h);
        return st;
    }
    *out = h;
    return DEFT_OK;
}

extern "C" void deft_block_destroy(deft_block_t *h) { free_handle(h); }

extern "C" deft_status_t deft_block_get_info(const deft_block_t *h, deft_block_info_t *info)
{
    if (!h || !info) return DEFT_ERR_INVALID_ARG;
    info->scratch_bytes = h->ffn.scratch_bytes;
    info->compute_units = h->compute_units;
    return DEFT_OK;
}

extern "C" deft_status_t deft_checkpoint(deft_block_t *h, const deft_checkpoint_call_t *a)
{
    if (!h || !a) return DEFT_ERR_INVALID_ARG;
    const deft_status_t s = checkpoint_sizes_ok(h, DEFT_BLOCK_CHECKPOINT, a->n_rows, a->width);
    if (s != DEFT_OK) return s;
    if (a->n_rows == 0) return DEFT_OK;
    if (!rows_ok(h, a->x, a->width, a->x_stride) || !checkpoint_ok(a->out, a->width)) return DEFT_ERR_INVALID_ARG;
    DeviceGuard g(h->cfg.device);
    if (!g.ok) return DEFT_ERR_DEVICE;
    return done(checkpoint_launch(h->cfg.dtype, *a, static_cast<hipStream_t>(a->stream)));
}

extern "C" deft_status_t deft_restore(deft_block_t *h, const deft_restore_call_t *a)
{
    if (!h || !a) return DEFT_ERR_INVALID_ARG;
    const deft_status_t s = checkpoint_sizes_ok(h, DEFT_BLOCK_RESTORE, a->n_rows, a->width);
    if (s != DEFT_OK) return s;
    if (a->n_rows == 0) return DEFT_OK;
    if (!rows_ok(h, a->out, a->width, a->out_stride) || !checkpoint_ok(a->from, a->width)) return DEFT_ERR_INVALID_ARG;
    DeviceGuard g(h->cfg.device);
    if (!g.ok) return DEFT_ERR_DEVICE;
    return done(restore_launch(h->cfg.dtype, *a, static_cast<hipStream_t>(a->stream)));
}

extern "C" deft_status_t deft_ffn(deft_block_t *h, const deft_ffn_t *a)
{
    if (!h || !a) return DEFT_ERR_INVALID_ARG;
    const deft_status_t s = ffn_sizes_ok(h, DEFT_BLOCK_FFN, a->n_rows, a->hidden, a->inner, a->activation);
    if (s != DEFT_OK) return s;
    if (a->n_rows == 0) return DEFT_OK;
    if (!rows_ok(h, a->x, a->hidden, a->x_stride) || !rows_ok(h, a->w_gate, a->hidden, a->w_gate_stride) ||
        !rows_ok(h, a->w_up, a->hidden, a->w_up_stride) || !rows_ok(h, a->w_down, a->inner, a->w_down_stride) ||
        !rows_ok(h, a->y, a->hidden, a->y_stride) || !saved_ok(h, a->save, a->inner))
        return DEFT_ERR_INVALID_ARG;
    DeviceGuard g(h->cfg.device);
    if (!g.ok) return DEFT_ERR_DEVICE;
    return done(ffn_launch(h->ffn, h->cfg.dtype, *a, h->scratch, h->compute_units, static_cast<hipStream_t>(a->stream)));
}

extern "C" deft_status_t deft_ffn_grad(deft_block_t *h, const deft_ffn_grad_t *a)
{
    if (!h || !a) return DEFT_ERR_INVALID_ARG;
    const deft_status_t s = ffn_sizes_ok(h, DEFT_BLOCK_FFN_GRAD, a->n_rows, a->hidden, a->inner, a->activation);
    if (s != DEFT_OK) return s;
    if ((a->accumulate & ~1) != 0 || (!a->grad_x && !a->grad_gate && !a->grad_up && !a->grad_down)) return DEFT_ERR_INVALID_ARG;
    if (a->n_rows > 0 &&
        (!rows_ok(h, a->grad_y, a->hidden, a->grad_y_stride) ||
         !(a->x ? rows_ok(h, a->x, a->hidden, a->x_stride) : checkpoint_ok(a->packed_x, a->hidden)) ||
         !rows_ok(h, a->w_gate, a->hidden, a->w_gate_stride) || !rows_ok(h, a->w_up, a->hidden, a->w_up_stride) ||
         !rows_ok(h, a->w_down, a->inner, a->w_down_stride) || !saved_ok(h, a->saved, a->inner) ||
         (a->grad_x && !rows_ok(h, a->grad_x, a->hidden, a->grad_x_stride))))
        return DEFT_ERR_INVALID_ARG;
    if ((a->grad_gate && !rows_ok(h, a->grad_gate, a->hidden, a->grad_gate_stride)) ||
        (a->grad_up && !rows_ok(h, a->grad_up, a->hidden, a->grad_up_stride)) ||
        (a->grad_down && !rows_ok(h, a->grad_down, a->inner, a->grad_down_stride)) || (a->events && (!a->events[0] || !a->events[1])))
        return DEFT_ERR_INVALID_ARG;
    DeviceGuard g(h->cfg.device);
    if (!g.ok) return DEFT_ERR_DEVICE;
    return done(ffn_grad_launch(h->ffn, h->cfg.dtype, *a, h->scratch, h->compute_units, static_cast<hipStream_t>(a->stream)));
}
