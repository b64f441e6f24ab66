// extern "C" boundary of the training operators: argument checks and the table of tensors.
#include <cmath>
#include <cstring>
#include "ftc_train.cuh"

namespace ftc {
namespace {

uint32_t size_of(uint32_t dtype) { return dtype == FTC_F32 ? 4u : 2u; }
bool is_float(uint32_t dtype) { return dtype == FTC_F32 || dtype == FTC_BF16 || dtype == FTC_F16; }
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int sm_count(int& n) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return FTC_ECUDA;
    return cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess ? FTC_OK : FTC_ECUDA;
}
int status(cudaError_t e) { return e == cudaSuccess ? FTC_OK : FTC_ECUDA; }

int check_norm(const ftc_norm_t* d, uint64_t rows) {
    if (!d) return FTC_EINVAL;
    if (!is_float(d->dtype) || (d->wdtype != FTC_F32 && d->wdtype != d->dtype)) return FTC_EUNSUPPORTED;
    if (d->H == 0 || d->H > (1u << 24) || d->P == 0 || d->P > (1u << 20) || d->k == 0 || d->k > (1u << 24) || !(d->eps >= 0.f) || rows > (1ull << 31))
        return FTC_EINVAL;
    if (((uint64_t)d->H + d->k + 31) / 32 * d->P > 0x7FFFFFFFull) return FTC_EINVAL;
    return FTC_OK;
}

size_t norm_workspace(const ftc_norm_t* d, uint64_t rows, int sms) {
    return ((size_t)norm_backward_groups(d->H, rows, sms) + d->P) * d->H * 2 * sizeof(float);
}

const TableHead* head_of(const void* h_table) {
    const TableHead* h = static_cast<const TableHead*>(h_table);
    return h && aligned(h, 8) && h->magic == kTableMagic ? h : nullptr;
}

// Entries that can be laid out: their blocks in all, or -1.
int64_t count_blocks(const ftc_param_t* p, uint32_t n) {
    if ((!p && n) || n > (1u << 30)) return -1;
    uint64_t blocks = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const ftc_param_t& t = p[i];
        if (t.n > (1ull << 40) || !is_float(t.param_dtype) || !is_float(t.grad_dtype) || t.reserved || !std::isfinite(t.lr_scale) || !std::isfinite(t.weight_decay)) return -1;
        if (t.n && !t.grad) return -1;
        if (!aligned(t.param, size_of(t.param_dtype)) || !aligned(t.grad, size_of(t.grad_dtype)) || !aligned(t.master, 4) || !aligned(t.status, 16)) return -1;
        if (t.status && (t.k == 0 || t.k > (1u << 30))) return -1;
        blocks += (t.n + FTC_STATE_BLOCK - 1) / FTC_STATE_BLOCK;
        if (blocks > (1ull << 32)) return -1;
    }
    return (int64_t)blocks;
}

// A state of such a beta changes by less than a 32nd a step. Rounded to the nearest code it would not fall any more below code 64 of 255
// (v), 32 of 127 (m), or further up. Root of v against that of 32-bit states, median, where gradients of 100 in 256 elements became a hundred times
// smaller: 1.03 after 1000 steps of 0.95, 1.11 after 1500 of 0.96875, 1.74 after 3000 of 0.99, 11.6 after 4000 of 0.999; dithered 0.99, 0.98, 1.00, 0.98.
bool long_memory(double beta) { return beta > 0.96875; }

size_t grad_norm_doubles(const TableHead* h, int sms) { return (size_t)grad_norm_warps(h->n_blocks, sms) + 2 * (size_t)h->n_params + 1; }

}  // namespace
}  // namespace ftc

using namespace ftc;

extern "C" {

int ftc_layernorm_forward(const ftc_norm_t* desc, uint64_t rows, const void* d_x, uint64_t x_stride, const void* d_gamma,
                          const void* d_beta, void* d_y, uint64_t y_stride, float* d_mean, float* d_rstd, void* cuda_stream) {
    int rc = check_norm(desc, rows), sms = 0;
    if (rc != FTC_OK || rows == 0) return rc;
    const uint32_t e = size_of(desc->dtype), w = size_of(desc->wdtype);
    if (!d_x || !d_y || x_stride < desc->H || y_stride < desc->H || x_stride > (1ull << 40) || y_stride > (1ull << 40)) return FTC_EINVAL;
    if (!aligned(d_x, e) || !aligned(d_y, e) || !aligned(d_gamma, w) || !aligned(d_beta, w) || !aligned(d_mean, 4) || !aligned(d_rstd, 4)) return FTC_EINVAL;
    if ((rc = sm_count(sms)) != FTC_OK) return rc;
    NormArgs a{};
    a.x = d_x; a.gamma = d_gamma; a.beta = d_beta; a.y = d_y; a.mean_out = d_mean; a.rstd_out = d_rstd;
    a.rows = (uint32_t)rows; a.x_stride = x_stride; a.y_stride = y_stride;
    a.H = desc->H; a.dtype = desc->dtype; a.wdtype = desc->wdtype; a.eps = desc->eps;
    return status(launch_norm_forward(a, sms, static_cast<cudaStream_t>(cuda_stream)));
}

size_t ftc_layernorm_workspace_bytes(const ftc_norm_t* desc, uint64_t rows) {
    if (check_norm(desc, rows) != FTC_OK) return 0;
    int sms = 0;
    if (sm_count(sms) != FTC_OK) sms = 148;
    return norm_workspace(desc, rows, sms);
}

int ftc_layernorm_backward(const ftc_norm_t* desc, uint64_t rows, const void* d_dy, uint64_t dy_stride, const void* d_x,
                           uint64_t x_stride, const void* d_gamma, const float* d_mean, const float* d_rstd,
                           const uint64_t* d_row_splits, void* d_dx, uint64_t dx_stride, float* d_dgamma, float* d_dbeta,
                           void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
    int rc = check_norm(desc, rows), sms = 0;
    if (rc != FTC_OK) return rc;
    const uint32_t e = size_of(desc->dtype);
    const uint64_t far = 1ull << 40;
    if (rows && (!d_dy || !d_x || !d_mean || !d_rstd || dy_stride < desc->H || x_stride < desc->H || dy_stride > far || x_stride > far)) return FTC_EINVAL;
    if (rows && d_dx && (dx_stride < desc->H || dx_stride > far)) return FTC_EINVAL;
    if (!aligned(d_dy, e) || !aligned(d_x, e) || !aligned(d_dx, e) || !aligned(d_gamma, size_of(desc->wdtype)) || !aligned(d_mean, 4) || !aligned(d_rstd, 4) ||
        !aligned(d_dgamma, 4) || !aligned(d_dbeta, 4) || !aligned(d_row_splits, 8)) return FTC_EINVAL;
    const bool weights = d_dgamma || d_dbeta;
    if (!weights && (!d_dx || rows == 0)) return FTC_OK;
    if ((rc = sm_count(sms)) != FTC_OK) return rc;
    if (weights && (!d_workspace || !aligned(d_workspace, 16) || workspace_bytes < norm_workspace(desc, rows, sms))) return FTC_EWORKSPACE;
    NormArgs a{};
    a.x = d_x; a.dy = d_dy; a.gamma = d_gamma; a.mean = d_mean; a.rstd = d_rstd; a.splits = d_row_splits; a.dx = d_dx;
    a.dgamma = d_dgamma; a.dbeta = d_dbeta; a.slots = weights ? static_cast<float*>(d_workspace) : nullptr;
    a.rows = (uint32_t)rows; a.x_stride = x_stride; a.dy_stride = dy_stride; a.dx_stride = dx_stride;
    a.H = desc->H; a.P = desc->P; a.k = desc->k; a.dtype = desc->dtype; a.wdtype = desc->wdtype; a.eps = desc->eps;
    a.direct = norm_backward_direct(a, sms);
    if (a.direct) a.slots = nullptr;
    a.groups = a.direct ? a.P : norm_backward_groups(desc->H, rows, sms);
    a.rows_per_group = a.groups ? (uint32_t)((rows + a.groups - 1) / a.groups) : 0;
    return status(launch_norm_backward(a, sms, static_cast<cudaStream_t>(cuda_stream)));
}

size_t ftc_param_table_bytes(const ftc_param_t* h_params, uint32_t n_params) {
    const int64_t blocks = count_blocks(h_params, n_params);
    return blocks < 0 ? 0 : sizeof(TableHead) + (size_t)n_params * sizeof(TableEntry) + (((size_t)blocks + 1) & ~(size_t)1) * 4;
}

int ftc_param_table_build(const ftc_param_t* h_params, uint32_t n_params, void* h_table, size_t table_bytes) {
    const int64_t blocks = count_blocks(h_params, n_params);
    if (blocks < 0 || !h_table || !aligned(h_table, 8) || table_bytes < ftc_param_table_bytes(h_params, n_params)) return FTC_EINVAL;
    TableHead* h = static_cast<TableHead*>(h_table);
    std::memset(h, 0, ftc_param_table_bytes(h_params, n_params));
    h->magic = kTableMagic; h->n_blocks = (uint64_t)blocks; h->n_params = n_params;
    TableEntry* en = reinterpret_cast<TableEntry*>(h + 1);
    uint32_t* map = reinterpret_cast<uint32_t*>(en + n_params);
    uint64_t at = 0, wide = 0;
    for (uint32_t i = 0; i < n_params; ++i) {
        const ftc_param_t& t = h_params[i];
        TableEntry& q = en[i];
        q.param = t.param; q.master = t.master; q.grad = t.grad; q.status = t.status; q.n = t.n; q.first_block = at;
        q.k = t.status ? t.k : 1; q.k_shift = q.k & (q.k - 1) ? 255 : (uint8_t)__builtin_ctz(q.k); q.param_dtype = (uint8_t)t.param_dtype; q.grad_dtype = (uint8_t)t.grad_dtype;
        q.wide = aligned(t.grad, 8 * size_of(t.grad_dtype)) && aligned(t.param, 8 * size_of(t.param_dtype)) && aligned(t.master, 32);   // 8 elements a load
        q.lr_scale = t.lr_scale; q.weight_decay = t.weight_decay;
        if (t.n && !t.param) h->flags |= 1u;
        if (t.status && (t.k % 8 || FTC_STATE_BLOCK % t.k || !aligned(t.grad, 8 * size_of(t.grad_dtype)))) h->flags |= 4u;
        if (q.wide) wide += t.n / FTC_STATE_BLOCK;
        for (const uint64_t end = at + (t.n + FTC_STATE_BLOCK - 1) / FTC_STATE_BLOCK; at < end; ++at) map[at] = i;
    }
    if (wide * 2 >= h->n_blocks) h->flags |= 2u;
    return FTC_OK;
}

uint64_t ftc_param_table_blocks(const void* h_table) {
    const TableHead* h = head_of(h_table);
    return h ? h->n_blocks : 0;
}

size_t ftc_grad_norm_workspace_bytes(const void* h_table) {
    const TableHead* h = head_of(h_table);
    if (!h) return 0;
    int sms = 0;
    if (sm_count(sms) != FTC_OK) sms = 148;
    return grad_norm_doubles(h, sms) * sizeof(double);
}

int ftc_grad_norm(const void* h_table, const void* d_table, float max_norm, float* d_norm, float* d_norms, void* d_workspace,
                  size_t workspace_bytes, void* cuda_stream) {
    const TableHead* h = head_of(h_table);
    if (!h || !d_table || !aligned(d_table, 256) || !(max_norm > 0.f) || !d_norm || !aligned(d_norm, 4) || !aligned(d_norms, 4)) return FTC_EINVAL;
    int sms = 0, rc = sm_count(sms);
    if (rc != FTC_OK) return rc;
    if (!d_workspace || !aligned(d_workspace, 16) || workspace_bytes < grad_norm_doubles(h, sms) * sizeof(double)) return FTC_EWORKSPACE;
    return status(launch_grad_norm(d_table, h->n_params, h->n_blocks, h->flags >> 2 & 1u, max_norm, d_norm, d_norms, static_cast<double*>(d_workspace), sms,
                                   static_cast<cudaStream_t>(cuda_stream)));
}

int ftc_adamw_step(const ftc_adamw_t* hyper, const void* h_table, const void* d_table, void* d_m, void* d_v, float* d_m_scale,
                   float* d_v_scale, const float* d_grad_scale, void* cuda_stream) {
    const TableHead* h = head_of(h_table);
    if (!hyper || !h || !d_table || !aligned(d_table, 256) || hyper->reserved || (h->flags & 1u)) return FTC_EINVAL;
    if (!(hyper->lr >= 0) || !std::isfinite((float)hyper->lr) || !(hyper->beta1 >= 0 && (float)hyper->beta1 < 1.f) || !(hyper->beta2 >= 0 && (float)hyper->beta2 < 1.f) ||
        !(hyper->eps >= 1e-30) || !std::isfinite((float)hyper->eps) || hyper->step == 0) return FTC_EINVAL;
    if (hyper->state_bits != 32 && hyper->state_bits != 8) return FTC_EUNSUPPORTED;
    if (h->n_blocks == 0) return FTC_OK;
    if (!d_m || !d_v || !aligned(d_m, 32) || !aligned(d_v, 32) || !aligned(d_grad_scale, 4)) return FTC_EINVAL;
    if (hyper->state_bits == 8 && (!d_m_scale || !d_v_scale || !aligned(d_m_scale, 4) || !aligned(d_v_scale, 4))) return FTC_EINVAL;
    int sms = 0, rc = sm_count(sms);
    if (rc != FTC_OK) return rc;
    AdamArgs a{};
    a.table = d_table; a.n_params = h->n_params; a.n_blocks = h->n_blocks;
    a.m = d_m; a.v = d_v; a.m_scale = d_m_scale; a.v_scale = d_v_scale; a.grad_scale = d_grad_scale; a.bits = hyper->state_bits; a.mostly_wide = h->flags >> 1 & 1u;
    const double t = (double)hyper->step;
    a.one = 1.f;
    if (a.bits == 8) a.dither = (long_memory(hyper->beta1) ? kDitherM : 0u) | (long_memory(hyper->beta2) ? kDitherV : 0u);
    a.phase = (uint32_t)hyper->step * kDitherStep;
    a.lr = (float)hyper->lr; a.eps = (float)hyper->eps;
    a.beta1 = (float)hyper->beta1; a.beta2 = (float)hyper->beta2; a.rest1 = (float)(1 - hyper->beta1); a.rest2 = (float)(1 - hyper->beta2);
    a.fix1 = (float)(1 / (1 - std::pow(hyper->beta1, t))); a.fix2 = (float)(1 / std::sqrt(1 - std::pow(hyper->beta2, t)));
    return status(launch_adamw(a, sms, static_cast<cudaStream_t>(cuda_stream)));
}

int ftc_adamw_states(uint64_t blocks, const void* d_m, const void* d_v, const float* d_m_scale, const float* d_v_scale, float* d_m_out,
                     float* d_v_out, void* cuda_stream) {
    if (blocks == 0) return FTC_OK;
    if (blocks > (1ull << 32) || !d_m || !d_v || !d_m_scale || !d_v_scale || !d_m_out || !d_v_out) return FTC_EINVAL;
    if (!aligned(d_m, 32) || !aligned(d_v, 32) || !aligned(d_m_out, 32) || !aligned(d_v_out, 32) || !aligned(d_m_scale, 4) || !aligned(d_v_scale, 4)) return FTC_EINVAL;
    return status(launch_adamw_states(blocks, d_m, d_v, d_m_scale, d_v_scale, d_m_out, d_v_out, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
