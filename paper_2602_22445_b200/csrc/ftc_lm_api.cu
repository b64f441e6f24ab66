// extern "C" boundary of the embedding, the token log probabilities and the orthogonalised update: argument checks, workspaces, the plan.
#include <algorithm>
#include <cmath>
#include <cstring>
#include "ftc_lm.cuh"

namespace ftc {
namespace {

uint32_t size_of(uint32_t dtype) { return dtype == FTC_F32 ? 4u : 2u; }
bool is_float(uint32_t dtype) { return dtype == FTC_F32 || dtype == FTC_BF16 || dtype == FTC_F16; }
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t rounded(size_t n, size_t to) { return (n + to - 1) / to * to; }
int status(cudaError_t e) { return e == cudaSuccess ? FTC_OK : FTC_ECUDA; }
int sm_count(int& n) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return FTC_ECUDA;
    return cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess ? FTC_OK : FTC_ECUDA;
}

constexpr uint64_t kFar = 1ull << 40;                            // strides

int check_embed(const ftc_embed_t* d, uint64_t n) {
    if (!d) return FTC_EINVAL;
    if (!is_float(d->dtype) || (d->wdtype != FTC_F32 && d->wdtype != d->dtype) || (d->token_bits != 32 && d->token_bits != 64)) return FTC_EUNSUPPORTED;
    if (d->V == 0 || d->V > (1u << 30) || d->H == 0 || d->H > (1u << 24) || d->P == 0 || d->P > (1u << 20) || d->k == 0 || d->k > (1u << 24) || n > (1ull << 31))
        return FTC_EINVAL;
    if ((uint64_t)d->V * d->H > kFar || !std::isfinite(d->scale) || ((uint64_t)d->V * d->H + d->k) > kFar / d->P) return FTC_EINVAL;
    return FTC_OK;
}
// Five lists of the tokens, then the sums of runs that leave their chunk; those are needed from the second chunk on.
size_t embed_list(uint64_t n) { return rounded(n * 4, 16); }
size_t embed_workspace(const ftc_embed_t* d, uint64_t n) {
    return n ? 5 * embed_list(n) + (n + FTC_EMBED_RUN - 1) / FTC_EMBED_RUN * 2 * rounded((size_t)d->H * 4, 16) : 0;
}

int check_logprob(const ftc_logprob_t* d, uint64_t rows) {
    if (!d) return FTC_EINVAL;
    if (!is_float(d->dtype) || (d->token_bits != 32 && d->token_bits != 64)) return FTC_EUNSUPPORTED;
    if (d->V == 0 || d->V > (1u << 30) || d->top > 32 || d->top > d->V || !(d->scale >= 1e-6f && d->scale <= 1e6f) || rows > 0x7FFFFFFFull) return FTC_EINVAL;
    return FTC_OK;
}

const PlanHead* plan_of(const void* h_plan) {
    const PlanHead* h = static_cast<const PlanHead*>(h_plan);
    return h && aligned(h, 8) && h->magic == kPlanMagic ? h : nullptr;
}

// Entries that can be laid out; what they need in all.
bool count_matrices(const ftc_matrix_t* q, uint32_t n, PlanHead& h) {
    h = PlanHead{};
    if ((!q && n) || n > (1u << 20)) return false;
    h.magic = kPlanMagic; h.n = n;
    uint64_t chunks = 0, blocks = 0, gram = 0, apply = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const ftc_param_t& t = q[i].tensor;
        const uint64_t rows = q[i].rows, cols = q[i].cols, m = rows < cols ? rows : cols, w = rows < cols ? cols : rows;
        if (m == 0 || m > (1u << 14) || w > (1u << 20) || rows * cols > (1ull << 31) || t.n != rows * cols) return false;
        if (!is_float(t.param_dtype) || !is_float(t.grad_dtype) || t.reserved || !std::isfinite(t.lr_scale) || !std::isfinite(t.weight_decay)) return false;
        if (!t.grad || !t.param) return false;
        if (!aligned(t.param, size_of(t.param_dtype)) || !aligned(t.grad, size_of(t.grad_dtype)) || !aligned(t.master, 4) || !aligned(t.status, 16)) return false;
        if (t.status && (t.k == 0 || t.k > (1u << 30))) return false;
        const uint64_t mb = (m + 127) / 128, nb = (w + 63) / 64, mb2 = (mb + 1) / 2;
        h.n_blocks += (t.n + FTC_STATE_BLOCK - 1) / FTC_STATE_BLOCK;
        blocks += mb * nb; h.a_blocks += mb * 2 * mb; h.diagonals += mb * 128;
        chunks += (t.n + kMuonChunk - 1) / kMuonChunk;
        const uint32_t size = plan_size(m, w);
        if (size < 2) ++h.items[kSmall];
        if (size > 0) { gram += mb2 * (mb2 + 1) / 2; apply += mb2 * ((nb + 3) / 4); }
        if (size == 1) { ++h.middle; h.gram_middle += (uint32_t)(mb2 * (mb2 + 1) / 2); h.apply_middle += (uint32_t)(mb2 * ((nb + 3) / 4)); }
        if (h.n_blocks > (1ull << 32) || blocks > 0x7FFFFFFFull || h.a_blocks > 0x7FFFFFFFull || chunks > 0x7FFFFFFFull || 16 * (2 * gram + apply) > 0x7FFFFFFFull) return false;   // tiles of 16 steps
    }
    h.items[kChunks] = (uint32_t)chunks; h.items[kBlocks] = (uint32_t)blocks; h.items[kGramTiles] = (uint32_t)gram; h.items[kApplyTiles] = (uint32_t)apply;
    return true;
}
size_t plan_bytes(const PlanHead& h) {
    return sizeof(PlanHead) + (size_t)h.n * sizeof(PlanEntry) + rounded(((size_t)h.items[kChunks] + h.items[kBlocks] + h.items[kGramTiles] + h.items[kApplyTiles] + h.items[kSmall] + h.n) * 4, 8);
}

struct MuonLayout { size_t sums, live, factor, written, diag_a, diag_b, x0, x1, a, b, x_bytes, a_bytes, total; };
MuonLayout muon_layout(const PlanHead& h, uint32_t products) {
    const size_t block = 128 * 64 * 2, numbers = products == 32 ? 2 : 1;
    MuonLayout l{};
    l.x_bytes = h.items[kBlocks] * block; l.a_bytes = h.a_blocks * block;
    size_t at = 1024;
    auto take = [&](size_t bytes) { const size_t here = at; at = rounded(at + bytes, 256); return here; };
    l.sums = take((size_t)h.items[kChunks] * 16); l.live = take((size_t)h.n * 4); l.factor = take((size_t)h.n * 4); l.written = take((size_t)h.n * 12);
    l.diag_a = take(h.diagonals * 4); l.diag_b = take(h.diagonals * 4);
    l.x0 = take(l.x_bytes * numbers); l.x1 = take(l.x_bytes * numbers); l.a = take(l.a_bytes * numbers); l.b = take(l.a_bytes * numbers);
    l.total = at;
    return l;
}

}  // namespace
}  // namespace ftc

using namespace ftc;

extern "C" {

int ftc_embedding_forward(const ftc_embed_t* desc, uint64_t n, const void* d_tokens, const void* d_table, uint64_t table_stride, void* d_y,
                          uint64_t y_stride, void* cuda_stream) {
    int rc = check_embed(desc, n), sms = 0;
    if (rc != FTC_OK || n == 0) return rc;
    if (!d_tokens || !d_table || !d_y || table_stride < desc->H || y_stride < desc->H || table_stride > kFar || y_stride > kFar) return FTC_EINVAL;
    if (!aligned(d_tokens, desc->token_bits / 8) || !aligned(d_table, size_of(desc->wdtype)) || !aligned(d_y, size_of(desc->dtype))) return FTC_EINVAL;
    if ((rc = sm_count(sms)) != FTC_OK) return rc;
    EmbedArgs a{};
    a.tokens = d_tokens; a.table = d_table; a.y = d_y; a.table_stride = table_stride; a.y_stride = y_stride;
    a.n = (uint32_t)n; a.V = desc->V; a.H = desc->H; a.dtype = desc->dtype; a.wdtype = desc->wdtype; a.token_bits = desc->token_bits; a.scale = desc->scale;
    return status(launch_embedding_forward(a, sms, static_cast<cudaStream_t>(cuda_stream)));
}

size_t ftc_embedding_workspace_bytes(const ftc_embed_t* desc, uint64_t n) { return check_embed(desc, n) == FTC_OK ? embed_workspace(desc, n) : 0; }

int ftc_embedding_backward(const ftc_embed_t* desc, uint64_t n, const void* d_tokens, const void* d_dy, uint64_t dy_stride,
                           const uint64_t* d_row_splits, float* d_dtable, void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
    int rc = check_embed(desc, n), sms = 0;
    if (rc != FTC_OK) return rc;
    if (!d_dtable || !aligned(d_dtable, 4) || !aligned(d_row_splits, 8)) return FTC_EINVAL;
    if (n && (!d_tokens || !d_dy || dy_stride < desc->H || dy_stride > kFar || !aligned(d_tokens, desc->token_bits / 8) || !aligned(d_dy, size_of(desc->dtype)))) return FTC_EINVAL;
    if ((n + FTC_EMBED_RUN - 1) / FTC_EMBED_RUN * ((desc->H + 63) / 64) > 0x7FFFFFFFull) return FTC_ETOOLARGE;
    if (n && (!d_workspace || !aligned(d_workspace, 16) || workspace_bytes < embed_workspace(desc, n))) return FTC_EWORKSPACE;
    if ((rc = sm_count(sms)) != FTC_OK) return rc;
    EmbedArgs a{};
    a.tokens = d_tokens; a.dy = d_dy; a.dy_stride = dy_stride; a.splits = d_row_splits; a.dtable = d_dtable;
    a.n = (uint32_t)n; a.V = desc->V; a.H = desc->H; a.P = desc->P; a.k = desc->k; a.dtype = desc->dtype; a.token_bits = desc->token_bits; a.scale = desc->scale;
    a.out_floats = ((uint64_t)a.V * a.H + a.k - 1) / a.k * a.k * a.P;
    unsigned char* ws = static_cast<unsigned char*>(d_workspace);
    uint32_t** lists[5] = {&a.keys[0], &a.keys[1], &a.index[0], &a.index[1], &a.process};
    for (int i = 0; i < 5; ++i) *lists[i] = reinterpret_cast<uint32_t*>(ws + i * embed_list(n));
    a.parts = reinterpret_cast<float*>(ws + 5 * embed_list(n));
    return status(launch_embedding_backward(a, sms, static_cast<cudaStream_t>(cuda_stream)));
}

int ftc_token_logprobs(const ftc_logprob_t* desc, uint64_t rows, const void* d_logits, uint64_t stride, const void* d_tokens,
                       float* d_logprob, float* d_entropy, float* d_lse, float* d_top_logprob, int32_t* d_top_token, void* cuda_stream) {
    int rc = check_logprob(desc, rows), sms = 0;
    if (rc != FTC_OK || rows == 0) return rc;
    if (!d_logits || stride < desc->V || stride > kFar || (d_logprob && !d_tokens) || (desc->top > 0) != (d_top_logprob != nullptr) || (desc->top > 0) != (d_top_token != nullptr))
        return FTC_EINVAL;
    if (!aligned(d_logits, size_of(desc->dtype)) || !aligned(d_tokens, desc->token_bits / 8) || !aligned(d_logprob, 4) || !aligned(d_entropy, 4) || !aligned(d_lse, 4) ||
        !aligned(d_top_logprob, 4) || !aligned(d_top_token, 4)) return FTC_EINVAL;
    if (!d_logprob && !d_entropy && !d_lse && !desc->top) return FTC_OK;
    if ((rc = sm_count(sms)) != FTC_OK) return rc;
    LogprobArgs a{};
    a.logits = d_logits; a.stride = stride; a.tokens = d_tokens; a.logprob = d_logprob; a.entropy = d_entropy; a.lse = d_lse; a.top_logprob = d_top_logprob; a.top_token = d_top_token;
    a.rows = (uint32_t)rows; a.V = desc->V; a.dtype = desc->dtype; a.token_bits = desc->token_bits; a.top = desc->top; a.scale = desc->scale;
    return status(launch_token_logprobs(a, sms, static_cast<cudaStream_t>(cuda_stream)));
}

int ftc_token_logprobs_backward(const ftc_logprob_t* desc, uint64_t rows, const void* d_logits, uint64_t stride, const void* d_tokens,
                                const float* d_lse, const float* d_entropy, const float* d_dlogprob, const float* d_dentropy, void* d_dlogits,
                                uint64_t dstride, void* cuda_stream) {
    int rc = check_logprob(desc, rows), sms = 0;
    if (rc != FTC_OK || rows == 0) return rc;
    if (!d_logits || !d_dlogits || !d_lse || stride < desc->V || dstride < desc->V || stride > kFar || dstride > kFar || (d_dlogprob && !d_tokens) || (d_dentropy && !d_entropy))
        return FTC_EINVAL;
    if (d_logits == d_dlogits && stride != dstride) return FTC_EINVAL;
    const uint32_t e = size_of(desc->dtype);
    if (!aligned(d_logits, e) || !aligned(d_dlogits, e) || !aligned(d_tokens, desc->token_bits / 8) || !aligned(d_lse, 4) || !aligned(d_entropy, 4) || !aligned(d_dlogprob, 4) ||
        !aligned(d_dentropy, 4)) return FTC_EINVAL;
    if ((rc = sm_count(sms)) != FTC_OK) return rc;
    LogprobArgs a{};
    a.logits = d_logits; a.stride = stride; a.tokens = d_tokens; a.lse_in = d_lse; a.entropy_in = d_entropy; a.dlogprob = d_dlogprob; a.dentropy = d_dentropy;
    a.dlogits = d_dlogits; a.dstride = dstride;
    a.rows = (uint32_t)rows; a.V = desc->V; a.dtype = desc->dtype; a.token_bits = desc->token_bits; a.scale = desc->scale;
    return status(launch_token_logprobs_backward(a, sms, static_cast<cudaStream_t>(cuda_stream)));
}

size_t ftc_muon_plan_bytes(const ftc_matrix_t* h_matrices, uint32_t n) {
    PlanHead h;
    return count_matrices(h_matrices, n, h) ? plan_bytes(h) : 0;
}

int ftc_muon_plan_build(const ftc_matrix_t* h_matrices, uint32_t n, void* h_plan, size_t bytes) {
    PlanHead h;
    if (!count_matrices(h_matrices, n, h) || !h_plan || !aligned(h_plan, 8) || bytes < plan_bytes(h)) return FTC_EINVAL;
    std::memset(h_plan, 0, plan_bytes(h));
    *static_cast<PlanHead*>(h_plan) = h;
    PlanEntry* e = const_cast<PlanEntry*>(plan_entries(h_plan));
    uint64_t blocks = 0, x = 0, a = 0, diagonal = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const ftc_param_t& t = h_matrices[i].tensor;
        PlanEntry& q = e[i];
        q.param = t.param; q.master = t.master; q.grad = t.grad; q.status = t.status; q.n = t.n;
        q.rows = h_matrices[i].rows; q.cols = h_matrices[i].cols; q.tall = q.rows > q.cols;
        q.k = t.status ? t.k : 1; q.k_shift = q.k & (q.k - 1) ? 255 : (uint8_t)__builtin_ctz(q.k);
        q.param_dtype = (uint8_t)t.param_dtype; q.grad_dtype = (uint8_t)t.grad_dtype; q.lr_scale = t.lr_scale; q.weight_decay = t.weight_decay;
        q.m = q.tall ? q.cols : q.rows; q.w = q.tall ? q.rows : q.cols;
        q.mb = (q.m + 127) / 128; q.nb = (q.w + 63) / 64; q.kb = (q.m + 63) / 64;
        q.first_block = blocks; q.x_block = x; q.a_block = a; q.diagonal = diagonal;
        blocks += (t.n + FTC_STATE_BLOCK - 1) / FTC_STATE_BLOCK; x += (uint64_t)q.mb * q.nb; a += (uint64_t)q.mb * 2 * q.mb; diagonal += q.mb * 128;
        q.wide = aligned(t.grad, 16) && aligned(t.param, 16) && aligned(t.master, 16);
    }
    // The maps.
    uint32_t* map = reinterpret_cast<uint32_t*>(e + n);
    uint32_t* const order = map + h.items[kChunks] + h.items[kBlocks] + h.items[kGramTiles] + h.items[kApplyTiles] + h.items[kSmall];      // room for the sorting
    for (uint32_t i = 0; i < n; ++i) order[i] = i;
    for (int w = 0; w < kLists; ++w) {
        // chunks and blocks as the caller has them; tiles and small matrices: middle sizes last, those of many steps first
        if (w >= kGramTiles)
            std::sort(order, order + n, [e, w](uint32_t i, uint32_t j) {
                const bool late = plan_size(e[i].m, e[i].w) == 1, late_j = plan_size(e[j].m, e[j].w) == 1;
                const uint32_t s = w == kGramTiles ? e[i].nb : e[i].kb, s_j = w == kGramTiles ? e[j].nb : e[j].kb;
                return late != late_j ? late_j : s != s_j ? s > s_j : i < j;
            });
        uint32_t at = 0;
        for (uint32_t o = 0; o < n; ++o) {
            const uint32_t i = order[o];
            PlanEntry& q = e[i];
            const uint32_t mb2 = (q.mb + 1) / 2;
            const uint32_t count = w == kChunks ? (uint32_t)((q.n + kMuonChunk - 1) / kMuonChunk) : w == kBlocks ? q.mb * q.nb : w == kSmall ? plan_size(q.m, q.w) < 2 : plan_size(q.m, q.w) == 0 ? 0 : w == kGramTiles ? mb2 * (mb2 + 1) / 2 : mb2 * ((q.nb + 3) / 4);
            q.first[w] = at;
            for (const uint32_t end = at + count; at < end; ++at) map[at] = i;
        }
        map += at;
    }
    return FTC_OK;
}

uint64_t ftc_muon_plan_blocks(const void* h_plan) {
    const PlanHead* h = plan_of(h_plan);
    return h ? h->n_blocks : 0;
}

size_t ftc_muon_workspace_bytes(const void* h_plan, uint32_t products) {
    const PlanHead* h = plan_of(h_plan);
    return h && (products == 16 || products == 32) ? muon_layout(*h, products).total : 0;
}

int ftc_muon_step(const ftc_muon_t* hyper, const void* h_plan, const void* d_plan, float* d_momentum, const float* d_grad_scale,
                  void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
    const PlanHead* h = plan_of(h_plan);
    if (!hyper || !h || !d_plan || !aligned(d_plan, 256) || hyper->reserved || hyper->nesterov > 1) return FTC_EINVAL;
    if (!(hyper->lr >= 0) || !std::isfinite((float)hyper->lr) || !(hyper->momentum >= 0 && (float)hyper->momentum < 1.f) || !(hyper->eps >= 1e-30) ||
        !std::isfinite((float)hyper->eps) || hyper->steps == 0 || hyper->steps > 16) return FTC_EINVAL;
    if (hyper->products != 16 && hyper->products != 32) return FTC_EUNSUPPORTED;
    if (h->n == 0) return FTC_OK;
    if (!d_momentum || !aligned(d_momentum, 32) || !aligned(d_grad_scale, 4)) return FTC_EINVAL;
    const MuonLayout l = muon_layout(*h, hyper->products);
    if (!d_workspace || !aligned(d_workspace, 256) || workspace_bytes < l.total) return FTC_EWORKSPACE;
    int sms = 0, rc = sm_count(sms);
    if (rc != FTC_OK) return rc;
    unsigned char* ws = static_cast<unsigned char*>(d_workspace);
    MuonArgs a{};
    a.plan = d_plan; a.n = h->n; a.momentum = d_momentum; a.grad_scale = d_grad_scale; a.word = reinterpret_cast<uint32_t*>(ws);
    a.sums = reinterpret_cast<double2*>(ws + l.sums); a.live = reinterpret_cast<uint32_t*>(ws + l.live); a.factor = reinterpret_cast<float*>(ws + l.factor); a.written = reinterpret_cast<uint32_t*>(ws + l.written);
    a.diag_a = reinterpret_cast<float*>(ws + l.diag_a); a.diag_b = reinterpret_cast<float*>(ws + l.diag_b);
    a.x[0] = ws + l.x0; a.x[1] = ws + l.x1; a.a = ws + l.a; a.b = ws + l.b; a.x_bytes = l.x_bytes; a.a_bytes = l.a_bytes;
    const uint32_t* map = reinterpret_cast<const uint32_t*>(plan_entries(d_plan) + h->n);
    for (int w = 0; w < kLists; ++w) { a.items[w] = h->items[w]; a.maps[w] = map; map += h->items[w]; }
    if (hyper->products == 16) { a.items[kGramTiles] -= h->gram_middle; a.items[kApplyTiles] -= h->apply_middle; }
    else a.items[kSmall] -= h->middle;
    a.steps = hyper->steps; a.nesterov = hyper->nesterov; a.split = hyper->products == 32;
    a.lr = (float)hyper->lr; a.mu = (float)hyper->momentum; a.eps = (float)hyper->eps;
    return status(launch_muon(a, sms, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
