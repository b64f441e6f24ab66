// Shared by the operators at the two ends of a language model and of its matrices' update.
#pragma once
#include "ftc_train.cuh"

namespace ftc {

struct EmbedArgs {
    const void *tokens, *table, *dy;
    void* y;
    const uint64_t* splits;
    float* dtable;
    uint32_t *keys[2], *index[2], *process;      // the sorted tokens and their positions (two sides of the passes), their processes
    float* parts;                                // [chunks][2][H]: sums of runs that leave their chunk
    uint64_t table_stride, y_stride, dy_stride, out_floats;
    uint32_t n, V, H, P, k, dtype, wdtype, token_bits, k_shift, k_inverse;       // k = 2^k_shift, or 32; ceil(2^32 / k), as 32 bits
    float scale;
};
cudaError_t launch_embedding_forward(const EmbedArgs& a, int sms, cudaStream_t st);
cudaError_t launch_embedding_backward(const EmbedArgs& a, int sms, cudaStream_t st);

struct LogprobArgs {
    const void *logits, *tokens;
    float *logprob, *entropy, *lse, *top_logprob;
    int32_t* top_token;
    const float *lse_in, *entropy_in, *dlogprob, *dentropy;
    void* dlogits;
    uint64_t stride, dstride;
    uint32_t rows, V, dtype, token_bits, top;
    float scale;
};
cudaError_t launch_token_logprobs(const LogprobArgs& a, int sms, cudaStream_t st);
cudaError_t launch_token_logprobs_backward(const LogprobArgs& a, int sms, cudaStream_t st);

// Token i, or -1 where it is not in 0 .. V-1.
__device__ __forceinline__ int32_t token_at(const void* tokens, uint32_t bits, uint64_t i, uint32_t V) {
    if (bits == 64) {
        const uint64_t t = static_cast<const uint64_t*>(tokens)[i];
        return t < V ? (int32_t)t : -1;
    }
    const uint32_t t = static_cast<const uint32_t*>(tokens)[i];
    return t < V ? (int32_t)t : -1;
}

// ---- the plan of matrices: header, entries, then the matrix of each chunk, block and tile ----

constexpr uint64_t kPlanMagic = 0x316E4C5054435446ull;
constexpr uint32_t kMuonChunk = 4096;                            // elements of a block of the momentum kernel
enum { kChunks, kBlocks, kGramTiles, kApplyTiles, kSmall, kLists };    // kSmall: matrices that one block takes through all steps
// Matrices of at most 128 x 256 are small; of at most 128 x 512 where operands are one number each. The latter come last in the lists.
inline uint32_t plan_size(uint64_t m, uint64_t w) { return m <= 128 && w <= 256 ? 0 : m <= 128 && w <= 512 ? 1 : 2; }
struct PlanHead { uint64_t magic, n_blocks, a_blocks, diagonals; uint32_t items[kLists], n, middle, gram_middle, apply_middle, pad; };     // ..middle: matrices and tiles of size 1, the lists' last
struct PlanEntry {
    void* param; float* master; const void* grad; const uint32_t* status;
    uint64_t n, first_block, x_block, a_block, diagonal;         // x_block, a_block: in blocks of 128 x 64 float16; diagonal: in numbers
    uint32_t k, rows, cols;
    uint8_t param_dtype, grad_dtype, tall, k_shift;
    float lr_scale, weight_decay;
    uint32_t m, w, mb, nb, kb, wide;                             // X is m x w (m <= w): mb blocks of 128 rows, nb of 64 columns; A: kb of 64 columns. wide: addresses allow eights
    uint32_t first[kLists];                                      // where its chunks, blocks, tiles begin
    uint32_t pad;
};
static_assert(sizeof(PlanHead) == 72 && sizeof(PlanEntry) == 144, "plan layout");
__host__ __device__ inline const PlanEntry* plan_entries(const void* p) {
    return reinterpret_cast<const PlanEntry*>(static_cast<const char*>(p) + sizeof(PlanHead));
}

struct MuonArgs {
    const void* plan; const uint32_t* maps[kLists]; uint32_t n;
    float* momentum; const float* grad_scale;
    uint32_t* word;                              // first of the workspace: not 0 once a wait has given up
    double2* sums; uint32_t* live; float* factor; // [chunks]: squares of U, messages delivered; [n]: was anything delivered, 2^14 / (|U| + eps)
    float *diag_a, *diag_b; uint32_t* written;            // [3][n]: warps' parts of tiles that have been written, by product
    unsigned char *x[2], *a, *b;                 // blocks of 128 x 64 float16; with two numbers for each, the low ones x_bytes / a_bytes further on
    uint64_t x_bytes, a_bytes;
    uint32_t items[kLists], steps, nesterov, split;
    float lr, mu, eps;
};
cudaError_t launch_muon(const MuonArgs& a, int sms, cudaStream_t st);

}  // namespace ftc
