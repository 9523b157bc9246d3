// The operators that a training step runs on a rank's shard between two
// collectives: argument structs and launchers of adamw.hip, rmsnorm.hip and
// balance.hip.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

#include "../../include/hoccl.h"

namespace hoccl {

constexpr int kOpThreads = 256;  // per workgroup, of every kernel but the wide rows of rmsnorm.hip

// ---- AdamW ------------------------------------------------------------------

struct AdamTensor {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    void *copy;
    uint64_t n;
};
// The same in 48 bits a word, which holds a user's address and any n of a call
// (fewer than 2^31 tiles): 76 tensors fit into the 4 KiB of a launch's arguments instead
// of 60.
struct AdamSeg {
    uint32_t lo[8], hi[4];  // hi: bits 32 to 47 of two words each
    void set(const AdamTensor &t) {
        const uint64_t w[8] = {(uint64_t)t.param, (uint64_t)t.grad,    (uint64_t)t.m,    (uint64_t)t.v,
                               (uint64_t)t.m_scale, (uint64_t)t.v_scale, (uint64_t)t.copy, t.n};
        for (int i = 0; i < 8; ++i) lo[i] = (uint32_t)w[i];
        for (int i = 0; i < 4; ++i) hi[i] = (uint32_t)(w[2 * i] >> 32) | (uint32_t)(w[2 * i + 1] >> 32) << 16;
    }
};

struct AdamStep {
    float b1, c1, b2, c2;            // beta1, 1 - beta1, beta2, 1 - beta2
    float decay, rate, root, eps;    // 1 - lr wd, lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    double lr, weight_decay, log_b1, log_b2, t;  // where lr or t is on the device
    const float *lr_dev;
    const int32_t *t_dev;
    const float *grad_scale;
};
// One launch's tensors.  first[i] is the tile at which tensor i starts.
template <int CAP>
struct AdamArgsT {
    AdamSeg seg[CAP];
    uint32_t first[CAP + 1];
    int nseg;
    AdamStep step;
};
constexpr int kAdamSegs = 76;
constexpr int kAdamFewSegs = 8;
using AdamArgs = AdamArgsT<kAdamSegs>;
static_assert(sizeof(AdamArgs) <= 4096, "the arguments of a launch");

uint32_t adamw_tile(int state_bits);  // elements of one tile
hipError_t launch_adamw(const AdamArgs &a, hoccl_dtype_t param, hoccl_dtype_t grad, int state_bits, int wg,
                        hipStream_t s);

// ---- RMSNorm -----------------------------------------------------------------

constexpr size_t kMaxHidden = 32768;

struct RmsArgs {
    const void *x, *residual, *weight;
    void *residual_out, *y;   // y: T, or e4m3 bytes with `scale`
    float *scale;
    uint64_t rows;
    uint32_t hidden;
    int weight_bf16;
    float eps;
    uint32_t threads;         // of a row; set at the launch
};
struct RmsBackArgs {
    const void *dy, *dres, *h, *weight;
    void *dx;
    float *partial;           // [blocks][hidden], or null: no weight gradient
    uint64_t rows;
    uint32_t hidden, blocks;
    int weight_bf16;
    float eps;
    uint32_t threads;         // of a row; set at the launch
};

// Workgroups of the automatic launch.
unsigned long long rmsnorm_workgroups(size_t rows, size_t hidden, hoccl_dtype_t dt, int cus);
// `bytes`: what the call moves.
hipError_t launch_rmsnorm(RmsArgs a, hoccl_dtype_t dt, unsigned long long bytes, int wg, hipStream_t s);
// Partial sums of the weight's gradient: a number that goes by the sizes
// alone, so that the result does not depend on the workgroups.
uint32_t rmsnorm_backward_blocks(size_t rows, size_t hidden, hoccl_dtype_t dt);
hipError_t launch_rmsnorm_backward(RmsBackArgs a, hoccl_dtype_t dt, int wg, hipStream_t s);
uint32_t rmsnorm_grad_workgroups(size_t hidden);
hipError_t launch_rmsnorm_weight_grad(const float *partial, uint32_t blocks, uint32_t hidden, float *dweight, int wg,
                                      hipStream_t s);

// ---- balance loss -------------------------------------------------------------

constexpr int kMaxExperts = 1024;
constexpr int kMaxTopk = 64;
constexpr int kMaxBatches = 64;

struct BalanceSeg {
    const void *logits;
    const void *experts;
    void *dlogits;
    uint64_t tokens;
};
struct BalanceArgs {
    BalanceSeg seg[kMaxBatches];
    uint32_t first[kMaxBatches + 1];  // first block of each batch
    int nseg, E, k, D;
    int index64;
    uint32_t rank_mul;     // e * rank_mul >> 21 is the rank of expert e < 1024
    int32_t *partial;      // [blocks][balance_columns]: sums of p (floats), choices, tokens a rank, tokens
    float *loss;           // [nseg]
    int32_t *expert_tokens, *rank_tokens;  // [nseg][E], [nseg][D]
    float *coef;           // [nseg][E]
    const float *grad;     // [nseg] or null
    // w times the tokens: of a choice, of a choice of the rank's, of a token
    // that goes to the rank.
    double expert_scale, rank_scale, traffic_scale;
};

// Words of a block's sums: E of p, E + D + 1 counts, and up to four's multiple.
constexpr int balance_columns(int E, int D) { return (2 * E + D + 1 + 3) & ~3; }
// Fills first[0 .. batches] with the blocks of the forward pass, a division
// that goes by the sizes alone.
void balance_blocks(const size_t *tokens, int E, hoccl_dtype_t dt, int batches, uint32_t *first);
// Whether every batch is one workgroup's: it then finishes it as well, and
// needs no workspace.
inline bool balance_is_one(const uint32_t *first, int batches) { return first[batches] == (uint32_t)batches; }
hipError_t launch_balance(const BalanceArgs &a, hoccl_dtype_t dt, int wg, hipStream_t s);
hipError_t launch_balance_finish(const BalanceArgs &a, int wg, hipStream_t s);
uint32_t balance_backward_blocks(size_t tokens, int E, hoccl_dtype_t dt);
hipError_t launch_balance_backward(const BalanceArgs &a, hoccl_dtype_t dt, int wg, hipStream_t s);

}  // namespace hoccl
