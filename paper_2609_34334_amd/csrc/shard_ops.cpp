// Entry points of the operators on a rank's shard (adamw.hip, rmsnorm.hip,
// balance.hip): validation, launch shapes and statistics.
#include "shard_ops.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <utility>
#include <vector>

#include "call.h"
#include "errors.h"
#include "hoccl_internal.h"

namespace hoccl {
namespace {

#define TRY(expr)                          \
    do {                                   \
        hoccl_status_t st_ = (expr);       \
        if (st_ != HOCCL_OK) return st_;   \
    } while (0)

template <typename... A>
hoccl_status_t invalid(const char *fmt, A... a) {
    format_error(fmt, a...);
    return HOCCL_ERR_INVALID_ARG;
}
hoccl_status_t invalid(const char *msg) {
    set_error_message(msg);
    return HOCCL_ERR_INVALID_ARG;
}

// No exception leaves a C entry point.
template <typename F>
hoccl_status_t guarded(F &&f) {
    try {
        return f();
    } catch (const std::bad_alloc &) {
        set_error_message("out of host memory");
        return HOCCL_ERR_NO_MEMORY;
    } catch (...) {
        set_error_message("unexpected host error");
        return HOCCL_ERR_INTERNAL;
    }
}

bool float_type(hoccl_dtype_t dt) { return dt == HOCCL_FP32 || dt == HOCCL_BF16; }
size_t size_of(hoccl_dtype_t dt) { return dt == HOCCL_BF16 ? 2 : 4; }

// The memory of one call's operands.  Written ones may overlap no other, but
// for the pairs that a call allows by not adding the second of them.
class Operands {
public:
    explicit Operands(size_t most = 16) { all_.reserve(most); }
    // `align`: the element size.
    hoccl_status_t add(const void *p, size_t bytes, size_t align, bool written, const char *name, long index = -1) {
        if (!p && bytes) return index < 0 ? invalid("%s is NULL", name) : invalid("%s[%ld] is NULL", name, index);
        if ((uintptr_t)p % align)
            return index < 0 ? invalid("%s is not aligned to its elements", name)
                             : invalid("%s[%ld] is not aligned to its elements", name, index);
        if (((uintptr_t)p + bytes) >> 48)
            return index < 0 ? invalid("%s ends behind the address space", name)
                             : invalid("%s[%ld] ends behind the address space", name, index);
        if (bytes) all_.push_back({(uintptr_t)p, (uintptr_t)p + bytes, written, name, index});
        return HOCCL_OK;
    }
    hoccl_status_t check() {
        std::vector<Key> order(all_.size());
        for (size_t i = 0; i < all_.size(); ++i) order[i] = {all_[i].lo, i};
        by_address(order);
        // The furthest reach of what came before, and of what is written of it.
        const Span *any = nullptr, *out = nullptr;
        for (const Key &k : order) {
            const Span &s = all_[k.span];
            const Span *bad = out && out->hi > s.lo ? out : s.written && any && any->hi > s.lo ? any : nullptr;
            if (bad)
                return invalid("%s and %s overlap (%ld, %ld)", bad->name, s.name, bad->index, s.index);
            if (!any || s.hi > any->hi) any = &s;
            if (s.written && (!out || s.hi > out->hi)) out = &s;
        }
        return HOCCL_OK;
    }

private:
    struct Span {
        uintptr_t lo, hi;
        bool written;
        const char *name;
        long index;
    };
    struct Key {
        uint64_t lo;
        size_t span;
    };
    // Many by radix, byte by byte from the lowest, without the bytes that are
    // the same everywhere (the 900 of 150 tensors: 9.5 us by comparisons, 6.5 so).
    static void by_address(std::vector<Key> &keys) {
        if (keys.size() < 64) {
            std::sort(keys.begin(), keys.end(), [](const Key &a, const Key &b) { return a.lo < b.lo; });
            return;
        }
        uint64_t differ = 0;
        for (const Key &k : keys) differ |= k.lo ^ keys[0].lo;
        std::vector<Key> other(keys.size());
        for (int shift = 0; shift < 64; shift += 8) {
            if ((differ >> shift & 0xff) == 0) continue;
            size_t at[256] = {};
            for (const Key &k : keys) ++at[k.lo >> shift & 0xff];
            size_t before = 0;
            for (size_t &n : at) before += std::exchange(n, before);
            for (const Key &k : keys) other[at[k.lo >> shift & 0xff]++] = k;
            keys.swap(other);
        }
    }
    std::vector<Span> all_;
};

bool product_fits(size_t a, size_t b, size_t c) {
    return (b == 0 || a <= SIZE_MAX / 2 / b) && (c == 0 || a * b <= SIZE_MAX / 2 / c);
}

// ---- AdamW ----------------------------------------------------------------------

hoccl_status_t check_adamw(const hoccl_adamw_t &o) {
    if (!float_type(o.param_dtype) || !float_type(o.grad_dtype))
        return invalid("parameters and gradients are fp32 or bf16");
    if (o.state_bits != 8 && o.state_bits != 32) return invalid("state_bits is 8 or 32, not %d", o.state_bits);
    if (!o.step_dev && o.step < 1) return invalid("steps count from 1, not %lld", o.step);
    if (!o.lr_dev && !(o.lr >= 0 && std::isfinite(o.lr))) return invalid("lr = %g", o.lr);
    if (!(o.beta1 >= 0 && o.beta1 < 1) || !(o.beta2 >= 0 && o.beta2 < 1))
        return invalid("betas %g, %g outside [0, 1)", o.beta1, o.beta2);
    if (!(o.eps >= 0 && std::isfinite(o.eps)) || !(o.weight_decay >= 0 && std::isfinite(o.weight_decay)))
        return invalid("eps %g or weight_decay %g negative or not finite", o.eps, o.weight_decay);
    if (o.eps > 0 && o.eps < FLT_MIN) return invalid("eps = %g is neither 0 nor a normal fp32 number", o.eps);
    if ((uintptr_t)o.lr_dev % 4 || (uintptr_t)o.step_dev % 4 || (uintptr_t)o.grad_scale % 4)
        return invalid("lr_dev, step_dev and grad_scale are 4-byte elements");
    return HOCCL_OK;
}

hoccl_status_t adamw(const hoccl_adamw_tensor_t *ts, int count, const hoccl_adamw_t *op, hipStream_t stream) {
    if (!op || count < 0 || (count > 0 && !ts)) return invalid("tensors or options are NULL, or a negative count");
    const hoccl_adamw_t &o = *op;
    TRY(check_adamw(o));
    const size_t ps = size_of(o.param_dtype), gs = size_of(o.grad_dtype), ss = o.state_bits == 8 ? 1 : 4;
    unsigned long long bytes = 0, tiles = 0;
    const uint32_t tile = adamw_tile(o.state_bits);
    Operands mem(7 * (size_t)count + 3);
    for (int i = 0; i < count; ++i) {
        const hoccl_adamw_tensor_t &t = ts[i];
        if (t.n == 0) continue;
        if (!product_fits(t.n, 8, 1)) return invalid("tensor %d: %zu elements do not fit in size_t", i, t.n);
        TRY(mem.add(t.param, t.n * ps, ps, true, "param", i));
        TRY(mem.add(t.grad, t.n * gs, gs, false, "grad", i));
        TRY(mem.add(t.exp_avg, t.n * ss, ss, true, "exp_avg", i));
        TRY(mem.add(t.exp_avg_sq, t.n * ss, ss, true, "exp_avg_sq", i));
        size_t b = t.n * (2 * ps + gs + 4 * ss);
        if (o.state_bits == 8) {
            const size_t blocks = (t.n + HOCCL_BLOCK - 1) / HOCCL_BLOCK;
            TRY(mem.add(t.exp_avg_scale, blocks * 4, 4, true, "exp_avg_scale", i));
            TRY(mem.add(t.exp_avg_sq_scale, blocks * 4, 4, true, "exp_avg_sq_scale", i));
            b += blocks * 16;
        }
        if (t.copy) {
            TRY(mem.add(t.copy, t.n * 2, 2, true, "copy", i));
            b += t.n * 2;
        }
        bytes += b;
        tiles += (t.n + tile - 1) / tile;
    }
    if (tiles == 0) return HOCCL_OK;
    if (tiles >= 1ull << 31) return invalid("more elements than one call takes");
    if (o.lr_dev) TRY(mem.add(o.lr_dev, 4, 4, false, "lr_dev"));
    if (o.step_dev) TRY(mem.add(o.step_dev, 4, 4, false, "step_dev"));
    if (o.grad_scale) TRY(mem.add(o.grad_scale, 4, 4, false, "grad_scale"));
    TRY(mem.check());

    OpCall call;
    TRY(call.open(stream));
    AdamArgs a;
    AdamStep &s = a.step;
    const double t = o.step_dev ? 1.0 : (double)o.step, lr = o.lr_dev ? 0.0 : o.lr;
    s.b1 = (float)o.beta1, s.c1 = (float)(1.0 - o.beta1);
    s.b2 = (float)o.beta2, s.c2 = (float)(1.0 - o.beta2);
    s.log_b1 = std::log(o.beta1), s.log_b2 = std::log(o.beta2);
    s.decay = (float)(1.0 - lr * o.weight_decay);
    s.rate = (float)(lr / -std::expm1(t * s.log_b1));
    s.root = (float)(1.0 / std::sqrt(-std::expm1(t * s.log_b2)));
    s.eps = (float)o.eps;
    s.lr = lr, s.weight_decay = o.weight_decay, s.t = t;
    s.lr_dev = o.lr_dev, s.t_dev = o.step_dev, s.grad_scale = o.grad_scale;
    for (int i = 0; i < count;) {
        a.nseg = 0;
        a.first[0] = 0;
        for (; i < count && a.nseg < kAdamSegs; ++i) {
            const hoccl_adamw_tensor_t &x = ts[i];
            if (x.n == 0) continue;
            a.seg[a.nseg].set({x.param, x.grad, x.exp_avg, x.exp_avg_sq, x.exp_avg_scale, x.exp_avg_sq_scale, x.copy, x.n});
            a.first[a.nseg + 1] = a.first[a.nseg] + (uint32_t)((x.n + tile - 1) / tile);
            ++a.nseg;
        }
        if (a.nseg == 0) break;
        const int wg = call.budget(a.first[a.nseg]);
        TRY(call.launch(wg, [&] { return launch_adamw(a, o.param_dtype, o.grad_dtype, o.state_bits, wg, stream); }));
    }
    call.done(bytes);
    return HOCCL_OK;
}

// ---- RMSNorm ----------------------------------------------------------------------

hoccl_status_t check_rows(size_t rows, size_t hidden, double eps, hoccl_dtype_t dt, hoccl_dtype_t wdt) {
    if (!float_type(dt) || !float_type(wdt)) return invalid("rows and weight are fp32 or bf16");
    if (hidden < 1 || hidden > kMaxHidden) return invalid("hidden = %zu outside [1, %zu]", hidden, kMaxHidden);
    if (!(eps >= 0 && std::isfinite(eps))) return invalid("eps = %g", eps);
    if (!product_fits(rows, hidden, 4)) return invalid("%zu rows of %zu do not fit in size_t", rows, hidden);
    return HOCCL_OK;
}

hoccl_status_t rmsnorm(const void *x, const void *residual, const void *weight, void *residual_out, void *y,
                       float *scale, size_t rows, size_t hidden, double eps, hoccl_dtype_t dt, hoccl_dtype_t wdt,
                       hipStream_t stream) {
    TRY(check_rows(rows, hidden, eps, dt, wdt));
    if (rows == 0) return HOCCL_OK;
    const size_t es = size_of(dt), bytes = rows * hidden * es, blocks = (hidden + HOCCL_BLOCK - 1) / HOCCL_BLOCK;
    Operands mem;
    // An output may be an input of its own size, which it then replaces.
    auto replaces = [&](const void *out) { return out == x || (out == residual && out); };
    const bool h_in = residual_out && replaces(residual_out), y_in = !scale && y && replaces(y);
    TRY(mem.add(x, bytes, es, x == residual_out || (!scale && x == y), "x"));
    if (residual && residual != x)
        TRY(mem.add(residual, bytes, es, residual == residual_out || (!scale && residual == y), "residual"));
    TRY(mem.add(weight, hidden * size_of(wdt), size_of(wdt), false, "weight"));
    if (residual_out && !h_in) TRY(mem.add(residual_out, bytes, es, true, "residual_out"));
    if (y && y == residual_out) return invalid("y and residual_out are the same buffer");
    if (!y_in) TRY(mem.add(y, scale ? rows * hidden : bytes, scale ? 1 : es, true, "y"));
    if (scale) TRY(mem.add(scale, rows * blocks * 4, 4, true, "scale"));
    TRY(mem.check());

    OpCall call;
    TRY(call.open(stream));
    const RmsArgs a = {x, residual, weight, residual_out, y, scale, rows, (uint32_t)hidden, wdt == HOCCL_BF16, (float)eps, 0};
    const unsigned long long moved = (unsigned long long)bytes * (1 + (residual != nullptr) + (residual_out != nullptr)) +
                                     (scale ? rows * (hidden + blocks * 4) : bytes) + hidden * size_of(wdt);
    const int wg = call.budget(rmsnorm_workgroups(rows, hidden, dt, call.cus()));
    TRY(call.launch(wg, [&] { return launch_rmsnorm(a, dt, moved, wg, stream); }));
    call.done(moved);
    return HOCCL_OK;
}

hoccl_status_t rmsnorm_backward(const void *dy, const void *dres, const void *h, const void *weight, void *dx,
                                float *dweight, void *workspace, size_t workspace_bytes, size_t rows, size_t hidden,
                                double eps, hoccl_dtype_t dt, hoccl_dtype_t wdt, hipStream_t stream) {
    TRY(check_rows(rows, hidden, eps, dt, wdt));
    if (rows == 0 && !dweight) return HOCCL_OK;
    const size_t es = size_of(dt), bytes = rows * hidden * es;
    const uint32_t blocks = rmsnorm_backward_blocks(rows, hidden, dt);
    const size_t need = dweight ? (size_t)blocks * hidden * 4 : 0;
    if (workspace_bytes < need)
        return invalid("a workspace of %zu bytes where %zu are needed", workspace_bytes, need);
    Operands mem;
    // Inputs may be the same buffer, and dx one of them; a NULL, which dres may
    // be, is no buffer.
    auto is = [](const void *a, const void *b) { return a && a == b; };
    TRY(mem.add(dy, bytes, es, is(dy, dx), "dy"));
    if (dres && !is(dres, dy)) TRY(mem.add(dres, bytes, es, is(dres, dx), "dresidual"));
    if (!is(h, dy) && !is(h, dres)) TRY(mem.add(h, bytes, es, is(h, dx), "h"));
    TRY(mem.add(weight, hidden * size_of(wdt), size_of(wdt), false, "weight"));
    if (!is(dx, dy) && !is(dx, dres) && !is(dx, h)) TRY(mem.add(dx, bytes, es, true, "dx"));
    if (dweight) TRY(mem.add(dweight, hidden * 4, 4, true, "dweight"));
    TRY(mem.add(workspace, need, 4, true, "workspace"));
    TRY(mem.check());

    OpCall call;
    TRY(call.open(stream));
    if (rows > 0) {
        const RmsBackArgs a = {dy, dres, h, weight, dx, dweight ? (float *)workspace : nullptr, rows, (uint32_t)hidden,
                               blocks, wdt == HOCCL_BF16, (float)eps, 0};
        const int wg = call.budget(blocks);
        TRY(call.launch(wg, [&] { return launch_rmsnorm_backward(a, dt, wg, stream); }));
    }
    if (dweight) {
        const int wg = call.budget(rmsnorm_grad_workgroups(hidden));
        TRY(call.launch(wg, [&] {
            return launch_rmsnorm_weight_grad((const float *)workspace, blocks, (uint32_t)hidden, dweight, wg, stream);
        }));
    }
    call.done((unsigned long long)bytes * (dres ? 4 : 3) + hidden * size_of(wdt) + (dweight ? hidden * 4 : 0));
    return HOCCL_OK;
}

// ---- balance loss --------------------------------------------------------------------

hoccl_status_t check_balance(const hoccl_balance_t *op, const size_t *tokens, int batches) {
    if (!op) return invalid("options are NULL");
    const hoccl_balance_t &o = *op;
    if (batches < 1 || batches > kMaxBatches) return invalid("%d batches outside [1, %d]", batches, kMaxBatches);
    if (o.logits_dtype != HOCCL_FP32 && o.logits_dtype != HOCCL_BF16) return invalid("logits are fp32 or bf16");
    if (o.index_bytes != 4 && o.index_bytes != 8) return invalid("choices take 4 or 8 bytes, not %d", o.index_bytes);
    if (o.experts < 1 || o.experts > kMaxExperts) return invalid("%d experts outside [1, %d]", o.experts, kMaxExperts);
    if (o.topk < 1 || o.topk > kMaxTopk) return invalid("topk = %d outside [1, %d]", o.topk, kMaxTopk);
    if (o.ranks < 1 || o.ranks > kMaxRanks || o.experts % o.ranks)
        return invalid("%d ranks outside [1, %d], or they do not divide %d experts", o.ranks, kMaxRanks, o.experts);
    if (o.max_ranks < 0) return invalid("max_ranks = %d", o.max_ranks);
    if (!std::isfinite(o.expert_weight) || !std::isfinite(o.rank_weight) || !std::isfinite(o.traffic_weight))
        return invalid("a weight of the loss is not finite");
    if (!tokens) return invalid("tokens is NULL");
    for (int b = 0; b < batches; ++b)
        // Counts are 32-bit integers.
        if (tokens[b] >= ((size_t)1 << 31) / (size_t)o.topk) return invalid("batch %d: %zu tokens are too many", b, tokens[b]);
    return HOCCL_OK;
}

size_t balance_workspace(const hoccl_balance_t &o, const size_t *tokens, int batches) {
    uint32_t first[kMaxBatches + 1];
    balance_blocks(tokens, o.experts, o.logits_dtype, batches, first);
    if (balance_is_one(first, batches)) return 0;
    return (size_t)first[batches] * (size_t)balance_columns(o.experts, o.ranks) * 4;
}

// The operands that both directions have.
hoccl_status_t fill_balance(const hoccl_balance_t &o, const void *const *logits, const void *const *choices,
                            const size_t *tokens, int batches, Operands &mem, BalanceArgs &a, unsigned long long &bytes) {
    if (!logits || !choices) return invalid("the arrays of logits and choices must not be NULL");
    std::memset(&a, 0, sizeof a);
    const size_t es = size_of(o.logits_dtype);
    for (int b = 0; b < batches; ++b) {
        const size_t n = tokens[b] * (size_t)o.experts * es, m = tokens[b] * (size_t)o.topk * (size_t)o.index_bytes;
        TRY(mem.add(logits[b], n, es, false, "logits", b));
        TRY(mem.add(choices[b], m, (size_t)o.index_bytes, false, "choices", b));
        a.seg[b].logits = logits[b];
        a.seg[b].experts = choices[b];
        a.seg[b].tokens = tokens[b];
        bytes += n + m;
    }
    a.nseg = batches;
    a.E = o.experts, a.k = o.topk, a.D = o.ranks;
    a.index64 = o.index_bytes == 8;
    // 2^21 over the experts of a rank, rounded up: e times it is off by less
    // than 2^10, which keeps e / experts-of-a-rank exact below 1024.
    const uint32_t per = (uint32_t)(o.experts / o.ranks);
    a.rank_mul = ((1u << 21) + per - 1) / per;
    const int max_ranks = o.max_ranks > 0 ? o.max_ranks : std::min(o.topk, o.ranks);
    a.expert_scale = o.expert_weight * o.experts / o.topk;
    a.rank_scale = o.rank_weight * o.experts / ((double)o.topk * per);
    a.traffic_scale = o.traffic_weight * o.ranks / max_ranks;
    return HOCCL_OK;
}

hoccl_status_t balance_loss(const void *const *logits, const void *const *choices, const size_t *tokens, int batches,
                            const hoccl_balance_t *op, float *loss, int32_t *expert_tokens, int32_t *rank_tokens,
                            float *coef, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    TRY(check_balance(op, tokens, batches));
    const hoccl_balance_t &o = *op;
    const size_t need = balance_workspace(o, tokens, batches), nb = (size_t)batches;
    if (workspace_bytes < need)
        return invalid("a workspace of %zu bytes where %zu are needed", workspace_bytes, need);
    Operands mem;
    BalanceArgs a;
    unsigned long long bytes = 0;
    TRY(fill_balance(o, logits, choices, tokens, batches, mem, a, bytes));
    TRY(mem.add(loss, nb * 4, 4, true, "loss"));
    TRY(mem.add(expert_tokens, nb * (size_t)o.experts * 4, 4, true, "expert_tokens"));
    TRY(mem.add(rank_tokens, nb * (size_t)o.ranks * 4, 4, true, "rank_tokens"));
    TRY(mem.add(coef, nb * (size_t)o.experts * 4, 4, true, "coef"));
    TRY(mem.add(workspace, need, 4, true, "workspace"));
    TRY(mem.check());
    balance_blocks(tokens, o.experts, o.logits_dtype, batches, a.first);
    a.partial = (int32_t *)workspace;
    a.loss = loss, a.expert_tokens = expert_tokens, a.rank_tokens = rank_tokens, a.coef = coef;

    OpCall call;
    TRY(call.open(stream));
    const int wg = call.budget(a.first[batches]);
    TRY(call.launch(wg, [&] { return launch_balance(a, o.logits_dtype, wg, stream); }));
    if (!balance_is_one(a.first, batches)) {
        const int fwg = call.budget((unsigned long long)batches);
        TRY(call.launch(fwg, [&] { return launch_balance_finish(a, fwg, stream); }));
    }
    call.done(bytes + nb * 4 * (size_t)(1 + 2 * o.experts + o.ranks));
    return HOCCL_OK;
}

hoccl_status_t balance_backward(const void *const *logits, const void *const *choices, const size_t *tokens,
                                int batches, const hoccl_balance_t *op, const float *coef, const float *dloss,
                                void *const *dlogits, hipStream_t stream) {
    TRY(check_balance(op, tokens, batches));
    const hoccl_balance_t &o = *op;
    if (!dlogits) return invalid("the array of dlogits must not be NULL");
    Operands mem;
    BalanceArgs a;
    unsigned long long bytes = 0;
    TRY(fill_balance(o, logits, choices, tokens, batches, mem, a, bytes));
    const size_t nb = (size_t)batches, es = size_of(o.logits_dtype);
    TRY(mem.add(coef, nb * (size_t)o.experts * 4, 4, false, "coef"));
    if (dloss) TRY(mem.add(dloss, nb * 4, 4, false, "dloss"));
    unsigned long long blocks = 0;
    for (int b = 0; b < batches; ++b) {
        const size_t n = tokens[b] * (size_t)o.experts * es;
        TRY(mem.add(dlogits[b], n, es, true, "dlogits", b));
        a.seg[b].dlogits = dlogits[b];
        bytes += n;
        blocks += balance_backward_blocks(tokens[b], o.experts, o.logits_dtype);
        a.first[b + 1] = (uint32_t)blocks;
    }
    TRY(mem.check());
    a.coef = (float *)coef;
    a.grad = dloss;
    OpCall call;
    TRY(call.open(stream));
    const int wg = call.budget(blocks);
    TRY(call.launch(wg, [&] { return launch_balance_backward(a, o.logits_dtype, wg, stream); }));
    call.done(bytes + nb * 4 * (size_t)o.experts);
    return HOCCL_OK;
}

}  // namespace
}  // namespace hoccl

using namespace hoccl;

extern "C" {

hoccl_status_t hoccl_adamw(const hoccl_adamw_tensor_t *tensors, int count, const hoccl_adamw_t *options,
                           hipStream_t stream) {
    return guarded([&] { return adamw(tensors, count, options, stream); });
}

hoccl_status_t hoccl_rmsnorm(const void *x, const void *residual, const void *weight, void *residual_out, void *y,
                             float *scale, size_t rows, size_t hidden, double eps, hoccl_dtype_t dtype,
                             hoccl_dtype_t weight_dtype, hipStream_t stream) {
    return guarded([&] {
        return rmsnorm(x, residual, weight, residual_out, y, scale, rows, hidden, eps, dtype, weight_dtype, stream);
    });
}

hoccl_status_t hoccl_rmsnorm_backward_workspace(size_t rows, size_t hidden, hoccl_dtype_t dtype, size_t *bytes) {
    return guarded([&]() -> hoccl_status_t {
        if (!bytes) return invalid("bytes must not be NULL");
        TRY(check_rows(rows, hidden, 0.0, dtype, dtype));
        *bytes = (size_t)rmsnorm_backward_blocks(rows, hidden, dtype) * hidden * 4;
        return HOCCL_OK;
    });
}

hoccl_status_t hoccl_rmsnorm_backward(const void *dy, const void *dresidual, const void *h, const void *weight,
                                      void *dx, float *dweight, void *workspace, size_t workspace_bytes, size_t rows,
                                      size_t hidden, double eps, hoccl_dtype_t dtype, hoccl_dtype_t weight_dtype,
                                      hipStream_t stream) {
    return guarded([&] {
        return rmsnorm_backward(dy, dresidual, h, weight, dx, dweight, workspace, workspace_bytes, rows, hidden, eps,
                                dtype, weight_dtype, stream);
    });
}

hoccl_status_t hoccl_balance_workspace(const size_t *tokens, int batches, const hoccl_balance_t *options,
                                       size_t *bytes) {
    return guarded([&]() -> hoccl_status_t {
        if (!bytes) return invalid("bytes must not be NULL");
        TRY(check_balance(options, tokens, batches));
        *bytes = balance_workspace(*options, tokens, batches);
        return HOCCL_OK;
    });
}

hoccl_status_t hoccl_balance_loss(const void *const *logits, const void *const *choices, const size_t *tokens,
                                  int batches, const hoccl_balance_t *options, float *loss, int32_t *expert_tokens,
                                  int32_t *rank_tokens, float *coef, void *workspace, size_t workspace_bytes,
                                  hipStream_t stream) {
    return guarded([&] {
        return balance_loss(logits, choices, tokens, batches, options, loss, expert_tokens, rank_tokens, coef,
                            workspace, workspace_bytes, stream);
    });
}

hoccl_status_t hoccl_balance_loss_backward(const void *const *logits, const void *const *choices,
                                           const size_t *tokens, int batches, const hoccl_balance_t *options,
                                           const float *coef, const float *dloss, void *const *dlogits,
                                           hipStream_t stream) {
    return guarded([&] {
        return balance_backward(logits, choices, tokens, batches, options, coef, dloss, dlogits, stream);
    });
}

}  // extern "C"
