"""The operators on a rank's shard between the collectives they belong to:
a sharded data-parallel step, the norm of sequence parallelism and an
expert-parallel dispatch, over virtual ranks."""
import concurrent.futures
import math

import pytest
import torch

import paper_2609_34334_amd as hc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def randn(seed, *shape, dt=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dt)


@pytest.mark.parametrize("bits", [32, 8])
def test_sharded_steps(bits):
    """reduce-scatter of bf16 gradients -> AdamW on each rank's fp32 shard
    -> all-gather of the bf16 copies, three steps, every rank's shard one
    tensor of the same call."""
    R, n = 4, 3001
    whole = randn(1, R * n, scale=0.1)
    shards = [whole[r * n:(r + 1) * n].clone() for r in range(R)]
    state = hc.adamw_state(shards, bits=bits)
    copies = [torch.empty(n, dtype=torch.bfloat16, device="cuda") for _ in range(R)]
    m = v = torch.zeros(R * n, dtype=torch.float64, device="cuda")
    p = whole.double()
    lr, (b1, b2), decay = 1e-2, (0.9, 0.99), 0.1
    for step in (1, 2, 3):
        grads = [randn(10 * step + r, R * n, dt=torch.bfloat16) for r in range(R)]
        mine = hc.reduce_scatter(grads)
        hc.adamw(shards, mine, *state, step=step, lr=lr, betas=(b1, b2), weight_decay=decay, copies=copies,
                 grad_scale=torch.tensor([1 / R], device="cuda"))
        full = hc.allgather(copies)
        torch.cuda.synchronize()
        for f in full[1:]:
            assert torch.equal(f, full[0])
        got = torch.cat(shards)
        assert torch.equal(full[0], got.bfloat16())
        # the formulas in 64 bits on the reduced gradients
        g = torch.cat(mine).double() / R
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        p = p * (1 - lr * decay) - lr * (m / (1 - b1 ** step)) / ((v / (1 - b2 ** step)).sqrt() + 1e-8)
        if bits == 32 or step == 1:      # later 8-bit steps start from rounded states
            # each step: 4 roundings of the parameter, about 20 of the update, of at most lr / sqrt(1 - b2) or so
            assert ((got.double() - p).abs() <= step * (4 * U * (p.abs() + 0.2) + 40 * U * lr * 10)).all()
        else:
            # m to 2^-4 of its block's largest part by part, the root to 2^-4 and its floor: the update
            # stays within a small multiple of lr
            assert ((got.double() - p).abs() <= step * 12 * lr).all()


def test_sharded_8bit_steps_from_what_each_finds():
    """The same with 8-bit states, every step against the formulas in 64 bits
    from the states that the step before has left: to the roundings of fp32."""
    R, n = 4, 3001
    whole = randn(1, R * n, scale=0.1)
    shards = [whole[r * n:(r + 1) * n].clone() for r in range(R)]
    state = hc.adamw_state(shards, bits=8)
    copies = [torch.empty(n, dtype=torch.bfloat16, device="cuda") for _ in range(R)]
    lr, (b1, b2), decay, eps = 1e-2, (0.9, 0.99), 0.1, 1e-8

    def held(codes, scales):
        each = [s.repeat_interleave(128)[:n] for s in scales]
        return torch.cat([q.float() * s for q, s in zip(codes, each)])

    for step in range(1, 6):
        p, m, root = torch.cat(shards).double(), held(state[0], state[2]).double(), held(state[1], state[3])
        v = (root * root).double()                       # as the kernel takes it, in fp32
        mine = hc.reduce_scatter([randn(10 * step + r, R * n, dt=torch.bfloat16) for r in range(R)])
        hc.adamw(shards, mine, *state, step=step, lr=lr, betas=(b1, b2), eps=eps, weight_decay=decay, copies=copies,
                 grad_scale=torch.tensor([1 / R], device="cuda"))
        torch.cuda.synchronize()
        g = torch.cat(mine).double() / R
        m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        den, rate = v1.sqrt() / math.sqrt(1 - b2 ** step) + eps, lr / (1 - b1 ** step)
        want = p * (1 - lr * decay) - rate * m1 / den
        # m: scale and product, beta, its product and the sum; the update: rate, its product, root (half of v's 6.1,
        # and 1), factor, product, eps and sum, reciprocal and product, last difference; the parameter: 1 - lr wd, product, sum
        err_m = 4.1 * U * (b1 * m.abs() + (1 - b1) * g.abs())
        err = 3.1 * U * p.abs() + 13.1 * U * (rate * m1 / den).abs() + rate * err_m / den + 1e-30
        got = torch.cat(shards)
        assert ((got.double() - want).abs() <= err).all(), step
        assert torch.equal(torch.cat(copies), got.bfloat16())
        # the states that it leaves: half a step of e4m3, and the root's floor
        for x, codes, scales, floor in ((m1, state[0], state[2], 0.0), (v1.sqrt(), state[1], state[3], 2.0 ** -9)):
            each = torch.cat([s.repeat_interleave(128)[:n] for s in scales]).double()
            now = held(codes, scales).double()
            assert ((now - x).abs() <= (2.0 ** -4 + 20 * U) * x.abs() + (2.0 ** -10 + floor) * each + err_m).all(), step


def test_sequence_parallel_norm():
    """reduce-scatter of partial outputs -> residual + RMS norm in 8 bits on
    each rank's rows -> all-gather of the bytes and of the scales; the
    gradients the other way round."""
    R, rows, H = 4, 24, 1000
    partial = [randn(r, R * rows * H, dt=torch.bfloat16) for r in range(R)]
    residual = [randn(20 + r, rows, H, dt=torch.bfloat16) for r in range(R)]
    w = randn(30, H)
    mine = [t.view(rows, H) for t in hc.reduce_scatter(partial)]
    q, s, h = [], [], []
    for r in range(R):
        (a, b), c = hc.rmsnorm(mine[r], w, residual[r], quantize=True)
        q.append(a)
        s.append(b)
        h.append(c)
    bytes_ = hc.allgather([t.view(torch.uint8).flatten() for t in q])
    scales = hc.allgather([t.flatten() for t in s])
    torch.cuda.synchronize()
    want_h = torch.cat([(a.float() + b.float()).bfloat16() for a, b in zip(mine, residual)])
    assert torch.equal(torch.cat(h), want_h)
    d = want_h.double()
    want = d / (d.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
    for r in range(R):
        got = bytes_[r].view(torch.float8_e4m3fn).view(R * rows, H).double()
        each = scales[r].view(R * rows, 8).double().repeat_interleave(128, -1)[:, :H]
        assert ((got * each - want).abs() <= (2.0 ** -4 + 100 * U) * want.abs() + 2.0 ** -10 * each).all()
    # backward: every rank's gradient of the gathered rows summed to its owner, then the norm's
    up = [randn(40 + r, R * rows * H, dt=torch.bfloat16, scale=0.1) for r in range(R)]
    dy = [t.view(rows, H) for t in hc.reduce_scatter(up)]
    dx, dw = zip(*[hc.rmsnorm_backward(dy[r], h[r], w) for r in range(R)])
    total = hc.allreduce([t.clone() for t in dw])
    torch.cuda.synchronize()
    gw = torch.cat(dy).double() * w.double()
    rms = (d.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    exact = (gw - d * (gw * d).mean(-1, keepdim=True) / rms ** 2) / rms
    big = (gw.abs() + d.abs() * (gw * d).abs().mean(-1, keepdim=True) / rms ** 2) / rms
    assert ((torch.cat(dx).double() - exact).abs() <= 200 * U * big + 2.0 ** -8 * (exact.abs() + 200 * U * big)).all()
    terms = torch.cat(dy).double() * d / rms
    assert ((total[0].double() - terms.sum(0)).abs() <= 150 * U * terms.abs().sum(0)).all()


def test_expert_parallel_dispatch():
    """Router logits -> balance loss and counts -> all-to-all(v) by those
    counts -> the loss's gradient."""
    import workloads as W
    R, T, E, k, hidden = 4, 96, 16, 2, 64
    logits = [randn(r, T, E) for r in range(R)]
    experts = [x.topk(k, -1).indices for x in logits]
    out = hc.balance_loss(logits, experts, R, expert_weight=0.01, traffic_weight=0.02)
    counts = (out.rank_tokens.cpu().long() * hidden).flatten().tolist()
    tokens, plan, sd, rd = W.a2a_plan([e.cpu().numpy() for e in experts], R, E, hidden)
    assert counts == plan
    acts = [randn(50 + r, T, hidden, dt=torch.bfloat16) for r in range(R)]
    send = [torch.cat([acts[s][torch.from_numpy(tokens[s][d]).cuda()] for d in range(R)]).flatten() for s in range(R)]
    recv = [torch.zeros(sum(counts[s * R + d] for s in range(R)), dtype=torch.bfloat16, device="cuda") for d in range(R)]
    hc.alltoallv(send, counts, sd, recv, rd)
    grads = hc.balance_loss_backward(logits, experts, out.coef)
    torch.cuda.synchronize()
    for d in range(R):
        want = torch.cat([acts[s][torch.from_numpy(tokens[s][d]).cuda()] for s in range(R)])
        assert torch.equal(recv[d].view(-1, hidden), want)
    for x, e, g, loss in zip(logits, experts, grads, out.loss):
        z = x.double().requires_grad_()
        p = torch.softmax(z, -1).mean(0)
        f = torch.zeros(E, dtype=torch.float64, device="cuda").index_add_(
            0, e.flatten(), torch.ones(T * k, dtype=torch.float64, device="cuda")) * E / (k * T)
        sent = torch.zeros(T, R, device="cuda").scatter_(1, e // (E // R), 1.0).sum(0).double() * R / (min(k, R) * T)
        want = (0.01 * f * p).sum() + 0.02 * (sent * p.view(R, -1).sum(1)).sum()
        want.backward()
        # tokens' softmax to about 100 roundings each, of terms as large as the loss over the tokens
        assert abs(loss.double() - want) <= 300 * U * want
        assert ((g.double() - z.grad).abs() <= 300 * U * float(want.detach()) / T).all()


def test_threads_with_streams_of_their_own():
    """Four host threads call the operators at once, each on its own stream
    and tensors: the results are those of one after another."""
    def work(seed, stream):
        x, r, w = randn(seed, 300, 1000, dt=torch.bfloat16), randn(seed + 1, 300, 1000, dt=torch.bfloat16), randn(seed + 2, 1000)
        p, g = [randn(seed + k, 700 * k + 1) for k in range(1, 20)], [randn(seed - k, 700 * k + 1) for k in range(1, 20)]
        logits = [randn(seed + 7, 900, 64), randn(seed + 8, 333, 64)]
        experts = [t.topk(4, -1).indices for t in logits]
        states = hc.adamw_state(p, bits=8)
        torch.cuda.synchronize()
        for step in range(1, 21):
            y, h = hc.rmsnorm(x, w, r, stream=stream)
            dx, dw = hc.rmsnorm_backward(y, h, w, stream=stream)
            hc.adamw(p, g, *states, step=step, lr=1e-2, stream=stream)
            b = hc.balance_loss(logits, experts, 8, rank_weight=0.1, stream=stream)
            d = hc.balance_loss_backward(logits, experts, b.coef, stream=stream)
        stream.synchronize()
        return [y, h, dx, dw, *p, *(t.view(torch.uint8) for s in states[:2] for t in s), *b, *d]

    seeds = [1000, 2000, 3000, 4000]
    alone = [work(s, torch.cuda.Stream()) for s in seeds]
    with concurrent.futures.ThreadPoolExecutor(len(seeds)) as pool:
        together = list(pool.map(lambda s: work(s, torch.cuda.Stream()), seeds))
    for a, b in zip(alone, together):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
