"""Residual addition with RMS norm (hoccl_rmsnorm) and its gradients against
the formulas in 64 bits.

Tolerances count roundings of at most half a step (U = 2^-24 in fp32, 2^-8 of
the value in bf16).  A row's sum of squares adds at most 32 values a thread
and then joins lanes and waves: 32 + 6 + 16 additions and one rounding for
each square, 55 U; half of it, with the mean, eps, root and reciprocal, is in
1 / rms: 32 U."""
import math

import pytest
import torch

import paper_2609_34334_amd as hc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
RMS = 32 * U


@pytest.fixture(autouse=True)
def _defaults():
    saved = hc.get_config()
    yield
    hc.set_config(**saved)


def tensor(seed, *shape, dt=torch.float32, scale=1.0, shift=0, guard=24):
    """A seeded tensor on the GPU, `shift` elements into a buffer whose other
    elements are a guard."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = math.prod(shape)
    whole = torch.full((shift + n + guard,), 55.0, dtype=dt, device="cuda")
    x = whole[shift:shift + n]
    x.copy_(torch.randn(n, generator=g, device="cuda") * scale)
    x = x.view(shape)
    x.guard = (whole, shift, n)
    return x


def check_guard(x):
    whole, shift, n = x.guard
    assert (whole[:shift] == 55).all() and (whole[shift + n:] == 55).all(), "written outside"


def reference(x, r, w, eps):
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    d = h.double()
    rms = (d.square().mean(-1, keepdim=True) + eps).sqrt()
    return h, d / rms * w.double(), rms


def check_forward(x, r, w, y, h, eps=1e-6):
    want_h, want, _ = reference(x, r, w, eps)
    if r is not None:
        assert torch.equal(h, want_h)
    # 1 / rms and two products, then one rounding to the type
    err = (RMS + 2 * U) * want.abs()
    assert ((y.double() - want).abs() <= err + HALF[x.dtype] * (want.abs() + err) + SMALLEST[x.dtype]).all()


def check_8bit(x, r, w, q, scale, h, eps=1e-6):
    want_h, want, _ = reference(x, r, w, eps)
    if r is not None:
        assert torch.equal(h, want_h)
    H = x.shape[-1]
    nb = -(-H // 128)
    assert scale.shape == x.shape[:-1] + (nb,)
    pad = torch.nn.functional.pad(want.abs(), (0, nb * 128 - H)).unflatten(-1, (nb, 128))
    top = pad.amax(-1)
    err = RMS + 3 * U
    assert ((scale.double() - top / 448).abs() <= err * top / 448).all()
    each = scale.double().repeat_interleave(128, -1)[..., :H]
    # half a step of e4m3, and the roundings before it
    assert ((q.double() * each - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -10 * each + 2 * err * want.abs()).all()


# Hidden sizes around the changes of shape: 8 to 64 lanes a row, a workgroup a row, several vectors a thread; odd ones.
HIDDEN = [1, 3, 7, 9, 32, 33, 64, 100, 127, 128, 130, 250, 256, 257, 384, 512, 513, 1024, 1025, 2048, 2049, 4096, 5003, 8192, 8193, 16384, 16390, 32767, 32768]


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("hidden", HIDDEN)
def test_formulas(hidden, dt):
    t = DT[dt]
    for rows, shift, wdt, with_r in ((5, 0, t, True), (3, 1, torch.float32, False), (1, 3, torch.bfloat16, True)):
        x = tensor(hidden, rows, hidden, dt=t, scale=3.0, shift=shift)
        r = tensor(hidden + 1, rows, hidden, dt=t, shift=shift) if with_r else None
        w = tensor(hidden + 2, hidden, dt=wdt, shift=shift)
        x0 = x.clone()
        got = hc.rmsnorm(x, w, r)
        y, h = got if with_r else (got, None)
        check_forward(x0, r, w, y, h)
        got = hc.rmsnorm(x, w, r, quantize=True)
        (q, scale), h = got if with_r else (got, None)
        check_8bit(x0, r, w, q, scale, h)
        assert torch.equal(x, x0)
        assert hc.last_stats()["reduce_launches"] == 1


def check_backward(h, dy, dres, w, dx, dw, eps=1e-6):
    H, rows = h.shape[-1], h.numel() // h.shape[-1]
    d, gw = h.double().view(rows, H), (dy.double() * w.double()).view(rows, H)
    rms = (d.square().mean(-1, keepdim=True) + eps).sqrt()
    c = (gw * d).mean(-1, keepdim=True) / rms ** 2
    want = (gw - d * c) / rms
    big = (gw * d).abs().mean(-1, keepdim=True) / rms ** 2
    # gy w and 1 / rms; the mean of products of two roundings in 55 additions, over rms twice, times h
    err = (gw.abs() * (RMS + 3 * U) + d.abs() * big * (57 * U + 3 * RMS + 4 * U)) / rms
    if dres is not None:
        want = want + dres.double().view(rows, H)
    err = err + U * want.abs()
    t = h.dtype
    assert ((dx.double().view(rows, H) - want).abs() <= err + HALF[t] * (want.abs() + err) + SMALLEST[t]).all()
    if dw is None:
        return
    terms = dy.double().view(rows, H) * d / rms
    # at most 1024 partial sums: rows a thread adds, a workgroup's rows, 32 partials in each of 32 lots
    adds = -(-rows // 1024) + 4 + 32 + 32
    assert ((dw.double() - terms.sum(0)).abs() <= (RMS + 2 * U + adds * U) * terms.abs().sum(0) + 1e-37).all()


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("hidden", HIDDEN)
def test_gradients(hidden, dt):
    t = DT[dt]
    for rows, shift, wdt, with_r in ((6, 0, t, True), (3, 1, torch.float32, False), (1, 3, torch.bfloat16, True)):
        h = tensor(hidden, rows, hidden, dt=t, scale=2.0, shift=shift)
        dy = tensor(hidden + 1, rows, hidden, dt=t, scale=0.1, shift=shift)
        dres = tensor(hidden + 2, rows, hidden, dt=t, scale=0.1, shift=shift) if with_r else None
        w = tensor(hidden + 3, hidden, dt=wdt, shift=shift)
        dx, dw = hc.rmsnorm_backward(dy, h, w, dres)
        check_backward(h, dy, dres, w, dx, dw)
        assert dw.dtype == torch.float32
        dx2, none = hc.rmsnorm_backward(dy, h, w, dres, weight_grad=False)
        assert none is None and torch.equal(dx2, dx)
        assert hc.last_stats()["reduce_launches"] == 1


@pytest.mark.parametrize("rows,hidden", [(5000, 64), (4099, 300), (3001, 2050), (1030, 8200)])
def test_many_rows(rows, hidden):
    """More rows than workgroups and partial sums."""
    x, r = (tensor(i, rows, hidden, dt=torch.bfloat16) for i in (1, 2))
    w = tensor(3, hidden)
    y, h = hc.rmsnorm(x, w, r)
    check_forward(x, r, w, y, h)
    (q, scale), h = hc.rmsnorm(x, w, r, quantize=True)
    check_8bit(x, r, w, q, scale, h)
    dy = tensor(4, rows, hidden, dt=torch.bfloat16)
    dx, dw = hc.rmsnorm_backward(dy, h, w, r)
    check_backward(h, dy, r, w, dx, dw)


def test_gradients_against_differences():
    """The gradients of sum(y * dy) + sum(h * dres), by central differences of
    the formula in 64 bits along random directions."""
    rows, H, eps = 5, 200, 1e-5
    h, dy, dres = (tensor(i, rows, H) for i in (1, 2, 3))
    w = tensor(4, H)
    dx, dw = hc.rmsnorm_backward(dy, h, w, dres, eps=eps)

    def f(x, weight):
        y = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight
        return (y * dy.double()).sum() + (x * dres.double()).sum()

    g = torch.Generator(device="cuda").manual_seed(9)
    for _ in range(4):
        ux = torch.randn(rows, H, generator=g, device="cuda", dtype=torch.float64)
        uw = torch.randn(H, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-5
        num = (f(h.double() + e * ux, w.double() + e * uw) - f(h.double() - e * ux, w.double() - e * uw)) / (2 * e)
        ana = (dx.double() * ux).sum() + (dw.double() * uw).sum()
        size = (dx.double() * ux).abs().sum() + (dw.double() * uw).abs().sum()
        # differences: e^2 of a third derivative of order one a term, and 2^-53 / e; the kernel: about 100 U a term
        assert abs(num - ana) <= (1e-8 + 200 * U) * size


def test_in_place_forms():
    rows, H = 37, 4100
    for t in (torch.bfloat16, torch.float32):
        w = tensor(3, H, dt=t)
        fresh = lambda: (tensor(1, rows, H, dt=t), tensor(2, rows, H, dt=t))
        x, r = fresh()
        y0, h0 = hc.rmsnorm(x, w, r)
        for pick in ("yx hr", "yr hx", "hx", "hr", "yx", "yr"):
            x, r = fresh()
            at = {"x": x, "r": r}
            kw = {}
            for p in pick.split():
                kw["out" if p[0] == "y" else "residual_out"] = at[p[1]]
            y, h = hc.rmsnorm(x, w, r, **kw)
            assert torch.equal(y, y0) and torch.equal(h, h0), pick
            check_guard(x)
            check_guard(r)
        x, _ = fresh()
        y1 = hc.rmsnorm(x, w)
        assert hc.rmsnorm(x, w, out=x) is x and torch.equal(x, y1)
        dy, dres = tensor(5, rows, H, dt=t), tensor(6, rows, H, dt=t)
        dx0, dw0 = hc.rmsnorm_backward(dy, h0, w, dres)
        for k in range(3):
            ts = [dy.clone(), h0.clone(), dres.clone()]
            dx, dw = hc.rmsnorm_backward(ts[0], ts[1], w, ts[2], out=ts[k])
            assert torch.equal(dx, dx0) and torch.equal(dw, dw0), k


def test_rows_of_nothing():
    for t in (torch.bfloat16, torch.float32):
        x, w = torch.empty(0, 64, dtype=t, device="cuda"), torch.ones(64, device="cuda")
        assert hc.rmsnorm(x, w).shape == (0, 64)
        q, s = hc.rmsnorm(x, w, quantize=True)
        assert q.shape == (0, 64) and s.shape == (0, 1)
        dx, dw = hc.rmsnorm_backward(x, x, w)
        assert dx.shape == (0, 64) and torch.equal(dw, torch.zeros(64, device="cuda"))


def test_shapes_of_more_and_fewer_dimensions():
    x, w = tensor(1, 2, 3, 160, dt=torch.bfloat16), tensor(2, 160)
    check_forward(x, None, w, hc.rmsnorm(x, w), None)
    q, s = hc.rmsnorm(x, w, quantize=True)
    assert q.shape == (2, 3, 160) and s.shape == (2, 3, 2)
    one = tensor(3, 160, dt=torch.bfloat16)
    y = hc.rmsnorm(one, w)
    assert y.shape == (160,)
    check_forward(one, None, w, y, None)
    dx, dw = hc.rmsnorm_backward(x, x, w)
    assert dx.shape == x.shape
    check_backward(x, x, None, w, dx, dw)


def test_zeros_and_what_is_not_finite():
    H = 300
    w = torch.ones(H, device="cuda")
    x = torch.zeros(4, H, device="cuda")
    x[1, 7] = math.nan
    x[2, 200] = math.inf
    x[3] = 1.0
    y = hc.rmsnorm(x, w)
    assert torch.equal(y[0], torch.zeros(H, device="cuda"))
    assert torch.isnan(y[1]).all()
    assert torch.isnan(y[2, 200]) and (torch.cat([y[2, :200], y[2, 201:]]) == 0).all()
    q, s = hc.rmsnorm(x, w, quantize=True)
    held = q.float() * s.repeat_interleave(128, -1)[:, :H]
    assert (held[0] == 0).all() and (s[0] == 0).all()
    assert torch.isnan(held[1]).all()
    assert torch.isnan(held[2, 128:256]).all() and (held[2, :128] == 0).all() and (held[2, 256:] == 0).all()
    assert torch.isfinite(held[3]).all()
    # eps = 0: a row of zeros is 0 / 0, and the other rows stay what they are, short blocks too
    y, (q, s) = hc.rmsnorm(x, w, eps=0.0), hc.rmsnorm(x, w, eps=0.0, quantize=True)
    assert torch.isnan(y[0]).all() and (y[3] == 1).all()
    assert torch.isfinite(s[3]).all() and (q[3].float() == 448).all()


def test_large_calls():
    """Calls of more bytes than the caches hold, whole and ragged rows."""
    for rows, H in ((70_001, 1024), (70_001, 1001)):
        x, r = (tensor(i, rows, H, dt=torch.bfloat16) for i in (1, 2))
        w = tensor(3, H)
        y, h = hc.rmsnorm(x, w, r)
        (q, s), h2 = hc.rmsnorm(x, w, r, quantize=True)
        assert torch.equal(h, h2)
        for at in (slice(0, 500), slice(rows - 500, rows)):
            check_forward(x[at], r[at], w, y[at], h[at])
            check_8bit(x[at], r[at], w, q[at], s[at], h[at])
        assert torch.equal(y[1000:3000], hc.rmsnorm(x[1000:3000], w, r[1000:3000])[0])


@pytest.mark.parametrize("hidden", [40, 100, 2500, 20000])
def test_budgets_and_streams_give_the_same_bits(hidden):
    rows, t = 700, torch.bfloat16
    x, r, dy = (tensor(i, rows, hidden, dt=t) for i in (1, 2, 3))
    w = tensor(4, hidden)
    runs = []
    for wg, own in ((0, False), (1, False), (5, True), (0, True)):
        hc.set_config(workgroups_per_step=wg)
        stream = torch.cuda.Stream() if own else None
        torch.cuda.synchronize()
        y, h = hc.rmsnorm(x, w, r, stream=stream)
        q, s = hc.rmsnorm(x, w, r, quantize=True, stream=stream)[0]
        dx, dw = hc.rmsnorm_backward(dy, x, w, r, stream=stream)
        assert wg == 0 or hc.last_stats()["workgroups_per_step"] <= wg
        torch.cuda.synchronize()
        runs.append((y, h, q.view(torch.uint8), s, dx, dw))
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("H", [90, 2100, 20000])
def test_replays(H):
    rows, t = 300, torch.bfloat16
    x, r, dy = (tensor(i, rows, H, dt=t) for i in (1, 2, 3))
    w = tensor(4, H)
    hc.init()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, h = hc.rmsnorm(x, w, r)
        q, s = hc.rmsnorm(x, w, r, quantize=True)[0]
        dx, dw = hc.rmsnorm_backward(dy, h, w, r)
    for k in range(3):
        x.copy_(tensor(100 + k, rows, H, dt=t))
        graph.replay()
        torch.cuda.synchronize()
        ey, eh = hc.rmsnorm(x, w, r)
        (eq, es), _ = hc.rmsnorm(x, w, r, quantize=True)
        edx, edw = hc.rmsnorm_backward(dy, eh, w, r)
        torch.cuda.synchronize()
        for a, b in ((y, ey), (h, eh), (q.view(torch.uint8), eq.view(torch.uint8)), (s, es), (dx, edx), (dw, edw)):
            assert torch.equal(a, b), k
    del graph


def test_offsets_past_32_bits():
    """2.2 G elements: rows behind 4 GiB."""
    rows, H = 131100, 16400
    x = torch.zeros(rows, H, dtype=torch.bfloat16, device="cuda")
    w = tensor(1, H)
    for at in (0, 65600, rows - 1):
        x[at] = tensor(2 + at, H, dt=torch.bfloat16)
    y = hc.rmsnorm(x, w)
    for at in (0, 65600, rows - 1):
        check_forward(x[at], None, w, y[at], None)
    assert not y[1:65600].any() and not y[65601:-1].any()
    dx, dw = hc.rmsnorm_backward(x, x, w, out=y)
    for at in (0, 65600, rows - 1):
        check_backward(x[at], x[at], None, w, dx[at], None)


def test_outputs_that_are_given_count_as_written():
    """A graph that saved a tensor which a call then writes is refused."""
    x, r, w = (torch.randn(6, 40, device="cuda") for _ in range(3))
    w = w[0].contiguous()
    pair = (torch.empty(6, 40, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(6, 1, device="cuda"))
    fresh = torch.empty(6, 40, device="cuda")
    for out, call in (([fresh], lambda: hc.rmsnorm(x, w, out=fresh)),
                      ([x, r], lambda: hc.rmsnorm(x, w, r, out=x, residual_out=r)),
                      ([*pair, r], lambda: hc.rmsnorm(x, w, r, quantize=True, out=pair, residual_out=r)),
                      ([fresh], lambda: hc.rmsnorm_backward(x, r, w, out=fresh)),
                      ([], lambda: hc.rmsnorm(x, w, r)), ([], lambda: hc.rmsnorm_backward(x, r, w))):
        every = [x, r, w, fresh, *pair]
        versions = [t._version for t in every]
        call()
        for t, v in zip(every, versions):
            assert (t._version > v) == any(t is o for o in out)
    leaf = torch.randn(6, 40, device="cuda", requires_grad=True)
    mid = leaf * 2
    loss = (mid * mid).sum()
    hc.rmsnorm(x, w, out=mid.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_the_reciprocal_root_is_rounded_once():
    """Rows (1, k / 64): their squares' sum and mean are exact, and so are the
    products with 1, so that y of the first and its weight's gradient are
    1 / rms itself: off by half a step, and 2^-10 of one for a Newton step's
    remainder (1.5 times the square of 2^-22)."""
    k = torch.arange(4096, device="cuda")
    h = torch.stack([torch.ones(4096, device="cuda"), k / 64], 1)
    w = torch.ones(2, device="cuda")
    want = 1 / ((1 + (k.double() / 64) ** 2) / 2).sqrt()
    y = hc.rmsnorm(h, w, eps=0.0)
    assert ((y[:, 0].double() - want).abs() <= (1 + 2.0 ** -10) * U * want).all()
    for i in (0, 1, 63, 64, 777, 4095):
        _, dw = hc.rmsnorm_backward(torch.ones(1, 2, device="cuda"), h[i:i + 1], w, eps=0.0)
        assert abs(dw[0].double() - want[i]) <= (1 + 2.0 ** -10) * U * want[i]


def test_magnitudes_near_the_ends_of_fp32():
    """Rows whose mean of squares lies from 2^-120 to 2^120."""
    w = torch.ones(64, device="cuda")
    base = tensor(5, 64)
    for e in (-60, -51, -50, -49, -30, 30, 49, 50, 51, 57):
        x = (base * 2.0 ** e).view(1, 64)
        check_forward(x, None, w, hc.rmsnorm(x, w, eps=0.0), None, eps=0.0)
        dx, dw = hc.rmsnorm_backward(x * 2.0 ** -e, x, w, eps=0.0)
        check_backward(x, x * 2.0 ** -e, None, w, dx, dw, eps=0.0)
    # single powers of two, whose squares are exact down to 2^-148: y is 1
    x = torch.ldexp(torch.ones(138), torch.arange(-74, 64)).view(-1, 1).cuda()
    y = hc.rmsnorm(x, torch.ones(1, device="cuda"), eps=0.0)
    assert torch.equal(y, torch.ones_like(y))
    # squares that vanish, or pass the range: 1 / rms is infinite, or 0
    for dt in (torch.float32, torch.bfloat16):
        x = torch.tensor([[2.0 ** -100] * 8, [2.0 ** 100] * 8], device="cuda").to(dt)
        y = hc.rmsnorm(x, torch.ones(8, device="cuda"), eps=0.0)
        assert torch.isposinf(y[0]).all() and (y[1] == 0).all()
