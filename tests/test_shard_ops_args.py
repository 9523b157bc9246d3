"""The operators' refusals (CPU: bad arguments are found before a device is
touched), through the C ABI with made-up pointers and through Python."""
import ctypes
import os
import re
import shutil
import subprocess
import sys

import pytest
import torch

import paper_2609_34334_amd as hc

L = hc.lib()
BAD, OK = hc.ERR_INVALID_ARG, hc.OK
P = 0x100000


def error():
    return L.hoccl_last_error_string().decode()


# ---- AdamW -------------------------------------------------------------------


def adamw(rows, **kw):
    """hoccl_adamw over rows of (param, grad, m, v, m scale, v scale, copy, n)."""
    o = dict(param_dtype=hc.FP32, grad_dtype=hc.FP32, state_bits=32, step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
             weight_decay=0.0)
    o.update(kw)
    flat = [x for r in rows for x in r]
    return L.hoccl_adamw((ctypes.c_uint64 * max(1, len(flat)))(*flat), len(rows), ctypes.byref(hc._AdamW(**o)), None)


ROW = (P, 2 * P, 3 * P, 4 * P, 0, 0, 0, 64)


@pytest.mark.parametrize("kw", [
    dict(param_dtype=hc.INT32), dict(grad_dtype=hc.UINT8), dict(param_dtype=9), dict(state_bits=16), dict(step=0),
    dict(step=-3), dict(lr=-1.0), dict(lr=float("nan")), dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1),
    dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1e-8), dict(eps=float("nan")), dict(eps=1e-40), dict(weight_decay=-1.0),
    dict(weight_decay=float("inf")), dict(lr_dev=P + 2), dict(step_dev=P + 1), dict(grad_scale=P + 3)])
def test_adamw_options(kw):
    assert adamw([ROW], **kw) == BAD
    assert error()


@pytest.mark.parametrize("at,value,word", [(0, 0, "param[0] is NULL"), (1, 0, "grad[0]"), (2, 0, "exp_avg[0]"),
                                           (3, 0, "exp_avg_sq[0]"), (0, P + 2, "aligned"), (2, P + 16, "overlap"),
                                           (1, P, "overlap"), (3, 3 * P + 252, "overlap"), (6, 2 * P, "overlap"),
                                           (7, (1 << 64) - 1, "fit"), (1, 1 << 48, "address space"),
                                           (7, 1 << 47, "address space")])
def test_adamw_tensors(at, value, word):
    row = list(ROW)
    row[at] = value
    assert adamw([row]) == BAD
    assert word in error()


def test_adamw_lists():
    assert adamw([ROW, ROW]) == BAD and "overlap" in error()          # the same tensor twice
    assert adamw([]) == OK
    assert adamw([(0, 0, 0, 0, 0, 0, 0, 0)] * 3) == OK                # tensors of no elements
    assert L.hoccl_adamw(None, 1, ctypes.byref(hc._AdamW(hc.FP32, hc.FP32, 32, 1)), None) == BAD
    assert L.hoccl_adamw(None, 0, None, None) == BAD
    assert L.hoccl_adamw(None, -1, ctypes.byref(hc._AdamW(hc.FP32, hc.FP32, 32, 1)), None) == BAD
    assert adamw([ROW], state_bits=8) == BAD and "exp_avg_scale[0] is NULL" in error()
    eight = (P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 0, 129)
    assert adamw([eight[:5] + (5 * P + 4,) + eight[6:]], state_bits=8) == BAD and "overlap" in error()
    # many tensors, in any order, of which two share a byte
    for count in (3, 16, 17, 200):
        for i, at in ((0, 0), (count // 2, 3), (count - 1, 1)):
            rows = [[P * (1 + c * 1024 + (j * 37) % count) + 4 * j for c in range(4)] + [0, 0, 0, 65] for j in range(count)]
            rows[i][at] = rows[(i + 1) % count][2] + 256
            assert adamw(rows) == BAD and "overlap" in error()
    # a scalar that the call writes over
    assert adamw([ROW], grad_scale=P + 8) == BAD and "overlap" in error()


def test_versions_of_written_tensors():
    """What an operator writes by address counts as written for autograd."""
    a, b = torch.zeros(4), torch.zeros(3, requires_grad=True)
    with torch.inference_mode():
        c = torch.zeros(2)                                            # has no version
    versions = a._version, b._version
    hc._tensors.wrote([a, c], None, (b, a))
    assert (a._version, b._version) == (versions[0] + 2, versions[1] + 1)
    flat, alone = torch.zeros(12), torch.zeros(2)
    views = [*flat.split(4), alone, flat[1:3]]                        # views share the version of what they are cut from
    versions = flat._version, alone._version
    hc._tensors.wrote(views)
    assert flat._version > versions[0] and alone._version == versions[1] + 1
    assert all(v._version == flat._version for v in views if v is not alone)
    with pytest.raises(TypeError):
        hc._tensors.wrote([a, None])
    with pytest.raises(TypeError):
        hc._tensors.wrote(3)


def test_adamw_python():
    p, g = [torch.zeros(4)], [torch.zeros(4)]
    m, v, _, _ = hc.adamw_state(p)
    with pytest.raises(ValueError, match="GPU"):
        hc.adamw(p, g, m, v, step=1, lr=0.1)
    with pytest.raises(ValueError, match="grads has 2"):
        hc.adamw(p, g * 2, m, v, step=1, lr=0.1)
    with pytest.raises(TypeError, match="fp32 or bf16"):
        hc.adamw([p[0].half()], g, m, v, step=1, lr=0.1)
    with pytest.raises(TypeError, match="exp_avgs"):
        hc.adamw(p, g, [m[0].half()], v, step=1, lr=0.1)
    with pytest.raises(ValueError, match="elements"):
        hc.adamw(p, [torch.zeros(5)], m, v, step=1, lr=0.1)
    with pytest.raises(ValueError, match="contiguous"):
        hc.adamw(p, [torch.zeros(8)[::2]], m, v, step=1, lr=0.1)
    with pytest.raises(TypeError, match="tensors"):
        hc.adamw(p, g, [None], v, step=1, lr=0.1)
    with pytest.raises(ValueError, match="exp_avg_sqs has 2"):
        hc.adamw(p, g, m, v * 2, step=1, lr=0.1)
    with pytest.raises(ValueError, match="scales of both"):
        hc.adamw(p, g, m, v, [torch.zeros(1)], step=1, lr=0.1)
    with pytest.raises(ValueError, match="bits"):
        hc.adamw_state(p, bits=16)
    assert hc.adamw([], [], [], [], step=1, lr=0.1) == []
    q, r, qs, rs = hc.adamw_state([torch.zeros(129), torch.zeros(2, 64)], bits=8)
    assert q[0].dtype == torch.float8_e4m3fn and r[1].shape == (2, 64)
    assert [len(s) for s in qs + rs] == [2, 1, 2, 1]


# ---- RMSNorm -------------------------------------------------------------------


def rmsnorm(x=P, res=2 * P, w=3 * P, h=4 * P, y=5 * P, scale=0, rows=4, hidden=64, eps=1e-6, dt=hc.BF16, wdt=hc.FP32):
    return L.hoccl_rmsnorm(x, res, w, h, y, scale, rows, hidden, eps, dt, wdt, None)


@pytest.mark.parametrize("kw", [
    dict(dt=hc.INT32), dict(wdt=hc.UINT8), dict(hidden=0), dict(hidden=32769), dict(eps=-1.0), dict(eps=float("nan")),
    dict(x=0), dict(w=0), dict(y=0), dict(x=P + 1), dict(w=3 * P + 2), dict(rows=1 << 60), dict(y=4 * P),
    dict(y=P + 2), dict(h=2 * P + 64), dict(y=3 * P), dict(h=P, y=P), dict(scale=P), dict(scale=6 * P + 1),
    dict(y=P, scale=6 * P), dict(h=3 * P)])
def test_rmsnorm_arguments(kw):
    assert rmsnorm(**kw) == BAD
    assert error()


def test_rmsnorm_of_no_rows():
    assert rmsnorm(0, 0, 0, 0, 0, rows=0) == OK


def backward(dy=P, dres=2 * P, h=3 * P, w=4 * P, dx=5 * P, dw=6 * P, ws=7 * P, size=1 << 19, rows=4, hidden=64, eps=1e-6,
             dt=hc.BF16, wdt=hc.FP32):
    return L.hoccl_rmsnorm_backward(dy, dres, h, w, dx, dw, ws, size, rows, hidden, eps, dt, wdt, None)


@pytest.mark.parametrize("kw", [
    dict(dt=hc.INT32), dict(hidden=0), dict(hidden=1 << 20), dict(eps=-1.0), dict(dy=0), dict(h=0), dict(w=0), dict(dx=0),
    dict(ws=0), dict(size=100), dict(dw=6 * P + 2), dict(ws=6 * P), dict(dw=4 * P), dict(dx=P + 64), dict(dx=4 * P)])
def test_rmsnorm_backward_arguments(kw):
    assert backward(**kw) == BAD
    assert error()


@pytest.mark.parametrize("kw,word", [(dict(h=0), "h is NULL"), (dict(dx=0), "dx is NULL"), (dict(dy=0), "dy is NULL"),
                                     (dict(h=0, dx=0), "h is NULL"), (dict(dx=0, dw=0, ws=0, size=0), "dx is NULL")])
def test_rmsnorm_backward_without_a_residual_gradient(kw, word):
    """No residual gradient (NULL) does not stand for another operand that is missing."""
    assert backward(dres=0, **kw) == BAD
    assert word in error()


def test_rmsnorm_backward_workspace():
    n = ctypes.c_size_t()
    assert L.hoccl_rmsnorm_backward_workspace(8, 64, hc.BF16, ctypes.byref(n)) == OK and n.value >= 256
    assert n.value <= 8 * 64 * 4
    assert L.hoccl_rmsnorm_backward_workspace(0, 64, hc.BF16, ctypes.byref(n)) == OK and n.value == 0
    assert L.hoccl_rmsnorm_backward_workspace(1 << 40, 64, hc.BF16, ctypes.byref(n)) == OK and n.value < 1 << 30
    assert L.hoccl_rmsnorm_backward_workspace(8, 0, hc.BF16, ctypes.byref(n)) == BAD
    assert L.hoccl_rmsnorm_backward_workspace(8, 64, hc.BF16, None) == BAD
    assert backward(0, 0, 0, 0, 0, 0, 0, 0, rows=0) == OK


def test_rmsnorm_python():
    x, w = torch.zeros(3, 8), torch.ones(8)
    for call in (lambda: hc.rmsnorm(x, w), lambda: hc.rmsnorm_backward(x, x, w)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(TypeError, match="x must be"):
        hc.rmsnorm(x.half(), w)
    with pytest.raises(ValueError, match="weight has the shape"):
        hc.rmsnorm(x, torch.ones(7))
    with pytest.raises(TypeError, match="residual must be"):
        hc.rmsnorm(x, w, x.bfloat16())
    with pytest.raises(ValueError, match="contiguous"):
        hc.rmsnorm(torch.zeros(8, 3).t(), w)
    with pytest.raises(ValueError, match="dimension"):
        hc.rmsnorm(torch.zeros(()), w)
    with pytest.raises(ValueError, match="grad_residual"):
        hc.rmsnorm_backward(x, x, w, torch.zeros(2, 8))


# ---- balance loss -------------------------------------------------------------


def options(**kw):
    o = dict(logits_dtype=hc.FP32, index_bytes=4, experts=8, topk=2, ranks=4, max_ranks=0, expert_weight=1.0)
    o.update(kw)
    return hc._Balance(**o)


def balance(o, tokens=(20000,), logits=(P,), choices=(2 * P,), loss=3 * P, n=4 * P, s=5 * P, coef=6 * P, ws=7 * P,
            size=1 << 19):
    b = len(tokens)
    vp = ctypes.c_void_p * max(1, b)
    return L.hoccl_balance_loss(vp(*logits), vp(*choices), (ctypes.c_size_t * max(1, b))(*tokens), b, ctypes.byref(o), loss,
                                n, s, coef, ws, size, None)


@pytest.mark.parametrize("kw", [
    dict(logits_dtype=hc.INT32), dict(index_bytes=2), dict(experts=0), dict(experts=1025), dict(topk=0), dict(topk=65),
    dict(ranks=0), dict(ranks=3), dict(ranks=16), dict(max_ranks=-1), dict(expert_weight=float("nan")),
    dict(rank_weight=float("inf")), dict(traffic_weight=float("nan")), dict(experts=130, ranks=65)])
def test_balance_options(kw):
    assert balance(options(**kw)) == BAD
    assert error()
    n = ctypes.c_size_t()
    assert L.hoccl_balance_workspace((ctypes.c_size_t * 1)(16), 1, ctypes.byref(options(**kw)), ctypes.byref(n)) == BAD


@pytest.mark.parametrize("kw", [
    dict(tokens=()), dict(tokens=(1,) * 65, logits=(P,) * 65, choices=(P,) * 65), dict(tokens=(1 << 30,)),
    dict(logits=(0,)), dict(choices=(0,)), dict(choices=(2 * P + 2,)), dict(loss=0), dict(n=0), dict(s=0), dict(coef=0),
    dict(ws=0), dict(size=64), dict(loss=P), dict(n=2 * P), dict(coef=4 * P), dict(ws=6 * P), dict(ws=7 * P + 2)])
def test_balance_arguments(kw):
    assert balance(options(), **kw) == BAD
    assert error()


def test_balance_workspace():
    n = ctypes.c_size_t()
    for tokens, some in ((16, False), (20000, True)):
        assert L.hoccl_balance_workspace((ctypes.c_size_t * 1)(tokens), 1, ctypes.byref(options()), ctypes.byref(n)) == OK
        assert (n.value > 0) == some and n.value % 4 == 0
    assert L.hoccl_balance_workspace(None, 1, ctypes.byref(options()), ctypes.byref(n)) == BAD
    assert L.hoccl_balance_workspace((ctypes.c_size_t * 1)(16), 1, ctypes.byref(options()), None) == BAD


@pytest.mark.parametrize("dt,experts,most", [
    (hc.FP32, 1, 2048), (hc.FP32, 8, 2048), (hc.FP32, 9, 1536), (hc.FP32, 16, 1536), (hc.FP32, 32, 768), (hc.FP32, 64, 512),
    (hc.FP32, 256, 128), (hc.FP32, 1024, 64), (hc.BF16, 8, 2048), (hc.BF16, 32, 768), (hc.BF16, 128, 256),
    (hc.BF16, 256, 256), (hc.BF16, 512, 128)])
def test_balance_batches_of_one_workgroup(dt, experts, most):
    """The longest batch that one workgroup finishes, which needs no
    workspace: a few passes, fewer where one lane counts for a token."""
    n = ctypes.c_size_t()
    o = options(logits_dtype=dt, experts=experts, topk=1, ranks=1)
    for tokens, some in ((most, False), (most + 1, True)):
        for others in ((), (1, most)):
            t = (*others, tokens)
            assert L.hoccl_balance_workspace((ctypes.c_size_t * len(t))(*t), len(t), ctypes.byref(o), ctypes.byref(n)) == OK
            assert (n.value > 0) == some


@pytest.mark.parametrize("coef,dlogits", [(0, 4 * P), (3 * P, 0), (3 * P, P), (3 * P, 2 * P), (3 * P, 3 * P), (3 * P, 4 * P + 2)])
def test_balance_backward_arguments(coef, dlogits):
    vp = ctypes.c_void_p * 1
    t = (ctypes.c_size_t * 1)(16)
    assert L.hoccl_balance_loss_backward(vp(P), vp(2 * P), t, 1, ctypes.byref(options()), coef, None, vp(dlogits), None) == BAD


def test_balance_python():
    x, e = [torch.zeros(4, 8)], [torch.zeros(4, 2, dtype=torch.int64)]
    with pytest.raises(ValueError, match="GPU"):
        hc.balance_loss(x, e, 4)
    with pytest.raises(ValueError, match="same length"):
        hc.balance_loss(x, e * 2, 4)
    with pytest.raises(ValueError, match="same length"):
        hc.balance_loss([], [], 4)
    with pytest.raises(TypeError, match="int32 or int64"):
        hc.balance_loss(x, [e[0].short()], 4)
    with pytest.raises(ValueError, match="same tokens"):
        hc.balance_loss(x * 2, [e[0], e[0][:3]], 4)
    with pytest.raises(ValueError, match=r"logits\[1\] must have the shape"):
        hc.balance_loss([x[0], torch.zeros(4, 9)], e * 2, 4)
    with pytest.raises(ValueError, match=r"experts\[1\] must have the shape"):
        hc.balance_loss(x * 2, [e[0], e[0][0]], 4)
    with pytest.raises(ValueError, match="contiguous"):
        hc.balance_loss([torch.zeros(8, 4).t()], e, 4)
    with pytest.raises(ValueError, match="tokens"):
        hc.balance_loss([torch.zeros(4)], e, 4)
    with pytest.raises(ValueError, match="coef"):
        hc.balance_loss_backward(x, e, torch.zeros(2, 8))


# ---- what is not built ----------------------------------------------------------


@pytest.mark.parametrize("there", [[], ["libhoccl.so"]])
def test_the_import_names_a_build_command_that_runs(tmp_path, there):
    """Without one of the two built files the import says how to build them;
    the command does not need the package that cannot be imported yet."""
    package = tmp_path / "paper_2609_34334_amd"
    package.mkdir()
    home = os.path.dirname(hc.__file__)
    for name in ["__init__.py", "build.py", *there]:
        shutil.copy(os.path.join(home, name), package)
    env = dict(os.environ, PYTHONPATH=str(tmp_path), HIPCC="/bin/false", CXX="/bin/false")
    r = subprocess.run([sys.executable, "-c", "import paper_2609_34334_amd"], cwd=tmp_path, env=env, capture_output=True,
                       text=True)
    assert r.returncode != 0 and "is not built" in r.stderr
    command = re.search("`python (.*?)`", r.stderr).group(1)
    r = subprocess.run([sys.executable, *command.split()], cwd=tmp_path, env=env, capture_output=True, text=True)
    assert r.returncode != 0 and "compiling" in r.stderr and "is not built" not in r.stderr
