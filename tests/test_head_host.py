"""CPU-only checks of the calls at the output head: refusals on the host before anything touches the GPU, workspace sizes, and
the float64 oracle itself (closed forms, gradients against differences)."""
import ctypes
import math
import subprocess
import sys
from pathlib import Path

import pytest
import torch

from oracle import head as oh
from paper_2603_05168_b200 import build as sbn_build

NULL, SHAPE, ALIGN, UNSUP, WS = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def L():
    sbn_build.build()
    from paper_2603_05168_b200 import binding
    return binding.lib()


p, q, r = (ctypes.c_void_p(a << 12) for a in (0x10, 0x20, 0x30))      # fake, never dereferenced, well aligned
odd = ctypes.c_void_p(0x10002)
BIG = 1 << 40


def _ce(L, **k):
    return L.sbn_head_cross_entropy(k.get("x", p), k.get("T", 4), k.get("K", 256), k.get("head", q), k.get("N", 1000), k.get("labels", p),
                                    k.get("loss", p), k.get("lse", p), k.get("ws", p), k.get("wsb", BIG), None)


def _ceb(L, **k):
    return L.sbn_head_cross_entropy_backward(k.get("x", p), k.get("T", 4), k.get("K", 256), k.get("head", q), k.get("N", 1000), k.get("labels", p),
                                             k.get("lse", p), k.get("dloss", p), k.get("dx", r), k.get("dhead", r), k.get("ws", p), k.get("wsb", BIG), None)


def _kd(L, **k):
    return L.sbn_head_distill(k.get("x", p), k.get("T", 4), k.get("K", 256), k.get("head", q), k.get("N", 1000), k.get("index", p), k.get("logits", p),
                              k.get("dt", 0), k.get("top", 8), k.get("tau", 1.0), k.get("labels", p), k.get("kd", p), k.get("ce", p), k.get("lse", p),
                              k.get("ws", p), k.get("wsb", BIG), None)


def _kdb(L, **k):
    return L.sbn_head_distill_backward(k.get("x", p), k.get("T", 4), k.get("K", 256), k.get("head", q), k.get("N", 1000), k.get("index", p),
                                       k.get("logits", p), k.get("dt", 0), k.get("top", 8), k.get("tau", 1.0), k.get("labels", p), k.get("lse", p),
                                       k.get("dkd", p), k.get("dce", p), k.get("dx", r), k.get("dhead", r), k.get("ws", p), k.get("wsb", BIG), None)


@pytest.mark.parametrize("call", [_ce, _ceb, _kd, _kdb])
def test_refusals_that_all_calls_share(L, call):
    for name in ("x", "head", "lse"):
        assert call(L, **{name: None}) == NULL, name
    for bad in (dict(T=0), dict(T=-1), dict(N=0), dict(K=0), dict(K=100), dict(K=64), dict(K=(1 << 20) + 128), dict(T=(1 << 30) + 1), dict(N=(1 << 30) + 1)):
        assert call(L, **bad) == SHAPE, bad
    assert call(L, ws=None) == WS
    assert call(L, wsb=100) == WS
    for name in ("x", "head", "ws", "labels"):
        assert call(L, **{name: odd}) == ALIGN, name
    assert call(L, ws=ctypes.c_void_p(0x10080)) == ALIGN                # workspaces start on 256 bytes
    assert call(L, lse=odd) == ALIGN


def test_refusals_of_each_call(L):
    assert _ce(L, labels=None) == NULL and _ce(L, loss=None) == NULL and _ce(L, loss=odd) == ALIGN
    assert _ceb(L, labels=None) == NULL and _ceb(L, dloss=None) == NULL and _ceb(L, dloss=odd) == ALIGN
    for call in (_ceb, _kdb):
        assert call(L, dx=None, dhead=None) == NULL
        assert call(L, dx=p) == UNSUP and call(L, dhead=q) == UNSUP    # the inputs' own buffers
        assert call(L, dx=odd) == ALIGN and call(L, dhead=odd) == ALIGN
    for call in (_kd, _kdb):
        assert call(L, index=None) == NULL and call(L, logits=None) == NULL
        assert call(L, index=ctypes.c_void_p(0x10004)) == ALIGN and call(L, logits=odd) == ALIGN
        for bad in (dict(top=0), dict(top=-3), dict(top=257), dict(dt=2), dict(tau=0.0), dict(tau=-1.0), dict(tau=math.inf), dict(tau=math.nan), dict(tau=1e-39)):
            assert call(L, **bad) == UNSUP, bad
    assert _kd(L, kd=None) == NULL and _kdb(L, dkd=None) == NULL
    assert _kd(L, labels=None) == NULL and _kd(L, ce=None) == NULL       # both or neither
    assert _kdb(L, labels=None) == NULL and _kdb(L, dce=None) == NULL
    assert _kd(L, kd=odd) == ALIGN and _kd(L, ce=odd) == ALIGN and _kdb(L, dkd=odd) == ALIGN and _kdb(L, dce=odd) == ALIGN


@pytest.mark.parametrize("call", [_ceb, _kdb])
def test_gradients_that_overlap_are_refused(L, call):
    # T x K and N x K values of 2 bytes: 2 KB and 500 KB
    x, head, ws, dx, dhead = 0x1000000, 0x2000000, 0x3000000, 0x4000000, 0x5000000
    at = ctypes.c_void_p

    def run(**k):
        return call(L, **{"x": at(x), "head": at(head), "ws": at(ws), "dx": at(dx), "dhead": at(dhead), **k})

    for where in (x, x + 16, x + 2048 - 16, x - 2048 + 16, head + 16, head - 16, head + 512000 - 16, ws, ws - 16, dhead, dhead - 16, dhead + 511984):
        assert run(dx=at(where)) == UNSUP, hex(where)
    for where in (head, head - 512000 + 16, x, x - 16, x + 2032, ws + 256, dx, dx + 2032, dx - 511984):
        assert run(dhead=at(where)) == UNSUP, hex(where)
    assert run(dx=None, dhead=at(head + 16)) == UNSUP and run(dx=at(x + 16), dhead=None) == UNSUP


def test_smallest_temperature(L):
    for tau in (4.2e-39, 4.24e-39, 1e-45):                          # 1.45 / tau is no fp32 number
        assert _kd(L, tau=tau) == UNSUP and _kdb(L, tau=tau) == UNSUP


def test_workspace_sizes(L):
    from paper_2603_05168_b200 import binding as b
    for bad in ((0, 10, 128), (1, 0, 128), (1, 10, 100), (-1, 10, 128)):
        assert b.sbn_head_workspace_bytes(*bad) == 0
    assert b.sbn_head_workspace_bytes(4, 100, 128, top=257) == 0 and b.sbn_head_workspace_bytes(4, 100, 128, top=-1) == 0
    with pytest.raises(ValueError):
        b.alloc_head_ws(4, 100, 100, device="cpu")
    # far from the logits' T x N values, and no more for a larger vocabulary once it goes in pieces
    T, K = 8192, 4096
    small, large = (b.sbn_head_workspace_bytes(T, N, K, backward=True) for N in (65536, 1 << 20))
    assert large <= small * 1.05 and large < 0.1 * 2 * T * (1 << 20)
    assert b.sbn_head_workspace_bytes(T, 131072, K) < 0.1 * 4 * T * 131072
    assert b.sbn_head_workspace_bytes(T, 131072, K, top=64) < 0.15 * 4 * T * 131072
    # sizes past 32 bits are counted in 64
    assert b.sbn_head_workspace_bytes(1 << 20, 1 << 20, 4096, backward=True) > 1 << 34


def test_workspace_sizes_at_the_largest_sizes(L):
    # a child asks: an arithmetic fault would end the process
    ask = """
from paper_2603_05168_b200 import binding as b
for T in (1, 17, 300, 1 << 20, (1 << 30) - 5, 1 << 30):
    for N in (1, 1 << 20, 1 << 30):
        for K in (128, 1 << 16, 1 << 20):
            for top in (0, 256):
                for backward in (False, True):
                    n = b.sbn_head_workspace_bytes(T, N, K, top, backward)
                    assert (4 * T * K if backward else 8 * T) <= n < 1 << 62, (T, N, K, top, backward, n)
"""
    done = subprocess.run([sys.executable, "-c", ask], cwd=Path(__file__).resolve().parent.parent, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr[-500:]


def test_status_of_an_index_outside_the_vocabulary(L):
    from paper_2603_05168_b200 import binding as b
    assert "vocabulary" in b.status_string(9)


def test_binding_refuses_tensors_off_the_current_device(L):
    from paper_2603_05168_b200 import binding as b
    x, head = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(10, 128, dtype=torch.bfloat16)
    f = torch.zeros(4)
    with pytest.raises(ValueError):
        b.sbn_head_cross_entropy(x, head, torch.zeros(4, dtype=torch.int64), f, f)
    with pytest.raises(ValueError):
        b.sbn_head_cross_entropy(x[0], head, torch.zeros(4, dtype=torch.int64), f, f)


# ---- the oracle ----------------------------------------------------------------------------------
def _problem(T=6, N=11, K=5, top=4, seed=0):
    g = torch.Generator().manual_seed(seed)
    x, head = torch.randn(T, K, generator=g, dtype=torch.float64), torch.randn(N, K, generator=g, dtype=torch.float64)
    labels = torch.randint(0, N, (T,), generator=g)
    index = torch.randint(0, N, (T, top), generator=g)
    return dict(x=x, head=head, labels=labels, top_index=index, top_logits=torch.randn(T, top, generator=g, dtype=torch.float64), tau=1.7)


def test_oracle_closed_forms():
    c = _problem()
    c["head"] = torch.zeros_like(c["head"])                                # uniform: every loss is log N (less the teacher's entropy)
    o = oh.head_loss(**c)
    assert torch.allclose(o["ce"], torch.full_like(o["ce"], math.log(11)))
    Q, there, ne = oh.targets(c["top_index"], c["top_logits"], 11, 1.7)
    assert there.all() and torch.allclose(Q.sum(1), torch.ones(6, dtype=torch.float64))
    assert torch.allclose(o["distill"], ne + math.log(11))
    # a teacher that is the student itself, all of it: no loss, no gradient
    c = _problem(top=11)
    z = c["x"] @ c["head"].T
    c["top_index"], c["top_logits"] = torch.arange(11).repeat(6, 1), z
    o = oh.head_loss(**c, d_distill=torch.ones(6, dtype=torch.float64))
    assert o["distill"].abs().max() < 1e-12 and o["dx"].abs().max() < 1e-12
    # an index twice counts twice
    one = oh.targets(torch.tensor([[3, 3]]), torch.zeros(1, 2), 5, 1.0)
    assert one[0][0, 3] == 1.0 and abs(float(one[2][0]) - math.log(0.5)) < 1e-12


def test_oracle_gradients_against_differences():
    c = _problem(seed=3)
    c["labels"][2] = -1
    c["top_index"][4] = -1
    g = torch.Generator().manual_seed(9)
    d_ce, d_kd = torch.rand(6, generator=g, dtype=torch.float64), torch.rand(6, generator=g, dtype=torch.float64)
    o = oh.head_loss(**c, d_ce=d_ce, d_distill=d_kd)

    def total(**change):
        v = oh.head_loss(**dict(c, **change))
        return float((v["ce"] * d_ce + v["distill"] * d_kd).sum())

    h = 1e-5
    for name, grad in (("x", o["dx"]), ("head", o["dhead"])):
        for at in [(0, 0), (2, 3), (4, 1), (5, 4)]:
            step = torch.zeros_like(c[name])
            step[at] = h
            slope = (total(**{name: c[name] + step}) - total(**{name: c[name] - step})) / (2 * h)
            assert abs(slope - float(grad[at])) < 1e-8, (name, at)


@pytest.mark.parametrize("call", [_ce, _ceb, _kd, _kdb])
def test_nothing_written_may_lie_on_anything_else(L, call):
    # T x K and N x K values of 2 bytes: 2 KB and 500 KB; per token 4 bytes (lse twice beside a teacher) or 8; 4 tokens x 8 entries
    distill, back = call in (_kd, _kdb), call in (_ceb, _kdb)
    size = dict(x=2048, head=512000, labels=32, lse=32 if distill else 16, ws=L.sbn_head_workspace_bytes(int(back), 4, 1000, 256, 8 if distill else 0))
    if distill:
        size.update(index=256, logits=128)
    reads = {_ceb: ["lse", "dloss"], _kdb: ["lse", "dkd", "dce"]}.get(call, [])
    writes = {_ce: ["loss", "lse"], _kd: ["kd", "ce", "lse"]}.get(call, ["dx", "dhead"])
    for name in reads + writes:
        size.setdefault(name, dict(dx=2048, dhead=512000).get(name, 16))
    at = {name: (i + 1) << 28 for i, name in enumerate(size)}
    inputs = [name for name in size if name not in writes and name != "ws"]

    def run(**k):
        return call(L, **{name: ctypes.c_void_p(k.get(name, where)) for name, where in at.items()})

    pairs = [(w, o) for w in writes for o in size if o != w] + [("ws", o) for o in inputs]
    for w, o in pairs:
        step = 256 if "ws" in (w, o) else 16
        for moved, still in ((w, o), (o, w)):
            for where in (at[still], at[still] + (size[still] - 1) // step * step, at[still] - (size[moved] - 1) // step * step):
                assert run(**{moved: where}) == UNSUP, (moved, still, hex(where))


@pytest.mark.parametrize("big", [(1 << 32) + 4, (1 << 31) + 4, -(1 << 32) + 4, 1 << 70])
def test_workspace_of_sizes_past_32_bits(L, big):
    # no size that only its low 32 bits make look possible
    from paper_2603_05168_b200 import binding as b
    for at in range(3):
        sizes = [4, 1000, 256]
        sizes[at] = big
        assert b.sbn_head_workspace_bytes(*sizes) == 0
        with pytest.raises(ValueError):
            b.alloc_head_ws(*sizes, device="cpu")
    assert b.sbn_head_workspace_bytes(4, 1000, 256, top=big) == 0


def test_smallest_temperature_of_the_gradient(L):
    # (the forward call goes on to the workspace, which is too small here)
    for tau in (2.0 ** -10 * (1 - 2.0 ** -24), 1e-4, 1e-8, 1e-30):
        assert _kdb(L, tau=tau) == UNSUP and _kd(L, tau=tau, wsb=100) == WS
    assert _kdb(L, tau=2.0 ** -10, wsb=100) == WS


def test_messages_fit_the_calls_at_the_head(L):
    # any N is right there, a workspace starts on 256 bytes, overlapping buffers are unsupported
    from paper_2603_05168_b200 import binding as b
    assert "output head" in b.status_string(SHAPE)
    assert not b.status_string(ALIGN).startswith("pointer not 16-byte") and "overlap" in b.status_string(UNSUP)
