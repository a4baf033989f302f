"""The losses at the output head (cross entropy, distillation) and their gradients on the GPU, through the C ABI, against the
float64 definitions of ``oracle/head.py`` within the bounds derived there."""
import pytest
import torch

from oracle import head as oh
from paper_2603_05168_b200 import binding as b

pytestmark = pytest.mark.gpu

F32, BF16, I64 = torch.float32, torch.bfloat16, torch.int64
NAN, INF = float("nan"), float("inf")


@pytest.fixture(autouse=True)
def _clean_status():
    b.sbn_set_gemm_tuning(0, 0)
    yield
    b.sbn_set_gemm_tuning(0, 0)
    b.sbn_check_status()


def make(T, N, K, seed, ignored=0.3, lean=1.0, scale=0.02, top=0, dtype=F32, labels=True, absent=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    head = (randn(N, K) * scale).to(BF16)
    y = torch.randint(0, N, (T,), generator=g, device="cuda")
    x = (randn(T, K) + lean * rand(T, 1) * 5.0 / (scale * K) * head[y].float() / scale).to(BF16)
    c = dict(T=T, N=N, K=K, x=x, head=head, tau=1.0)
    if labels:
        c["labels"] = torch.where(rand(T) < ignored, torch.full_like(y, -100), y)
        c["d_ce"] = (rand(T) + 0.5) / T
    if top:
        idx = torch.randint(0, N, (T, top), generator=g, device="cuda")          # an index may come twice
        idx[:, 0] = y
        idx = torch.where(rand(T, top) < absent, -1 - idx % 7, idx)
        idx[rand(T) < ignored] = -1
        c["top_index"], c["top_logits"] = idx, (randn(T, top) * 3.0).to(dtype)
        c["d_distill"] = (rand(T) + 0.5) / T
    return c


def forward(c, ws=None, dirty=True):
    T, N, K = c["T"], c["N"], c["K"]
    out = {}
    top = c["top_index"].shape[1] if "top_index" in c else 0
    ws = b.alloc_head_ws(T, N, K, top=top) if ws is None else ws
    if dirty:
        ws.fill_(0xFF)                                     # NaN everywhere: contents need no initialisation
    if not top:
        loss, lse = torch.full((T,), NAN, device="cuda"), torch.full((T,), NAN, device="cuda")
        b.sbn_head_cross_entropy(c["x"], c["head"], c["labels"], loss, lse, ws=ws)
        return dict(ce=loss, lse_ce=lse, lse=lse)
    labels = c.get("labels")
    lse = torch.full((1 if labels is None else 2, T), NAN, device="cuda")
    out["distill"] = torch.full((T,), NAN, device="cuda")
    if labels is not None:
        out["ce"] = torch.full((T,), NAN, device="cuda")
    b.sbn_head_distill(c["x"], c["head"], c["top_index"], c["top_logits"], c["tau"], out["distill"], lse, labels=labels,
                       ce_loss=out.get("ce"), ws=ws)
    out["lse"], out["lse_distill"] = lse, lse[0]
    if labels is not None:
        out["lse_ce"] = lse[1]
    return out


def backward(c, lse, dx=True, dhead=True, ws=None, dirty=True):
    T, N, K = c["T"], c["N"], c["K"]
    top = c["top_index"].shape[1] if "top_index" in c else 0
    ws = b.alloc_head_ws(T, N, K, top=top, backward=True) if ws is None else ws
    if dirty:
        ws.fill_(0xFF)
    dx = torch.full((T, K), NAN, dtype=BF16, device="cuda") if dx else None
    dhead = torch.full((N, K), NAN, dtype=BF16, device="cuda") if dhead else None
    if not top:
        b.sbn_head_cross_entropy_backward(c["x"], c["head"], c["labels"], lse, c["d_ce"], dx=dx, dhead=dhead, ws=ws)
    else:
        b.sbn_head_distill_backward(c["x"], c["head"], c["top_index"], c["top_logits"], c["tau"], lse, c["d_distill"],
                                    labels=c.get("labels"), d_ce=c.get("d_ce") if "labels" in c else None, dx=dx, dhead=dhead, ws=ws)
    return dx, dhead


def reference(c):
    kw = dict(tau=c["tau"], d_ce=c.get("d_ce"), d_distill=c.get("d_distill"))
    o = oh.head_loss(c["x"], c["head"], c.get("labels"), c.get("top_index"), c.get("top_logits"), **kw)
    return o, oh.bounds(o, **kw)


def assert_near(name, got, want, bound):
    err = (got.double() - want).abs()
    bad = torch.nonzero(~(err <= bound))
    assert bad.numel() == 0, (f"{name}: {bad.shape[0]} of {err.numel()} beyond the bound, first at {bad[0].tolist()}: got "
                              f"{got[tuple(bad[0])].item()}, want {want[tuple(bad[0])].item()}, bound {bound[tuple(bad[0])].item()}")


def check(c, o=None, bd=None):
    if o is None:
        o, bd = reference(c)
    f = forward(c)
    for name in ("ce", "distill", "lse_ce", "lse_distill"):
        if name in f and name in o:
            assert_near(name, f[name], o[name], bd[name])
    dx, dhead = backward(c, f["lse"])
    b.sbn_check_status()
    assert_near("dx", dx, o["dx"], bd["dx"])
    assert_near("dhead", dhead, o["dhead"], bd["dhead"])
    assert not dx[~o["counts"]].any()
    return f, dx, dhead


# one token, one word, widths that leave part of a tile, of a chunk, of a stage; rows around the tile's 32, 64, 128, 256
CE_SHAPES = [(1, 1, 128), (1, 2, 128), (1, 1009, 256), (2, 33, 128), (5, 31, 384), (31, 64, 128), (33, 65, 256), (64, 129, 128), (65, 255, 256), (127, 257, 128),
             (129, 300, 640), (255, 511, 128), (257, 1000, 384), (300, 4099, 640), (513, 1537, 256), (700, 333, 1152), (1030, 2050, 512)]


@pytest.mark.parametrize("T,N,K", CE_SHAPES)
def test_cross_entropy(T, N, K):
    check(make(T, N, K, seed=T + N + K))


@pytest.mark.parametrize("T,N,K", [(1, 130, 128), (77, 500, 256), (300, 700, 256)])
def test_cross_entropy_no_row_left_out(T, N, K):
    check(make(T, N, K, seed=7 + T, ignored=0.0))


# few tokens: the register-fed kernels' widths (up to 8 or 16 tokens; K in one, two, five, eight shares of 512, ragged) and the
# sizes on either side of them
@pytest.mark.parametrize("top", [0, 7, 64, 65, 100])
@pytest.mark.parametrize("T,N,K", [(16, 4001, 128), (8, 1300, 256), (1, 4099, 1024), (1, 17, 4096), (3, 2500, 640), (7, 1000, 2560), (8, 16, 512), (8, 5003, 1152), (8, 999, 3200), (9, 15, 128),
                                   (9, 3000, 2560), (13, 1601, 1024), (16, 2401, 2560), (16, 700, 2688), (9, 700, 4096), (8, 300, 4224), (17, 333, 512)])
def test_few_tokens(T, N, K, top):
    check(make(T, N, K, seed=T + N + K, top=top))


# up to 256 tokens words are on the lanes: token groups of 32 and more, tiles of 256 words, more tiles than CTA pairs; sizes beyond that, too
@pytest.mark.parametrize("top", [0, 11])
@pytest.mark.parametrize("T,N,K", [(17, 129, 128), (32, 20001, 256), (47, 1000, 2560), (49, 19007, 384), (96, 128, 1024), (161, 5000, 128), (192, 301, 4224),
                                   (250, 38500, 128), (256, 2049, 640), (257, 2049, 640), (320, 19001, 256), (333, 900, 384), (385, 38500, 128), (448, 3000, 512), (449, 700, 256)])
def test_words_on_the_lanes(T, N, K, top):
    check(make(T, N, K, seed=T + N + K, top=top))


# the vocabulary in several pieces, the last one short; dx from several slices of each piece, from one, and from half tiles
@pytest.mark.parametrize("T,N,K", [(3, 12007, 4096), (200, 11009, 4096), (400, 24001, 2048), (5000, 30011, 256), (2100, 70001, 128)])
def test_cross_entropy_in_pieces(T, N, K):
    c = make(T, N, K, seed=T + K)
    assert b.sbn_head_workspace_bytes(T, N, K, backward=True) < 2 * T * N + 10 * T * K * 4 + (160 << 20)
    check(c)


# every tile shape of logits and gradients, at sizes that leave part of a tile, of its halves, of its last 128 columns
@pytest.mark.parametrize("tile", [64, 128, 256, 512])
@pytest.mark.parametrize("T,N,K,top", [(500, 1500, 128, 0), (1100, 513, 640, 0), (700, 3333, 896, 5), (2600, 2560, 512, 3)])
def test_every_tile_shape(tile, T, N, K, top):
    b.sbn_set_gemm_tuning(-tile, 0)
    check(make(T, N, K, seed=tile + T, top=top))


def test_cross_entropy_wide_token_groups():
    # more than 16 row tiles: the second group of row tiles goes over the vocabulary again
    check(make(4500, 1100, 128, seed=3))


@pytest.mark.parametrize("T", [1, 64, 300, 600])
def test_every_row_left_out(T):
    c = make(T, 200, 256, seed=5)
    c["labels"].fill_(-1)
    c["x"].fill_(NAN)
    f = forward(c)
    dx, dhead = backward(c, f["lse"])
    b.sbn_check_status()
    assert not f["ce"].any() and not f["lse"].any() and not dx.any() and not dhead.any()


@pytest.mark.parametrize("T", [12, 200, 700])
@pytest.mark.parametrize("hold", [NAN, INF, -INF, 3.3895e38])
def test_rows_left_out_reach_nothing(hold, T):
    c = make(T, 400, 256, seed=11)
    out = c["labels"] < 0
    assert 0 < int(out.sum()) < T
    o, bd = reference(c)
    clean = check(c, o, bd)
    c["x"][out] = hold
    c["d_ce"][out] = NAN
    dirty = check(c, o, bd)
    for p, q in zip(clean[1:], dirty[1:]):
        assert torch.equal(p, q)
    assert torch.equal(clean[0]["ce"], dirty[0]["ce"])


@pytest.mark.parametrize("where", ["first", "last", "one", "alternate"])
def test_which_rows_count(where):
    T = 730
    c = make(T, 500, 128, seed=13, ignored=0.0)
    drop = torch.zeros(T, dtype=torch.bool, device="cuda")
    if where == "first":
        drop[:200] = True
    elif where == "last":
        drop[100:] = True
    elif where == "one":
        drop[:] = True
        drop[257] = False
    else:
        drop[::2] = True
    c["labels"][drop] = -(2 ** 40)
    check(c)


@pytest.mark.parametrize("T", [9, 100, 700])
def test_labels_outside_the_vocabulary_are_reported(T):
    c = make(T, 300, 128, seed=17, ignored=0.1)
    o, bd = reference(c)
    bad = torch.tensor([3, T // 2, T - 1], device="cuda")
    c["labels"][bad] = torch.tensor([300, 2 ** 31, 2 ** 40], device="cuda")
    f = forward(c)
    with pytest.raises(b.SbnError) as err:
        b.sbn_check_status()
    assert err.value.code == 9
    b.sbn_check_status()                                            # reported once
    assert torch.isnan(f["ce"][bad]).all() and not f["lse"][bad].any()
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[bad] = False
    assert_near("ce", f["ce"][rest], o["ce"][rest], bd["ce"][rest])
    dx, dhead = backward(c, f["lse"])
    with pytest.raises(b.SbnError):
        b.sbn_check_status()
    ref = dict(c, labels=torch.where(rest, c["labels"], torch.full_like(c["labels"], -1)))
    o, bd = reference(ref)
    assert_near("dx", dx, o["dx"], bd["dx"])
    assert_near("dhead", dhead, o["dhead"], bd["dhead"])


def test_extreme_logits():
    # logits of several hundred: the maximum has to come off before exp
    c = make(70, 300, 128, seed=19, scale=4.0, lean=0.0)
    o, bd = reference(c)
    assert float(o["Z"].abs().max()) > 100
    check(c, o, bd)


def test_sure_rows():
    # one word far ahead of all others: loss next to zero, gradient next to zero
    c = make(40, 500, 256, seed=23, ignored=0.0, lean=30.0)
    check(c)


DISTILL = [  # T, N, K, top, teacher type, tau, with labels
    (1, 1, 128, 1, F32, 1.0, False), (1, 7, 128, 9, F32, 1.0, True), (2, 1000, 128, 3, BF16, 2.0, False), (33, 65, 256, 1, F32, 0.5, True),
    (64, 300, 128, 256, F32, 1.0, True), (100, 4099, 256, 255, BF16, 4.0, True), (129, 513, 384, 17, BF16, 1.5, False), (257, 2000, 256, 32, F32, 2.0, True),
    (300, 1111, 640, 64, F32, 2.0, False), (1030, 700, 128, 5, F32, 1.0, True)]


@pytest.mark.parametrize("T,N,K,top,dtype,tau,labels", DISTILL)
def test_distill(T, N, K, top, dtype, tau, labels):
    c = make(T, N, K, seed=T + N + K + top, top=top, dtype=dtype, labels=labels)
    c["tau"] = tau
    check(c)


@pytest.mark.parametrize("T,N,K,top", [(260, 24001, 2048, 40), (3000, 50021, 128, 12)])
def test_distill_in_pieces(T, N, K, top):
    c = make(T, N, K, seed=29, top=top)
    c["tau"] = 2.0
    check(c)


def test_distill_masked_entries():
    # -inf and the type's lowest value as teacher logits; rows with nothing but those; a single entry; one index in every place
    T, N, K, top = 40, 300, 128, 12
    for dtype in (F32, BF16):
        for tau in (0.25, 1.0):
            c = make(T, N, K, seed=31, top=top, dtype=dtype, ignored=0.0, absent=0.0)
            c["tau"] = tau
            low = torch.finfo(dtype).min
            c["top_logits"][0:4, 3:] = -INF
            c["top_logits"][4:8, 3:] = low
            c["top_logits"][8, :] = -INF                            # left out (its label stays)
            c["top_logits"][9, :] = low                             # uniform
            c["top_index"][10, 1:] = -1
            c["top_index"][11, :] = -5                              # left out
            c["top_index"][12, :] = 299
            c["top_logits"][13, :6] = low
            c["top_index"][14, ::2] = -1
            c["top_logits"][14, ::2] = NAN                          # not there: not looked at
            c["labels"][[8, 11, 20]] = -1                           # 8 and 11: nothing asked of the row
            c["x"][8] = NAN
            f, dx, dhead = check(c)
            assert float(f["distill"][8]) == 0.0 and float(f["distill"][11]) == 0.0 and float(f["ce"][20]) == 0.0
            assert not dx[8].any() and not dx[11].any()


@pytest.mark.parametrize("T", [14, 50, 600])
def test_distill_index_outside_the_vocabulary(T):
    c = make(T, 300, 128, seed=37, top=6, ignored=0.0, absent=0.0)
    ref = dict(c, top_index=c["top_index"].clone())
    c["top_index"][7, 2] = 300
    c["top_index"][8, 0] = 2 ** 40
    c["labels"][9] = 300
    ref["top_index"][[7, 8]] = -1
    ref["labels"] = c["labels"].clone()
    ref["labels"][9] = -1
    f = forward(c)
    with pytest.raises(b.SbnError) as err:
        b.sbn_check_status()
    assert err.value.code == 9
    assert torch.isnan(f["distill"][[7, 8]]).all() and torch.isnan(f["ce"][9]) and torch.isfinite(f["ce"][[7, 8]]).all()
    o, bd = reference(ref)
    dx, dhead = backward(c, f["lse"])
    with pytest.raises(b.SbnError):
        b.sbn_check_status()
    assert_near("dx", dx, o["dx"], bd["dx"])
    assert_near("dhead", dhead, o["dhead"], bd["dhead"])


@pytest.mark.parametrize("T", [5, 16, 90, 400])
def test_a_teacher_logit_that_is_no_number_stays_in_its_row(T):
    c = make(T, 600, 128, seed=91, top=5, ignored=0.0, absent=0.0)
    clean, o = forward(c), None
    bad = [1, T - 1]
    c["top_logits"][bad[0], 2] = NAN
    c["top_logits"][bad[1], :] = INF
    f = forward(c)
    b.sbn_check_status()
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[bad] = False
    assert torch.isnan(f["distill"][bad]).all() and torch.equal(f["distill"][rest], clean["distill"][rest])
    assert torch.equal(f["ce"], clean["ce"]) and torch.equal(f["lse"], clean["lse"])
    dx, _ = backward(c, f["lse"], dhead=False)
    assert torch.isfinite(dx[rest]).all()


@pytest.mark.parametrize("T", [3, 20, 300])
def test_heads_past_two_to_the_31_elements(T):
    N, K = 540001, 4096
    g = torch.Generator(device="cuda").manual_seed(97)
    head = torch.empty(N, K, dtype=BF16, device="cuda").normal_(0.0, 0.02, generator=g)
    x = torch.randn(T, K, generator=g, device="cuda").to(BF16)
    labels = torch.randint(0, N, (T,), generator=g, device="cuda")
    labels[0], labels[1] = N - 1, -1
    d = torch.rand(T, generator=g, device="cuda")
    c = dict(T=T, N=N, K=K, x=x, head=head, labels=labels, d_ce=d)
    f = forward(c, dirty=False)
    dx, dhead = backward(c, f["lse"], dirty=False)
    b.sbn_check_status()
    X = torch.where((labels >= 0)[:, None], x, torch.zeros_like(x)).double()
    Z = torch.cat([X @ head[a:a + 40000].double().T for a in range(0, N, 40000)], 1)
    lse = torch.logsumexp(Z, 1)
    has = labels >= 0
    want = torch.where(has, lse - Z.gather(1, labels.clamp(min=0)[:, None])[:, 0], 0.0)
    # one rounding or cut to 24 bits per 16 columns, of running sums below 8: 256 * 2^-23 * 8 = 2.5e-4, for lse and for the label's logit
    assert float((f["ce"].double() - want).abs().max()) < 5e-4
    P = torch.exp(Z - lse[:, None]) * torch.where(has, d, 0.0).double()[:, None]
    P[torch.arange(T, device="cuda")[has], labels[has]] -= d[has].double()
    ref = sum(P[:, a:a + 40000] @ head[a:a + 40000].double() for a in range(0, N, 40000))
    assert float((dx.double() - ref).norm() / ref.norm()) < 2.0 ** -7 and not dx[1].any()
    for a, e in ((0, 300), (N // 2, N // 2 + 300), (N - 300, N)):
        r = P[:, a:e].T @ X
        assert float((dhead[a:e].double() - r).norm() / r.norm()) < 2.0 ** -7, (a, e)


def test_two_streams_at_once():
    # two steps on two streams with workspaces of their own, no order between them: both right
    cs = [make(300, 5000, 512, seed=101), make(60, 9000, 1024, seed=103, top=6), make(4, 7000, 512, seed=107)]
    refs = [reference(c) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = []
    for rep in range(3):
        for c, s in zip(cs, streams):
            with torch.cuda.stream(s):
                f = forward(c, dirty=False)
                got.append((c, f, *backward(c, f["lse"], dirty=False)))
    torch.cuda.synchronize()
    for i, (c, f, dx, dhead) in enumerate(got):
        o, bd = refs[i % 3]
        assert_near("ce", f["ce"], o["ce"], bd["ce"])
        assert_near("dx", dx, o["dx"], bd["dx"])
        assert_near("dhead", dhead, o["dhead"], bd["dhead"])


def test_distill_with_one_entry_is_cross_entropy():
    # top = 1, tau = 1: q = 1 at the label, so both losses are the same up to where the label's logit comes from (the products for a
    # teacher's entry, a sum of its own for a label; check() holds both to the bound), and the gradients are the same bits
    c = make(130, 900, 256, seed=41, ignored=0.2)
    d = dict(c, top_index=c["labels"][:, None].contiguous(), top_logits=torch.zeros(130, 1, device="cuda"), d_distill=c["d_ce"])
    del d["labels"], d["d_ce"]
    f, dx, dhead = check(c)
    g, ex, ehead = check(d)
    assert torch.equal(f["lse"], g["lse"][0]) and torch.equal(dx, ex) and torch.equal(dhead, ehead)


@pytest.mark.parametrize("top", [0, 5])
@pytest.mark.parametrize("T,N,K", [(140, 700, 256), (5, 3000, 384), (14, 2700, 1152), (400, 3000, 384), (1100, 20000, 640)])
def test_either_gradient_alone(T, N, K, top):
    c = make(T, N, K, seed=43, top=top)
    f = forward(c)
    dx, dhead = backward(c, f["lse"])
    only_dx, none = backward(c, f["lse"], dhead=False)
    assert none is None and torch.equal(dx, only_dx)
    none, only_dhead = backward(c, f["lse"], dx=False)
    assert none is None and torch.equal(dhead, only_dhead)


def test_gradient_is_the_slope_of_the_loss():
    # central differences of the library's own losses along a direction: bf16 steps that are exact
    c = make(64, 300, 128, seed=47, ignored=0.2)
    c["x"] = torch.round(c["x"].float() * 16).clamp(-64, 64).div(16).to(BF16)
    f = forward(c)
    dx, _ = backward(c, f["lse"], dhead=False)
    step = torch.randint(-1, 2, c["x"].shape, generator=torch.Generator().manual_seed(1)).to("cuda").float() / 16
    up, down = (dict(c, x=(c["x"].float() + s * step).to(BF16)) for s in (1, -1))
    assert torch.equal(up["x"].float() - c["x"].float(), step)
    fu, fd = forward(up), forward(down)
    slope = (fu["ce"].double() - fd["ce"].double()) / 2 * c["d_ce"].double()
    o, bd = reference(c)
    u = step.double() @ c["head"].double().T                        # change of the logits
    third = (u.max(1).values - u.min(1).values) ** 3                # |f'''| of log-sum-exp along a line, over 6 below
    want = (dx.double() * step.double()).sum(1)
    tol = (bd["dx"] * step.abs().double()).sum(1) + c["d_ce"].double() * (third / 6 + bd["ce"] * 2)
    has = c["labels"] >= 0
    assert bool(((slope - want).abs() <= tol)[has].all()), ((slope - want).abs() / tol)[has].max()
    assert float(slope[has].abs().max()) > 5 * float(tol[has].median())


def test_same_bits_from_call_to_call_and_on_another_stream():
    c = make(500, 3001, 512, seed=53, top=9)
    f = forward(c)
    dx, dhead = backward(c, f["lse"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = forward(c)
        ex, ehead = backward(c, g["lse"])
    torch.cuda.current_stream().wait_stream(s)
    for k in f:
        assert torch.equal(f[k], g[k]), k
    assert torch.equal(dx, ex) and torch.equal(dhead, ehead)


def test_calls_back_to_back_on_one_workspace():
    # no synchronisation in between: each call overwrites the workspace the one before it used
    cs = [make(T, N, K, seed=59 + T, top=top) for T, N, K, top in ((300, 2000, 256, 0), (70, 900, 512, 4), (300, 2000, 256, 7), (1, 500, 128, 0))]
    n = max(b.sbn_head_workspace_bytes(c["T"], c["N"], c["K"], c["top_index"].shape[1] if "top_index" in c else 0, w) for c in cs for w in (False, True))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    got = []
    for c in cs:
        f = forward(c, ws=ws, dirty=False)
        got.append((f, *backward(c, f["lse"], ws=ws, dirty=False)))
    for c, (f, dx, dhead) in zip(cs, got):
        o, bd = reference(c)
        for name in ("ce", "distill"):
            if name in f and name in o:
                assert_near(name, f[name], o[name], bd[name])
        assert_near("dx", dx, o["dx"], bd["dx"])
        assert_near("dhead", dhead, o["dhead"], bd["dhead"])


@pytest.mark.parametrize("top", [0, 6])
@pytest.mark.parametrize("T,N,K", [(200, 1500, 256), (7, 2000, 512), (900, 1500, 256), (1300, 9000, 1024)])
def test_captured_into_a_graph(T, N, K, top):
    # a whole step in a graph, replayed on other inputs (other rows left out) in the same buffers
    c = make(T, N, K, seed=61, top=top)
    ws = [b.alloc_head_ws(T, N, K, top=top, backward=w) for w in (False, True)]
    f = forward(c, ws=ws[0])
    backward(c, f["lse"], ws=ws[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f = forward(c, ws=ws[0])
        dx, dhead = backward(c, f["lse"], ws=ws[1])
    for seed in (67, 71):
        new = make(T, N, K, seed=seed, top=top, ignored=0.6 if seed == 67 else 0.0)
        for k, v in new.items():
            if torch.is_tensor(v):
                c[k].copy_(v)
        g.replay()
        o, bd = reference(c)
        for name in ("ce", "distill"):
            if name in f and name in o:
                assert_near(name, f[name], o[name], bd[name])
        assert_near("dx", dx, o["dx"], bd["dx"])
        assert_near("dhead", dhead, o["dhead"], bd["dhead"])


@pytest.mark.parametrize("T,N,K", [(3, 33, 128), (130, 700, 256), (300, 1000, 384), (600, 1000, 384)])
def test_nothing_is_written_outside_the_outputs(T, N, K):
    c = make(T, N, K, seed=73)
    pad = 4096

    def guarded(shape, dtype):
        n = shape[0] * (shape[1] if len(shape) > 1 else 1)
        buf = torch.full((n + 2 * pad,), 7.0, dtype=dtype, device="cuda")
        return buf, buf[pad:pad + n].view(shape)

    bufs = {k: guarded(s, d) for k, s, d in (("loss", (T,), F32), ("lse", (T,), F32), ("dx", (T, K), BF16), ("dhead", (N, K), BF16))}
    wss = []
    for back in (False, True):
        n = b.sbn_head_workspace_bytes(T, N, K, backward=back)
        wss.append((n, torch.full((n + 2 * pad,), 0x5A, dtype=torch.uint8, device="cuda")))
    b.sbn_head_cross_entropy(c["x"], c["head"], c["labels"], bufs["loss"][1], bufs["lse"][1], ws=wss[0][1][pad:pad + wss[0][0]])
    b.sbn_head_cross_entropy_backward(c["x"], c["head"], c["labels"], bufs["lse"][1], c["d_ce"], dx=bufs["dx"][1], dhead=bufs["dhead"][1],
                                      ws=wss[1][1][pad:pad + wss[1][0]])
    b.sbn_check_status()
    for k, (buf, view) in bufs.items():
        assert bool((buf[:pad] == 7).all()) and bool((buf[pad + view.numel():] == 7).all()), k
        assert bool(torch.isfinite(view).all())
    for n, ws in wss:
        assert bool((ws[:pad] == 0x5A).all()) and bool((ws[pad + n:] == 0x5A).all())


def test_waits_are_bounded():
    c = make(300, 700, 256, seed=79)
    f = forward(c)
    try:
        b.sbn_set_wait_test(True, 1000)
        forward(c)
        with pytest.raises(b.SbnError) as err:
            b.sbn_check_status()
        assert err.value.code == 7
        backward(c, f["lse"])
        with pytest.raises(b.SbnError) as err:
            b.sbn_check_status()
        assert err.value.code == 7
    finally:
        b.sbn_set_wait_test(False, 0)
    check(c)


def test_a_training_step_together():
    """Quantiser, sparse layer, head, loss, the head's gradients, the layer's gradients: one chain on one stream, its losses and
    gradients against the same chain in float64 from the layer's own output on."""
    T, K, H, V = 192, 256, 384, 1237
    g = torch.Generator(device="cuda").manual_seed(83)
    W = torch.randn(H, K, generator=g, device="cuda") * 0.05
    x = torch.randn(T, K, generator=g, device="cuda").to(BF16)
    head = (torch.randn(V, H, generator=g, device="cuda") * 0.05).to(BF16)
    labels = torch.randint(-300, V, (T,), generator=g, device="cuda")
    p = b.alloc_packed(H, K)
    xq, sc = b.alloc_xq(T, K), torch.empty(T, device="cuda")
    y = torch.empty(T, H, dtype=BF16, device="cuda")
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dy, dhead = torch.empty_like(y), torch.empty_like(head)
    dX, dW = torch.empty_like(x), torch.empty_like(W)
    d = torch.full((T,), 1.0, device="cuda") / (labels >= 0).sum()
    b.sbn_quantize_mask_pack(W, p["vals"], p["meta"], p["w_scale"], p["ws"])
    b.sbn_quant_act(x, xq, sc)
    b.sbn_sparse_bitlinear(xq, sc, p["vals"], p["meta"], p["w_scale"], y, ws=b.alloc_gemm_ws(b.OP_SPARSE_BITLINEAR, T, H, K))
    b.sbn_head_cross_entropy(y, head, labels, loss, lse, ws=b.alloc_head_ws(T, V, H))
    b.sbn_head_cross_entropy_backward(y, head, labels, lse, d, dx=dy, dhead=dhead, ws=b.alloc_head_ws(T, V, H, backward=True))
    ws = torch.empty(b.sbn_workspace_bytes(b.OP_BACKWARD, T, H, K), dtype=torch.uint8, device="cuda")
    b.sbn_bitlinear_backward(dy, xq, sc, p["vals"], p["meta"], p["w_scale"], H, K, dX=dX, dW=dW, ws=ws)
    b.sbn_check_status()
    o = oh.head_loss(y, head, labels, d_ce=d)
    bd = oh.bounds(o, d_ce=d)
    assert_near("loss", loss, o["ce"], bd["ce"])
    assert_near("dy", dy, o["dx"], bd["dx"])
    assert_near("dhead", dhead, o["dhead"], bd["dhead"])
    # dW = dy^T x_q: the fake-quantised activations are the input within half a quantisation step
    want = dy.double().T @ x.double()
    step = sc.double()
    assert bool(((dW.double() - want).abs() <= dy.double().abs().T @ ((0.51 * step + 2.0 ** -8 * 127 * step)[:, None].expand(T, K)) + 1e-30).all())
    assert float(want.abs().max()) > 0 and bool(torch.isfinite(dX).all())


@pytest.mark.parametrize("change", ["x_dtype", "x_strided", "labels_int32", "labels_short", "loss_dtype", "head_cols", "cpu_head", "ws_cpu"])
def test_binding_refuses_wrong_tensors(change):
    c = make(20, 100, 128, seed=89)
    loss, lse, ws = torch.empty(20, device="cuda"), torch.empty(20, device="cuda"), b.alloc_head_ws(20, 100, 128)
    x, head, labels = c["x"], c["head"], c["labels"]
    if change == "x_dtype":
        x = x.float()
    elif change == "x_strided":
        x = torch.cat([x, x], 1)[:, :128]
    elif change == "labels_int32":
        labels = labels.int()
    elif change == "labels_short":
        labels = labels[:-1]
    elif change == "loss_dtype":
        loss = loss.double()
    elif change == "head_cols":
        head = head[:, :64].contiguous()
    elif change == "cpu_head":
        head = head.cpu()
    else:
        ws = ws.cpu()
    n = b.sbn_launch_count()
    with pytest.raises(ValueError):
        b.sbn_head_cross_entropy(x, head, labels, loss, lse, ws=ws)
    assert b.sbn_launch_count() == n


@pytest.mark.parametrize("top", [0, 4])
@pytest.mark.parametrize("T", [9, 100, 700])
def test_a_bad_index_does_not_hide_a_timeout(T, top):
    # a wait that ran out leaves results that are no results: that is what the status has to say, whichever came first
    broken, bad = make(300, 700, 256, seed=113), make(T, 300, 128, seed=109, top=top, ignored=0.0, absent=0.0)
    bad["top_index" if top else "labels"][T // 2] = 300

    def time_out():
        try:
            b.sbn_set_wait_test(True, 1000)
            forward(broken)
        finally:
            b.sbn_set_wait_test(False, 0)

    for order in ((time_out, lambda: forward(bad)), (lambda: forward(bad), time_out)):
        for call in order:
            call()
        with pytest.raises(b.SbnError) as err:
            b.sbn_check_status()
        assert err.value.code == 7
        b.sbn_check_status()
    forward(bad)
    with pytest.raises(b.SbnError) as err:
        b.sbn_check_status()
    assert err.value.code == 9


@pytest.mark.parametrize("T", [6, 16, 90, 400])
def test_nan_shows_in_both_losses(T):
    # a token that is no number, and words that are none: a whole share of the partial sums then has no maximum
    N, K = 3000, 256
    c = make(T, N, K, seed=127, top=5, ignored=0.0, absent=0.0)
    clean = forward(c)
    c["x"][3] = NAN
    f = forward(c)
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[3] = False
    for name in ("distill", "ce", "lse_distill", "lse_ce"):
        assert torch.isnan(f[name][3]) and torch.equal(f[name][rest], clean[name][rest]), name
    c = make(T, N, K, seed=127, top=5, ignored=0.0, absent=0.0)
    c["head"][512:1024] = NAN
    f = forward(c)
    for name in ("distill", "ce", "lse_distill", "lse_ce"):
        assert torch.isnan(f[name]).all(), name


def sure(T, N, K, seed, label_logit, top=0):
    """Tokens that know their label: its logit is near `label_logit`, the others are N(0, 1).  The teacher is as sure."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    head = (randn(N, K) * 0.02).to(BF16)
    y = torch.randint(0, N, (T,), generator=g, device="cuda")
    rows = head[y].float()
    x = (randn(T, K) + label_logit * rows / (rows * rows).sum(1, keepdim=True)).to(BF16)
    c = dict(T=T, N=N, K=K, x=x, head=head, tau=1.0, labels=y, d_ce=torch.full((T,), 1.0 / T, device="cuda"))
    if top:
        index = (y[:, None] + torch.arange(top, device="cuda") * (N // top)) % N        # the label's entry is the first
        c["top_index"], c["top_logits"] = index, torch.where(torch.arange(top, device="cuda") == 0, label_logit, 0.0) + randn(T, top)
        c["d_distill"] = c["d_ce"]
    return c


@pytest.mark.parametrize("top", [0, 5])
@pytest.mark.parametrize("label_logit", [20.0, 30.0, 40.0])
@pytest.mark.parametrize("T,K", [(4, 2560), (16, 2560), (8, 4096), (40, 2560), (200, 4096), (300, 2560), (1100, 4096)])
def test_losses_of_sure_tokens(T, K, label_logit, top):
    """A sure token's loss is what the other words add to a sum of 1: with S = 1 + rest in fp32, each of at most 64 additions a thread's
    and a row's sums go through once the label is in (40 for its 4 chunks of 32 words, 16 + 8 to put them together) is rounded by at
    most 2^-24 of something below 2, so rest is off by 64 * 2^-23 = 7.7e-6 at worst.  Beside that only what the logits
    themselves are off by, relative to the loss.  A cross entropy is never below 0; a divergence not by more than its q are rounded
    (2^-24 per entry and one for log q)."""
    c = sure(T, 5000, K, 131 + T, label_logit, top)
    o, bd = reference(c)
    bz = K * 2.0 ** -23 * (o["X"].abs() @ o["W"].abs().T).max(1).values            # as in oracle/head.py
    f = forward(c)
    b.sbn_check_status()
    # exp(2 bz) - 1 of the loss, and ex2's and its argument's error of every term (2^-16)
    tol = o["ce"] * (torch.expm1(2 * bz) + 2.0 ** -16) + 64 * 2.0 ** -23
    assert float(f["ce"].min()) >= 0.0, float(f["ce"].min())
    assert_near("ce", f["ce"], o["ce"], tol)
    if top:
        kd = o["distill"].abs() + (o["Q"] * (o["Z"] - o["Z"].max(1, keepdim=True).values).abs()).sum(1)
        tol = kd * (torch.expm1(2 * bz) + 2.0 ** -16) + 64 * 2.0 ** -23 + (top + 2) * 2.0 ** -24
        assert float(f["distill"].min()) >= -(top + 2) * 2.0 ** -24, float(f["distill"].min())
        assert_near("distill", f["distill"], o["distill"], tol)


@pytest.mark.parametrize("big", [(1 << 32) + 4, -(1 << 32) + 4, 1 << 70])
def test_workspace_of_sizes_past_32_bits(big):
    forward(make(4, 100, 128, seed=137))                    # the extension is there
    for at in range(3):
        sizes = [4, 1000, 256]
        sizes[at] = big
        with pytest.raises(ValueError):
            b.alloc_head_ws(*sizes)


@pytest.mark.parametrize("tau", [0.1, 0.01, 2.0 ** -10])
@pytest.mark.parametrize("T", [6, 60, 400])
def test_small_temperatures(T, tau):
    # logits up to 8: z / tau up to 8192, and p 2^-24 * 8192 = 5e-4 off beside bf16's own roundings (2^-8 at most, each)
    c = make(T, 700, 256, seed=5 + T, top=5, labels=False, ignored=0.0, scale=0.1)
    c["tau"] = tau
    o, _ = reference(c)
    f, dx, dhead = check(c)
    for got, want in ((dx, o["dx"]), (dhead, o["dhead"])):
        assert float((got.double() - want).norm() / want.norm()) < 2 * 2.0 ** -8 + 2.0 ** -10


@pytest.mark.parametrize("T", [6, 60, 400])
def test_temperatures_that_only_the_loss_has(T):
    c = make(T, 700, 256, seed=5 + T, top=5, labels=False, ignored=0.0, scale=0.1)
    for tau in (1e-4, 1e-8):
        c["tau"] = tau
        o, bd = reference(dict(c, d_distill=None))
        f = forward(c)
        assert_near("distill", f["distill"], o["distill"], bd["distill"])
        with pytest.raises(b.SbnError) as err:
            backward(c, f["lse"])
        assert err.value.code == 4


# ---- how near the results are, beside the worst case that check() allows ----
# T, N, K, tile: up to 16 tokens (dz in two parts where `two`), words on the lanes, row tiles with narrow and with wide gradients
ACCURACY = [(8, 5003, 2560, 0, True), (8, 5003, 4096, 0, True), (16, 5003, 1024, 0, True), (16, 5003, 2560, 0, False), (40, 5003, 2560, 0, False),
            (200, 9001, 2560, 0, False), (600, 9001, 2560, -256, False), (2100, 5003, 2560, -512, False), (300, 5003, 4096, 0, False)]
# One rounding to bf16 is off by something even between -2^(e-8) and 2^(e-8) for values from 2^e to 2^(e+1): 2^-8 / sqrt(3) of the value in the
# 2-norm at most (values just above a power of two).  5 % for what the logits' own errors and the small entries of dz add
ONE_ROUNDING = 1.05 * 2.0 ** -8 / 3 ** 0.5


def relative(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("T,N,K,tile,two", ACCURACY)
def test_gradients_of_a_mean_are_off_by_one_rounding(T, N, K, tile, two):
    # no token knows its label: its dz is -d (1 - p), p around 1 / N.  All d alike, half way between two bf16 numbers: the unit that dz is
    # kept in makes it -1, else every target would be off by 2^-8 in the same direction (2-norm 4e-3 instead of 1.7e-3)
    b.sbn_set_gemm_tuning(tile, 0)
    c = make(T, N, K, seed=139 + T, ignored=0.0, lean=0.0)
    c["d_ce"].fill_((0.5 + 2.0 ** -9) / 1024)
    o, _ = reference(c)
    dx, dhead = backward(c, forward(c)["lse"])
    b.sbn_check_status()
    assert relative(dx, o["dx"]) < ONE_ROUNDING
    assert relative(dhead, o["dhead"]) < ONE_ROUNDING


@pytest.mark.parametrize("T,N,K,tile,two", ACCURACY)
def test_gradients_with_weights_of_their_own(T, N, K, tile, two):
    # every second token's weight is half way between two bf16 numbers even in the call's unit.  Two parts of dz: the results' own rounding is
    # all there is.  One part: that and at most 2^-8 of every entry of dz, independent of each other and of it
    b.sbn_set_gemm_tuning(tile, 0)
    c = make(T, N, K, seed=149 + T, ignored=0.0, lean=0.0)
    c["d_ce"].fill_(1.0 / 1024)
    c["d_ce"][1::2] = (0.5 + 2.0 ** -9) / 1024
    o, _ = reference(c)
    dx, dhead = backward(c, forward(c)["lse"])
    b.sbn_check_status()
    tol = ONE_ROUNDING if two else 1.05 * 2.0 ** -8 * (4 / 3) ** 0.5
    assert relative(dx, o["dx"]) < tol
    assert relative(dhead, o["dhead"]) < tol
    if two:                                                 # token by token: one part would be 4e-3 off in every second
        rows = (dx.double() - o["dx"]).norm(dim=1) / o["dx"].norm(dim=1)
        assert float(rows.max()) < tol, rows


@pytest.mark.parametrize("top", [0, 7])
@pytest.mark.parametrize("T,N,K,tile,two", ACCURACY)
def test_losses_are_not_off_in_one_direction(T, N, K, tile, two, top):
    # logits N(0, 3^2): what the tensor cores cut off would make lse, and with it every loss, K 2^-30 E_p[z] too small on average (2e-5 at
    # 2560 columns); the factor that takes it back leaves a fifth of it or less.  Half of it is the line here, for the rounding of c0 and the losses (less than 2^-24 of lse each) besides
    b.sbn_set_gemm_tuning(tile, 0)
    c = make(T, N, K, seed=151 + T, ignored=0.0, lean=0.0, scale=3.0 / K ** 0.5, top=top, absent=0.0)
    o, _ = reference(c)
    f = forward(c)
    b.sbn_check_status()
    P = torch.softmax(o["Z"], 1)
    bias = K * 2.0 ** -30 * float((P * o["Z"]).sum(1).mean())
    for name in ("ce", "distill") if top else ("ce",):
        err = f[name].double() - o[name]
        assert abs(float(err.mean())) < 0.5 * bias + 2.0 ** -23 * float(o["lse_ce"].abs().mean()), (name, float(err.mean()), bias)
        # a single loss: the bias once more, and the label's (or the entries') logit in fp32: sqrt(24) additions of at most |z| (12) / 2^24
        assert float(err.pow(2).mean().sqrt()) < bias + 5 * 12 * 2.0 ** -24 + 2.0 ** -23 * float(o["lse_ce"].abs().mean()) + \
            (K * 2.0 ** -30 * 3.0 if top else 0.0), name


@pytest.mark.parametrize("kind", ["whole", "sparse", "steady"])
@pytest.mark.parametrize("T,K,tile", [(8, 2560, 0), (16, 2560, 0), (60, 2560, 0), (256, 8192, 0), (300, 2560, 0), (700, 8192, -512)])
def test_logits_that_nothing_or_much_is_cut_off(T, K, tile, kind):
    """The factor is made for sums of changing sign.  Sums that fit 24 bits ("whole": small whole numbers; "sparse": a few entries that are not 0) lose
    nothing and come out K 2^-30 too large; sums that only grow ("steady") lose more than it gives back: an MMA of 16 columns cuts off less
    than 2^-23 of the running sum, which is half of the logit on average, K / 16 times: K 2^-28 of the logit at most."""
    N = 3001
    b.sbn_set_gemm_tuning(tile, 0)
    g = torch.Generator(device="cuda").manual_seed(157 + T)
    whole = lambda lo, hi, *s: torch.randint(lo, hi + 1, s, generator=g, device="cuda").float()
    if kind == "whole":
        x, head = whole(-3, 3, T, K), whole(-2, 2, N, K) / 64
    elif kind == "sparse":
        at = torch.randint(0, K, (T, 4), generator=g, device="cuda")
        x, head = torch.zeros(T, K, device="cuda").scatter_(1, at, whole(-4, 4, T, 4) * 4), whole(-8, 8, N, K) / 16
    else:
        x, head = torch.rand(T, K, generator=g, device="cuda"), torch.rand(N, K, generator=g, device="cuda") * 80 / K
    y = torch.randint(0, N, (T,), generator=g, device="cuda")
    c = dict(T=T, N=N, K=K, x=x.to(BF16), head=head.to(BF16), tau=1.0, labels=y, d_ce=torch.full((T,), 1.0 / T, device="cuda"))
    if kind == "sparse":
        c["x"][::2, 5] = 24.0                               # tokens that know their label: its logit is 24, exactly
        c["head"][:, 5] = 0.0
        c["head"][y[::2], 5] = 1.0
        c["x"][::2, :5] = 0.0
        c["x"][::2, 6:] = 0.0
    o, _ = reference(c)
    f = forward(c)
    b.sbn_check_status()
    Z = o["Z"]
    share = 2.0 ** -28 if kind == "steady" else 2.0 ** -30
    # and what lse and loss have besides: 64 additions of the sum, ex2 (2^-22), c0 and its product (2^-24 of the logits' range each), the
    # results' rounding and the label's logit in fp32 (5 of them)
    rest = 64 * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -23 * (Z.max(1).values - Z.min(1).values) + 5 * 2.0 ** -24 * (o["lse_ce"].abs() + Z.abs().max(1).values)
    tol = K * share * Z.abs().max(1).values + rest
    assert_near("lse", f["lse"], o["lse_ce"], tol)
    assert_near("ce", f["ce"], o["ce"], tol)
    assert float(f["ce"].min()) >= 0.0


@pytest.mark.parametrize("T,K,tile", [(8, 2560, 0), (16, 2560, 0), (60, 2560, 0), (256, 8192, 0), (300, 2560, 0), (700, 8192, -512)])
def test_sure_tokens_whose_logits_are_exact(T, K, tile):
    # one entry of x per token, in a column of its own where only the label's word is not 0: its logit is 24 exactly, all others are 0, and the loss
    # is log(1 + 3000 exp(-24)) = 1.1e-7, up to 64 additions to a sum of 1 (see test_losses_of_sure_tokens)
    N = 3001
    b.sbn_set_gemm_tuning(tile, 0)
    at = torch.arange(T, device="cuda")
    y = (at * 7 + 3) % N
    x, head = torch.zeros(T, K, device="cuda"), torch.zeros(N, K, device="cuda")
    x[at, at * 3 + 5], head[y, at * 3 + 5] = 24.0, 1.0
    f = forward(dict(T=T, N=N, K=K, x=x.to(BF16), head=head.to(BF16), labels=y))
    b.sbn_check_status()
    want = torch.full((T,), 3000.0, dtype=torch.float64, device="cuda").mul(torch.exp(torch.tensor(-24.0, dtype=torch.float64))).log1p()
    assert float(f["ce"].min()) >= 0.0
    assert_near("ce", f["ce"], want, torch.full_like(want, 64 * 2.0 ** -23))


# 1 to 16 tokens with more columns than the register-fed kernels take; several groups of tokens, the last one with a token or a few
@pytest.mark.parametrize("top", [0, 9])
@pytest.mark.parametrize("T,N,K", [(1, 300, 4224), (3, 1, 5120), (8, 2000, 8192), (16, 1000, 4224), (97, 1000, 384), (225, 513, 256), (193, 4100, 128), (129, 9001, 256)])
def test_words_on_the_lanes_in_groups(T, N, K, top):
    check(make(T, N, K, seed=T + N + K, top=top))


# tokens of a whole batch: pieces of the vocabulary at their narrowest (1024 words), many row tiles, dx added up piece by piece
@pytest.mark.parametrize("T,N,K,top", [(20011, 5000, 256, 0), (66001, 2100, 128, 0), (9001, 4200, 384, 3)])
def test_tokens_of_a_whole_batch(T, N, K, top):
    check(make(T, N, K, seed=163, top=top))


@pytest.mark.parametrize("T,tile", [(100, 0), (256, 0), (600, -512)])
def test_waits_are_bounded_with_words_on_the_lanes_and_wide_tiles(T, tile):
    b.sbn_set_gemm_tuning(tile, 0)
    c = make(T, 1700, 640, seed=167, top=3)
    f = forward(c)
    try:
        b.sbn_set_wait_test(True, 1000)
        for call in (lambda: forward(c), lambda: backward(c, f["lse"]), lambda: backward(c, f["lse"], dx=False), lambda: backward(c, f["lse"], dhead=False)):
            call()
            with pytest.raises(b.SbnError) as err:
                b.sbn_check_status()
            assert err.value.code == 7
    finally:
        b.sbn_set_wait_test(False, 0)
    check(c)


@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("T,N,K", [(9, 2003, 1152), (12, 5003, 2048), (16, 5003, 2560)])
def test_gradients_of_few_tokens_are_off_by_their_own_rounding(T, N, K, top):
    # as test_gradients_with_weights_of_their_own, token by token and for the labels' words: dz in one part is 4e-3 off there
    c = make(T, N, K, seed=173 + T, ignored=0.0, lean=0.0, top=top, absent=0.0)
    c["labels"] = torch.arange(T, device="cuda") * (N // T) + 5
    c["d_ce"].fill_(1.0 / 1024)
    c["d_ce"][1::2] = (0.5 + 2.0 ** -9) / 1024
    if top:
        c["d_distill"] = c["d_ce"] / 2
    o, _ = reference(c)
    dx, dhead = backward(c, forward(c)["lse"])
    b.sbn_check_status()
    for got, want in ((dx, o["dx"]), (dhead[c["labels"]], o["dhead"][c["labels"]])):
        rows = (got.double() - want).norm(dim=1) / want.norm(dim=1)
        assert float(rows.max()) < ONE_ROUNDING, rows


@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("T,N,K", [(9, 2003, 2688), (17, 2003, 1152), (33, 5003, 2560), (64, 1300, 1024), (65, 1300, 1024), (97, 5003, 512), (128, 19001, 384)])
def test_gradients_of_up_to_128_tokens_are_off_by_their_own_rounding(T, N, K, top):
    c = make(T, N, K, seed=179 + T, ignored=0.0, lean=0.0, top=top, absent=0.0)
    c["labels"] = torch.arange(T, device="cuda") * (N // T) + 5
    c["d_ce"].fill_(1.0 / 1024)
    c["d_ce"][1::2] = (0.5 + 2.0 ** -9) / 1024
    if top:
        c["d_distill"] = c["d_ce"] / 2
    o, _ = reference(c)
    dx, dhead = backward(c, forward(c)["lse"])
    b.sbn_check_status()
    for got, want in ((dx, o["dx"]), (dhead[c["labels"]], o["dhead"][c["labels"]])):
        rows = (got.double() - want).norm(dim=1) / want.norm(dim=1)
        assert float(rows.max()) < ONE_ROUNDING * 1.03, rows       # (a row of 384 values: 3 % more than its expectation)


@pytest.mark.parametrize("T", [20, 64, 65, 128, 129])
def test_rows_left_out_of_both_parts(T):
    # tokens that nothing is asked of in every place of a 64, gradients of either kind alone, and NaN in them
    c = make(T, 900, 384, seed=181 + T, ignored=0.5)
    c["x"][c["labels"] < 0] = NAN
    f, dx, dhead = check(c)
    assert torch.equal(backward(c, f["lse"], dhead=False)[0], dx) and torch.equal(backward(c, f["lse"], dx=False)[1], dhead)


@pytest.mark.parametrize("top", [0, 6])
@pytest.mark.parametrize("T,N,K", [(12, 2000, 1152), (50, 700, 384), (64, 1500, 256), (128, 1500, 256)])
def test_two_parts_captured_and_within_their_buffers(T, N, K, top):
    # a step in a graph, replayed on other inputs; outputs and workspaces between guards
    c, pad = make(T, N, K, seed=191, top=top), 4096
    n = [b.sbn_head_workspace_bytes(T, N, K, top, w) for w in (False, True)]
    held = [torch.full((m + 2 * pad,), 0x5A, dtype=torch.uint8, device="cuda") for m in n]
    ws = [h[pad:pad + m] for h, m in zip(held, n)]
    outs = {k: torch.full((m * K + 2 * pad,), 7.0, dtype=BF16, device="cuda") for k, m in (("dx", T), ("dhead", N))}
    dx, dhead = outs["dx"][pad:pad + T * K].view(T, K), outs["dhead"][pad:pad + N * K].view(N, K)

    def step():
        f = forward(c, ws=ws[0], dirty=False)
        if top:
            b.sbn_head_distill_backward(c["x"], c["head"], c["top_index"], c["top_logits"], c["tau"], f["lse"], c["d_distill"], labels=c["labels"],
                                        d_ce=c["d_ce"], dx=dx, dhead=dhead, ws=ws[1])
        else:
            b.sbn_head_cross_entropy_backward(c["x"], c["head"], c["labels"], f["lse"], c["d_ce"], dx=dx, dhead=dhead, ws=ws[1])
        return f

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f = step()
    for seed in (193, 197):
        new = make(T, N, K, seed=seed, top=top, ignored=0.6 if seed == 193 else 0.0)
        for k, v in new.items():
            if torch.is_tensor(v):
                c[k].copy_(v)
        g.replay()
        o, bd = reference(c)
        for name in ("ce", "distill"):
            if name in f and name in o:
                assert_near(name, f[name], o[name], bd[name])
        assert_near("dx", dx, o["dx"], bd["dx"])
        assert_near("dhead", dhead, o["dhead"], bd["dhead"])
    for h, m in zip(held, n):
        assert bool((h[:pad] == 0x5A).all()) and bool((h[pad + m:] == 0x5A).all())
    for k, m in (("dx", T), ("dhead", N)):
        assert bool((outs[k][:pad] == 7).all()) and bool((outs[k][pad + m * K:] == 7).all()), k
