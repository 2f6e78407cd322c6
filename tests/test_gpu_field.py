"""The operators over the candidates of a field against the oracle in 64 bits.

Tolerances come from the arithmetic.  e = 2^-24.  A logit of K products in fp32 in any order is off by at most
(K + 2) e (|w_j| + sum_k |G_ik v_jk|) =: ez_ij.  Scaled and shifted, x = scale z is off by
a_i = scale max_j ez_ij + 4 e max_j |x_ij|.  2^x of the hardware is good to 2^-22, a sum of C positive terms, independent
roundings, to 4 sqrt(C) e.  So lse is off by a_i + 2^-21 + 4 sqrt(C) e + 4 e |lse|, and a probability, relatively, by
D_i = 2 a_i + 2^-20 + 4 sqrt(C) e + 4 e |lse|; the entropy by (1 + H) D_i.  A gradient is a sum of terms d_ij v_jk or d_ij G_ik
whose factors are off by D_i; adding m of them costs another 4 sqrt(m) e + 2^-20 of the sum of their absolute values."""
import numpy as np
import pytest

from oracle import field_oracle as F

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


def _torch():
    import torch
    return torch


def _bits(allowed):
    """[rows x C] truth values as int32 words."""
    rows, C = allowed.shape
    pad = np.zeros((rows, (C + 31) // 32 * 32), np.uint8)
    pad[:, :C] = allowed
    return np.packbits(pad, axis=1, bitorder="little").view(np.int32).copy()


def _data(seed, n, C, K, T, vtype, mask, grid):
    """Inputs as the GPU gets them, on the host.  grid: values whose logits are exact in fp32."""
    torch = _torch()
    rng = np.random.default_rng(seed)
    V = (rng.normal(size=(C, K)) * 0.4).astype(np.float32)
    G = (rng.normal(size=(n, K)) * (4 / np.sqrt(K))).astype(np.float32)
    w = (rng.normal(size=C) - 0.3 * np.log1p(np.arange(C))).astype(np.float32)
    if grid:
        V, G, w = (np.clip(np.round(x * s), -m, m).astype(np.float32) / s for x, s, m in
                   ((V, 64, 255), (G, 32, 511), (w, 64, 2047)))  # a coarse grid: many logits are equal
    Vd = torch.from_numpy(V).to(getattr(torch, vtype))
    allowed = None
    if mask == "shared":
        allowed = rng.random((1, C)) < 0.8
    elif mask == "rows":
        allowed = rng.random((n, C)) < 0.6
        allowed[n // 2] = False            # nothing left
        if n > 2:
            allowed[n - 1] = False
            allowed[n - 1, C - 1] = True   # one candidate left, the last one
    ids = np.stack([rng.permutation(C)[:T] if C >= T else rng.integers(0, C, T) for _ in range(n)]) if T else np.zeros((n, 0), int)
    ids = np.where(rng.random(ids.shape) < 0.15, -1, ids).astype(np.int32)
    if T and n > 3:
        ids[1] = -1
        ids[3, 0] = C  # outside
    teacher = (rng.normal(size=(n, T)) * 3).astype(np.float32)
    weight = (rng.random(n) * (rng.random(n) < 0.9)).astype(np.float32)
    return dict(V=Vd, G=G, w=w, allowed=allowed, ids=ids, teacher=teacher, weight=weight)


def _exact(d, scale):
    V = d["V"].double().numpy()
    z = F.logits(d["G"], V, d["w"], d["allowed"])
    return V, z


def _off(d, V, z, scale):
    """a_i and D_i above, and lse's own bound."""
    n, C = z.shape
    K = V.shape[1]
    live = z > -np.inf
    size = np.abs(d["G"].astype(np.float64)) @ np.abs(V).T + np.abs(d["w"].astype(np.float64))
    x = np.where(live, np.abs(scale * np.where(live, z, 0)), 0).max(1)
    a = scale * (K + 2) * E * np.where(live, size, 0).max(1) + 4 * E * x
    lse = F.log_softmax(z, scale)[1]
    lse = np.where(np.isfinite(lse), np.abs(lse), 0)
    return a, 2 * a + 2.0 ** -20 + 4 * np.sqrt(C) * E + 4 * E * lse, a + 2.0 ** -21 + 4 * np.sqrt(C) * E + 4 * E * lse


def _near(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=what)
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)], err_msg=what)
    bad = fine & ~(np.abs(got - np.where(fine, want, 0)) <= np.broadcast_to(tol, got.shape))
    if bad.any():
        at = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}{at}: got {got[at]:.9e}, want {want[at]:.9e}, tolerance {np.broadcast_to(tol, got.shape)[at]:.2e}; {bad.sum()} of {bad.size}")


def _dev(x):
    return None if x is None else _torch().from_numpy(np.ascontiguousarray(x)).cuda()


def _field(C, K, n, top=0):
    from paper_2004_13940_amd import binding as B
    return B.Field(C, K, max_rows=max(n, 1), max_top=top)


def _run_logprobs(d, scale, top, field=None, V=None, G=None):
    torch = _torch()
    n, K = d["G"].shape
    C, T = d["V"].shape[0], d["ids"].shape[1]
    f = field or _field(C, K, n, top)
    out = dict(lse=torch.full((n,), 7.0), entropy=torch.full((n,), 7.0), logprob=torch.full((n, T), 7.0))
    if top:
        out.update(top_ids=torch.full((n, top), 7, dtype=torch.int32), top_logprob=torch.full((n, top), 7.0))
    out = {k: v.cuda() for k, v in out.items()}
    f.fm_field_logprobs(_dev(d["G"]) if G is None else G, d["V"].cuda() if V is None else V, w=_dev(d["w"]),
                        mask=None if d["allowed"] is None else _dev(_bits(d["allowed"])), scale=scale, ids=_dev(d["ids"]), **out)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in out.items()}


def _run_distill(d, scale, field=None, V=None, G=None, weight=True):
    torch = _torch()
    n, K = d["G"].shape
    C = d["V"].shape[0]
    f = field or _field(C, K, n)
    out = {k: torch.full(s, 7.0, device="cuda") for k, s in
           dict(loss=(n,), grad_G=(n, K), grad_V=(C, K), grad_w=(C,)).items()}
    f.fm_field_distill(_dev(d["G"]) if G is None else G, d["V"].cuda() if V is None else V, _dev(d["ids"]), _dev(d["teacher"]),
                       w=_dev(d["w"]), mask=None if d["allowed"] is None else _dev(_bits(d["allowed"])), scale=scale,
                       weight=_dev(d["weight"]) if weight else None, **out)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in out.items()}


def _check_logprobs(got, d, scale, top):
    V, z = _exact(d, scale)
    want = F.logprobs(z, scale, d["ids"], top)
    a, D, tol = _off(d, V, z, scale)
    _near(got["lse"], want["lse"], tol, "lse")
    _near(got["entropy"], want["entropy"], (1 + np.abs(np.nan_to_num(want["entropy"]))) * D, "entropy")
    _near(got["logprob"], want["logprob"], (a + tol)[:, None], "logprob")
    if top:
        np.testing.assert_array_equal(got["top_ids"], want["top_ids"])
        _near(got["top_logprob"], want["top_logprob"], (a + tol)[:, None], "top_logprob")


def _check_distill(got, d, scale, weight=True):
    V, z = _exact(d, scale)
    n, C = z.shape
    G = d["G"].astype(np.float64)
    want = F.distill(z, G, V, scale, d["ids"], d["teacher"], d["weight"] if weight else None)
    a, D, tol = _off(d, V, z, scale)
    q = want["q"]
    Dq = 2.0 ** -20 + 8 * E * scale * np.abs(d["teacher"]).max()
    logp, _ = F.log_softmax(z, scale)
    r = scale * (d["weight"] if weight else np.ones(n)) * (q.sum(1) > 0)
    _near(got["loss"], want["loss"], (a + tol + 2 * Dq) * (q.sum(1) > 0) + 2 * Dq * np.abs(np.nan_to_num(want["loss"])) + 4 * Dq * np.log(1 + q.shape[1]) * (q.sum(1) > 0), "loss")
    p = np.where(np.isfinite(logp), np.exp(np.where(np.isfinite(logp), logp, 0)), 0)
    Q = np.zeros((n, C))
    for i in range(n):
        ok = q[i] > 0
        np.add.at(Q[i], d["ids"][i][ok], q[i][ok])
    off = r[:, None] * (p * D[:, None] + Q * Dq)
    size = r[:, None] * (p + Q)
    addC, addn = 4 * np.sqrt(C) * E + 2.0 ** -20, 4 * np.sqrt(n) * E + 2.0 ** -20
    _near(got["grad_G"], want["grad_G"], (off + addC * size) @ np.abs(V) + 1e-30, "grad_G")
    _near(got["grad_V"], want["grad_V"], (off + addn * size).T @ np.abs(G) + 1e-30, "grad_V")
    _near(got["grad_w"], want["grad_w"], (off + addn * size).sum(0) + 1e-30, "grad_w")


SIZES = [  # n, C, K, T
    (1, 1, 1, 1), (1, 2, 16, 1), (2, 33, 5, 3), (5, 64, 8, 4), (16, 63, 16, 16), (17, 65, 16, 7), (33, 257, 13, 8),
    (64, 1000, 8, 1), (65, 1023, 32, 33), (1, 20_011, 16, 2), (3, 4_097, 64, 20), (130, 515, 33, 9), (31, 777, 64, 64),
    (48, 300, 100, 5), (19, 129, 256, 3), (257, 2_050, 20, 10), (300, 96, 128, 96), (1000, 31, 16, 3), (129, 6_000, 4, 1)]


@pytest.mark.parametrize("n,C,K,T", SIZES)
@pytest.mark.parametrize("vtype,mask", [("float32", "none"), ("float32", "rows"), ("float16", "shared"), ("bfloat16", "rows")])
def test_logprobs(n, C, K, T, vtype, mask):
    print("logprobs", n, C, K, T, vtype, mask, flush=True)
    d = _data(n * 7 + C, n, C, K, T, vtype, mask, False)
    _check_logprobs(_run_logprobs(d, 0.7, 0), d, 0.7, 0)
    d = _data(n * 7 + C, n, C, K, T, vtype, mask, True)
    for top in (1, 7, 64):
        _check_logprobs(_run_logprobs(d, 1.0, top), d, 1.0, top)


@pytest.mark.parametrize("n,C,K,T", SIZES)
@pytest.mark.parametrize("vtype,mask", [("float32", "none"), ("float32", "rows"), ("float16", "rows"), ("bfloat16", "shared")])
def test_distill(n, C, K, T, vtype, mask):
    print("distill", n, C, K, T, vtype, mask, flush=True)
    d = _data(n * 5 + C, n, C, K, min(T, C), vtype, mask, False)
    _check_distill(_run_distill(d, 0.7), d, 0.7)
    _check_distill(_run_distill(d, 1.0, weight=False), d, 1.0, weight=False)


@pytest.mark.parametrize("n,C", [(7, 300), (1, 5000), (200, 1111)])
def test_what_is_left_out_may_hold_anything(n, C):
    """Masked candidates with NaN and infinities, rows without weight or candidates whose aggregates are NaN: the same values,
    bit for bit, as with ordinary numbers there."""
    K = 16
    d = _data(11, n, C, K, 5, "float32", "shared", False)
    clean = (_run_logprobs(d, 1.0, 9), _run_distill(d, 1.0))
    dirty = dict(d, V=d["V"].clone(), w=d["w"].copy())
    out = np.flatnonzero(~d["allowed"][0])
    dirty["V"][out[::3]] = float("nan")
    dirty["V"][out[1::3]] = float("inf")
    dirty["w"][out[2::3]] = np.inf
    for a, b in zip(clean, (_run_logprobs(dirty, 1.0, 9), _run_distill(dirty, 1.0))):
        for k in a:
            np.testing.assert_array_equal(a[k], b[k], err_msg=k)
    if n > 2:
        d["allowed"] = np.repeat(d["allowed"], n, 0)
        d["allowed"][2] = False
        clean = _run_distill(d, 1.0)
        d["G"][2] = np.nan
        dirty = _run_distill(d, 1.0)
        for k in clean:
            np.testing.assert_array_equal(clean[k], dirty[k], err_msg=k)


def test_a_candidate_masked_in_some_rows_only():
    """NaN in V of a candidate that one row allows and the others do not: that row is NaN, the others are not."""
    d = _data(12, 40, 500, 16, 5, "float32", "none", False)
    d["allowed"] = np.ones((40, 500), bool)
    d["allowed"][:, 77] = False
    d["allowed"][9, 77] = True
    V = d["V"].numpy()
    V[77, 3] = np.nan
    got = _run_logprobs(d, 1.0, 4)
    assert np.isnan(got["lse"][9]) and (got["top_ids"][9] == -1).all() and np.isnan(got["top_logprob"][9]).all()
    rest = np.arange(40) != 9
    for k in ("lse", "entropy", "top_logprob"):
        assert np.isfinite(got[k][rest]).all()
    got = _run_distill(d, 1.0)
    assert np.isfinite(got["loss"][rest]).all() and np.isfinite(got["grad_G"][rest]).all()
    assert d["weight"][9] == 0 or np.isnan(got["grad_G"][9]).all()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_infinite_logits(bad):
    """A weight of -inf leaves a candidate out like a mask; NaN and +inf make every row NaN."""
    d = _data(13, 20, 300, 8, 4, "float32", "none", True)
    d["w"][5] = bad
    if bad == -np.inf:
        d["ids"][0, 0] = 5
    _check_logprobs(_run_logprobs(d, 1.0, 6), d, 1.0, 6)
    if bad == -np.inf:
        _check_distill(_run_distill(d, 1.0), d, 1.0)
    else:
        got = _run_distill(d, 1.0)
        some = (d["ids"] >= 0) & (d["ids"] < 300)
        assert np.isnan(got["loss"][some.any(1)]).all()


@pytest.mark.parametrize("spread", [1e-6, 30.0, 1e4])
def test_flat_and_steep_rows(spread):
    """Logits that hardly differ, and such that all but one probability underflow."""
    d = _data(14, 37, 700, 16, 6, "float32", "none", False)
    d["G"] = (d["G"] * spread).astype(np.float32)
    d["w"] = (d["w"] * spread).astype(np.float32)
    _check_logprobs(_run_logprobs(d, 1.0, 0), d, 1.0, 0)
    if spread < 100:
        _check_distill(_run_distill(d, 1.0), d, 1.0)


def test_ascending_logits():
    """The running maximum changes all along the row."""
    d = _data(15, 40, 5000, 16, 6, "float32", "none", True)
    d["w"] = (np.arange(5000) / 64).astype(np.float32)
    _check_logprobs(_run_logprobs(d, 1.0, 20), d, 1.0, 20)
    d["w"] = (np.arange(5000) / 640).astype(np.float32)
    _check_distill(_run_distill(d, 1.0), d, 1.0)


@pytest.mark.parametrize("vtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("K", [16, 13])
def test_strides_and_alignment(vtype, K):
    """Rows of V, G and the masks that are parts of wider ones, aligned like one value."""
    torch = _torch()
    n, C = 70, 900
    d = _data(16, n, C, K, 5, vtype, "rows", True)
    V = torch.zeros(C, K + 5, dtype=d["V"].dtype, device="cuda")[:, 1:K + 1]
    V.copy_(d["V"])
    G = torch.zeros(n, K + 3, device="cuda")[:, 3:]
    G.copy_(_dev(d["G"]))
    _check_logprobs(_run_logprobs(d, 1.0, 5, V=V, G=G), d, 1.0, 5)
    d = _data(17, n, C, K, 5, vtype, "rows", False)
    V.copy_(d["V"])
    G.copy_(_dev(d["G"]))
    _check_distill(_run_distill(d, 1.0, V=V, G=G), d, 1.0)
    words = torch.zeros(n, (C + 31) // 32 + 2, dtype=torch.int32, device="cuda")[:, 1:-1]
    words.copy_(_dev(_bits(d["allowed"])))
    lse = torch.empty(n, device="cuda")
    _field(C, K, n).fm_field_logprobs(G, V, w=_dev(d["w"]), mask=words, lse=lse)
    z = _exact(d, 1.0)[1]
    _near(lse.cpu().numpy(), F.log_softmax(z)[1], _off(d, d["V"].double().numpy(), z, 1.0)[2], "lse")


def test_a_handle_serves_calls_of_every_size():
    """One handle, calls with fewer rows, other outputs and other parameters; the same call twice gives the same bits."""
    K, C = 16, 3001
    f = _field(C, K, 500, 8)
    for n in (500, 1, 77, 500):
        d = _data(n, n, C, K, 4, "float32", "none", True)
        a, b = _run_logprobs(d, 1.0, 8, field=f), _run_logprobs(d, 1.0, 8, field=f)
        _check_logprobs(a, d, 1.0, 8)
        c, e = _run_distill(d, 0.5, field=f), _run_distill(d, 0.5, field=f)
        _check_distill(c, d, 0.5)
        for x, y in ((a, b), (c, e)):
            for k in x:
                np.testing.assert_array_equal(x[k], y[k], err_msg=k)
    # single outputs, no rows
    torch = _torch()
    lse = torch.empty(500, device="cuda")
    f.fm_field_logprobs(_dev(d["G"]), d["V"].cuda(), w=_dev(d["w"]), lse=lse)
    np.testing.assert_array_equal(lse.cpu().numpy(), a["lse"])
    only = torch.full((500, K), 7.0, device="cuda")
    f.fm_field_distill(_dev(d["G"]), d["V"].cuda(), _dev(d["ids"]), _dev(d["teacher"]), w=_dev(d["w"]), weight=_dev(d["weight"]),
                       scale=0.5, grad_G=only)
    np.testing.assert_array_equal(only.cpu().numpy(), c["grad_G"])
    gw = torch.full((C,), 7.0, device="cuda")
    f.fm_field_distill(torch.empty(0, K, device="cuda"), d["V"].cuda(), torch.empty(0, 4, dtype=torch.int32, device="cuda"),
                       torch.empty(0, 4, device="cuda"), grad_w=gw)
    assert (gw == 0).all()


def test_gradient_is_the_difference_of_the_loss():
    """Central differences of the fp32 losses themselves, along random directions: a step h along directions of unit size changes
    the loss by about h |gradient|, a loss of size L is known to about 2^-19 L, the third derivative is of the order of 1."""
    torch = _torch()
    d = _data(18, 24, 200, 8, 5, "float32", "rows", False)
    V = d["V"].numpy()
    got = _run_distill(d, 1.0)
    rng = np.random.default_rng(5)
    h = 2.0 ** -6
    weight = d["weight"].astype(np.float64)
    for name, x in (("grad_G", d["G"]), ("grad_V", V), ("grad_w", d["w"])):
        u = rng.normal(size=x.shape)
        u = (u / np.linalg.norm(u)).astype(np.float32)
        keep = x.copy()
        total = []
        for sign in (1, -1):
            x[...] = keep + np.float32(sign * h) * u
            total.append((weight * _run_distill(d, 1.0)["loss"]).sum())
        x[...] = keep
        slope, want = (total[0] - total[1]) / (2 * h), (got[name].astype(np.float64) * u).sum()
        size = (weight * np.abs(got["loss"])).sum()
        assert abs(slope - want) <= 2.0 ** -19 * size / h + 10 * h * h, (name, slope, want)


def test_another_stream_and_graph_replay():
    """Work goes to the given stream; a captured call gives the eager call's bits at every replay."""
    torch = _torch()
    d = _data(19, 100, 2000, 16, 4, "float32", "none", True)
    want, grads = _run_logprobs(d, 1.0, 5), _run_distill(d, 1.0)
    f = _field(2000, 16, 100, 5)
    s = torch.cuda.Stream()
    G, V, w, ids, teacher, weight = _dev(d["G"]), d["V"].cuda(), _dev(d["w"]), _dev(d["ids"]), _dev(d["teacher"]), _dev(d["weight"])
    out = dict(lse=torch.empty(100, device="cuda"), top_ids=torch.empty(100, 5, dtype=torch.int32, device="cuda"))
    back = dict(grad_V=torch.empty(2000, 16, device="cuda"), loss=torch.empty(100, device="cuda"))
    torch.cuda.synchronize()

    def calls():
        f.fm_field_logprobs(G, V, w=w, **out)
        f.fm_field_distill(G, V, ids, teacher, w=w, weight=weight, **back)

    def same():
        for k, v in out.items():
            np.testing.assert_array_equal(v.cpu().numpy(), want[k], err_msg=k)
        for k, v in back.items():
            np.testing.assert_array_equal(v.cpu().numpy(), grads[k], err_msg=k)

    with torch.cuda.stream(s):
        calls()
    s.synchronize()
    same()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for _ in range(3):
        for v in (*out.values(), *back.values()):
            v.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        same()


def test_offsets_beyond_32_bits():
    """A table whose rows lie further apart than 2^32 bytes in all: the last candidates are the best ones."""
    torch = _torch()
    C, K = 70_000, 16
    rng = np.random.default_rng(20)
    wide = torch.empty(C * 16_500, dtype=torch.float32, device="cuda")  # 4.6 GB, 66,000 bytes from row to row
    V = wide.view(C, 16_500)[:, 16_484:]
    small = torch.from_numpy((np.round(rng.normal(size=(C, K)) * 32) / 64).astype(np.float32)).cuda()
    V.copy_(small)
    G = torch.from_numpy((np.round(rng.normal(size=(20, K)) * 32) / 32).astype(np.float32)).cuda()
    a, b = (dict(lse=torch.empty(20, device="cuda"), top_ids=torch.empty(20, 9, dtype=torch.int32, device="cuda")) for _ in range(2))
    f = _field(C, K, 20, 9)
    f.fm_field_logprobs(G, V, **a)
    f.fm_field_logprobs(G, small, **b)
    ids = torch.randint(0, C, (20, 3), device="cuda", dtype=torch.int32)
    teacher = torch.randn(20, 3, device="cuda")
    ga, gb = (dict(grad_G=torch.empty(20, K, device="cuda"), grad_V=torch.empty(C, K, device="cuda")) for _ in range(2))
    f.fm_field_distill(G, V, ids, teacher, **ga)
    f.fm_field_distill(G, small, ids, teacher, **gb)
    for x, y in ((a, b), (ga, gb)):
        for k in x:
            assert torch.equal(x[k], y[k]), k


def test_refusals():
    from paper_2004_13940_amd import binding as B
    torch = _torch()
    for args in ((0, 8, 1, 0), (1 << 31, 8, 1, 0), (10, 0, 1, 0), (10, 65, 1, 0), (10, 8, 0, 0), (10, 8, 1, 65), (10, 8, 1, -1)):
        with pytest.raises(B.FMError):
            B.Field(*args)
    f = B.Field(100, 8, 10, 4)
    G, V, w = torch.zeros(10, 8, device="cuda"), torch.zeros(100, 8, device="cuda"), torch.zeros(100, device="cuda")
    lse = torch.empty(10, device="cuda")
    f.fm_field_logprobs(G, V, w=w, lse=lse)
    ids, teacher = torch.zeros(10, 2, dtype=torch.int32, device="cuda"), torch.zeros(10, 2, device="cuda")

    def refused(error, call, *args, **kw):
        with pytest.raises(error):
            call(*args, **kw)

    lp, ds = f.fm_field_logprobs, f.fm_field_distill
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        refused(B.FMError, lp, G, V, scale=scale, lse=lse)
        refused(B.FMError, ds, G, V, ids, teacher, scale=scale)
    refused(B.FMError, lp, torch.zeros(11, 8, device="cuda"), V, lse=torch.empty(11, device="cuda"))       # too many rows
    refused(B.FMError, lp, G, V, top_ids=torch.empty(10, 5, dtype=torch.int32, device="cuda"))             # top > max_top
    refused(B.FMError, lp, G, V, logprob=torch.empty(10, 0, device="cuda"), mask=None, scale=-1.0)
    refused(ValueError, lp, G, V[:99], lse=lse)
    refused(ValueError, lp, G[:, :7], V, lse=lse)
    refused(TypeError, lp, G.double(), V, lse=lse)
    refused(TypeError, lp, G, V.double(), lse=lse)
    refused(TypeError, lp, G.cpu(), V, lse=lse)
    refused(TypeError, lp, G, torch.zeros(8, 100, device="cuda").t(), lse=lse)
    refused(ValueError, lp, G, V, lse=torch.empty(9, device="cuda"))
    refused(TypeError, lp, G, V, lse=torch.empty(10, device="cuda", dtype=torch.float64))
    refused(ValueError, lp, G, V, lse=lse, mask=torch.zeros(10, 3, dtype=torch.int32, device="cuda"))
    refused(ValueError, lp, G, V, lse=lse, mask=torch.zeros(9, 4, dtype=torch.int32, device="cuda"))
    refused(TypeError, lp, G, V, lse=lse, mask=torch.zeros(10, 4, device="cuda"))
    refused(ValueError, lp, G, V, logprob=torch.empty(10, 2, device="cuda"))                               # without ids
    refused(TypeError, ds, G, V, ids.long(), teacher)
    refused(ValueError, ds, G, V, ids, teacher[:, :1].contiguous())
    refused(B.FMError, ds, G, V, ids[:, :0].contiguous(), teacher[:, :0].contiguous())                     # no entries
    refused(ValueError, ds, G, V, ids, teacher, grad_V=torch.empty(99, 8, device="cuda"))
    # through the C entry: strides, types and null pointers
    lib, st = B.load(), torch.cuda.current_stream().cuda_stream
    import ctypes

    def entry(n=10, g_stride=8, top=0, G=G.data_ptr(), handle=f._h, **kw):
        c = B.fm_candidates(V.data_ptr(), w.data_ptr(), None, 8, 0, B.FM_TYPE_F32, 1.0)
        for k, v in kw.items():
            setattr(c, k, v)
        return lib.fm_field_logprobs(handle, ctypes.byref(c), n, G, g_stride, 0, None, None, lse.data_ptr(), None, top, None, None, st)

    assert entry() == B.FM_OK and entry(n=0) == B.FM_OK
    for kw in (dict(n=-1), dict(n=11), dict(top=5)):
        assert entry(**kw) == B.FM_ERANGE, kw
    for kw in (dict(g_stride=7), dict(v_stride=7), dict(v_stride=1 << 50), dict(v_type=3), dict(v_type=-1), dict(V=None), dict(G=None),
               dict(V=V.data_ptr() + 2), dict(w=w.data_ptr() + 1), dict(mask=w.data_ptr(), mask_stride=3), dict(handle=None)):
        assert entry(**kw) == B.FM_EINVAL, kw
    assert b"mask_stride" in lib.fm_field_last_error(f._h) or lib.fm_field_last_error(f._h)
    torch.cuda.synchronize()


@pytest.mark.parametrize("n,C,K,T,vtype,mask", [
    (1700, 20_011, 16, 7, "float32", "rows"), (1700, 20_011, 16, 7, "float16", "shared"), (300, 30_001, 64, 33, "bfloat16", "rows"),
    (330, 12_345, 100, 5, "float32", "none"), (230, 9_000, 200, 5, "float32", "rows"), (230, 9_001, 256, 5, "bfloat16", "none"),
    (1700, 9_999, 20, 10, "float16", "rows"), (3000, 5_003, 33, 1, "float32", "shared")])
def test_from_the_packed_table(n, C, K, T, vtype, mask):
    """Calls with so many products that the table is laid out first, at every number of chunks and parts."""
    print("packed", n, C, K, T, vtype, mask, flush=True)
    d = _data(n + C, n, C, K, T, vtype, mask, True)
    _check_logprobs(_run_logprobs(d, 1.0, 9), d, 1.0, 9)
    d = _data(n + C, n, C, K, T, vtype, mask, False)
    _check_logprobs(_run_logprobs(d, 0.6, 0), d, 0.6, 0)
    _check_distill(_run_distill(d, 0.6), d, 0.6)


@pytest.mark.parametrize("n", [1, 2, 3, 4])
@pytest.mark.parametrize("C,K,vtype", [(70_001, 16, "float16"), (30_000, 16, "float32"), (9_999, 8, "float32"), (40_003, 8, "bfloat16"),
                                       (25_000, 32, "bfloat16"), (66_000, 4, "float32"), (33_333, 64, "float16")])
def test_few_rows_of_a_large_field(n, C, K, vtype):
    print("few", n, C, K, vtype, flush=True)
    for mask in ("none", "shared", "rows"):
        d = _data(n + C, n, C, K, 3, vtype, mask, True)
        _check_logprobs(_run_logprobs(d, 1.0, 10), d, 1.0, 10)
        d = _data(n + C, n, C, K, 3, vtype, mask, False)
        _check_logprobs(_run_logprobs(d, 0.7, 0), d, 0.7, 0)


def test_every_row_names_the_same_candidates():
    """More entries in a block of candidates than lanes, and all of them at the same few candidates."""
    d = _data(31, 500, 9_000, 16, 40, "float32", "none", False)
    d["ids"] = np.tile(np.arange(40, dtype=np.int32), (500, 1))
    d["ids"][::3] += 8_950
    _check_distill(_run_distill(d, 0.7), d, 0.7)


@pytest.mark.parametrize("n,C", [(1, 300_000), (20, 300_000), (2100, 20_000)])
def test_equal_logits_go_to_the_lowest_numbers(n, C):
    """All logits equal, or equal in long runs: the best are the first ones."""
    torch = _torch()
    K = 4
    f = _field(C, K, n, 20)
    V, G = torch.ones(C, K, device="cuda"), torch.ones(n, K, device="cuda")
    ids = torch.empty(n, 20, dtype=torch.int32, device="cuda")
    f.fm_field_logprobs(G, V, top_ids=ids)
    assert (ids.cpu() == torch.arange(20)).all()
    w = torch.zeros(C, device="cuda")
    w[C // 2 + 3:] = 1.0
    f.fm_field_logprobs(G, V, w=w, top_ids=ids)
    assert (ids.cpu() == C // 2 + 3 + torch.arange(20)).all()
    w[C - 7] = 2.0
    f.fm_field_logprobs(G, V, w=w, top_ids=ids)
    assert (ids.cpu()[:, 0] == C - 7).all() and (ids.cpu()[:, 1:] == C // 2 + 3 + torch.arange(19)).all()


def test_handles_without_distillation_and_too_many_entries():
    from paper_2004_13940_amd import binding as B
    torch = _torch()
    f = B.Field(100, 8, 10, max_entries=0)
    G, V = torch.zeros(10, 8, device="cuda"), torch.zeros(100, 8, device="cuda")
    lse = torch.empty(10, device="cuda")
    f.fm_field_logprobs(G, V, lse=lse)
    assert abs(lse.cpu().numpy() - np.log(100)).max() < 1e-5
    ids, teacher = torch.zeros(10, 2, dtype=torch.int32, device="cuda"), torch.zeros(10, 2, device="cuda")
    for h in (f, B.Field(100, 8, 10, max_entries=1)):
        with pytest.raises(B.FMError):
            h.fm_field_distill(G, V, ids, teacher)
    B.Field(100, 8, 10, max_entries=2).fm_field_distill(G, V, ids, teacher)
    torch.cuda.synchronize()


def test_a_model_of_a_field_learns_from_its_teacher():
    from paper_2004_13940_amd import next_item
    losses, hit = next_item.run(N=3_000, held_out=500, fields=6, width=100, C=600, K=8, T=8, steps=40, eta=5.0)
    assert np.isfinite(losses).all() and losses[-1] < 0.95 * losses[0]
    assert hit > 3 * 10 / 600  # three times what ten items drawn at random would have
