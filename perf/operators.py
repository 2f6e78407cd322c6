"""The operators over the candidates of a field, as timed cases.

A row that holds everything but one one-hot field scores candidate j of that field as  z_ij = w_j + <G_i, v_j>  plus a
constant of the row: G are its aggregates, v_j and w_j the parameters of the field's columns.  Over the candidates this
is a softmax, and the operators are

  logprobs   log probabilities of given candidates, log-sum-exp, entropy and the best candidates of every row
  distill    the loss against a teacher's top logits and its gradient by G, V and w

`listed()` holds the cases, `draw()` more of the same ranges, `prepare()` makes what a program has in hand before the
call, `run()` is one pass, `exact()` the same from the definitions in 64 bits.  Fields of a case:
  op, n rows, C candidates, K latent size, type of V (f32, f16, bf16), T given candidates or teacher entries to a row,
  top best candidates to return, mask: none, shared (one for all rows: what is in stock) or rows (one to each row: what
  it has not seen yet; some rows have nothing left), scale: 1 / temperature.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LOG_MIN = -math.inf  # the logit of a candidate that is left out


def listed():
    return [
        # One user, the tiny workload's thousand features as the field: launches and latency.
        dict(name="lp_one_tiny", op="logprobs", n=1, C=1_000, K=8, type="f32", T=1, top=5, mask="none", scale=1.0),
        # One user against all columns of the click-style workload, its table held in half precision.
        dict(name="lp_one_click", op="logprobs", n=1, C=1_000_000, K=16, type="f16", T=1, top=10, mask="none",
             scale=1.0),
        # A few users over a hashed table whose V is far beyond the caches.
        dict(name="lp_few_hashed", op="logprobs", n=3, C=4_000_000, K=64, type="f32", T=1, top=20, mask="shared",
             scale=1.0),
        # A batch of requests for one field of the click-style workload, with what is out of stock left out.
        dict(name="lp_requests", op="logprobs", n=64, C=38_461, K=16, type="f32", T=1, top=10, mask="shared",
             scale=0.7),
        # Requests with lists of what each user has seen, and several given candidates to a row.
        dict(name="lp_seen", op="logprobs", n=501, C=20_000, K=16, type="f16", T=4, top=8, mask="rows", scale=1.0),
        # Evaluation of the text-like workload: the probability of the held-out term of every row, and the entropy.
        dict(name="lp_eval_text", op="logprobs", n=50_000, C=20_000, K=16, type="f32", T=1, top=0, mask="none",
             scale=1.0),
        # Evaluation with the best ten, large latent size, table in bfloat16.
        dict(name="lp_eval_wide", op="logprobs", n=8_191, C=38_461, K=64, type="bf16", T=1, top=10, mask="none",
             scale=1.0),
        # Smallest training step: some rows of the tiny workload.
        dict(name="ds_tiny", op="distill", n=33, C=1_000, K=8, type="f32", T=8, mask="none", scale=1.0),
        # A batch over the text-like workload's terms.
        dict(name="ds_text", op="distill", n=2_000, C=20_000, K=16, type="f32", T=16, mask="none", scale=0.5),
        # Large batch over one field of the click-style workload.
        dict(name="ds_click", op="distill", n=16_384, C=38_461, K=16, type="f32", T=32, mask="none", scale=0.5),
        # Odd sizes, candidates left out row by row, table in half precision.
        dict(name="ds_seen", op="distill", n=1_025, C=9_999, K=20, type="f16", T=10, mask="rows", scale=1.0),
        # Many candidates and a large latent size, table in bfloat16, many teacher entries to a row.
        dict(name="ds_wide", op="distill", n=4_096, C=100_001, K=64, type="bf16", T=64, mask="shared", scale=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "distill"])
    K = rng.choice([4, 8, 10, 13, 16, 16, 20, 24, 32, 33, 48, 64, 64, 100, 128])
    most = 1_000_000 if op == "logprobs" else 100_000
    while True:
        n, C = _log_int(rng, 1, 20_000), _log_int(rng, 100, most)
        if n * C <= 400_000_000 and n * C * K <= 9_000_000_000 and 3072 not in (n, C):
            break
    case = dict(op=op, n=n, C=C, K=K, type=rng.choice(["f32", "f32", "f16", "bf16"]),
                T=rng.choice([1, 1, 4, 7, 16]) if op == "logprobs" else rng.choice([1, 5, 8, 16, 33, 64]),
                mask=rng.choice(["none", "none", "shared", "rows"]), scale=rng.choice([1.0, 0.5, 0.7, 1.3]))
    if op == "logprobs":
        case["top"] = rng.choice([0, 1, 5, 8, 10, 20, 32])
    return case


def _on_grid(x, step, most):
    return (x / step).round().clamp(-most, most) * step


def _bits(allowed):
    """Truth values [rows, C] as words of 32 bits, candidate j in bit j % 32 of word j / 32."""
    rows, C = allowed.shape
    words = (C + 31) // 32
    out = torch.zeros(rows, words, dtype=torch.int32, device=allowed.device)
    for b in range(32):
        part = allowed[:, b::32].to(torch.int32)
        out[:, :part.shape[1]] |= part << b
    return out


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    n, C, K, T = case["n"], case["C"], case["K"], case["T"]
    top = case.get("top", 0)

    def normal(*size):
        return torch.randn(*size, generator=g, device=dev)

    def uniform(*size):
        return torch.rand(*size, generator=g, device=dev)

    # A trained table: factors of some tenths, aggregates that make the logits' spread about 2, and linear weights that
    # fall off with the candidates' popularity.
    V = normal(C, K) * 0.3
    G = normal(n, K) * (2.0 / (0.3 * math.sqrt(K)))
    w = -0.9 * torch.log1p(torch.arange(C, device=dev, dtype=torch.float32)) + 0.3 * normal(C)
    if top:
        # Which candidates are the best is a whole number: factors as a table of 8 bits in fixed point holds them, and
        # aggregates and weights on a grid, so that every logit is exact in 32 bits in whatever order it is summed and
        # equal logits are really equal.
        V, G, w = _on_grid(V, 2.0 ** -7, 255), _on_grid(G, 2.0 ** -6, 1023), _on_grid(w, 2.0 ** -13, 2 ** 18)
    s = dict(case=case, G=G, V=V.to(TYPES[case["type"]]), w=w, mask=None)
    if case["mask"] == "shared":
        s["mask"] = _bits(uniform(1, C) < 0.9)
    elif case["mask"] == "rows":
        words = (C + 31) // 32
        a, b = (torch.randint(-2 ** 31, 2 ** 31, (n, words), generator=g, device=dev, dtype=torch.int64).to(torch.int32)
                for _ in range(2))
        s["mask"] = (a | b) * (torch.arange(n, device=dev, dtype=torch.int32) % 97 != 5).to(torch.int32)[:, None]
    # Candidates that rows name are mostly popular ones: log-uniform, distinct and ascending in a row.
    t = torch.arange(T, device=dev, dtype=torch.float64)
    u = (t + uniform(n, T).double()) / max(T, 1)
    ids = (max(C - T, 1) ** u).floor().to(torch.int64) - 1 + t.long()
    ids = ids.clamp(0, C - 1)
    count = torch.where(uniform(n, 1) < 0.8, torch.full((n, 1), T, device=dev),
                        (uniform(n, 1) * (T + 1)).floor().long())
    s["ids"] = torch.where(torch.arange(T, device=dev)[None, :] < count, ids, -1).to(torch.int32)
    if case["op"] == "distill":
        s["teacher"] = 2.0 * normal(n, T) + 1.0
        s["weight"] = (uniform(n) * 2.0 / n) * (uniform(n) > 0.05)
        s["out"] = dict(loss=torch.empty(n, device=dev), grad_G=torch.empty(n, K, device=dev),
                        grad_V=torch.empty(C, K, device=dev), grad_w=torch.empty(C, device=dev))
    else:
        s["out"] = dict(lse=torch.empty(n, device=dev), entropy=torch.empty(n, device=dev),
                        logprob=torch.empty(n, T, device=dev))
        if top:
            s["out"].update(top_ids=torch.empty(n, top, device=dev, dtype=torch.int32),
                            top_logprob=torch.empty(n, top, device=dev))
    if own:
        from paper_2004_13940_amd import binding as B
        s["field"] = B.Field(C, K, max_rows=n, max_top=top)
    return s


def run(s):
    case, out = s["case"], s["out"]
    if own:
        if case["op"] == "logprobs":
            s["field"].fm_field_logprobs(s["G"], s["V"], w=s["w"], mask=s["mask"], scale=case["scale"], ids=s["ids"],
                                         **out)
        else:
            s["field"].fm_field_distill(s["G"], s["V"], s["ids"], s["teacher"], w=s["w"], mask=s["mask"],
                                        scale=case["scale"], weight=s["weight"], **out)
        return out
    return _plain_logprobs(s) if case["op"] == "logprobs" else _plain_distill(s)


def _plain_allowed(mask, C):
    j = torch.arange(C, device=mask.device)
    return (mask[:, j >> 5] >> (j & 31).to(torch.int32)) & 1 != 0


def _plain_softmax(s):
    """Logits with -inf where a candidate is left out, their scaled values less the row's maximum, the exponentials of
    these, their sums and the log-sum-exp."""
    case = s["case"]
    z = s["G"] @ s["V"].float().t() + s["w"]
    if s["mask"] is not None:
        z = torch.where(_plain_allowed(s["mask"], case["C"]), z, LOG_MIN)
    x = z * case["scale"]
    m = x.amax(1, keepdim=True)
    m = torch.where(m == LOG_MIN, torch.zeros_like(m), m)
    x = x - m
    e = torch.exp(x)
    S = e.sum(1, keepdim=True)
    return z, x, e, S, (m + torch.log(S))[:, 0]


def _plain_logprobs(s):
    case = s["case"]
    z, x, e, S, lse = _plain_softmax(s)
    U = torch.where(e > 0, e * x, torch.zeros_like(e)).sum(1)
    S = S[:, 0]
    entropy = torch.where(S > 0, torch.log(S) - U / S, torch.zeros_like(S))
    del x, e
    ids = s["ids"].long()
    given = z.gather(1, ids.clamp(min=0)) * case["scale"]
    none = lse == LOG_MIN
    logprob = torch.where(none[:, None], torch.full_like(given, LOG_MIN), given - lse[:, None])
    out = dict(lse=lse, entropy=entropy, logprob=torch.where(ids < 0, torch.zeros_like(logprob), logprob))
    if case["top"]:
        # One whole number to a logit: its order above, the candidate's below, lower ones first.
        b = (z + 0.0).view(torch.int32)
        key = torch.where(b < 0, b ^ 0x7FFFFFFF, b).long()
        key = (key << 32) + (case["C"] - 1 - torch.arange(case["C"], device=z.device))
        most = min(case["top"], case["C"])
        at = case["C"] - 1 - (key.topk(most, 1).values & 0xFFFFFFFF)
        best = z.gather(1, at)
        left = best == LOG_MIN
        out["top_ids"] = torch.full((case["n"], case["top"]), -1, device=z.device, dtype=torch.int32)
        out["top_ids"][:, :most] = torch.where(left, torch.full_like(at, -1), at).to(torch.int32)
        out["top_logprob"] = torch.full((case["n"], case["top"]), LOG_MIN, device=z.device)
        out["top_logprob"][:, :most] = torch.where(left, best, best * case["scale"] - lse[:, None])
    return out


def _plain_distill(s):
    case = s["case"]
    C, scale = case["C"], case["scale"]
    z, x, e, S, lse = _plain_softmax(s)
    del x
    ids = s["ids"].long()
    at = ids.clamp(min=0)
    student = z.gather(1, at)
    del z
    there = (ids >= 0) & (student != LOG_MIN)
    t = torch.where(there, s["teacher"] * scale, LOG_MIN)
    m = t.amax(1, keepdim=True)
    m = torch.where(m == LOG_MIN, torch.zeros_like(m), m)
    f = torch.exp(t - m)
    Q = f.sum(1, keepdim=True)
    some = Q > 0
    q = torch.where(some, f / Q, torch.zeros_like(f))
    log_q = torch.where(there, t - m - torch.log(Q), torch.zeros_like(t))
    log_p = torch.where(there, student * scale - lse[:, None], torch.zeros_like(t))
    loss = (q * (log_q - log_p)).sum(1)
    r = torch.where(some, (s["weight"] * scale)[:, None], torch.zeros_like(S))
    d = e * torch.where(some, r / S, torch.zeros_like(S))
    del e
    d.scatter_add_(1, at, -r * q)
    return dict(loss=loss, grad_G=d @ s["V"].float(), grad_V=d.t() @ s["G"], grad_w=d.sum(0))


def work(case):
    n, C, K, T, top = case["n"], case["C"], case["K"], case["T"], case.get("top", 0)
    words = (C + 31) // 32
    read = 4 * n * K + (4 if case["type"] == "f32" else 2) * C * K + 4 * C + 4 * n * T
    read += {"none": 0, "shared": 4 * words, "rows": 4 * n * words}[case["mask"]]
    if case["op"] == "logprobs":
        # a logit: K multiply-adds; scaled and shifted, exponential, its sum, the entropy's multiply-add
        return {"bytes": read + 8 * n + 4 * n * T + 8 * n * top, "flops": n * C * (2 * K + 6)}
    # logits, their gradient by G and by V; scaled and shifted, exponential, its sum, times the row's weight, grad_w
    return {"bytes": read + 4 * n * T + 4 * n + 4 * n + 4 * n * K + 4 * C * K + 4 * C, "flops": n * C * (6 * K + 6)}


def exact(case, seed):
    s = prepare(case, seed)
    n, C, T, top, scale = case["n"], case["C"], case["T"], case.get("top", 0), case["scale"]
    G, V, w = s["G"].double(), s["V"].double(), s["w"].double()
    step = max(1, min(n, 100_000_000 // C))
    columns = torch.arange(C, device=G.device)
    got = []
    grad_V, grad_w = torch.zeros_like(V), torch.zeros_like(w)
    for lo in range(0, n, step):
        rows = slice(lo, min(n, lo + step))
        z = torch.addmm(w[None, :], G[rows], V.t())
        if s["mask"] is not None:
            words = s["mask"] if s["mask"].shape[0] == 1 else s["mask"][rows]
            z.masked_fill_(((words.long()[:, columns // 32] >> (columns % 32)) & 1) == 0, LOG_MIN)
        lse = torch.logsumexp(z * scale, 1)
        empty = torch.isneginf(lse)
        logp = z * scale - torch.where(empty, torch.zeros_like(lse), lse)[:, None]
        p = logp.exp()
        p[empty] = 0
        ids = s["ids"][rows].long()
        named = logp.gather(1, ids.clamp(min=0))
        if case["op"] == "logprobs":
            part = dict(lse=lse, entropy=-torch.xlogy(p, p).sum(1),
                        logprob=named.masked_fill(ids < 0, 0.0))
            if top:
                best = torch.full((z.shape[0], top), LOG_MIN, device=G.device, dtype=torch.float64)
                k = min(top, C)
                best[:, :k] = logp.topk(k, 1).values
                part["top_logprob"] = best
            got.append(part)
            continue
        q = (s["teacher"][rows].double() * scale).masked_fill((ids < 0) | torch.isneginf(named), LOG_MIN)
        none = torch.isneginf(q).all(1)
        q = torch.softmax(q, 1).masked_fill(none[:, None], 0.0)
        loss = torch.where(q > 0, torch.xlogy(q, q) - q * named, torch.zeros_like(q)).sum(1)
        d = p
        d[none] = 0
        d.scatter_add_(1, ids.clamp(min=0), -q)
        d *= (s["weight"][rows].double() * scale)[:, None]
        grad_V += d.t() @ G[rows]
        grad_w += d.sum(0)
        got.append(dict(loss=loss, grad_G=d @ V))
    out = {k: torch.cat([part[k] for part in got]) for k in got[0]}
    if case["op"] == "distill":
        out.update(grad_V=grad_V, grad_w=grad_w)
    elif top:
        out["top_ids"] = None
    return out
