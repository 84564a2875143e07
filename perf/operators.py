"""What the speed of the operators around a head is measured on: sample, logit_error and orthogonalize.

The selection works on per-example gradients of a head, given by their factors: the error of the logits and the features.
These three stand before and after it.

  sample   a label for every row of logits, drawn from the model's own distribution with a given random number: for
           examples that have no label, and, one row at a time, for serving.
  error    the cross-entropy of every row and its gradient with respect to the logits, which is the factor E of
           fd_update_outer and score_outer: the loss of a training step and its backward pass at once.
  ortho    the gradient matrix of the kept rows, made orthogonal by Newton-Schulz products: the update of a weight matrix.

A case's "kind" says which. Sizes are those of this repository's heads (1000 classes, 2048 features and a bias, batches of
1024) and generic vocabularies and weight matrices.
"""
import math

import torch

own = False  # False: plain torch operations; True: the calls of the library

MUON = (3.4445, -4.7750, 2.0315)  # the usual quintic: singular values end between about 0.7 and 1.2
CUBIC = (1.5, -0.5, 0.0)          # converges to 1 from below


def _sample(name, rows, classes, dtype, temperature, top_k=0, top_p=1.0, min_p=0.0, mixed=False, pad=0, masked=False):
    """temperature .. min_p hold for every row, unless mixed: then every row has its own, as requests of a batch do. pad: columns
    behind the classes, which hold anything. masked: half of the classes are at -inf, in one row all."""
    return {"name": name, "kind": "sample", "rows": rows, "classes": classes, "dtype": dtype, "temperature": temperature,
            "top_k": top_k, "top_p": top_p, "min_p": min_p, "mixed": mixed, "pad": pad, "masked": masked}


def _error(name, rows, classes, dtype, weighted=False, ignored=0.0, pad=0):
    """weighted: rows have weights; ignored: this share of the rows has no label."""
    return {"name": name, "kind": "error", "rows": rows, "classes": classes, "dtype": dtype, "weighted": weighted,
            "ignored": ignored, "pad": pad}


def _ortho(name, batch, rows, cols, dtype, steps=5, cubic=False):
    return {"name": name, "kind": "ortho", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype, "steps": steps,
            "cubic": cubic}


def listed():
    return [
        # one token of one request: all latency
        _sample("sample_token", 1, 32_768, "bf16", 0.8, top_k=50, top_p=0.95),
        # a batch of requests, each with its own settings, odd vocabulary, padded rows, masked classes
        _sample("sample_requests", 37, 50_021, "f32", 1.0, mixed=True, pad=43, masked=True),
        # labels for a batch of examples of the repository's head of 1000 classes
        _sample("sample_head", 1024, 1000, "f32", 1.0),
        # ... and for a batch of tokens of a large vocabulary, the nucleus only
        _sample("sample_vocab", 1024, 131_072, "bf16", 1.0, top_p=0.9),
        # one row: the loss of a single token
        _error("error_token", 1, 32_768, "bf16"),
        # a batch of the repository's head
        _error("error_head", 1024, 1000, "bf16"),
        # odd vocabulary, padded rows, weights, rows without a label
        _error("error_odd", 777, 50_021, "f32", weighted=True, ignored=0.1, pad=43),
        # the tokens of a training step
        _error("error_vocab", 4096, 65_536, "bf16", weighted=True),
        # a small weight matrix: all latency
        _ortho("ortho_block", 1, 64, 256, "f32"),
        # the slices of a projection, one matrix a head
        _ortho("ortho_heads", 48, 128, 1024, "bf16"),
        # the repository's head: 1000 classes, 2048 features and the bias
        _ortho("ortho_head", 1, 1000, 2049, "f32"),
        # a large square projection
        _ortho("ortho_square", 1, 4096, 4096, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "error", "ortho"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "ortho":
        m, n = _log_int(rng, 8, 4096), _log_int(rng, 8, 4096)
        batch = max(1, min(_log_int(rng, 1, 64), 4096 ** 3 // (4 * m * n * min(m, n))))
        if dtype == "f32":                     # fp32 takes twice the products: no dearer than the largest listed case
            while m * n * min(m, n) > 4096 ** 3 // 2:
                m, n = m * 3 // 4, n * 3 // 4
        cubic = rng.random() < 0.25
        return {"kind": "ortho", "batch": batch, "rows": m, "cols": n, "dtype": dtype,
                "steps": rng.randint(2, 8) if cubic else rng.randint(3, 5), "cubic": cubic}
    classes = _log_int(rng, 2, 200_000)
    pad = rng.choice([0, 0, rng.randint(1, 64)])
    if kind == "error":
        rows = min(_log_int(rng, 1, 4096), 4096 * 65_536 // (2 * classes))
        return {"kind": "error", "rows": rows, "classes": classes, "dtype": dtype, "weighted": rng.random() < 0.5,
                "ignored": rng.choice([0.0, 0.1, 0.5]), "pad": pad}
    rows = min(_log_int(rng, 1, 1024), 1024 * 131_072 // (2 * classes))
    return {"kind": "sample", "rows": rows, "classes": classes, "dtype": dtype,
            "temperature": rng.choice([0.0, 0.3, 0.7, 1.0, 1.3]), "top_k": rng.choice([0, 0, 1, 20, 50, 1000]),
            "top_p": rng.choice([1.0, 1.0, 0.9, 0.95, 0.5]), "min_p": rng.choice([0.0, 0.0, 0.02, 0.1]),
            "mixed": rng.random() < 0.3, "pad": pad, "masked": rng.random() < 0.3}


# ---- inputs -----------------------------------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _logits(case, g):
    """Rows as a head gives them: a bulk of small logits and a few that stand out, more in some rows than in others. Columns
    behind the classes hold no numbers."""
    rows, V, pad = case["rows"], case["classes"], case["pad"]
    z = torch.full((rows, V + pad), math.nan, device="cuda", dtype=_type(case))
    for lo in range(0, rows, 512):
        n = min(512, rows - lo)
        x = 2.0 * torch.randn((n, V), generator=g, device="cuda")
        hot = torch.randint(0, V, (n, min(V, 24)), generator=g, device="cuda")
        lift = 4.0 * torch.rand((n, 1), generator=g, device="cuda")
        x.scatter_reduce_(1, hot, 4.0 + lift + 2.0 * torch.randn(hot.shape, generator=g, device="cuda"), "amax")
        z[lo:lo + n, :V] = x.to(z.dtype)
    return z


def prepare(case, seed):
    torch.cuda.set_device(0)
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + 41) % (1 << 62))
    if case["kind"] == "ortho":
        return {"case": case, "G": _gradients(case, g)}
    rows, V = case["rows"], case["classes"]
    z = _logits(case, g)[:, :V]
    state = {"case": case, "logits": z}
    if case["kind"] == "error":
        y = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
        likely = z.float().argmax(1).to(torch.int32)  # most examples are learnt already
        y = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.6, likely, y)
        y[torch.rand(rows, generator=g, device="cuda") < case["ignored"]] = -1
        state["labels"] = y
        state["weights"] = torch.rand(rows, generator=g, device="cuda") if case["weighted"] else None
        return state
    if case["masked"]:
        off = torch.rand((rows, V), generator=g, device="cuda") < 0.5
        off[rows // 2] = True
        z.masked_fill_(off, -math.inf)
    state["u"] = torch.rand(rows, generator=g, device="cuda")
    for name in ("temperature", "top_k", "top_p", "min_p"):
        state[name] = case[name]
    if case["mixed"]:
        def pick(values, dtype):
            v = torch.tensor(values, device="cuda", dtype=dtype)
            return v[torch.randint(0, len(values), (rows,), generator=g, device="cuda")]

        state["temperature"] = pick([0.0, 0.5, 0.8, 1.0, 1.5], torch.float32)
        state["top_k"] = pick([0, 1, 40, 50, 500], torch.int32)
        state["top_p"] = pick([1.0, 0.95, 0.9, 0.5], torch.float32)
        state["min_p"] = pick([0.0, 0.0, 0.05], torch.float32)
    return state


def _gradients(case, g):
    """Sums of outer products with a power law, as the gradient of a layer is, and noise."""
    b, m, n = case["batch"], case["rows"], case["cols"]
    G = torch.empty((b, m, n), device="cuda", dtype=_type(case))
    r = max(1, min(m, n) // 2)
    fall = torch.arange(1, r + 1, device="cuda", dtype=torch.float32) ** -0.5
    for i in range(b):
        E = torch.randn((m, r), generator=g, device="cuda") * fall
        H = torch.randn((r, n), generator=g, device="cuda")
        G[i] = (1e-3 * (E @ H + 0.2 * torch.randn((m, n), generator=g, device="cuda"))).to(G.dtype)
    return G


def _coefficients(case):
    return CUBIC if case["cubic"] else MUON


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        from paper_2510_02470_amd.binding import logit_error, orthogonalize, sample

        if case["kind"] == "sample":
            return sample(state["logits"], state["u"], temperature=state["temperature"], top_k=state["top_k"],
                          top_p=state["top_p"], min_p=state["min_p"])
        if case["kind"] == "error":
            return logit_error(state["logits"], state["labels"], weights=state["weights"])
        return orthogonalize(state["G"], steps=case["steps"], coefficients=_coefficients(case))
    if case["kind"] == "sample":
        return _plain_sample(state)
    if case["kind"] == "error":
        return _plain_error(state)
    return _plain_ortho(state)


UNIT = 2.0 ** 42  # the weight of the greatest class; weights are whole numbers, so that their sums do not depend on an order


def _column(value, rows, dtype):
    """A setting as a column, one entry a row."""
    if torch.is_tensor(value):
        return value.to(dtype)[:, None]
    return torch.full((rows, 1), value, device="cuda", dtype=dtype)


def _plain_sample(state):
    z = state["logits"].float()
    rows, V = z.shape
    # fp32 settings widened, as the call takes them
    T = _column(state["temperature"], rows, torch.float32).double()
    k = _column(state["top_k"], rows, torch.int32).long()
    p = _column(state["top_p"], rows, torch.float32).double()
    mp = _column(state["min_p"], rows, torch.float32).double()
    v, order = torch.sort(z, dim=1, descending=True, stable=True)  # equal values: the lower class first
    top = v[:, :1].double()
    usable = torch.isfinite(top) & ~torch.isnan(z).any(1, keepdim=True)
    top = torch.where(usable, top, 0.0)
    greedy = ~(T > 0)
    Ts = torch.where(greedy, 1.0, T)
    d = v.double() - top
    w = torch.round(torch.exp(d / Ts) * UNIT).nan_to_num(0.0, 0.0, 0.0).long()
    w = torch.where(v == -math.inf, 0, w)
    rank = torch.arange(V, device="cuda")[None, :]
    first = rank == 0
    keep = first | (k <= 0) | (rank < k)
    wk = torch.where(keep, w, 0)
    c = wk.cumsum(1)
    need = torch.ceil(p * c[:, -1:].double()).long()
    keep &= first | ~(p < 1) | (c - wk < need)
    keep &= first | ~(mp > 0) | (d >= Ts * torch.log(torch.clamp(mp, max=1.0)))
    wk = torch.where(keep, w, 0)
    c = torch.zeros_like(w).scatter_(1, order, wk).cumsum(1)  # in the order of the classes
    S = c[:, -1:]
    u = state["u"].double()[:, None]
    t = torch.minimum((u * S.double()).long(), S - 1)
    label = torch.where(greedy, order[:, :1], (c <= t).sum(1, keepdim=True))
    label = label.clamp(max=V - 1)
    logp = (z.gather(1, label).double() - top) / Ts - torch.log(S.double() / UNIT)
    logp = torch.where(greedy, 0.0, logp)
    label = torch.where(usable, label, -1)
    logp = torch.where(usable, logp, math.nan)
    return label[:, 0].int(), logp[:, 0].float()


def _plain_error(state):
    z = state["logits"]
    y = state["labels"].long()
    some = y >= 0
    at = torch.where(some, y, 0)[:, None]
    x = z.float()
    x = x - x.amax(1, keepdim=True)
    e = torch.exp(x)
    ey = e.gather(1, at)
    rest = e.scatter(1, at, 0.0).sum(1, keepdim=True)  # without the label: what is left of 1 - p, also where p is nearly 1
    S = rest + ey
    loss = torch.log1p(rest / ey)[:, 0]
    f = torch.where(some, 1.0 if state["weights"] is None else state["weights"], 0.0)[:, None]
    E = e.mul_(f / S).scatter_(1, at, -f * rest / S)
    return E.to(z.dtype), torch.where(some, loss, 0.0)


def _plain_ortho(state):
    case = state["case"]
    a, b, c = _coefficients(case)
    X = state["G"].float()
    X = X / (torch.sqrt((X.double() ** 2).sum((1, 2), keepdim=True)) + 1e-7).float()
    tall = X.shape[1] > X.shape[2]
    if tall:
        X = X.transpose(1, 2).contiguous()
    for _ in range(case["steps"]):
        A = X @ X.transpose(1, 2).contiguous()
        B = b * A
        if c != 0.0:
            B = B + c * (A @ A)
        X = a * X + B @ X
    return (X.transpose(1, 2) if tall else X).to(state["G"].dtype)


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "ortho":
        a, b, c = _coefficients(case)
        out = []
        for G in state["G"]:
            X = G.double()
            X = X / (torch.linalg.vector_norm(X) + 1e-7)
            if X.shape[0] > X.shape[1]:
                for _ in range(case["steps"]):       # X (a + b A + c A A), A = X'X, one factor at a time
                    A = X.T @ X
                    Y = X @ A
                    X = a * X + b * Y + c * (Y @ A)
            else:
                for _ in range(case["steps"]):
                    A = X @ X.T
                    Y = A @ X
                    X = a * X + b * Y + c * (A @ Y)
            out.append(X)
        return torch.stack(out)
    if case["kind"] == "error":
        z, y = state["logits"], state["labels"].long()
        E = torch.empty(z.shape, device="cuda", dtype=torch.float64)
        loss = torch.empty(z.shape[0], device="cuda", dtype=torch.float64)
        for lo in range(0, z.shape[0], 256):
            x, t = z[lo:lo + 256].double(), y[lo:lo + 256]
            n = torch.arange(len(t), device="cuda")
            x = x - x[n, t.clamp(min=0)][:, None]    # relative to the label's logit: loss = ln sum e^x
            x[n, t.clamp(min=0)] = -math.inf
            other = torch.logsumexp(x, 1)            # ln of the odds against the label
            loss[lo:lo + 256] = torch.where(t >= 0, torch.logaddexp(other, torch.zeros_like(other)), 0.0)
            f = torch.ones(len(t), device="cuda", dtype=torch.float64)
            if state["weights"] is not None:
                f = state["weights"][lo:lo + 256].double()
            f = torch.where(t >= 0, f, 0.0)
            total = torch.logaddexp(other, torch.zeros_like(other))
            p = torch.exp(x - total[:, None])
            p[n, t.clamp(min=0)] = -torch.exp(other - total)
            E[lo:lo + 256] = p * f[:, None]
        return E, loss
    if case["rows"] * case["classes"] > 1 << 22:
        return None
    import numpy as np

    z = state["logits"].float().cpu().numpy().astype(np.float64)
    u = state["u"].cpu().numpy().astype(np.float64)
    rows, V = z.shape

    def setting(name):
        s = state[name]
        s = s.cpu().numpy() if torch.is_tensor(s) else np.full(rows, s, np.int32 if name == "top_k" else np.float32)
        return s.astype(np.float64)

    T, K, P, M = (setting(name) for name in ("temperature", "top_k", "top_p", "min_p"))
    labels, logp = [], []
    for i in range(rows):
        if not np.isfinite(z[i].max()):
            labels.append(-1)
            logp.append(math.nan)
            continue
        if T[i] <= 0:
            labels.append(int(z[i].argmax()))
            logp.append(0.0)
            continue
        x = (z[i] - z[i].max()) / T[i]
        w = np.rint(np.exp(x) * UNIT).astype(np.int64)
        kept = np.lexsort((np.arange(V), -z[i]))     # the greatest first, of equals the lower class
        if K[i] > 0:
            kept = kept[:int(K[i])]
        if P[i] < 1:
            before = np.concatenate([[0], np.cumsum(w[kept])[:-1]])
            kept = kept[:max(1, int((before < math.ceil(P[i] * float(w[kept].sum()))).sum()))]
        if M[i] > 0:
            kept = kept[(z[i][kept] - z[i].max()) >= T[i] * math.log(min(1.0, M[i]))]
        kept = np.sort(kept)
        c = np.cumsum(w[kept])
        t = min(int(u[i] * float(c[-1])), int(c[-1]) - 1)
        j = int(kept[np.searchsorted(c, t, side="right")])
        labels.append(j)
        logp.append(x[j] - math.log(float(c[-1]) / UNIT))
    return (torch.tensor(labels, dtype=torch.int32), torch.tensor(logp, dtype=torch.float64))


def work(case):
    esz = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "ortho":
        m, n = sorted((case["rows"], case["cols"]))
        # a symmetric product needs half of its entries: X X' m^2 n, A A m^3, and B X 2 m^2 n
        step = 3 * m * m * n + (0 if case["cubic"] else m ** 3)
        return {"bytes": 2 * case["batch"] * m * n * esz, "flops": case["batch"] * case["steps"] * step}
    rows, V = case["rows"], case["classes"]
    if case["kind"] == "error":
        return {"bytes": 2 * rows * V * esz + rows * (8 + 4 * case["weighted"]), "flops": 4 * rows * V}
    settings = 16 * case["mixed"]
    return {"bytes": rows * (V * esz + 12 + settings), "flops": 4 * rows * V}
