"""Performance cases of the first-order operators that train a model's tail beside the
subspace path: Newton-Schulz orthogonalisation (alone, and as the Muon optimiser's update)
and layer normalisation, forward and backward.

Four kinds of work:

* ``ortho``   -- orthogonalise a set of matrices: X_0 = G / (||G||_F + eps), then five times
  A = X X^T, X <- a X + (b A + c A A) X (on the transpose where G is taller than wide), the
  result rounded to the matrix's type.  What the subspace moments (r x r) and a plain
  update go through.
* ``muon``    -- one optimiser step of a set of weight matrices: M <- mu M + G, the
  orthogonalised G + mu M, W <- (1 - lr wd) W - lr s O with s = sqrt(max(1, m / n)).
* ``ln_fwd``  -- y = (h - mean) rstd weight + bias over the rows of h = x (+ residual), with
  the statistics for the backward pass.
* ``ln_bwd``  -- the gradients of the input, the weight and the bias from dy (with the
  residual branch's gradient added to the input's where there is one).

A case is a dict of plain values.  ``shapes`` lists matrices as "m x n [* count], ...".
Where ``own`` is true the framework's kernels run, else the same arithmetic as elementary
torch operations in 32 bits.
"""

import math

import torch

own = False

DEVICE = "cuda"
NS_STEPS = 5
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315     # the Muon optimiser's quintic
NS_EPS = 1e-7
MU, LR, WD = 0.95, 0.02, 0.01
LN_EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------- cases

def listed():
    return [
        # the subspace moments of a 7B model's 224 matrices at an ordinary rank: one
        # orthogonalised direction per matrix and step
        dict(name="ortho 224 moments r32", kind="ortho", shapes="32x32*224", dtype="f32"),
        # the same at the largest rank
        dict(name="ortho 224 moments r128", kind="ortho", shapes="128x128*224", dtype="f32"),
        # one fp32 matrix of odd sizes with padded rows (a small adapter or a head)
        dict(name="ortho 1001x333 f32 padded", kind="ortho", shapes="1001x333", dtype="f32",
             pad=7),
        # the thin LoRA factors of ten layers of a 13B model
        dict(name="muon LoRA 13B x10 f32", kind="muon", shapes="8x5120*20,5120x8*20",
             dtype="f32"),
        # the last block of a 1.3B model
        dict(name="muon 1.3B block bf16", kind="muon", shapes="2048x2048*4,8192x2048,2048x8192",
             dtype="bf16"),
        # one attention and one up projection of a 7B model: the largest products
        dict(name="muon 7B pair bf16", kind="muon", shapes="4096x4096,11008x4096", dtype="bf16"),
        # a single token's row: latency
        dict(name="ln_fwd 1x5120 bf16", kind="ln_fwd", rows=1, cols=5120, dtype="bf16",
             wdtype="bf16", residual=False),
        # a full batch of a 7B-wide model with the residual sum fused in
        dict(name="ln_fwd 4096x4096 bf16 res", kind="ln_fwd", rows=4096, cols=4096, dtype="bf16",
             wdtype="bf16", residual=True),
        # many short rows of a small fp32 model
        dict(name="ln_fwd 50001x768 f32", kind="ln_fwd", rows=50001, cols=768, dtype="f32",
             wdtype="f32", residual=False),
        # one short example, odd sizes, fp32
        dict(name="ln_bwd 97x1001 f32", kind="ln_bwd", rows=97, cols=1001, dtype="f32",
             wdtype="f32", residual=False),
        # a batch of a 1.3B model, fp32 master weights beside bf16 activations
        dict(name="ln_bwd 2048x2048 bf16", kind="ln_bwd", rows=2048, cols=2048, dtype="bf16",
             wdtype="f32", residual=False),
        # the largest batch of a 13B-wide model with its residual branch
        dict(name="ln_bwd 16384x5120 bf16 res", kind="ln_bwd", rows=16384, cols=5120,
             dtype="bf16", wdtype="bf16", residual=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size spread over its logarithm: odd, a multiple of 8 or of 64."""
    v = _log_int(rng, lo, hi)
    step = rng.choice([1, 8, 64])
    return max(lo, v // step * step)


def draw(rng):
    """One more case of the listed kinds; no dearer than the 7B pair."""
    kind = rng.choice(["moments", "thin", "set", "set", "ln_fwd", "ln_fwd", "ln_bwd", "ln_bwd"])
    if kind == "moments":
        r = rng.choice([4, 8, 16, 32, 64, 128])
        return dict(kind="ortho", shapes=f"{r}x{r}*{_log_int(rng, 1, 448)}", dtype="f32")
    if kind == "thin":
        a, h = rng.choice([4, 8, 16, 32, 64]), _size(rng, 256, 8192)
        k = _log_int(rng, 1, 40)
        return dict(kind=rng.choice(["ortho", "muon"]), shapes=f"{a}x{h}*{k},{h}x{a}*{k}",
                    dtype=rng.choice(["bf16", "f32"]))
    if kind == "set":
        shapes, cost = [], 0.0
        for _ in range(rng.randint(1, 3)):
            m, n = _size(rng, 48, 8192), _size(rng, 48, 8192)
            p, c = min(m, n), max(m, n)
            each = p * p * (2.0 * c + p)
            left = 1.2e11 - cost
            if each > left:
                m, n = max(48, m // 4), max(48, n // 4)
                p, c = min(m, n), max(m, n)
                each = p * p * (2.0 * c + p)
                if each > left:
                    continue
            k = max(1, min(rng.choice([1, 1, 2, 4]), int(left / each)))
            cost += each * k
            shapes.append(f"{m}x{n}*{k}")
        if not shapes:
            shapes.append(f"{_size(rng, 48, 1024)}x{_size(rng, 48, 1024)}")
        case = dict(kind=rng.choice(["ortho", "muon"]), shapes=",".join(shapes),
                    dtype=rng.choice(["bf16", "f32"]))
        if rng.random() < 0.3:
            case["pad"] = rng.choice([1, 8, 24])
        return case
    rows, cols = _log_int(rng, 1, 50000), _size(rng, 48, 12288)
    rows = max(1, min(rows, 80_000_000 // cols))
    return dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(["bf16", "f32"]),
                wdtype=rng.choice(["bf16", "f32"]), residual=rng.random() < 0.4)


def _shapes(case):
    out = []
    for part in case["shapes"].split(","):
        size, _, count = part.strip().partition("*")
        m, n = size.split("x")
        out += [(int(m), int(n))] * int(count or 1)
    return out


# ------------------------------------------------------------------------- inputs

def _rng(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(1000003 * int(seed) + 17)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32)


def _gradients(g, m, n, count):
    """Gradients dY^T X of `count` linear layers, from tokens whose features have widely
    spread scales (a few strong ones), as a batch gives them.  (count, m, n) fp32."""
    if max(m, n) <= 128 and m == n:                # subspace moments: sums of Gaussians
        return _randn(g, count, m, n) * 0.7
    t = max(2 * min(m, n), 64)
    x = _randn(g, count, t, n) * torch.exp(_randn(g, count, 1, n))
    d = _randn(g, count, t, m) * torch.exp(_randn(g, count, 1, m))
    return torch.bmm(d.transpose(1, 2), x).mul_(1e-4 / math.sqrt(t))


def _padded(x, dtype, pad):
    """x in `dtype`, its rows `pad` elements apart from one another."""
    if not pad:
        return x.to(dtype).contiguous()
    buf = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=dtype, device=x.device)
    buf[:, :x.shape[1]] = x
    return buf[:, :x.shape[1]]


def _matrices(case, seed):
    g, dt, pad = _rng(seed), DTYPES[case["dtype"]], case.get("pad", 0)
    G, W, M = [], [], []
    muon = case["kind"] == "muon"
    shapes = _shapes(case)
    i = 0
    while i < len(shapes):
        m, n = shapes[i]
        k = 1
        while i + k < len(shapes) and shapes[i + k] == (m, n) and (k + 1) * m * n <= 1 << 24:
            k += 1
        grads = _gradients(g, m, n, k)
        G += [_padded(x, dt, pad) for x in grads]
        if muon:
            W += [_padded(x * 0.02, dt, pad) for x in _randn(g, k, m, n)]
            M += [x.mul_(8.0).contiguous() for x in _gradients(g, m, n, k)]
        else:
            W += [_padded(torch.zeros(m, n, device=DEVICE), dt, pad) for _ in range(k)]
        i += k
    return G, W, M


def _rows_of(case, seed):
    g, dt, wdt = _rng(seed), DTYPES[case["dtype"]], DTYPES[case["wdtype"]]
    r, c = case["rows"], case["cols"]
    s = {"x": (_randn(g, r, c) + 0.5 * _randn(g, 1, c)).to(dt),
         "weight": (1.0 + 0.2 * _randn(g, c)).to(wdt), "bias": (0.1 * _randn(g, c)).to(wdt)}
    if case["residual"]:
        s["residual"] = _randn(g, r, c).to(dt)
    if case["kind"] == "ln_bwd":
        # what the forward pass left: its input (the sum, where there is a residual) and the
        # rows' statistics
        h = s["x"].float()
        if case["residual"]:
            h = h + s.pop("residual").float()
            s["x"] = h.to(dt)
            h = s["x"].float()
            s["dresidual"] = (0.1 * _randn(g, r, c)).to(dt)
        s["mean"] = h.mean(1)
        s["rstd"] = torch.rsqrt((h - s["mean"][:, None]).square().mean(1) + LN_EPS)
        s["dy"] = (0.1 * _randn(g, r, c)).to(dt)
    return s


def prepare(case, seed):
    if case["kind"] in ("ln_fwd", "ln_bwd"):
        return dict(_rows_of(case, seed), kind=case["kind"])
    G, W, M = _matrices(case, seed)
    state = {"kind": case["kind"], "G": G, "W": W, "M": M}
    if own:
        # the handle over the program's buffers, which it keeps as long as they live
        from paper_2608_15665_gb300 import firstorder
        state["op"] = (firstorder.Muon(W, G, M) if case["kind"] == "muon"
                       else firstorder.Orthogonalizer(G, W))
    return state


# ---------------------------------------------------------------------- plain forms

def _orthogonalized(U):
    """Newton-Schulz on one stack of matrices (k, m, n), fp32."""
    tall = U.shape[1] > U.shape[2]
    X = U.transpose(1, 2) if tall else U
    X = X / (X.square().sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    for _ in range(NS_STEPS):
        A = torch.bmm(X, X.transpose(1, 2))
        X = NS_A * X + torch.bmm(NS_B * A + NS_C * torch.bmm(A, A), X)
    return X.transpose(1, 2) if tall else X


def _stacks(G):
    """Indices of neighbours of one shape, at most 2^26 elements together."""
    at, out = 0, []
    while at < len(G):
        k = 1
        while (at + k < len(G) and G[at + k].shape == G[at].shape
               and (k + 1) * G[at].numel() <= 1 << 26):
            k += 1
        out.append(slice(at, at + k))
        at += k
    return out


def _plain_matrices(s):
    G, W, M = s["G"], s["W"], s["M"]
    for k in _stacks(G):
        U = torch.stack(G[k]).float()
        if M:
            m_new = MU * torch.stack(M[k]) + U
            U = U + MU * m_new
        O = _orthogonalized(U)
        for i in range(O.shape[0]):
            w = W[k.start + i]
            if M:
                scale = math.sqrt(max(1.0, w.shape[0] / w.shape[1]))
                w.copy_((1.0 - LR * WD) * w.float() - (LR * scale) * O[i])
                M[k.start + i].copy_(m_new[i])
            else:
                w.copy_(O[i])
    return {"W": W[:30], "M": M[:30]}


def _plain_forward(s):
    x, dt = s["x"].float(), s["x"].dtype
    out = {}
    if "residual" in s:
        out["h"] = (x + s["residual"].float()).to(dt)
        x = out["h"].float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt(x.square().mean(1, keepdim=True) + LN_EPS)
    y = x * rstd * s["weight"].float() + s["bias"].float()
    return dict(out, y=y.to(dt), mean=mean[:, 0], rstd=rstd[:, 0])


def _plain_backward(s):
    x, dy, dt = s["x"].float(), s["dy"].float(), s["x"].dtype
    rstd = s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    g = dy * s["weight"].float()
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if "dresidual" in s:
        dx = dx + s["dresidual"].float()
    wdt = s["weight"].dtype
    return {"dx": dx.to(dt), "dweight": (dy * xh).sum(0).to(wdt), "dbias": dy.sum(0).to(wdt)}


# --------------------------------------------------------------------------- passes

def _own(s):
    from paper_2608_15665_gb300 import firstorder as fo
    if s["kind"] == "ortho":
        s["op"]()
        return {"W": s["W"][:30], "M": []}
    if s["kind"] == "muon":
        s["op"].step(lr=LR, momentum=MU, weight_decay=WD)
        return {"W": s["W"][:30], "M": s["M"][:30]}
    if s["kind"] == "ln_fwd":
        got = fo.layer_norm(s["x"], s["weight"], s["bias"], LN_EPS, residual=s.get("residual"))
        return {k: v for k, v in got._asdict().items() if v is not None}
    dx, dw, db = fo.layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"],
                                        dresidual=s.get("dresidual"))
    return {"dx": dx, "dweight": dw, "dbias": db}


def run(state):
    if own:
        return _own(state)
    if state["kind"] in ("ortho", "muon"):
        return _plain_matrices(state)
    return (_plain_forward if state["kind"] == "ln_fwd" else _plain_backward)(state)


# ----------------------------------------------------------------------------- work

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] in ("ortho", "muon"):
        params = flops = 0.0
        for m, n in _shapes(case):
            p, c = min(m, n), max(m, n)
            params += m * n
            # X X^T and A A are symmetric: half of each product is all there is to compute
            flops += NS_STEPS * (p * p * c + p * p * p + 2.0 * p * p * c)
        # G read and the result written; a step reads and writes W, and M in fp32
        return {"bytes": params * ((3 * e + 8) if case["kind"] == "muon" else 2 * e),
                "flops": flops}
    r, c = case["rows"], case["cols"]
    w = 2 if case["wdtype"] == "bf16" else 4
    if case["kind"] == "ln_fwd":      # x -> y; with a residual its row too, and the sum
        return {"bytes": r * c * e * (4 if case["residual"] else 2) + 2 * c * w + 8 * r,
                "flops": 8.0 * r * c}
    return {"bytes": r * c * e * (4 if case["residual"] else 3) + 3 * c * w + 8 * r,
            "flops": 14.0 * r * c}


# ---------------------------------------------------------------------------- exact

def _polar_like(U):
    """The five quintic steps in 64 bits.  They act on the singular values alone: small
    matrices go by their SVD, larger ones by Horner's form on the thin side's Gram matrix."""
    tall = U.shape[0] > U.shape[1]
    X = U.double().t() if tall else U.double()
    X = X / (torch.linalg.vector_norm(X) + NS_EPS)
    if X.shape[0] <= 128:
        left, s, right = torch.linalg.svd(X, full_matrices=False)
        for _ in range(NS_STEPS):
            s = s * (NS_A + s * s * (NS_B + NS_C * s * s))
        X = (left * s) @ right
    else:
        for _ in range(NS_STEPS):
            A = X @ X.t()
            Q = (NS_C * A) @ A
            Q.add_(A, alpha=NS_B)
            Q.diagonal().add_(NS_A)
            X = Q @ X
    return X.t() if tall else X


def exact(case, seed):
    if case["kind"] in ("ortho", "muon"):
        flops = sum(6.0 * NS_STEPS * min(s) ** 2 * max(s) for s in _shapes(case))
        if flops > 8e12:               # beyond ~20 s of 64-bit products
            return None
        G, W, M = _matrices(case, seed)
        outs, moms = [], []
        for i in range(min(30, len(G))):
            U, m, n = G[i].double(), G[i].shape[0], G[i].shape[1]
            if M:
                mom = MU * M[i].double() + U
                O = _polar_like(U + MU * mom)
                outs.append((1 - LR * WD) * W[i].double() - LR * max(1.0, m / n) ** 0.5 * O)
                moms.append(mom)
            else:
                outs.append(_polar_like(U))
        return {"W": outs, "M": moms}
    s = _rows_of(case, seed)
    x, dt = s["x"].double(), s["x"].dtype
    w = s["weight"].double()
    if case["kind"] == "ln_fwd":
        out = {}
        if case["residual"]:
            out["h"] = x + s["residual"].double()
            x = out["h"].to(dt).double()      # the sum is stored, and normalised, in x's type
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = 1.0 / torch.sqrt(var + LN_EPS)
        y = (x - mean[:, None]) * rstd[:, None] * w + s["bias"].double()
        return dict(out, y=y, mean=mean, rstd=rstd)
    dy, rstd = s["dy"].double(), s["rstd"].double()[:, None]
    xh = (x - s["mean"].double()[:, None]) * rstd
    n = x.shape[1]
    g = dy * w
    dx = rstd / n * (n * g - g.sum(1, keepdim=True) - xh * (g * xh).sum(1, keepdim=True))
    if case["residual"]:
        dx = dx + s["dresidual"].double()
    return {"dx": dx, "dweight": torch.einsum("ij,ij->j", dy, xh), "dbias": dy.sum(0)}
