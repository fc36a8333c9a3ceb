"""Performance cases of further operators that train a model's tail: the AdamW step over many
tensors, a preference loss over pairs of answers, and the gated linear block of a feed-forward
layer, the last two with their backward passes.

* ``adamw``    -- m <- b1 m + (1 - b1) g, v <- b2 v + (1 - b2) g^2,
  W <- (1 - lr wd) W - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps), with m and v in
  32 bits, or m and r = sqrt(v) as e4m3 values times a power of two per 256 elements.  A state
  in 8 bits is rounded up or down at random, by 16 bits of a Philox4x32-10 stream an element:
  a running mean that moves by a thousandth a step would otherwise never leave its code.
* ``pref_fwd`` -- log-probabilities of the labels under rows of logits, summed over each
  answer's counted rows; with the reference model's sums, the loss of every pair (chosen,
  rejected) and its mean; the rows' logsumexp and the loss's derivative by each row's
  log-probability for the backward pass.
* ``pref_bwd`` -- the gradient of the logits from those.
* ``gated_fwd`` -- H = act(X Wg^T) * (X Wu^T), with both products where they are kept for the
  backward pass.
* ``gated_bwd`` -- the gradients of X, Wg and Wu from that of H.

A case is a dict of plain values.  Where ``own`` is true the framework's kernels run, else the
same arithmetic as elementary torch operations in 32 bits.
"""

import math
import random

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LR, B1, B2, EPS, WD = 1e-3, 0.9, 0.999, 1e-8, 0.01
SEED = 1234                          # of the states' rounding
BLOCK = 256                          # elements of a power of two
BETA, SMOOTH = 0.1, 0.1
IGNORE = -100
F8 = torch.float8_e4m3fn


# ---------------------------------------------------------------------------- cases

def listed():
    return [
        # the last norms' weights and biases of a 13B model: a launch's latency
        dict(name="adamw norms 13B f32", kind="adamw", sizes="5120*4", dtype="f32", gdtype="f32",
             bits=32, t=7),
        # the LoRA factors of four layers' q and v, an odd-sized head beside them
        dict(name="adamw LoRA 13B x4 f32 8-bit", kind="adamw", sizes="40960*16,33333*1",
             dtype="f32", gdtype="f32", bits=8, t=100),
        # a block of a 1.3B model with states in 32 bits
        dict(name="adamw 1.3B block bf16", kind="adamw",
             sizes="4194304*4,16777216*2,2048*4,8192*1", dtype="bf16", gdtype="bf16", bits=32,
             t=1000),
        # the head (vocabulary 32000) of a 7B model and its last norm, states in 8 bits
        dict(name="adamw 7B head bf16 8-bit", kind="adamw", sizes="131072000*1,4096*2",
             dtype="bf16", gdtype="bf16", bits=8, t=1000),
        # one pair of short answers: latency
        dict(name="pref_fwd 1 pair 32000 bf16", kind="pref_fwd", pairs=1, tokens=24, vocab=32000,
             dtype="bf16", loss="sigmoid", prompt=0.0, pad=0, tail=0),
        # a batch of pairs whose prompts are not counted
        dict(name="pref_fwd 16 pairs 32000 bf16", kind="pref_fwd", pairs=16, tokens=600,
             vocab=32000, dtype="bf16", loss="sigmoid", prompt=0.3, pad=0, tail=100),
        # fp32 logits of an odd vocabulary in padded rows
        dict(name="pref_bwd 3 pairs 50257 f32", kind="pref_bwd", pairs=3, tokens=130, vocab=50257,
             dtype="f32", loss="square", prompt=0.2, pad=47, tail=5),
        # the largest batch
        dict(name="pref_bwd 8 pairs 32000 bf16", kind="pref_bwd", pairs=8, tokens=1000,
             vocab=32000, dtype="bf16", loss="sigmoid", prompt=0.1, pad=0, tail=0),
        # one token through a 7B model's feed-forward: the weights' way from memory
        dict(name="gated_fwd 1 token 7B", kind="gated_fwd", tokens=1, d=4096, f=11008, act="silu",
             save=False),
        # an odd number of tokens, kept for the backward pass, on the 13B shapes
        dict(name="gated_fwd 777 tokens 13B", kind="gated_fwd", tokens=777, d=5120, f=13824,
             act="gelu", save=True),
        # a training batch of a 7B model, forward and backward
        dict(name="gated_fwd 4096 tokens 7B", kind="gated_fwd", tokens=4096, d=4096, f=11008,
             act="silu", save=True),
        dict(name="gated_bwd 4096 tokens 7B", kind="gated_bwd", tokens=4096, d=4096, f=11008,
             act="silu"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed kinds; none dearer than the 4096 tokens' backward pass."""
    kind = rng.choice(["adamw", "pref_fwd", "pref_bwd", "gated_fwd", "gated_bwd"])
    if kind == "adamw":
        parts, left = [], 100_000_000
        for _ in range(rng.randint(1, 4)):
            n, step = min(_log_int(rng, 64, 50_000_000), left), rng.choice([1, 8, 256])
            n = max(1, n // step * step)
            k = max(1, min(rng.randint(1, 12), left // n))
            left -= n * k
            parts.append(f"{n}*{k}")
            if left < 64:
                break
        dtype = rng.choice(["bf16", "f32"])
        return dict(kind=kind, sizes=",".join(parts), dtype=dtype,
                    gdtype=rng.choice([dtype, "f32"]), bits=rng.choice([8, 32]),
                    t=_log_int(rng, 1, 20000))
    if kind in ("pref_fwd", "pref_bwd"):
        vocab = _log_int(rng, 500, 160_000)
        if rng.random() < 0.5:
            vocab = vocab // 64 * 64 + 64
        pairs = _log_int(rng, 1, 64)
        tokens = _log_int(rng, 1, 2000)
        tokens = max(1, min(tokens, 500_000_000 // (2 * pairs * vocab)))
        return dict(kind=kind, pairs=pairs, tokens=tokens, vocab=vocab,
                    dtype=rng.choice(["bf16", "f32"]),
                    loss=rng.choice(["sigmoid", "hinge", "square"]),
                    prompt=rng.choice([0.0, 0.3, 0.7]), pad=rng.choice([0, 0, 1, 8, 64]),
                    tail=rng.choice([0, 3]))
    d, f = _log_int(rng, 64, 8192) // 8 * 8, _log_int(rng, 64, 16384) // 8 * 8
    tokens = _log_int(rng, 1, 8192)
    tokens = max(1, min(tokens, 180_000_000_000 // (d * f)))
    case = dict(kind=kind, tokens=tokens, d=d, f=f, act=rng.choice(["silu", "gelu"]))
    if kind == "gated_fwd":
        case["save"] = rng.random() < 0.5
    return case


def _sizes(case):
    out = []
    for part in case["sizes"].split(","):
        n, _, count = part.partition("*")
        out += [int(n)] * int(count or 1)
    return out


def _lengths(case):
    """(answers' rows, their uncounted first rows) of a case: the chosen ones, then the rejected."""
    r = random.Random(case["pairs"] * 100003 + case["tokens"])
    rows = [max(1, int(case["tokens"] * r.uniform(0.4, 1.6))) for _ in range(2 * case["pairs"])]
    return rows, [int(n * case["prompt"]) for n in rows]


# ------------------------------------------------------------------------- inputs

def _rng(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(1000003 * int(seed) + 29)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32)


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device=DEVICE, dtype=torch.float32)


def _nearest_codes(x):
    """(e4m3 values, exponents) of a nonnegative or signed state, blocks of BLOCK, rounded to
    nearest: a state as earlier steps may have left it."""
    blocks = x.view(-1, BLOCK)
    top = blocks.abs().amax(1)
    e = torch.frexp(top)[1] + 126                         # the largest's biased exponent
    e = torch.where(top > 0, e, torch.zeros_like(e)).clamp(0, 254)
    q = torch.ldexp(blocks, (134 - e.clamp(min=40))[:, None]).to(F8)
    return q.view(-1), e.to(torch.uint8)


def _adamw_state(case, seed):
    """Tensors side by side in flat buffers, each from a multiple of BLOCK elements on."""
    g, sizes = _rng(seed), _sizes(case)
    dt, gdt = DTYPES[case["dtype"]], DTYPES[case["gdtype"]]
    counts = torch.tensor([-(-n // BLOCK) for n in sizes])
    first = (torch.cumsum(counts, 0) - counts) * BLOCK
    total = int(counts.sum()) * BLOCK
    inside = torch.zeros(total, dtype=torch.bool, device=DEVICE)
    for at, n in zip(first.tolist(), sizes):
        inside[at:at + n] = True
    scale = 1e-4 * torch.exp(_randn(g, total // 64)).repeat_interleave(64)    # as of rows
    s = {"kind": "adamw", "case": case, "sizes": sizes, "first": first.tolist()}
    s["W"] = (_randn(g, total) * 0.02 * inside).to(dt)
    s["G"] = (_randn(g, total) * scale * inside).to(gdt)
    m = _randn(g, total) * 0.3 * scale * inside
    r = (0.6 + 0.8 * _rand(g, total)) * scale * inside
    if case["bits"] == 8:
        s["m"], s["m_exp"] = _nearest_codes(m)
        s["v"], s["v_exp"] = _nearest_codes(r)
        # of every eight elements: their number within their tensor, and the tensor's
        words = counts.to(DEVICE) * (BLOCK // 8)
        start = (torch.cumsum(words, 0) - words).repeat_interleave(words)
        s["word"] = torch.arange(total // 8, device=DEVICE) - start
        s["tensor"] = torch.arange(len(sizes), device=DEVICE).repeat_interleave(words)
    else:
        s["m"], s["v"] = m, r * r
    return s


def _pref_state(case, seed):
    g, dt = _rng(seed), DTYPES[case["dtype"]]
    lengths, prompts = _lengths(case)
    rows, v = sum(lengths) + case["tail"], case["vocab"]
    buf = torch.zeros(rows, v + case["pad"], dtype=dt, device=DEVICE)
    logits = buf[:, :v]
    favour = 1.5 * _randn(g, 1, v)                       # frequent and rare words
    labels = torch.randint(0, v, (rows,), generator=g, device=DEVICE)
    lse = torch.empty(rows, device=DEVICE)
    for at in range(0, rows, 2048):
        part = _randn(g, min(2048, rows - at), v) * 1.5 + favour
        at_label = labels[at:at + 2048, None]
        part.scatter_add_(1, at_label, 6.0 + 2.0 * _randn(g, part.shape[0], 1))
        logits[at:at + 2048] = part.to(dt)
        lse[at:at + 2048] = torch.logsumexp(logits[at:at + 2048].float(), 1)
    ends = torch.cumsum(torch.tensor(lengths), 0)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), ends]).to(DEVICE)
    logp = logits.gather(1, labels[:, None])[:, 0].float() - lse
    at = 0
    for n, p in zip(lengths, prompts):                   # prompts count for nothing
        labels[at:at + p] = IGNORE
        at += n
    logp = torch.where(labels < 0, torch.zeros_like(logp), logp)
    sums = torch.cat([torch.zeros(1, device=DEVICE, dtype=torch.float64),
                      torch.cumsum(logp.double(), 0)])
    sums = sums[offsets[1:]] - sums[offsets[:-1]]
    s = {"kind": case["kind"], "case": case, "logits": logits, "labels": labels,
         "offsets": offsets, "ref": (sums + 4.0 * _randn(g, len(lengths))).float()}
    if case["kind"] == "pref_bwd":
        # what the forward pass left
        slope = torch.randn(len(lengths), generator=g, device=DEVICE).abs() * BETA
        slope[case["pairs"]:] *= -1.0
        seq = torch.bucketize(torch.arange(rows, device=DEVICE), offsets[1:], right=True)
        slope = torch.cat([slope, torch.zeros(1, device=DEVICE)])[seq] / case["pairs"]
        s["lse"] = torch.where(labels < 0, torch.zeros_like(lse), lse)
        s["dlogp"] = torch.where(labels < 0, torch.zeros_like(lse), slope)
        s["dloss"] = torch.tensor(-1.25, device=DEVICE)
    return s


def _gated_state(case, seed):
    g = _rng(seed)
    t, d, f = case["tokens"], case["d"], case["f"]
    # a norm's output: unit rows, a few features above the rest
    x = (_randn(g, t, d) * torch.exp(0.4 * _randn(g, 1, d))).to(torch.bfloat16)
    scale = 1.2 / math.sqrt(d)
    s = {"kind": case["kind"], "case": case, "x": x,
         "wg": (_randn(g, f, d) * scale).to(torch.bfloat16),
         "wu": (_randn(g, f, d) * scale).to(torch.bfloat16)}
    if case["kind"] == "gated_bwd":
        s["gate"] = (x.float() @ s["wg"].float().t()).to(torch.bfloat16)
        s["up"] = (x.float() @ s["wu"].float().t()).to(torch.bfloat16)
        s["dh"] = (0.01 * _randn(g, t, f)).to(torch.bfloat16)
    return s


def _inputs(case, seed):
    if case["kind"] == "adamw":
        return _adamw_state(case, seed)
    if case["kind"] in ("pref_fwd", "pref_bwd"):
        return _pref_state(case, seed)
    return _gated_state(case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["kind"] == "adamw":
        # the handle over the program's buffers, which it keeps as long as they live
        from paper_2608_15665_gb300 import firstorder as fo

        def parts(flat, step=1):
            return [flat[at // step:at // step + -(-n // step)]
                    for at, n in zip(s["first"], s["sizes"])]
        m, v = parts(s["m"]), parts(s["v"])
        if case["bits"] == 8:
            states = [fo.AdamWState(*p) for p in zip(m, v, parts(s["m_exp"], BLOCK),
                                                     parts(s["v_exp"], BLOCK))]
        else:
            states = [fo.AdamWState(*p) for p in zip(m, v)]
        s["op"] = fo.AdamW(parts(s["W"]), parts(s["G"]), states=states, bits=case["bits"],
                           seed=SEED)
    return s


# ---------------------------------------------------------------------- plain forms

def _philox(c0, c1, t):
    """The four words of Philox4x32-10 (Salmon et al., SC'11) at counter (c0, c1, t, 6 << 24)
    under key SEED, as 64-bit integers."""
    low = 0xFFFFFFFF
    c0, c1 = c0 & low, c1 & low
    c2, c3 = torch.full_like(c0, t & low), torch.full_like(c0, 6 << 24)
    k0, k1 = SEED & low, SEED >> 32
    p0, p1 = 0xD2511F53 * c0, 0xCD9E8D57 * c2
    c0, c1, c2, c3 = (p1 >> 32 & low) ^ c1 ^ k0, p1 & low, (p0 >> 32 & low) ^ c3 ^ k1, p0 & low
    for _ in range(9):
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
        p0, p1 = 0xD2511F53 * c0, 0xCD9E8D57 * c2
        c0, c1, c2, c3 = (p1 >> 32 & low) ^ c1 ^ k0, p1 & low, (p0 >> 32 & low) ^ c3 ^ k1, p0 & low
    return c0, c1, c2, c3


def _rounding_bits(s):
    """16 bits for every element: the halves of the words of its eight, low half first."""
    w = torch.stack(_philox(s["word"], s["tensor"], s["case"]["t"]), 1)
    return torch.stack([w & 0xFFFF, w >> 16], 2).view(-1)


def _wide(code, exponent):
    """The fp32 values of e4m3 values times their blocks' powers of two."""
    e = exponent.to(torch.int32).clamp(min=40) - 134
    return torch.ldexp(code.view(-1, BLOCK).float(), e[:, None]).view(-1)


def _exponent_of(bits):
    return (bits >> 23).to(torch.int64)


def _codes(x, exponent, bits16):
    """x as e4m3 values times 2^(exponent - 134), rounded by 16 random bits an element."""
    y = torch.ldexp(x.view(-1, BLOCK), (134 - exponent.clamp(min=40))[:, None]).view(-1)
    step = torch.ldexp(torch.ones_like(y), torch.frexp(y.abs())[1].clamp(min=-5) - 4)
    return torch.floor(y.abs() / step + bits16 / 65536.0) * step, y


def _plain_adamw(s):
    case = s["case"]
    g = s["G"].float()
    eight = case["bits"] == 8
    m = _wide(s["m"], s["m_exp"]) if eight else s["m"]
    m = B1 * m + (1.0 - B1) * g
    if eight:
        r = _wide(s["v"], s["v_exp"])
        v = B2 * (r * r) + (1.0 - B2) * (g * g)
    else:
        v = B2 * s["v"] + (1.0 - B2) * (g * g)
    root = torch.sqrt(v)
    c1, c2 = 1.0 - B1 ** case["t"], math.sqrt(1.0 - B2 ** case["t"])
    w = (1.0 - LR * WD) * s["W"].float() - (LR / c1) * m / (root / c2 + EPS)
    s["W"].copy_(w)
    if not eight:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return {"W": s["W"], "m": s["m"], "v": s["v"]}
    random16 = _rounding_bits(s)
    top = m.abs().view(-1, BLOCK).amax(1)
    m_exp = _exponent_of(top.view(torch.int32))
    # of the root: 2^k <= sqrt(v) < 2^(k + 1) where 2^2k <= v < 2^(2k + 2)
    v_exp = _exponent_of(v.view(-1, BLOCK).amax(1).view(torch.int32))
    v_exp = torch.where(v_exp > 0, (v_exp - 127 >> 1) + 127, torch.zeros_like(v_exp))
    q, y = _codes(m, m_exp, random16)
    s["m"].copy_(torch.copysign(q, y).to(F8))
    q, y = _codes(root, v_exp, random16)
    q = torch.where(v > 0, q.clamp(min=2.0 ** -9), q)    # above zero stays above zero
    s["v"].copy_(q.to(F8))
    s["m_exp"].copy_(m_exp.to(torch.uint8))
    s["v_exp"].copy_(v_exp.to(torch.uint8))
    return {"W": s["W"], "m": s["m"], "v": s["v"], "m_exp": s["m_exp"], "v_exp": s["v_exp"]}


def _pair_losses(case, delta):
    """(losses, their derivatives by delta)"""
    if case["loss"] == "square":
        d = delta - 0.5 / BETA
        return d * d, 2.0 * d
    z = BETA * delta
    if case["loss"] == "hinge":
        return (1.0 - z).clamp(min=0.0), torch.where(z < 1.0, -BETA, 0.0).to(z.dtype)
    # log(1 + exp(-|z|)) is common to both signs
    both = torch.log1p(torch.exp(-z.abs()))
    loss = (1.0 - SMOOTH) * (both - z.clamp(max=0.0)) + SMOOTH * (both + z.clamp(min=0.0))
    return loss, BETA * (1.0 / (1.0 + torch.exp(-z)) - (1.0 - SMOOTH))


def _plain_pref_fwd(s):
    case = s["case"]
    labels, offsets, pairs = s["labels"], s["offsets"], case["pairs"]
    rows = torch.arange(labels.shape[0], device=labels.device)
    counted = (labels >= 0) & (rows < offsets[-1])
    x = s["logits"].float()
    top = x.amax(1)
    lse = top + torch.log(torch.exp(x - top[:, None]).sum(1))
    logp = x.gather(1, labels.clamp(min=0)[:, None])[:, 0] - lse
    zero = torch.zeros_like(lse)
    lse, logp = torch.where(counted, lse, zero), torch.where(counted, logp, zero)
    sums = torch.cat([zero[:1].double(), torch.cumsum(logp.double(), 0)])
    logps = sums[offsets[1:]] - sums[offsets[:-1]]
    gain = logps - s["ref"].double()
    losses, slope = _pair_losses(case, gain[:pairs] - gain[pairs:])
    slope = torch.cat([slope, -slope, torch.zeros_like(slope[:1])]) / pairs
    dlogp = slope[torch.bucketize(rows, offsets[1:], right=True)].float()
    return {"loss": losses.mean().float(), "losses": losses.float(), "logps": logps.float(),
            "lse": lse, "dlogp": torch.where(counted, dlogp, zero)}


def _plain_pref_bwd(s):
    x, labels = s["logits"].float(), s["labels"]
    scale = torch.where(labels >= 0, s["dlogp"] * s["dloss"], torch.zeros_like(s["dlogp"]))
    d = -scale[:, None] * torch.exp(x - s["lse"][:, None])
    d = torch.where(scale[:, None] != 0, d, torch.zeros_like(d))
    d.scatter_add_(1, labels.clamp(min=0)[:, None], scale[:, None])
    return d.to(s["logits"].dtype)


def _act(case, g):
    """(act(g), act'(g))"""
    if case["act"] == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    c = math.sqrt(2.0 / math.pi)
    th = torch.tanh(c * (g + 0.044715 * g * g * g))
    return (0.5 * g * (1.0 + th),
            0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * c * (1.0 + 3 * 0.044715 * g * g))


def _plain_gated_fwd(s):
    x = s["x"].float()
    g, u = x @ s["wg"].float().t(), x @ s["wu"].float().t()
    out = {"h": (_act(s["case"], g)[0] * u).to(torch.bfloat16)}
    if s["case"]["save"]:
        out.update(gate=g.to(torch.bfloat16), up=u.to(torch.bfloat16))
    return out


def _plain_gated_bwd(s):
    x, dh = s["x"].float(), s["dh"].float()
    act, slope = _act(s["case"], s["gate"].float())
    dg, du = dh * s["up"].float() * slope, dh * act
    dx = dg @ s["wg"].float() + du @ s["wu"].float()
    return {"dx": dx.to(torch.bfloat16), "dw_gate": (dg.t() @ x).to(torch.bfloat16),
            "dw_up": (du.t() @ x).to(torch.bfloat16)}


# --------------------------------------------------------------------------- passes

def _own(s):
    from paper_2608_15665_gb300 import firstorder as fo
    case, kind = s["case"], s["kind"]
    if kind == "adamw":
        s["op"].step(lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, t=case["t"])
        out = {"W": s["W"], "m": s["m"], "v": s["v"]}
        if case["bits"] == 8:
            out.update(m_exp=s["m_exp"], v_exp=s["v_exp"])
        return out
    if kind == "pref_fwd":
        got = fo.preference_loss(s["logits"], s["labels"], s["offsets"], s["ref"], beta=BETA,
                                 kind=case["loss"],
                                 smoothing=SMOOTH if case["loss"] == "sigmoid" else 0.0)
        return got._asdict()
    if kind == "pref_bwd":
        return fo.preference_loss_backward(s["logits"], s["labels"], s["lse"], s["dlogp"],
                                           dloss=s["dloss"])
    if kind == "gated_fwd":
        got = fo.gated_linear(s["x"], s["wg"], s["wu"], act=case["act"], save=case["save"])
        return {k: v for k, v in got._asdict().items() if v is not None}
    dx, dwg, dwu = fo.gated_linear_backward(s["dh"], s["x"], s["wg"], s["wu"], s["gate"], s["up"],
                                            act=case["act"])
    return {"dx": dx, "dw_gate": dwg, "dw_up": dwu}


def run(state):
    if own:
        return _own(state)
    return {"adamw": _plain_adamw, "pref_fwd": _plain_pref_fwd, "pref_bwd": _plain_pref_bwd,
            "gated_fwd": _plain_gated_fwd, "gated_bwd": _plain_gated_bwd}[state["kind"]](state)


# ----------------------------------------------------------------------------- work

def work(case):
    if case["kind"] == "adamw":
        n = sum(_sizes(case))
        w = 2 if case["dtype"] == "bf16" else 4
        g = 2 if case["gdtype"] == "bf16" else 4
        states = 16.0 if case["bits"] == 32 else 4.0 + 4.0 / BLOCK
        return {"bytes": n * (2 * w + g + states), "flops": 16.0 * n}
    if case["kind"] in ("pref_fwd", "pref_bwd"):
        e = 2 if case["dtype"] == "bf16" else 4
        lengths, prompts = _lengths(case)
        counted, rows = sum(lengths) - sum(prompts), sum(lengths) + case["tail"]
        # only counted rows are read; the gradient's other rows are zeros to be written
        moved = counted * case["vocab"] * e + 16.0 * rows
        if case["kind"] == "pref_bwd":
            moved += rows * case["vocab"] * e
        return {"bytes": moved, "flops": 4.0 * counted * case["vocab"]}
    t, d, f = case["tokens"], case["d"], case["f"]
    if case["kind"] == "gated_fwd":
        return {"bytes": 2.0 * (t * d + 2 * d * f + t * f * (3 if case["save"] else 1)),
                "flops": 4.0 * t * d * f + 6.0 * t * f}
    return {"bytes": 2.0 * (2 * t * d + 4 * d * f + 3 * t * f), "flops": 8.0 * t * d * f + 12.0 * t * f}


# ---------------------------------------------------------------------------- exact

def _scaled64(codes, exps):
    e = exps.to(torch.int32).clamp(min=40) - 134
    return torch.ldexp(codes.double().view(-1, BLOCK), e[:, None]).view(-1)


def _rounded64(x, bits16):
    """x in 64 bits as multiples of its blocks' powers of two, rounded to e4m3 values by 16 random
    bits an element.  (The power of two is that of the block's largest value in 32 bits.)"""
    size = x.abs().view(-1, BLOCK)
    mantissa, k = torch.frexp(size.amax(1).float())
    exps = torch.where(mantissa > 0, k + 126, torch.zeros_like(k)).clamp(min=40)
    y = torch.ldexp(size, (134 - exps)[:, None]).view(-1)
    for power in range(-6, 9):                    # values of [2^power, 2^(power + 1)): 8 steps
        low = 2.0 ** power if power > -6 else 0.0
        here = (y >= low) & (y < 2.0 ** (power + 1))
        step = 2.0 ** (power - 3)
        y = torch.where(here, -torch.floor(y / step + bits16.double() / 65536) * step, y)
    return -y


def _exact_adamw(case, seed):
    s = _adamw_state(case, seed)
    g, w = s["G"].double(), s["W"].double()
    if case["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m, v = _scaled64(s["m"], s["m_exp"]), _scaled64(s["v"], s["v_exp"]).square()
    m.lerp_(g, 1.0 - B1)
    v.lerp_(g * g, 1.0 - B2)
    root = v.sqrt()
    hat = m / (1.0 - B1 ** case["t"])
    w = w - LR * WD * w - LR * hat / (root / math.sqrt(1.0 - B2 ** case["t"]) + EPS)
    if case["bits"] == 32:
        return {"W": w, "m": m, "v": v}
    bits16 = _rounding_bits(s)
    qm, qv = _rounded64(m, bits16), _rounded64(root, bits16)
    qv = torch.where(v > 0, qv.clamp(min=2.0 ** -9), qv)
    return {"W": w, "m": torch.where(m < 0, -qm, qm), "v": qv, "m_exp": None, "v_exp": None}


def _exact_pref(case, seed):
    s = _pref_state(case, seed)
    labels, rows = s["labels"], s["labels"].shape[0]
    if case["kind"] == "pref_bwd":
        out = torch.zeros(rows, case["vocab"], dtype=torch.float64, device=DEVICE)
        for r0 in range(0, rows, 2048):
            lab = labels[r0:r0 + 2048]
            p = torch.exp(s["logits"][r0:r0 + 2048].double() - s["lse"][r0:r0 + 2048, None].double())
            hit = torch.arange(case["vocab"], device=DEVICE)[None] == lab[:, None]
            scale = float(s["dloss"]) * s["dlogp"][r0:r0 + 2048].double() * (lab >= 0)
            out[r0:r0 + 2048] = torch.where(scale[:, None] == 0, 0.0, scale[:, None] * (hit.double() - p))
        return out
    lengths, _ = _lengths(case)
    lse = torch.zeros(rows, dtype=torch.float64, device=DEVICE)
    logp = torch.zeros_like(lse)
    for r0 in range(0, rows, 2048):
        x = s["logits"][r0:r0 + 2048].double()
        lse[r0:r0 + 2048] = torch.logsumexp(x, 1)
        logp[r0:r0 + 2048] = torch.log_softmax(x, 1).gather(1, labels[r0:r0 + 2048, None].clamp(min=0))[:, 0]
    end = sum(lengths)
    live = (labels[:end] >= 0).double()
    per = [(a * b).sum() for a, b in zip(logp[:end].split(lengths), live.split(lengths))]
    logps, n = torch.stack(per), case["pairs"]
    gain = logps - s["ref"].double()
    d = (gain[:n] - gain[n:]).requires_grad_()
    if case["loss"] == "square":
        losses = torch.square(d - 1.0 / (2.0 * BETA))
    elif case["loss"] == "hinge":
        losses = torch.relu(1.0 - BETA * d)
    else:
        ls = torch.nn.functional.logsigmoid
        losses = -(1.0 - SMOOTH) * ls(BETA * d) - SMOOTH * ls(-BETA * d)
    slope, = torch.autograd.grad(losses.mean(), d)
    by_seq = torch.cat([slope, -slope]).split(1)
    dlogp = torch.cat([c.expand(k) for c, k in zip(by_seq, lengths)]) * live
    pad = torch.zeros(rows - end, dtype=torch.float64, device=DEVICE)
    losses = losses.detach()
    return {"loss": losses.mean(), "losses": losses, "logps": logps,
            "lse": lse * torch.cat([live, pad]), "dlogp": torch.cat([dlogp, pad])}


def _exact_gated(case, seed):
    s = _gated_state(case, seed)
    x, wg, wu = s["x"].double(), s["wg"].double(), s["wu"].double()
    act = torch.nn.functional.silu if case["act"] == "silu" else (
        lambda g: torch.nn.functional.gelu(g, approximate="tanh"))
    if case["kind"] == "gated_fwd":
        g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
        out = {"h": act(g) * u}
        if case["save"]:
            out.update(gate=g, up=u)
        return out
    g = s["gate"].double().requires_grad_()
    u, dh = s["up"].double(), s["dh"].double()
    a = act(g)
    dg, = torch.autograd.grad(a, g, dh * u)
    du = dh * a.detach()
    return {"dx": torch.addmm(torch.mm(dg, wg), du, wu), "dw_gate": torch.mm(dg.t(), x),
            "dw_up": torch.mm(du.t(), x)}


def exact(case, seed):
    if case["kind"] == "adamw":
        return _exact_adamw(case, seed)
    if case["kind"] in ("pref_fwd", "pref_bwd"):
        return _exact_pref(case, seed)
    if 8.0 * case["tokens"] * case["d"] * case["f"] > 8e12:        # beyond ~20 s of products
        return None
    return _exact_gated(case, seed)
