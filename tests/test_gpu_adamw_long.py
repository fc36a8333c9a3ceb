"""AdamW's 8-bit steps of tensors that a warp goes through block by block, with the next block on its
way: 10M elements (two blocks of every warp to a chunk) and 75M (eight), with odd ends.  The same
values one element off 16 bytes take the general path, element by element, and have to give the same
bits; and those are the codes of fp32 arithmetic with the oracle's random words."""

import numpy as np
import pytest
import torch

from oracle import rng
from test_gpu_adamw import B1, B2, EPS, LR, TYPES, WD, f64, values

pytestmark = pytest.mark.gpu

f = np.float32


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def off(t):
    """The same values, one element behind a 16-byte boundary."""
    buf = torch.zeros(t.numel() + 64, dtype=t.dtype, device=t.device)
    at = 16 // t.element_size() + 1
    assert buf.data_ptr() % 16 == 0
    return buf[at:at + t.numel()].copy_(t)


def tensors(sizes, dtype, gdtype, dev):
    from paper_2608_15665_gb300 import firstorder as fo
    g = torch.Generator(device=dev).manual_seed(7)
    out = []
    for n in sizes:
        scale = 1e-3 * torch.exp(torch.randn(-(-n // 64), generator=g, device=dev))
        scale = scale.repeat_interleave(64)[:n]
        W = (torch.randn(n, generator=g, device=dev) * 0.02).to(TYPES[dtype])
        G = (torch.randn(n, generator=g, device=dev) * scale).to(TYPES[gdtype])
        s = fo.adamw_state(W, 8)
        for c in (s.m, s.v):
            c.view(torch.uint8).copy_(torch.randint(0, 0x79, (n,), generator=g, device=dev))
        for e in (s.m_exp, s.v_exp):
            e.copy_(torch.randint(115, 122, e.shape, generator=g, device=dev))
        out.append((W, G, s))
    return out


@pytest.mark.parametrize("sizes,dtype,gdtype", [
    ([10_000_133], "bf16", "bf16"), ([10_000_133], "f32", "f32"), ([10_000_133], "bf16", "f32"),
    ([10_000_133], "f32", "bf16"), ([75_000_069], "bf16", "bf16"),
    ([300, 9_000_001, 257, 2_000_000, 1, 4096], "bf16", "f32"),
    ([40_000_000, 33, 36_000_255, 70_000], "f32", "f32")])
def test_whole_blocks_and_the_general_path_give_the_same_bits(lib, gpu, sizes, dtype, gdtype):
    from paper_2608_15665_gb300 import firstorder as fo
    data = tensors(sizes, dtype, gdtype, gpu)
    W, G, S = (list(t) for t in zip(*data))
    first = [(w.clone(), s.m.clone(), s.v.clone(), s.m_exp.clone(), s.v_exp.clone()) for w, _, s in data]
    W2, G2 = [off(t) for t in W], [off(t) for t in G]
    S2 = [fo.AdamWState(*(off(c.view(torch.uint8)).view(torch.float8_e4m3fn) for c in (s.m, s.v)),
                        s.m_exp.clone(), s.v_exp.clone()) for s in S]
    a, b = (fo.AdamW(w, g, states=s, bits=8, seed=(3 << 32) + 9) for w, g, s in ((W, G, S), (W2, G2, S2)))
    for t in (5, 6):
        for op in (a, b):
            op.step(LR, (B1, B2), EPS, WD, t=t)
        for k in range(len(sizes)):
            assert same(W[k], W2[k])
            assert all(same(p, q) for p, q in zip(S[k], S2[k])), (t, k)
        if t == 5:
            # the codes and the update of pieces of the first step, the last elements among them
            for k, n in enumerate(sizes):
                for at in sorted({0, (n // 3) // 256 * 256, max(0, (n - 3000) // 256 * 256)}):
                    check_piece(first[k], G[k], W[k], S[k], k, at, min(n - at, 4000), t, dtype)
    a.close()
    b.close()


def check_piece(before, G, W, s, index, at, n, t, dtype):
    w0, m0, v0, em0, ev0 = before
    here, blocks = slice(at, at + n), slice(at // 256, (at + n - 1) // 256 + 1)
    m = values(m0[here], em0[blocks], (n,)).astype(f)
    r = values(v0[here], ev0[blocks], (n,)).astype(f)
    x = f64(G[here]).astype(f)
    m1, v1 = f(B1) * m + f(1.0 - B1) * x, f(B2) * (r * r) + f(1.0 - B2) * (x * x)
    c = np.arange(at // 8, -(-(at + n) // 8), dtype=np.uint64)      # eight elements to a counter
    ctr = np.stack([c] + [np.full(c.size, v, dtype=np.uint64) for v in (index, t, 6 << 24)], axis=-1)
    key = np.broadcast_to(np.array(rng.key_of_seed((3 << 32) + 9), dtype=np.uint64), (c.size, 2))
    words = rng.philox4x32_10(ctr, key).reshape(-1).astype(np.uint64)
    u = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], 1).reshape(-1)[:n] / 65536.0
    # (a block that the piece cuts off has its largest elsewhere)
    whole = n if at + n == G.numel() else n // 256 * 256
    pad = np.zeros(-(-whole // 256) * 256)
    for code, exps, y, roots in ((s.m, s.m_exp, m1, False), (s.v, s.v_exp, v1, True)):
        pad[:whole] = np.abs(y[:whole])
        E = np.frexp(pad.reshape(-1, 256).max(1))[1] - 1
        E = (E >> 1 if roots else E) + 127
        assert np.array_equal(exps[blocks].cpu().numpy()[:E.size], E)
        y = np.abs(np.sqrt(y) if roots else y)[:whole].astype(np.float64)
        y = y * 2.0 ** np.repeat(134.0 - np.maximum(E, 40), 256)[:whole]
        step = 2.0 ** (np.floor(np.log2(np.maximum(y, 1e-30))) - 3)
        normal = y >= 2.0 ** -6
        got = np.abs(f64(code[here]))[:whole]
        assert np.array_equal(got[normal], (np.floor(y / step + u[:whole]) * step)[normal])
    move = LR * m1.astype(np.float64) / (1 - B1 ** t) / (np.sqrt(v1.astype(np.float64) / (1 - B2 ** t)) + EPS)
    want = (1 - LR * WD) * f64(w0[here]) - move
    # 24 roundings of the update, two of W, and half an ulp of the result
    lim = 2.0 ** -24 * (24 * np.abs(move) + 2 * np.abs(f64(w0[here])))
    lim += 1.01 * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want)
    assert np.all(np.abs(f64(W[here]) - want) <= lim)
