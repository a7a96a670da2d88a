"""How exact the cache operators are: inputs whose scores are exact in fp32, so
that the tolerances count only the roundings that the operators document.

Steps of a rounding are counted as torch.finfo(t).eps / 2 relative to the value
(bf16 2^-8, fp32 2^-24); the hardware's exponential, reciprocal and square root
as 2^-22; sums inside matrix products as 2^-23 per term.
"""
import math

import numpy as np
import pytest

import _cache_ops as ref
import synth
from _support import to_device, torch_bf16_to_f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu tests need an MI355X")
    import paper_2608_29539_amd as pk
    pk.library()
    return pk


def cu_of(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def grid(rng, step, *shape):
    """bf16 bits of -4 .. 4 times step: products of two such numbers and sums
    of 128 of them are exact in fp32."""
    x = (rng.integers(-4, 5, shape) * step).astype(np.float32)
    return synth.bf16_bits_from_f32(x.reshape(-1)).reshape(shape)


def attend(q, k, v, c):
    """One token's heads in fp64: (o [Hq, d], sum of the weights times |v|, the
    largest |score| in the exp2 domain)."""
    hq, d = q.shape
    G = hq // k.shape[1]
    o, a, top = np.zeros((hq, d)), np.zeros((hq, d)), 0.0
    for h in range(hq):
        x = c * (k[:, h // G] @ q[h])
        w = np.exp2(x - x.max())
        w /= w.sum()
        o[h], a[h] = w @ v[:, h // G], w @ np.abs(v[:, h // G])
        top = max(top, float(np.abs(x).max()))
    return o, a, top


def normed(o, a, top, n, eps, gain):
    """ContextNorm of a branch of n keys, and the bound on its error before the
    last rounding.  Relative to sum w |v|: an exponent is a product with the
    rounded scale, a fused subtraction and, where parts are joined, differences
    of maxima (6 roundings of at most 2 top); four exponentials (of the weight
    and of three joins); the weight in two bf16 parts (2^-16); 2 n + 64 terms
    added up in the numerator and n + 64 in the denominator."""
    e = (math.log(2.0) * 12 * top * 2.0 ** -24 + 4 * 2.0 ** -22 + 2.0 ** -16
         + (2 * n + 64) * 2.0 ** -23 + (n + 64) * 2.0 ** -24)
    r = np.sqrt((o * o).mean(-1, keepdims=True) + eps)
    dr = e * np.sqrt((a * a).mean(-1, keepdims=True))
    y = o / r * gain
    return y, (e * a / r + np.abs(o) * dr / r ** 2) * gain + 2.0 ** -21 * np.abs(y)


PRECISION = [
    # (prefix, group, own rows, Hq, Hkv, d, window): few rows a KV head, many
    # rows, the window inside the prefix and inside the own rows, no prefix
    (200, 3, (1, 30, 17), 8, 2, 128, 64), (200, 20, tuple(range(1, 21)), 8, 2, 128, 40),
    (130, 2, (60, 5), 4, 4, 64, 16), (150, 40, (7,) * 40, 4, 2, 64, 300),
    (0, 2, (90, 200), 8, 2, 128, 50), (257, 9, (3,) * 9, 16, 4, 64, 100),
]


@pytest.mark.parametrize("distinct", [False, True], ids=["shared", "own-global"])
@pytest.mark.parametrize("ci", range(len(PRECISION)))
def test_prefix_rounds_once(pk, ci, distinct):
    """The step's output is the 64-bit one rounded once to bf16, but for fp32
    roundings: the weights keep 16 bits or more for the product with V."""
    import torch
    P, n, own, hq, hkv, d, win = PRECISION[ci]
    rng = np.random.default_rng(4000 + ci)
    N, cu = sum(own), cu_of(own)
    x = dict(q=grid(rng, 0.5, n, hq, d), k=grid(rng, 0.25, N, hkv, d),
             k_pre=grid(rng, 0.25, P, hkv, d))
    if distinct:
        x.update(q_g=grid(rng, 0.5, n, hq, d), k_g=grid(rng, 0.25, N, hkv, d),
                 k_pre_g=grid(rng, 0.25, P, hkv, d))
    for name, rows in (("v", N), ("v_pre", P), ("v_g", N), ("v_pre_g", P)):
        if distinct or name in ("v", "v_pre"):
            x[name] = synth.bf16_bits_from_f32(
                rng.standard_normal(rows * hkv * d).astype(np.float32)).reshape(rows, hkv, d)
    gate = (0.2 + 0.6 * (np.arange(n) % 2) + 0.1 * rng.random(n)).astype(np.float32)
    gains = rng.uniform(0.5, 1.5, (2, hq, d)).astype(np.float32)
    eps, scale = 1e-6, 2.0 / math.sqrt(d)
    dev = to_device(dict(cu=cu, cp=cu_of([P]), cg=cu_of([n]), gate=gate, gl=gains[0], gg=gains[1],
                         **x))
    prob = pk.Problem(dev["cu"], hq, hkv, d, win, cu_seqlens_host=cu, softmax_scale=scale)
    pre = pk.Prefix(dev["cp"], dev["cg"], cu_prefix_host=[0, P], cu_group_host=[0, n])
    got = pk.logo_decode_prefix(prob, pre, dev["q"], dev["k_pre"], dev["v_pre"], dev["k"], dev["v"],
                                dev["gate"], threshold=0.5, eps=eps, gain_local=dev["gl"],
                                gain_global=dev["gg"],
                                **{t: dev[t] for t in x if t.endswith("_g")})[0]
    torch.cuda.synchronize()
    got = torch_bf16_to_f64(got)
    f = {t: ref.f64(a) for t, a in x.items()}
    c = float(np.float32(scale)) * math.log2(math.e)
    worst = 0.0
    for b in range(n):
        keys = {t: np.concatenate([f[t.replace("K", "k_pre")], f[t.replace("K", "k")][cu[b]:cu[b + 1]]])
                for t in ("K",) + (("K_g",) if distinct else ())}
        vals = {t: np.concatenate([f[t.replace("V", "v_pre")], f[t.replace("V", "v")][cu[b]:cu[b + 1]]])
                for t in ("V",) + (("V_g",) if distinct else ())}
        L = len(keys["K"])
        lo = max(0, L - win)
        o, a, top = attend(f["q"][b], keys["K"][lo:], vals["V"][lo:], c)
        want, slack = normed(o, a, top, L - lo, eps, gains[0])
        p = float(gate[b])
        if p > 0.5:
            g = "_g" if distinct else ""
            o, a, top = attend(f["q" + g][b], keys["K" + g], vals["V" + g], c)
            yg, sg = normed(o, a, top, L, eps, gains[1])
            # (1 - p, two products and a sum: 4 fp32 roundings)
            slack = (1 - p) * slack + p * sg + 2.0 ** -22 * ((1 - p) * np.abs(want) + p * np.abs(yg))
            want = (1 - p) * want + p * yg
        tol = 2.0 ** -8 * np.abs(want) + (1 + 2.0 ** -8) * slack
        worst = max(worst, float((np.abs(got[b] - want) / tol).max()))
    print(f"[prefix precision case{ci}] worst/tol={worst:.3g}", flush=True)
    assert worst <= 1.0


# --- the sums of weights ----------------------------------------------------------
LONG = [
    # (tokens, last rows, Hq, Hkv, d): 64, 128 and 256 keys per workgroup
    (4100, 4100, 8, 1, 64), (9001, 3000, 16, 4, 128), (8200, 4000, 32, 8, 64),
]


@pytest.mark.parametrize("kind", ["one-large", "spread"])
@pytest.mark.parametrize("ci", range(len(LONG)))
def test_long_sums_keep_their_small_terms(pk, ci, kind):
    """Scores of zero and whole log-sum-exps: every weight is a power of two,
    and a key's sum is off by the roundings of one block of rows (16 terms in a
    lane), of the sum itself, and of joining two lanes, four waves and what was
    there before (8) -- not by one for each of its thousands of blocks."""
    import torch
    N, n, hq, hkv, d = LONG[ci]
    rng = np.random.default_rng(5000 + ci)
    if kind == "one-large":                      # 1 in the first rows, then terms below its steps
        lse = np.full((hq, n), 24.0, np.float32)
        lse[:, :40] = 0.0
    else:
        lse = rng.integers(0, 20, (hq, n)).astype(np.float32)
    sel = np.arange(N - n, N).astype(np.int32)
    dev = to_device(dict(cu=cu_of([N]), sel=sel, cu_sel=cu_of([n]), lse=lse))
    q = torch.zeros((N, hq, d), dtype=torch.bfloat16, device="cuda")
    k = torch.ones((N, hkv, d), dtype=torch.bfloat16, device="cuda")
    prob = pk.Problem(dev["cu"], hq, hkv, d, 64, cu_seqlens_host=cu_of([N]))
    got = pk.logo_cache_score(prob, q, k, sel_idx=dev["sel"], cu_sel=dev["cu_sel"], lse=dev["lse"])
    got = got.cpu().numpy().astype(np.float64)
    w = np.exp2(-lse.astype(np.float64)).reshape(hkv, hq // hkv, n).sum(1)
    later = np.cumsum(w[:, ::-1], axis=1)[:, ::-1]             # rows at or after each
    want = np.concatenate([np.repeat(later[:, :1], N - n, 1), later], 1)
    tol = (16 + 2 + 8) * 2.0 ** -24 * want
    worst = float((np.abs(got - want) / tol).max())
    print(f"[score sums {kind} case{ci}] worst/tol={worst:.3g}", flush=True)
    assert worst <= 1.0
