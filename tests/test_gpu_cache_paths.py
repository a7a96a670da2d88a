"""GPU tests of the variants that larger prompts and longer caches take: the
prompt score's 128- and 256-key workgroups, whole and partly seen steps; the
step score's 512- and 1024-key chunks, whose waves refill their rings."""
import math

import numpy as np
import pytest

import _cache_shapes as shapes

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


def normal(g, *shape, std=1.0):
    import torch
    return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)


def weights(q, k, pos, lse=None):
    """fp64 softmax weights of rows q [n, G, d] on the keys k [L, d] up to
    pos [n], summed over the heads [n, L], and the largest sum |q k| of a score
    in the exp2 domain."""
    import torch
    n, G, d = q.shape
    c = math.log2(math.e) / math.sqrt(d)
    q, kt = q.reshape(n * G, d), k.t().contiguous()
    x = (torch.matmul(q, kt) * c).view(n, G, -1)
    size = float(torch.matmul(q.abs(), kt.abs()).max()) * c
    if pos is not None:
        hidden = torch.arange(k.shape[0], device=k.device)[None, :] > pos[:, None]
        x.masked_fill_(hidden[:, None, :], -math.inf)
    if lse is None:
        top = x.amax(-1, keepdim=True)
        w = torch.exp2(x - top)
        w /= w.sum(-1, keepdim=True)
    else:
        w = torch.exp2(x - lse[:, :, None])
    return w.sum(1), size


def tolerance(total, terms, d, size):
    """As _cache_ops.score_tolerance: a term's exponent is a sum of d products,
    scaled, less a log-sum-exp of the same size (2^-24 of sum |q k| each), the
    exponential and logarithm 2^-22, the terms added one after the other."""
    return ((math.log(2.0) * (2 * d + 8) * size + terms + 16) * 2.0 ** -24) * total + 1e-30


@pytest.mark.parametrize("ci", range(len(shapes.SCORES)))
def test_cache_score_of_larger_prompts(pk, ci):
    import torch
    (lens, n_rows, hq, hkv, d), _ = shapes.SCORES[ci]
    g = torch.Generator(device="cuda")
    g.manual_seed(700 + ci)
    rng = np.random.default_rng(700 + ci)
    N, cu, G = sum(lens), cu_of(lens), hq // hkv
    q, k = normal(g, N, hq, d, std=2.0), normal(g, N, hkv, d)
    before = torch.rand((hkv, N), generator=g, device="cuda")
    rows = []
    for T, n in zip(lens, n_rows):
        early = rng.choice(max(T - n, 0), min(n // 5, max(T - n, 0)), replace=False)
        rows.append(np.concatenate([np.sort(early), np.arange(T - n + len(early), T)]))
    cu_sel = cu_of([len(r) for r in rows])
    sel = np.concatenate([r + c for r, c in zip(rows, cu)]).astype(np.int32)
    dsel, dcs, dcu = (torch.from_numpy(x).cuda() for x in (sel, cu_sel, cu))
    prob = pk.Problem(dcu, hq, hkv, d, 64, cu_seqlens_host=cu)
    lse = torch.rand((hq, len(sel)), generator=g, device="cuda") * 8 + 4
    for given in (None, lse):
        want, size = before.double(), 0.0
        for b in range(len(lens)):
            s0, s1, c0, c1 = cu_sel[b], cu_sel[b + 1], cu[b], cu[b + 1]
            tok = dsel[s0:s1].long()
            for h in range(hkv if s1 > s0 else 0):
                hs = slice(h * G, (h + 1) * G)
                w, x = weights(q[tok, hs].double(), k[c0:c1, h].double(), tok - int(c0),
                               None if given is None else given[hs, s0:s1].t().double())
                want[h, c0:c1] += w.sum(0)
                size = max(size, x)
        got = pk.logo_cache_score(prob, q, k, sel_idx=dsel, cu_sel=dcs, lse=given, score_in=before)
        e = (got.double() - want).abs()
        worst = float((e / tolerance(want, max(n_rows) * G, d, size + (0 if given is None else 12))).max())
        print(f"[larger score case{ci} lse {'given' if given is not None else 'computed'}] "
              f"worst/tol={worst:.3g} rel={float((e.norm() / want.norm())):.3g}", flush=True)
        assert worst <= 1.0
        again = pk.logo_cache_score(prob, q, k, sel_idx=dsel, cu_sel=dcs, lse=given, score_in=before)
        assert torch.equal(again, got)


@pytest.mark.parametrize("ci", range(len(shapes.STEPS)))
def test_decode_score_of_longer_caches(pk, ci):
    import torch
    (lens, hq, hkv, d), _ = shapes.STEPS[ci]
    g = torch.Generator(device="cuda")
    g.manual_seed(800 + ci)
    N, B, cu, G = sum(lens), len(lens), cu_of(lens), hq // hkv
    q, k = normal(g, B, hq, d, std=2.0), normal(g, N, hkv, d)
    gate = torch.rand(B, generator=g, device="cuda") * 0.4 + 0.6
    gate[3] = 0.1
    prob = pk.Problem(torch.from_numpy(cu).cuda(), hq, hkv, d, 64, cu_seqlens_host=cu)
    want, size = torch.zeros((hkv, N), dtype=torch.float64, device="cuda"), 0.0
    for b in range(B):
        for h in range(hkv if b != 3 else 0):
            w, x = weights(q[b:b + 1, h * G:(h + 1) * G].double(), k[cu[b]:cu[b + 1], h].double(), None)
            want[h, cu[b]:cu[b + 1]] = w[0]
            size = max(size, x)
    got = pk.logo_decode_score(prob, q, k, gate, threshold=0.5)
    e = (got.double() - want).abs()
    worst = float((e / tolerance(want, G, d, size)).max())
    print(f"[longer step case{ci}] worst/tol={worst:.3g} rel={float(e.norm() / want.norm()):.3g}",
          flush=True)
    assert worst <= 1.0
    for _ in range(3):
        assert torch.equal(pk.logo_decode_score(prob, q, k, gate, threshold=0.5), got)
