"""The serving operators of long caches, as their users call them, with plain
forms to compare them with.

  prefix  one decoding step of the layer for groups of sequences that share a
          long prefix (``logo_decode_prefix``)
  score   the attention weight that every cached key has received from a
          prompt's queries (``logo_cache_score``): with the log-sum-exp that
          the forward kept, or without it
  step    the same for one decoding step (``logo_decode_score``)
  evict   the caches cut down to a budget of rows per KV head, the newest rows
          and those with the largest weight (``logo_cache_evict``)

Tensors are bf16 with fp32 gates, weights and log-sum-exps (the types that the
entry points take).  With ``own`` false, ``run`` computes the operators from
elementary torch operations in fp32.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
LOG2E = 1.4426950408889634


# --- the cases ---------------------------------------------------------------
def _case(name, op, lens, hq, hkv, d, **kw):
    """lens: cache lengths (op prefix: the sequences' own caches)."""
    c = dict(op=op, lens=lens, hq=hq, hkv=hkv, d=d)
    if op == "prefix":          # prefixes' lengths, sequences per prefix
        c.update(prefixes="0", groups="1", window=128, ratio=0.125, device_thr=False,
                 distinct=False, gains=False)
    if op == "score":           # share of the rows that are queries, or the last `last` of each
        c.update(ratio=0.125, last=0, lse=True)
    if op == "step":
        c.update(ratio=1.0)
    if op == "evict":
        c.update(budget=1024, recent=128)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # few requests behind a short system prompt, just started: latency
        _case("prefix-4x1k-mha-d64", "prefix", "1,17,5,64", 4, 4, 64, prefixes="1024", groups="4",
              window=128, ratio=0.25),
        # a serving batch behind a long document, an eighth of the tokens global
        _case("prefix-32x16k-gqa", "prefix", ",".join(str(37 + 61 * i) for i in range(32)), 32, 8,
              128, prefixes="16384", groups="32", window=1024, ratio=0.125),
        # many samples of one 32K prompt, every token global, learned gains
        _case("prefix-64x32k-gqa-all", "prefix", ",".join(str(200 + 3 * i) for i in range(64)),
              32, 8, 128, prefixes="32768", groups="64", window=1024, ratio=1.0, gains=True),
        # three prompts of odd lengths, one of them shorter than the window,
        # the threshold on the device, the global branch's own tensors
        _case("prefix-3groups-odd", "prefix", ",".join(str(1 + 97 * i % 1009) for i in range(23)),
              16, 2, 128, prefixes="5001,12345,257", groups="5,17,1", window=512, ratio=0.5,
              device_thr=True, distinct=True),
        # a short prompt's global branch
        _case("score-1k-d64", "score", "1024", 8, 2, 64, ratio=0.25),
        # the last 64 queries of three prompts of odd lengths, no forward behind them
        _case("score-last64", "score", "8192,5001,131", 32, 8, 128, last=64, lse=False),
        # the headline layer's prompt, the selected rows' weights with the
        # forward's log-sum-exp
        _case("score-32k-gqa", "score", "32768", 32, 8, 128, ratio=0.125),
        # serving: few short caches, every new token global
        _case("step-4x2k-mha", "step", "2047,513,1200,31", 16, 16, 128),
        # serving: 16 long caches, every new token global
        _case("step-16x32k-gqa", "step", ",".join(["32768"] * 16), 32, 8, 128),
        # a few chats' caches cut to a quarter
        _case("evict-4x2k-d64", "evict", "2048,2048,1999,300", 8, 2, 64, budget=512, recent=128),
        # a serving batch's long caches cut to an eighth
        _case("evict-16x32k", "evict", ",".join(["32768"] * 16), 32, 8, 128, budget=4096,
              recent=1024),
        # one context of the longest kind, odd lengths
        _case("evict-130k", "evict", "131071", 16, 4, 128, budget=16001, recent=4096),
    ]


_HEADS = ((4, 4), (8, 8), (16, 16), (8, 4), (16, 8), (8, 2), (16, 4), (32, 8), (16, 2))


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _join(xs):
    return ",".join(str(x) for x in xs)


def draw(rng):
    while True:
        op = rng.choice(["prefix", "prefix", "score", "score", "step", "evict"])
        hq, hkv = rng.choice(_HEADS)
        d = rng.choice([64, 128, 128])
        if op == "prefix":
            r = rng.choice([1, 1, 1, 2, 3])
            groups = [_log_int(rng, 1, 64) for _ in range(r)]
            if sum(groups) > 64:
                continue
            c = _case(None, op, _join(_log_int(rng, 1, 2048) for _ in range(sum(groups))), hq,
                      hkv, d, prefixes=_join(_log_int(rng, 64, 32768) for _ in range(r)),
                      groups=_join(groups), window=_log_int(rng, 16, 4096),
                      ratio=rng.choice([0.125, 0.5, 1.0]), device_thr=rng.random() < 0.4,
                      distinct=rng.random() < 0.4, gains=rng.random() < 0.4)
        elif op == "score":
            lens = [_log_int(rng, 64, 32768) for _ in range(rng.randint(1, 4))]
            last = rng.choice([0, 0, _log_int(rng, 1, 256)])
            c = _case(None, op, _join(lens), hq, hkv, d, ratio=rng.choice([0.0625, 0.125, 0.25]),
                      last=last, lse=rng.random() < 0.5)
        elif op == "step":
            lens = [_log_int(rng, 16, 32768) for _ in range(rng.randint(1, 16))]
            c = _case(None, op, _join(lens), hq, hkv, d, ratio=rng.choice([0.25, 0.5, 1.0]))
        else:
            lens = [_log_int(rng, 64, 131072) for _ in range(rng.randint(1, 8))]
            if sum(lens) * hkv * d > 524288 * 8 * 128:
                continue
            budget = _log_int(rng, 64, 16384)
            c = _case(None, op, _join(lens), hq, hkv, d, budget=budget,
                      recent=rng.choice([0, budget // 4, budget // 2]))
        if work(c)["flops"] <= 6e11 and work(c)["bytes"] <= 1.2e9:
            return c


# --- inputs ------------------------------------------------------------------
def _ints(s):
    return [int(x) for x in s.split(",")]


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _n_pass(n, ratio):
    """How many of a group's n new tokens are global: ratio of them, at least one."""
    return max(1, int(round(ratio * n)))


def _gates(rng, groups, ratio):
    """Gates of which _n_pass per group are above 1/2, in random places."""
    out = []
    for n in groups:
        z = np.zeros(n, bool)
        z[rng.permutation(n)[:_n_pass(n, ratio)]] = True
        u = rng.uniform(0.02, 0.48, n)
        out.append(np.where(z, 0.5 + u, u))
    return np.concatenate(out).astype(np.float32)


def _selected(case, rng=None):
    """The query rows of op score, ascending within each sequence: a random
    share of the rows, or the last ones; without rng only how many they are."""
    rows = []
    for T in _ints(case["lens"]):
        n = min(T, case["last"]) if case["last"] else max(1, int(case["ratio"] * T))
        if rng is None:
            rows.append(n)
        elif case["last"]:
            rows.append(np.arange(T - n, T))
        else:
            rows.append(np.sort(rng.choice(T, n, replace=False)))
    return rows


def _visible(rows, cu, dev):
    """Positions of packed query rows (fp32 [n, 1]) for the causal comparison."""
    return (rows - cu).to(torch.float32).view(-1, 1).to(dev)


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    op, lens, hq, hkv, d = case["op"], _ints(case["lens"]), case["hq"], case["hkv"], case["d"]
    N, B = sum(lens), len(lens)

    def normal(*shape, std=1.0):
        x = torch.randn(shape, generator=g, device=dev, dtype=torch.float32)
        return (x * std).to(torch.bfloat16)

    s = dict(case=case, cu_host=_cu(lens))
    s["cu"] = torch.from_numpy(s["cu_host"]).to(dev)
    if op != "evict":
        # scores of standard deviation 2, so that some keys get most of the weight
        s["k"] = normal(N, hkv, d)
        s["q"] = normal(N if op == "score" else B, hq, d, std=2.0)
    if op == "prefix":
        pre, groups = _ints(case["prefixes"]), _ints(case["groups"])
        P = sum(pre)
        s["v"] = normal(N, hkv, d)
        s["k_pre"], s["v_pre"] = normal(P, hkv, d), normal(P, hkv, d)
        s["kw"] = {}
        if case["distinct"]:
            s["kw"].update(q_g=normal(B, hq, d, std=2.0), k_g=normal(N, hkv, d),
                           v_g=normal(N, hkv, d), k_pre_g=normal(P, hkv, d),
                           v_pre_g=normal(P, hkv, d))
        if case["gains"]:
            for nm in ("gain_local", "gain_global"):
                s["kw"][nm] = 0.5 + torch.rand((hq, d), generator=g, device=dev)
        s["gate"] = torch.from_numpy(_gates(rng, groups, case["ratio"])).to(dev)
        s["cu_pre_host"], s["cu_group_host"] = _cu(pre), _cu(groups)
        s["thr"] = (dict(threshold_device=torch.full((1,), 0.5, device=dev))
                    if case["device_thr"] else dict(threshold=0.5))
    if op == "step":
        s["gate"] = torch.from_numpy(_gates(rng, [B], case["ratio"])).to(dev)
    if op in ("score", "step"):
        # the weights that earlier queries left
        s["score_in"] = torch.rand((hkv, N), generator=g, device=dev)
    if op == "score":
        rows = _selected(case, rng)
        s["cu_sel_host"] = _cu([len(r) for r in rows])
        sel = np.concatenate([r + c for r, c in zip(rows, s["cu_host"])]).astype(np.int32)
        s["sel_idx"] = torch.from_numpy(sel).to(dev)
        s["cu_sel"] = torch.from_numpy(s["cu_sel_host"]).to(dev)
        s["lse"] = None
        if case["lse"]:
            s["lse"] = _plain_lse(s)
    if op == "evict":
        s["k"], s["v"] = normal(N, hkv, d), normal(N, hkv, d)
        # heavy-tailed weights; a tenth of the rows never got any
        w = torch.randn((hkv, N), generator=g, device=dev).mul_(2.0).exp_()
        w[torch.rand((hkv, N), generator=g, device=dev) < 0.1] = 0.0
        s["score"] = w
    if own:
        import paper_2608_29539_amd as pk
        window = case.get("window", max(lens))
        prob = pk.Problem(s["cu"], hq, hkv, d, window, cu_seqlens_host=s["cu_host"])
        s["pk"], s["prob"] = pk, prob
        if op == "prefix":
            s["prefix"] = pk.Prefix(torch.from_numpy(s["cu_pre_host"]).to(dev),
                                    torch.from_numpy(s["cu_group_host"]).to(dev),
                                    cu_prefix_host=s["cu_pre_host"],
                                    cu_group_host=s["cu_group_host"])
            need = pk.logo_decode_prefix_workspace_bytes(prob, s["prefix"])
            s["out"] = torch.empty_like(s["q"])
        elif op == "score":
            need = pk.logo_workspace_bytes(prob, pk.LOGO_ENTRY_CACHE_SCORE,
                                           int(s["cu_sel_host"][-1]))
            s["out"] = torch.empty_like(s["score_in"])
        elif op == "step":
            need = pk.logo_workspace_bytes(prob, pk.LOGO_ENTRY_DECODE_SCORE)
            s["out"] = torch.empty_like(s["score_in"])
        else:
            cap = pk.logo_cache_keep_capacity(prob, case["budget"])
            need = pk.logo_workspace_bytes(prob, pk.LOGO_ENTRY_CACHE_EVICT)
            s["out"] = dict(k_out=torch.empty((cap, hkv, d), dtype=torch.bfloat16, device=dev),
                            v_out=torch.empty((cap, hkv, d), dtype=torch.bfloat16, device=dev),
                            score_out=torch.empty((hkv, cap), device=dev),
                            keep_idx=torch.empty((hkv, cap), dtype=torch.int32, device=dev),
                            cu_keep=torch.empty(B + 1, dtype=torch.int32, device=dev))
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    return s


# --- the plain forms ---------------------------------------------------------
def _plain_weights(q, k, pos):
    """2^(base-2 logits - their maximum) of query rows q [n, G, d] on keys
    k [L, d], zero past pos [n, 1], with the maximum and the sum."""
    x = (q.reshape(-1, q.shape[-1]) @ k.t()) * (LOG2E / math.sqrt(q.shape[-1]))
    x = x.view(q.shape[0], q.shape[1], -1)
    key = torch.arange(k.shape[0], device=k.device, dtype=torch.float32)
    x = torch.where((key <= pos).unsqueeze(1), x, -math.inf)
    m = x.amax(-1, keepdim=True)
    w = torch.exp2(x - m)
    return w, m, w.sum(-1, keepdim=True)


def _score_blocks(s):
    """(sequence, KV head, slice of ranks) of op score, in blocks of rows that
    keep the weights under 1 GiB."""
    case, cu, cs = s["case"], s["cu_host"], s["cu_sel_host"]
    G = case["hq"] // case["hkv"]
    for b in range(len(cu) - 1):
        L = int(cu[b + 1] - cu[b])
        step = max(1, (1 << 28) // max(1, L * G))
        for r0 in range(int(cs[b]), int(cs[b + 1]), step):
            r1 = min(r0 + step, int(cs[b + 1]))
            for h in range(case["hkv"]):
                yield int(cu[b]), int(cu[b + 1]), h, r0, r1


def _plain_lse(s):
    """Base-2 log-sum-exp of every selected row and head, fp32 [Hq, rows]."""
    case = s["case"]
    G = case["hq"] // case["hkv"]
    out = torch.empty((case["hq"], int(s["cu_sel_host"][-1])), device="cuda")
    for c0, c1, h, r0, r1 in _score_blocks(s):
        sel = s["sel_idx"][r0:r1].long()
        w, m, l = _plain_weights(s["q"][sel, h * G:(h + 1) * G].float(),
                                 s["k"][c0:c1, h].float(), _visible(sel, c0, "cuda"))
        out[h * G:(h + 1) * G, r0:r1] = (m + torch.log2(l)).squeeze(-1).t()
    return out


def _plain_score(s):
    case = s["case"]
    G = case["hq"] // case["hkv"]
    out = s["score_in"].clone()
    for c0, c1, h, r0, r1 in _score_blocks(s):
        sel = s["sel_idx"][r0:r1].long()
        w, m, l = _plain_weights(s["q"][sel, h * G:(h + 1) * G].float(),
                                 s["k"][c0:c1, h].float(), _visible(sel, c0, "cuda"))
        if s["lse"] is None:
            w = w / l
        else:
            lse = s["lse"][h * G:(h + 1) * G, r0:r1].t().unsqueeze(-1)
            w = w * torch.exp2(m - lse)
        out[h, c0:c1] += w.sum((0, 1))
    return out


def _plain_step(s):
    case, cu = s["case"], s["cu_host"]
    hkv, d = case["hkv"], case["d"]
    out = s["score_in"].clone()
    z = (s["gate"] > 0.5).to(torch.float32)
    for b in range(len(cu) - 1):
        k = s["k"][cu[b]:cu[b + 1]].float().transpose(0, 1)              # [Hkv, L, d]
        q = s["q"][b].float().view(hkv, -1, d)                           # [Hkv, G, d]
        x = torch.bmm(q, k.transpose(1, 2)) * (LOG2E / math.sqrt(d))
        w = torch.exp2(x - x.amax(-1, keepdim=True))
        out[:, cu[b]:cu[b + 1]] += (w / w.sum(-1, keepdim=True)).sum(1) * z[b]
    return out


def _plain_attend(q, k, v):
    """Softmax attention of one token's heads q [Hq, d] on rows k, v [L, Hkv, d]."""
    hkv, d = k.shape[1], k.shape[2]
    x = torch.bmm(q.view(hkv, -1, d), k.permute(1, 2, 0)) * (LOG2E / math.sqrt(d))
    w = torch.exp2(x - x.amax(-1, keepdim=True))
    o = torch.bmm(w, v.transpose(0, 1)) / w.sum(-1, keepdim=True)
    return o.reshape(-1, d)


def _plain_prefix(s):
    case, kw = s["case"], s["kw"]
    cu, cp, cg, w = s["cu_host"], s["cu_pre_host"], s["cu_group_host"], case["window"]
    names = ("q", "k", "v", "k_pre", "v_pre")
    loc = {n: s[n].float() for n in names}
    glb = {n: kw[n + "_g"].float() for n in names} if case["distinct"] else loc
    gl, gg = kw.get("gain_local", 1.0), kw.get("gain_global", 1.0)

    def norm(o, gain):
        return o * torch.rsqrt((o * o).mean(-1, keepdim=True) + EPS) * gain

    rows = []
    for r in range(len(cp) - 1):
        p0, p1 = int(cp[r]), int(cp[r + 1])
        for b in range(int(cg[r]), int(cg[r + 1])):
            c0, c1 = int(cu[b]), int(cu[b + 1])
            lo = max(p0, p1 - max(0, w - (c1 - c0)))      # the window's part of the prefix
            s0 = max(c0, c1 - w)
            ol = _plain_attend(loc["q"][b], torch.cat([loc["k_pre"][lo:p1], loc["k"][s0:c1]]),
                               torch.cat([loc["v_pre"][lo:p1], loc["v"][s0:c1]]))
            og = _plain_attend(glb["q"][b], torch.cat([glb["k_pre"][p0:p1], glb["k"][c0:c1]]),
                               torch.cat([glb["v_pre"][p0:p1], glb["v"][c0:c1]]))
            p = s["gate"][b]
            nl = norm(ol, gl)
            rows.append(torch.where(p > 0.5, (1 - p) * nl + p * norm(og, gg), nl))
    return torch.stack(rows).to(torch.bfloat16)


def _plain_evict(s):
    case, cu = s["case"], s["cu_host"]
    idx, lens = [], []
    for b in range(len(cu) - 1):
        L = int(cu[b + 1] - cu[b])
        n = min(L, case["budget"])
        rec = min(case["recent"], n)
        old = s["score"][:, cu[b]:cu[b + 1] - rec]
        top = torch.sort(old, dim=1, descending=True, stable=True)[1][:, :n - rec]
        new = torch.arange(L - rec, L, device=old.device).expand(case["hkv"], rec)
        idx.append(torch.cat([torch.sort(top, dim=1)[0], new], 1) + int(cu[b]))
        lens.append(n)
    idx = torch.cat(idx, 1)                                              # [Hkv, kept]
    rows = idx.t().unsqueeze(-1).expand(-1, -1, case["d"])
    cu_keep = torch.zeros(len(cu), dtype=torch.int32)
    cu_keep[1:] = torch.cumsum(torch.tensor(lens), 0)
    return dict(k_out=s["k"].gather(0, rows), v_out=s["v"].gather(0, rows),
                score_out=s["score"].gather(1, idx), keep_idx=idx.to(torch.int32),
                cu_keep=cu_keep.to(idx.device))


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"prefix": _plain_prefix, "score": _plain_score, "step": _plain_step,
                "evict": _plain_evict}[op](state)
    s, pk, prob = state, state["pk"], state["prob"]
    if op == "prefix":
        return pk.logo_decode_prefix(prob, s["prefix"], s["q"], s["k_pre"], s["v_pre"], s["k"],
                                     s["v"], s["gate"], out=s["out"], ws=s["ws"], eps=EPS,
                                     **s["thr"], **s["kw"])[0]
    if op == "score":
        return pk.logo_cache_score(prob, s["q"], s["k"], sel_idx=s["sel_idx"],
                                   cu_sel=s["cu_sel"], lse=s["lse"], score_in=s["score_in"],
                                   score=s["out"], ws=s["ws"])
    if op == "step":
        return pk.logo_decode_score(prob, s["q"], s["k"], s["gate"], threshold=0.5,
                                    score_in=s["score_in"], score=s["out"], ws=s["ws"])
    case = s["case"]
    pk.logo_cache_evict(prob, s["score"], case["budget"], recent=case["recent"], k=s["k"],
                        v=s["v"], ws=s["ws"], **s["out"])
    return s["out"]


# --- what a pass cannot do without -------------------------------------------
def work(case):
    op, lens, hq, hkv, d = case["op"], _ints(case["lens"]), case["hq"], case["hkv"], case["d"]
    N, B = sum(lens), len(lens)
    row = 2 * hkv * d                                    # bytes of one K or V row
    if op == "evict":
        kept = sum(min(L, case["budget"]) for L in lens)
        return {"bytes": 4 * hkv * N + kept * (4 * row + 8 * hkv), "flops": hkv * N}
    if op == "score":
        pairs = read = 0
        for L, n in zip(lens, _selected(case)):
            pairs += n * (L - (n - 1) / 2 if case["last"] else (L + 1) / 2)
            read += n * (2 * hq * d + (4 * hq if case["lse"] else 0))
        return {"bytes": N * row + 8 * hkv * N + read, "flops": int(2 * d * hq * pairs)}
    if op == "step":
        share = _n_pass(B, case["ratio"]) / B
        return {"bytes": int(share * N * row) + 8 * hkv * N + 2 * B * hq * d,
                "flops": int(share * 2 * d * hq * N)}
    # prefix: the window's rows for every token, all rows for the selected ones
    # (of the average length), a prefix's rows once for its group
    w, b0, rows, pairs = case["window"], 0, 0.0, 0.0
    for P, n in zip(_ints(case["prefixes"]), _ints(case["groups"])):
        own_len, z = lens[b0:b0 + n], _n_pass(n, case["ratio"])
        b0 += n
        tail = [min(P, max(0, w - S)) for S in own_len]
        near = [min(S, w) for S in own_len]
        pairs += sum(near) + sum(tail) + z * (P + sum(own_len) / n)
        rows += P + sum(near) + z / n * sum(own_len)
        rows += max(tail) if case["distinct"] else -z / n * sum(near)
    return {"bytes": int(rows * 2 * row) + 4 * B * hq * d + 4 * B, "flops": int(4 * d * hq * pairs)}


# --- the definitions in 64 bits ----------------------------------------------
def _softmax64(q, k, mask):
    """Weights in fp64 of q [n, d] on k [L, d]; mask [n, L] or None."""
    x = torch.matmul(q, k.t().contiguous()) / math.sqrt(q.shape[-1])
    if mask is not None:
        x = x.masked_fill(~mask, -math.inf)
    return torch.softmax(x, dim=-1), torch.logsumexp(x, dim=-1)


def _exact_rows(case, s):
    """Ops score and step: every query row adds its weights to its head's keys."""
    hq, hkv = case["hq"], case["hkv"]
    G = hq // hkv
    out = s["score_in"].double().clone()
    cu = [int(c) for c in s["cu_host"]]
    for b in range(len(cu) - 1):
        c0, c1 = cu[b], cu[b + 1]
        if case["op"] == "step":
            if float(s["gate"][b]) > 0.5:
                for h in range(hq):
                    wt, _ = _softmax64(s["q"][b:b + 1, h].double(),
                                       s["k"][c0:c1, h // G].double(), None)
                    out[h // G, c0:c1] += wt[0]
            continue
        r_end = int(s["cu_sel_host"][b + 1])
        for r0 in range(int(s["cu_sel_host"][b]), r_end, 1024):
            r1 = min(r_end, r0 + 1024)
            tok = s["sel_idx"][r0:r1].long()
            mask = torch.arange(c0, c1, device="cuda")[None, :] <= tok[:, None]
            for h in range(hq):
                wt, z = _softmax64(s["q"][tok, h].double(), s["k"][c0:c1, h // G].double(), mask)
                if s["lse"] is not None:
                    # the weights that the given log-sum-exp stands for
                    wt = wt * torch.exp(z - s["lse"][h, r0:r1].double() * math.log(2.0))[:, None]
                out[h // G, c0:c1] += wt.sum(0)
    return out


def _exact_prefix(case, s):
    hq, hkv, d, w = case["hq"], case["hkv"], case["d"], case["window"]
    G, kw = hq // hkv, s["kw"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    cu, cp, cg = ([int(c) for c in s[n]] for n in ("cu_host", "cu_pre_host", "cu_group_host"))

    def branch(b, r, suffix, count, gain):
        tensor = {n: kw.get(n + "_g") if suffix and case["distinct"] else s[n]
                  for n in ("q", "k", "v", "k_pre", "v_pre")}
        k = torch.cat([tensor["k_pre"][cp[r]:cp[r + 1]], tensor["k"][cu[b]:cu[b + 1]]])
        v = torch.cat([tensor["v_pre"][cp[r]:cp[r + 1]], tensor["v"][cu[b]:cu[b + 1]]])
        first = max(0, k.shape[0] - count)
        res = []
        for h in range(hkv):
            wt, _ = _softmax64(tensor["q"][b, h * G:(h + 1) * G].double(), k[first:, h].double(),
                               None)
            res.append(torch.matmul(wt, v[first:, h].double()))
        o = torch.cat(res)
        o = o / torch.sqrt(o.pow(2).sum(-1, keepdim=True) / d + EPS)
        return o if gain is None else o * gain.double()

    for r in range(len(cp) - 1):
        for b in range(cg[r], cg[r + 1]):
            p = float(s["gate"][b])
            o = branch(b, r, False, w, kw.get("gain_local"))
            if p > 0.5:
                o = (1.0 - p) * o + p * branch(b, r, True, 1 << 40, kw.get("gain_global"))
            out[b] = o
    return out


def _exact_evict(case, s):
    score, cu = s["score"].double().cpu().numpy(), s["cu_host"]
    idx, lens = [[] for _ in range(case["hkv"])], []
    for b in range(len(cu) - 1):
        L = int(cu[b + 1] - cu[b])
        n = min(L, case["budget"])
        rec = min(case["recent"], n)
        lens.append(n)
        for h in range(case["hkv"]):
            x = score[h, cu[b]:cu[b] + L - rec]
            best = np.lexsort((np.arange(L - rec), -x))[:n - rec]
            kept = np.zeros(L, bool)
            kept[best] = True
            kept[L - rec:] = True
            idx[h].append(np.nonzero(kept)[0] + int(cu[b]))
    idx = torch.from_numpy(np.stack([np.concatenate(x) for x in idx])).cuda()
    k = torch.stack([s["k"][idx[h], h] for h in range(case["hkv"])], 1)
    v = torch.stack([s["v"][idx[h], h] for h in range(case["hkv"])], 1)
    sc = torch.stack([s["score"][h, idx[h]] for h in range(case["hkv"])])
    return dict(k_out=k.double(), v_out=v.double(), score_out=sc.double(),
                keep_idx=idx.to(torch.int32), cu_keep=torch.from_numpy(_cu(lens)).cuda())


def exact(case, seed):
    global own
    kept, own = own, False                     # (the inputs alone)
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["op"] == "prefix":
        return _exact_prefix(case, s)
    if case["op"] == "evict":
        return _exact_evict(case, s)
    return _exact_rows(case, s)
