"""Beam search and the attention of sequences that share a prefix, as cases that can be timed.

Four operators of ``paper_2608_20530_gb300``:

``select``   the n best continuations of each request over its beams and the vocabulary, from logits
             (``beam_select``);
``merge``    the same from candidate lists that the program already has (``beam_merge``): the lists
             of ``topk_lse``, ``lm_head_topk`` or merged vocabulary shards;
``reorder``  the beams' caches moved, in place, to the beams that continue them (``beam_reorder``);
``attention`` the attention of sequences (beams, or drafted blocks under verification) that share
             their request's prefix and have a short cache of their own (``prefix_attention``).

With ``own`` false each is computed in its plain form, by elementary operations in 32 bits, or in 64
where totals of different beams are compared.
"""
import math

import numpy as np
import torch

own = False

V_FULL = 151936


def _select(name, R, W, V, n, dtype="bf16", done=False, banned=0):
    return {"name": name, "kind": "select", "R": R, "W": W, "V": V, "n": n, "dtype": dtype,
            "done": done, "banned": banned}


def _merge(name, R, W, K, n, done=False):
    return {"name": name, "kind": "merge", "R": R, "W": W, "K": K, "n": n, "done": done}


def _reorder(name, states, R, W, S, H, d, dtype="bf16", heads_first=False):
    return {"name": name, "kind": "reorder", "states": states, "R": R, "W": W, "S": S, "H": H,
            "d": d, "dtype": dtype, "heads_first": heads_first}


def _attention(name, G, W, T, Hq, Hkv, d, P, S, dtype="bf16", heads_first=False):
    return {"name": name, "kind": "attention", "G": G, "W": W, "T": T, "Hq": Hq, "Hkv": Hkv, "d": d,
            "P": P, "S": S, "dtype": dtype, "heads_first": heads_first}


def listed():
    return [
        # one request of four beams, twice as many continuations kept as beams: latency
        _select("select_b1", 1, 4, V_FULL, 8),
        # 32 requests of eight beams
        _select("select_b32", 32, 8, V_FULL, 16),
        # fp32 logits of an odd vocabulary, five beams, some finished, some tokens banned
        _select("select_f32_odd", 24, 5, 128257, 5, dtype="f32", done=True, banned=7),
        # the lists that the fused LM head leaves for one request's beams: latency
        _merge("merge_b1", 1, 4, 8, 8),
        # many requests with wide lists, finished beams and many equal totals
        _merge("merge_b512", 512, 16, 32, 32, done=True),
        # one request's caches of one layer, early in its answer: latency
        _reorder("reorder_b1", 2, 1, 4, 64, 8, 128),
        # two layers' caches of 32 requests of eight beams, up to 512 tokens each
        _reorder("reorder_b32", 4, 32, 8, 512, 8, 128),
        # a short prompt, four beams, small heads: latency
        _attention("attention_small", 1, 4, 1, 8, 2, 64, 200, 24),
        # a decoding step of eight requests of four beams on long prompts: the prefix's bytes
        _attention("attention_beams", 8, 4, 1, 32, 8, 128, 8192, 512),
        # four drafted blocks of 16 tokens verified for each of four requests, caches by head
        _attention("attention_verify", 4, 4, 16, 32, 8, 128, 16384, 48, heads_first=True),
        # 256 sequences behind one long instruction: the products bound it
        _attention("attention_shared", 1, 256, 1, 32, 8, 128, 12288, 256),
        # full precision, odd sizes
        _attention("attention_f32", 3, 5, 2, 8, 4, 96, 1777, 77, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["select", "merge", "reorder", "attention", "attention"])
    if kind == "select":
        W = rng.randint(1, 16)
        V = _log_int(rng, 1000, V_FULL)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 32 * 8 * V_FULL // (W * V * (2 if dtype == "f32" else 1))
        return _drop(_select("", min(_log_int(rng, 1, 128), max(1, most)), W, V,
                             min(32, rng.choice([W, 2 * W])), dtype, rng.random() < 0.4,
                             rng.choice([0, 0, rng.randint(1, 500)])))
    if kind == "merge":
        W, K = rng.randint(1, 24), rng.randint(1, 32)
        return _drop(_merge("", min(_log_int(rng, 1, 512), 512 * 16 * 32 // (W * K)), W, K,
                            rng.randint(1, min(32, W * K)), rng.random() < 0.4))
    if kind == "reorder":
        f32 = rng.random() < 0.3
        R, W, S = _log_int(rng, 1, 32), rng.randint(2, 12), _log_int(rng, 1, 600)
        H, d = rng.randint(1, 8), rng.choice([32, 64, 80, 96, 128])
        most = 4 * 32 * 8 * 512 * 1024 // (R * W * S * H * d * (2 if f32 else 1))
        return _drop(_reorder("", max(1, min(rng.randint(1, 6), most)), R, W, S, H, d,
                              "f32" if f32 else "bf16", rng.random() < 0.4))
    f32 = rng.random() < 0.25
    Hkv = rng.randint(1, 8)
    Hq = Hkv * rng.randint(1, 8 if Hkv < 5 else 4)
    d = rng.choice([32, 64, 80, 96, 128, 128])
    G, W, T = _log_int(rng, 1, 16), _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 5, 16])
    P, S = _log_int(rng, 1, 16384), _log_int(rng, T, 600)
    # no more than the largest listed case's operations (fp32 on the plain cores: 1/40 of them)
    most = 256 * 32 * 12288 * 128 // (40 if f32 else 1)
    W = max(1, min(W, most // (G * T * Hq * (P + S) * d)))
    P = max(1, min(P, most // (G * W * T * Hq * d)))
    return _drop(_attention("", G, W, T, Hq, Hkv, d, P, S, "f32" if f32 else "bf16",
                            rng.random() < 0.4))


def _drop(case):
    del case["name"]
    return case


def _type(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _spread(count, lo, hi):
    """`count` lengths spread evenly over lo..hi, in an order of their own."""
    at = (np.arange(1, count + 1) * 0.6180339887498949) % 1.0
    return (lo + np.floor(at * (hi - lo + 1))).astype(np.int32)


def _prefix_lens(case):
    return np.concatenate([[case["P"]], _spread(case["G"] - 1, max(1, case["P"] // 4), case["P"])])


def _seq_lens(case):
    N, T, S = case["G"] * case["W"], case["T"], case["S"]
    return np.concatenate([[S], _spread(N - 1, min(T, S), S)])


def _reorder_lens(case):
    return np.concatenate([[case["S"]], _spread(case["R"] - 1, max(1, case["S"] // 8), case["S"])])


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    rand = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    kind = case["kind"]
    st = {"case": dict(case), "kind": kind, "keep": {}}
    if kind in ("select", "merge"):
        R, W, n = case["R"], case["W"], case["n"]
        done = rand(R, W) < 0.3 if case["done"] else None
        st.update(n=n, done=done, end_id=2 if case["done"] else -1)
        # running log-probabilities of beams that survived: near one another, best first
        scores = -(5.0 * rand(R, 1) + torch.cumsum(0.6 * rand(R, W), 1))
        if kind == "select":
            V = case["V"]
            # rows of mixed entropy, a few likely tokens in each
            x = randn(R, W, V).mul_(1.0 + 2.0 * rand(R, W, 1))
            likely = torch.randint(0, V, (R, W, 6), generator=g, device="cuda")
            x.scatter_add_(2, likely, 10.0 * rand(R, W, 6))
            if case["banned"]:
                x[:, :, torch.randint(0, V, (case["banned"],), generator=g, device="cuda")] = -math.inf
            if done is not None:
                x[done] = math.nan                      # nobody computes a finished beam's logits
            st.update(logits=x.to(_type(case)), scores=scores)
        else:
            K = case["K"]
            # log-probabilities on a grid, so that totals meet: lists in descending order
            lp = torch.sort(-torch.round(6.0 * rand(R, W, K) * 16) / 16, dim=2, descending=True)[0]
            ids = torch.argsort(rand(R, W, 64 + K), dim=2)[:, :, :K].int().contiguous()
            st.update(ids=ids, logp=lp.contiguous(), scores=torch.round(scores * 16) / 16)
        if W > 2:
            st["scores"][:, W - 1] = torch.where(rand(R) < 0.3, -math.inf, st["scores"][:, W - 1])
        return st
    if kind == "reorder":
        R, W, S, H, d = (case[k] for k in ("R", "W", "S", "H", "d"))
        shape = (R, W, H, S, d) if case["heads_first"] else (R, W, S, H, d)
        states = [randn(*shape).to(_type(case)) for _ in range(case["states"])]
        if case["heads_first"]:
            states = [s.transpose(2, 3) for s in states]
        st.update(states=states, lengths=_ints(_reorder_lens(case)),
                  parents=torch.randint(0, W, (R, W), generator=g, device="cuda").int())
        return st
    G, W, T, Hq, Hkv, d, P, S = (case[k] for k in ("G", "W", "T", "Hq", "Hkv", "d", "P", "S"))
    N, dt = G * W, _type(case)
    prefix_len, seq_len = _ints(_prefix_lens(case)), _ints(_seq_lens(case))

    def cache(B, L, lens):
        # what lies behind a cache's last token was never written
        c = randn(B, L, Hkv, d)
        c[torch.arange(L, device="cuda")[None, :] >= lens[:, None]] = math.nan
        c = c.to(dt)
        return c.transpose(1, 2).contiguous().transpose(1, 2) if case["heads_first"] else c

    st.update(q=(1.5 * randn(N, T, Hq, d)).to(dt), prefix_len=prefix_len, seq_len=seq_len,
              prefix_k=cache(G, P, prefix_len), prefix_v=cache(G, P, prefix_len),
              k=cache(N, S, seq_len), v=cache(N, S, seq_len), scale=d ** -0.5)
    return st


# ------------------------------------------------------------------------------- plain forms
def _pick(total, tokens, st, W):
    """The n largest of total [R, W, K] (64 bits), ties to the lower position."""
    R, _, K = total.shape
    order = torch.sort(total.flatten(1), dim=1, descending=True, stable=True)
    n = st["n"]
    best, at = order[0][:, :n], order[1][:, :n]
    there = best > -math.inf
    parents = torch.where(there, torch.div(at, K, rounding_mode="floor"), -1)
    toks = torch.where(there, torch.gather(tokens.flatten(1), 1, at).long(), -1)
    over = (toks == st["end_id"]) & there if st["end_id"] >= 0 else torch.zeros_like(there)
    if st["done"] is not None:
        over = over | (torch.gather(st["done"], 1, parents.clamp(min=0)) & there)
    return toks.int(), parents.int(), best.float(), over


def _finished(total, tokens, st):
    """Finished beams offer their end token at their own score, and nothing else."""
    if st["done"] is None:
        return total, tokens
    done = st["done"][:, :, None]
    first = torch.arange(total.shape[2], device=total.device) == 0
    score = st["scores"].double()[:, :, None]
    total = torch.where(done, torch.where(first, score, -math.inf), total)
    return total, torch.where(done, st["end_id"], tokens)


def _plain_select(st):
    x, scores = st["logits"].float(), st["scores"].double()
    R, W, V = x.shape
    live = scores > -math.inf
    if st["done"] is not None:
        live = live & ~st["done"]
    x = torch.where(live[:, :, None], x, 0.0) + 0.0           # -0 counts as +0
    xd = x.double()
    m = xd.amax(2, keepdim=True)
    lse = m + torch.log(torch.exp(xd - m).sum(2, keepdim=True))
    # a row's best in the order (logit, then lower id): one whole number for both
    bits = x.view(torch.int32)
    key = ((bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32) - torch.arange(V, device=x.device)
    ids = torch.gather(torch.arange(V, device=x.device).expand(R, W, V), 2,
                       torch.topk(key, min(st["n"], V), dim=2)[1])
    total = scores[:, :, None] + (torch.gather(xd, 2, ids) - lse)
    total, ids = _finished(total, ids, st)
    return _pick(total, ids, st, W)


def _plain_merge(st):
    total = st["scores"].double()[:, :, None] + st["logp"].double()
    total, ids = _finished(total, st["ids"].long(), st)
    return _pick(total, ids, st, total.shape[1])


def _moved(s, at, live):
    view = s.transpose(2, 3) if not s.is_contiguous() else s   # as it lies in memory
    keep = live if view is s else live.transpose(2, 3)
    taken = torch.gather(view, 1, at.expand(view.shape))
    view.copy_(torch.where(keep, taken, view))
    return s


def _plain_reorder(st):
    S = st["states"][0].shape[2]
    live = (torch.arange(S, device="cuda") < st["lengths"][:, None])[:, None, :, None, None]
    at = st["parents"].long()[:, :, None, None, None]
    return list(map(_moved, st["states"], [at] * len(st["states"]), [live] * len(st["states"])))


def _plain_attention(st):
    q = st["q"].float()
    N, T, Hq, d = q.shape
    G, P, Hkv, _ = st["prefix_k"].shape
    S, W, rep = st["k"].shape[1], N // G, Hq // Hkv
    ends = st["seq_len"][:, None] - (T - 1) + torch.arange(T, device=q.device)      # [N, T]
    seen_p = torch.arange(P, device=q.device) < st["prefix_len"][:, None]           # [G, P]
    held = torch.arange(S, device=q.device) < st["seq_len"][:, None]                # [N, S]
    seen_s = torch.arange(S, device=q.device) < ends[:, :, None]                    # [N, T, S]
    zeroed = lambda c, ok: torch.where(ok[:, :, None, None], c.float(), 0.0)  # noqa: E731
    pk, pv = zeroed(st["prefix_k"], seen_p), zeroed(st["prefix_v"], seen_p)
    k, v = zeroed(st["k"], held), zeroed(st["v"], held)
    # all rows that share a prefix's key head are one product: [G, Hkv, W * T * rep, d]
    qg = q.view(G, W * T, Hkv, rep, d).permute(0, 2, 1, 3, 4).reshape(G, Hkv, W * T * rep, d)
    sp = torch.matmul(qg, pk.permute(0, 2, 3, 1)) * st["scale"]
    sp = torch.where(seen_p[:, None, None, :], sp, -math.inf)
    qn = q.view(N, T, Hkv, rep, d).permute(0, 2, 1, 3, 4).reshape(N, Hkv, T * rep, d)
    ss = torch.matmul(qn, k.permute(0, 2, 3, 1)) * st["scale"]
    ok = seen_s[:, None, :, None, :].expand(N, 1, T, rep, S).reshape(N, 1, T * rep, S)
    ss = torch.where(ok, ss, -math.inf)
    sp = sp.view(G, Hkv, W, T * rep, P).transpose(1, 2).reshape(N, Hkv, T * rep, P)
    m = torch.maximum(sp.amax(3, keepdim=True), ss.amax(3, keepdim=True))
    base = torch.where(m > -math.inf, m, 0.0)
    ep, es = torch.exp(sp - base), torch.exp(ss - base)
    total = ep.sum(3, keepdim=True) + es.sum(3, keepdim=True)
    epg = ep.view(G, W, Hkv, T * rep, P).transpose(1, 2).reshape(G, Hkv, W * T * rep, P)
    op = torch.matmul(epg, pv.permute(0, 2, 1, 3)).view(G, Hkv, W, T * rep, d).transpose(1, 2)
    o = op.reshape(N, Hkv, T * rep, d) + torch.matmul(es, v.permute(0, 2, 1, 3))
    o = torch.where(total > 0, o / total, 0.0)
    lse = base + torch.log(total)
    o = o.view(N, Hkv, T, rep, d).transpose(1, 2).reshape(N, T, Hq, d)
    return o.to(st["q"].dtype), lse.view(N, Hkv, T, rep).transpose(1, 2).reshape(N, T, Hq)


def _own(st):
    import paper_2608_20530_gb300 as ll
    keep = st["keep"]                                # a program's workspace, made on its first call
    if st["kind"] == "select":
        if "ws" not in keep:
            R, W, V = st["logits"].shape
            keep["ws"] = ll.Workspace(ll.beam_select_workspace_bytes(R, W, V, st["n"]))
        return ll.beam_select(st["logits"], st["scores"], st["n"], done=st["done"],
                              end_id=st["end_id"], ws=keep["ws"])
    if st["kind"] == "merge":
        return ll.beam_merge(st["ids"], st["logp"], st["scores"], st["n"], done=st["done"],
                             end_id=st["end_id"])
    if st["kind"] == "reorder":
        return ll.beam_reorder(st["states"], st["parents"], st["lengths"])
    if "ws" not in keep:
        keep["ws"] = ll.Workspace(ll.prefix_attention_workspace_bytes(st["q"], st["prefix_k"], st["k"]))
    return ll.prefix_attention(st["q"], st["prefix_k"], st["prefix_v"], st["k"], st["v"],
                               st["prefix_len"], st["seq_len"], scale=st["scale"], ws=keep["ws"])


def run(state):
    if own:
        return _own(state)
    return {"select": _plain_select, "merge": _plain_merge, "reorder": _plain_reorder,
            "attention": _plain_attention}[state["kind"]](state)


# ------------------------------------------------------------------------------- work, exact values
def work(case):
    kind = case["kind"]
    if kind == "select":
        rows = case["R"] * case["W"]
        if case["done"]:
            rows *= 0.7                              # finished beams' logits are not read
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": rows * case["V"] * size + case["R"] * case["n"] * 13,
                "flops": 4 * rows * case["V"]}
    if kind == "merge":
        cand = case["R"] * case["W"] * case["K"]
        return {"bytes": 8 * cand + 4 * case["R"] * case["W"] + 13 * case["R"] * case["n"],
                "flops": 2 * cand}
    if kind == "reorder":
        W, size = case["W"], 4 if case["dtype"] == "f32" else 2
        # parents drawn alike: W - 1 beams move on average, from so many different sources
        beams = (W - 1) + W * (1 - (1 - 1 / W) ** (W - 1))
        return {"bytes": case["states"] * float(_reorder_lens(case).sum()) * case["H"] * case["d"] *
                size * beams + 4 * case["R"] * (W + 1), "flops": 0}
    G, W, T, Hq, Hkv, d = (case[k] for k in ("G", "W", "T", "Hq", "Hkv", "d"))
    size = 4 if case["dtype"] == "f32" else 2
    pl, sl = float(_prefix_lens(case).sum()), float(_seq_lens(case).sum())
    N = G * W
    return {"bytes": 2 * (pl + sl) * Hkv * d * size + N * T * Hq * (2 * d * size + 4),
            "flops": 4.0 * d * T * Hq * (W * pl + sl)}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "reorder":
        return None                                  # copies: nothing is computed
    if case["kind"] in ("select", "merge"):
        sc = st["scores"].to(torch.float64).unsqueeze(2)
        if case["kind"] == "select":
            gone = torch.isinf(sc[:, :, 0])
            if st["done"] is not None:
                gone = gone | st["done"]
            x = st["logits"].masked_fill(gone.unsqueeze(2), 0.0).to(torch.float64)
            lp = torch.log_softmax(x, dim=-1)
        else:
            lp = st["logp"].to(torch.float64)
        lp = lp + sc
        if st["done"] is not None:
            lp[st["done"]] = -math.inf
            lp[:, :, 0] = torch.where(st["done"], sc[:, :, 0], lp[:, :, 0])
        return None, None, torch.topk(lp.reshape(case["R"], -1), case["n"], dim=1)[0], None
    q, W, T, d = st["q"].to(torch.float64), case["W"], case["T"], case["d"]
    rep = case["Hq"] // case["Hkv"]
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(q.shape[:3], dtype=torch.float64, device="cuda")
    plen, slen = st["prefix_len"].tolist(), st["seq_len"].tolist()
    # request by request, sequence by sequence: only the keys that are there
    for n in range(case["G"] * W):
        gi = n // W
        kk = torch.cat([st["prefix_k"][gi, :plen[gi]], st["k"][n, :slen[n]]]).to(torch.float64)
        vv = torch.cat([st["prefix_v"][gi, :plen[gi]], st["v"][n, :slen[n]]]).to(torch.float64)
        kk, vv = kk.repeat_interleave(rep, 1), vv.repeat_interleave(rep, 1)
        s = torch.einsum("thd,jhd->htj", q[n], kk) * st["scale"]
        if T > 1:
            pos = torch.arange(plen[gi] + slen[n], device="cuda")
            last = plen[gi] + slen[n] - T + torch.arange(T, device="cuda")
            s = s.masked_fill((pos[None, :] > last[:, None]) & (pos[None, :] >= plen[gi]), -math.inf)
        lse[n] = torch.logsumexp(s, dim=2).T
        out[n] = torch.einsum("htj,jhd->thd", torch.softmax(s, dim=2), vv)
    return out, lse
