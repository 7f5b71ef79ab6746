"""Measured cases of two operators around the LM head, beside their plain forms in elementary torch operations: low-rank
adapters of many requests next to the shared projection, and log probabilities of given tokens with entropy, rank and top
alternatives.

`listed()` names the cases, `draw()` gives more of the same ranges; `prepare()` makes what a serving loop holds before a call
(inputs from a seed, the resident head and adapters, the context), `run()` is one pass, `exact()` the same outputs in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False      # False: run() computes the plain form; True: it calls the framework

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MOST_MACS = 384 * 128256 * 4096                 # the dearest listed adapter case
MOST_LOGITS = 2304 * 128256                     # the dearest listed scoring case


# ------------------------------------------------------------------------------------------------ cases
def _score(name, rows, V, dtype, tokens, n_top, rank=True, pad=0, inputs="spread", emitted_k=-1):
    """`tokens` per row; `pad`: entries from one row's end to the next; `emitted_k` >= 0: rows are the k + 1 positions of
    rows / (k + 1) sequences behind a verify call, whose logZ is at hand and whose emitted tokens are scored."""
    return {"name": name, "op": "score", "rows": rows, "V": V, "dtype": dtype, "tokens": tokens, "n_top": n_top,
            "rank": rank, "pad": pad, "inputs": inputs, "emitted_k": emitted_k}


def _adapt(name, B, k, H, V, slots, rank, active, bare, weights="bf16"):
    """`slots` resident adapters of rank `rank`, `active` of them used by the batch, `bare` sequences that use none."""
    return {"name": name, "op": "adapt", "B": B, "k": k, "H": H, "V": V, "slots": slots, "rank": rank, "active": active,
            "bare": bare, "weights": weights}


def listed():
    return [
        # one user, behind one verify round: log probabilities and five alternatives; all latency
        _score("score_one_user", 5, 32000, "f32", 1, 5),
        # a serving batch, emitted tokens of a verify call, whose logZ is there already
        _score("score_emitted", 384, 32000, "f32", 1, 5, emitted_k=5),
        # a large vocabulary, the most alternatives that serving interfaces hand out
        _score("score_large_vocab", 384, 128256, "f32", 1, 20),
        # a long prompt is scored: token, rank and entropy, no alternatives, 16-bit logits
        _score("score_prompt", 2304, 128256, "bf16", 1, 0),
        # odd sizes, rows of a padded buffer that start on no 16-byte boundary, several tokens asked per row
        _score("score_ragged", 69, 50003, "f16", 3, 10, pad=6),
        # constrained decoding: most entries masked to -inf, in some rows fewer left than alternatives asked for
        _score("score_constrained", 192, 32000, "bf16", 1, 8, inputs="masked"),
        # one user with one adapter on a 7B-class head
        _adapt("adapt_one_user", 1, 4, 4096, 32000, 4, 16, 1, 0),
        # a full serving batch, sixteen adapters, a quarter of the users on the bare model
        _adapt("adapt_batched", 64, 5, 4096, 32000, 16, 16, 16, 16),
        # large vocabulary, every sequence its own adapter: the dearest
        _adapt("adapt_large_vocab", 64, 5, 4096, 128256, 64, 16, 64, 0),
        # plain decoding, one token per sequence, higher rank
        _adapt("adapt_single_tokens", 32, 0, 4096, 128256, 32, 32, 16, 4),
        # odd sizes: ragged last K block, a vocabulary that is no multiple of 4, a rank that is no power of two
        _adapt("adapt_ragged", 23, 3, 1032, 50003, 8, 24, 5, 3),
        # the 8-bit head of the quantiser with small adapters beside it
        _adapt("adapt_int8_head", 16, 5, 4096, 32000, 8, 8, 8, 0, weights="int8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        while True:
            k = rng.randint(0, 8) if rng.random() < 0.3 else -1
            rows = _log_int(rng, 1, 2304)
            if k >= 0:
                rows = max(1, rows // (k + 1)) * (k + 1)
            V = _log_int(rng, 1000, 128256)
            n_top = 0 if rng.random() < 0.25 else _log_int(rng, 1, 32)
            # (the plain form sorts rows for their alternatives)
            if rows * V <= (MOST_LOGITS if n_top == 0 else 384 * 128256):
                break
        c = _score("", rows, V, rng.choice(["f32", "f32", "bf16", "f16"]), 1 if k >= 0 else rng.randint(1, 4), n_top,
                   rank=rng.random() < 0.75, pad=rng.choice([0, 0, 1, 6, 64]), inputs=rng.choice(["spread", "spread", "masked"]),
                   emitted_k=k)
    else:
        weights = rng.choice(["bf16", "bf16", "bf16", "int8"])
        step = 16 if weights == "int8" else 8
        while True:
            B, k, V = _log_int(rng, 1, 256), rng.randint(0, 8), _log_int(rng, 1000, 128256)
            H = max(step, _log_int(rng, 64, 8192) // step * step)
            if B * (k + 1) * V * H <= MOST_MACS:
                break
        slots = _log_int(rng, 1, 64)
        bare = rng.choice([0, 0, B // 4])
        active = rng.randint(1, max(1, min(slots, B - bare)))
        c = _adapt("", B, k, H, V, slots, rng.choice([8, 16, 16, 24, 32, 64]), active, bare, weights)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _score_inputs(case, seed):
    rows, V, T, k = case["rows"], case["V"], case["tokens"], case["emitted_k"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    pitch = V + case["pad"]
    # logits of a trained head: a spread of its own for each row, from flat to peaked
    spread = torch.exp(torch.empty((rows, 1), device="cuda").uniform_(math.log(0.7), math.log(4.0), generator=g))
    full = torch.empty((rows, pitch), dtype=DTYPES[case["dtype"]], device="cuda")
    step = max(1, (1 << 27) // pitch)
    sampled = torch.empty((rows, T), dtype=torch.int64, device="cuda")
    for r0 in range(0, rows, step):
        l = torch.randn((min(step, rows - r0), pitch), generator=g, device="cuda") * spread[r0:r0 + step]
        if case["inputs"] == "masked":
            share = torch.exp(torch.empty((l.shape[0], 1), device="cuda").uniform_(math.log(2.0 / V), 0.0, generator=g))
            keep = torch.rand(l.shape, generator=g, device="cuda") < share
            at = torch.randint(0, V, (l.shape[0], 1), generator=g, device="cuda")
            keep.scatter_(1, at, True)                                   # (something is always allowed)
            l = torch.where(keep, l, -math.inf)
        l = l.to(full.dtype)
        full[r0:r0 + step] = l
        # tokens drawn from the softmax (the largest of logits + Gumbel noise), further ones anywhere
        noise = -torch.log(-torch.log(torch.rand((l.shape[0], V), generator=g, device="cuda").clamp(1e-20, 1 - 1e-7)))
        sampled[r0:r0 + step] = torch.randint(0, V, (l.shape[0], T), generator=g, device="cuda")
        sampled[r0:r0 + step, 0] = (l[:, :V].float() + noise).argmax(dim=1)
    logits = full[:, :V]
    s = {"logits": logits, "tokens": sampled.to(torch.int32)}
    if k >= 0:
        B = rows // (k + 1)
        s["accept_len"] = torch.randint(0, k + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        by_row = s.pop("tokens")[:, 0].reshape(B, k + 1)
        s["draft_tok"] = by_row[:, :k].contiguous()
        s["next_tok"] = by_row.gather(1, s["accept_len"].long()[:, None])[:, 0].contiguous()
        s["logits"] = full.reshape(B, k + 1, pitch)[:, :, :V]
        s["logZ"] = torch.stack([torch.logsumexp(logits[r].double(), 0) for r in range(rows)]).float().reshape(B, k + 1)
    return s


def _adapt_inputs(case, seed):
    B, k, H, V, S, R = (case[n] for n in ("B", "k", "H", "V", "slots", "rank"))
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std):
        out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        for part in out.view(-1, shape[-1]).split(max(1, (1 << 26) // shape[-1])):
            part.copy_(torch.randn(part.shape, generator=g, device="cuda") * std)
        return out

    s = {"hidden": normal((B, k + 1, H), 1.0)}
    W = normal((V, H), 1.28 / math.sqrt(H))                 # logits with the spread of a trained head
    if case["weights"] == "int8":
        # one scale per vocabulary row, ties to even
        scale = W.float().abs().amax(dim=1) / 127.0
        s["W"] = torch.round(W.float() / scale[:, None]).clamp(-127, 127).to(torch.int8)
        s["w_scale"] = scale
    else:
        s["W"], s["w_scale"] = W, None
    # an update of about a quarter of the head's own logits
    s["A"] = normal((S, R, H), 1.0 / math.sqrt(H))
    s["Bup"] = normal((S, V, R), 0.32 / math.sqrt(R))
    s["scale"] = torch.empty((S,), device="cuda").uniform_(0.5, 2.0, generator=g)
    used = torch.randperm(S, generator=g, device="cuda")[:case["active"]]
    ids = torch.full((B,), -1, dtype=torch.int64, device="cuda")
    who = torch.randperm(B, generator=g, device="cuda")[case["bare"]:]
    ids[who] = used[torch.arange(who.numel(), device="cuda") % case["active"]]
    s["ids"] = ids.to(torch.int32)
    return s


def prepare(case, seed):
    s = (_score_inputs if case["op"] == "score" else _adapt_inputs)(case, seed)
    s["case"] = case
    if own:
        from paper_2506_18952_b200 import binding
        s["binding"] = binding
        if case["op"] == "adapt":
            s["ctx"] = binding.HolaVerify(case["B"], case["k"], case["H"], case["V"])
            s["bank"] = binding.AdapterBank(s.pop("A"), s.pop("Bup"), s.pop("scale"))
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _emitted_tokens(s):
    """[rows, 1] tokens of the rows of a verify call, -1 behind the last one that it emitted."""
    draft, n = s["draft_tok"], s["accept_len"]
    B, k = draft.shape
    at = torch.arange(k + 1, device=draft.device)[None, :]
    tok = torch.cat([draft, s["next_tok"][:, None]], dim=1)
    tok = torch.where(at == n[:, None], s["next_tok"][:, None], tok)
    return torch.where(at <= n[:, None], tok, -1).reshape(-1, 1)


def _score_plain(s):
    case = s["case"]
    V, n_top = case["V"], case["n_top"]
    l = s["logits"].reshape(-1, V).float()
    got = {}
    if "logZ" in s:
        tok, logZ = _emitted_tokens(s), s["logZ"].reshape(-1)
    else:
        tok = s["tokens"]
        d = (l - l.amax(dim=1, keepdim=True)).clamp_min_(-1e30)
        e = torch.exp(d)
        z = e.sum(dim=1)
        got["entropy"] = torch.log(z) - (e * d).sum(dim=1) / z
        logZ = got["logZ"] = l.amax(dim=1) + torch.log(z)
        del d, e
    have = tok >= 0
    lx = l.gather(1, tok.long().clamp_min(0))
    got["logprob"] = torch.where(have, lx - logZ[:, None], 0.0)
    if case["rank"]:
        ids = torch.arange(V, device=l.device)
        ranks = [((l > lx[:, j:j + 1]) | ((l == lx[:, j:j + 1]) & (ids < tok[:, j:j + 1]))).sum(dim=1) for j in range(tok.shape[1])]
        got["rank"] = torch.where(have, torch.stack(ranks, dim=1).int(), -1)
    if n_top:
        v, i = torch.sort(l, dim=1, descending=True, stable=True)
        seen = have if "logZ" in s else torch.ones_like(have[:, :1])
        got["top_ids"] = torch.where(seen, i[:, :n_top].int(), -1)
        got["top_logprobs"] = torch.where(seen, v[:, :n_top] - logZ[:, None], 0.0)
    shape = s["logits"].shape[:-1]
    return {n: t.reshape(*shape, *t.shape[1:]) if "logZ" not in s or n.startswith("top") else t.reshape(shape) for n, t in got.items()}


def _score_own(s):
    case = s["case"]
    emitted = (s["draft_tok"], s["accept_len"], s["next_tok"]) if "logZ" in s else None
    out = s["binding"].hola_token_logprobs(s["logits"], s.get("tokens"), n_top=case["n_top"], logZ=s.get("logZ"), emitted=emitted,
                                           want_rank=case["rank"])
    got = {"logprob": out.logprob}
    if emitted is None:
        got.update(entropy=out.entropy, logZ=out.logZ)
    if case["rank"]:
        got["rank"] = out.rank
    if case["n_top"]:
        got.update(top_ids=out.top_ids, top_logprobs=out.top_logprobs)
    return got


def _adapt_plain(s):
    case = s["case"]
    B, k, H, V = (case[n] for n in ("B", "k", "H", "V"))
    x = s["hidden"].float()
    W = s["W"].float()
    if s["w_scale"] is not None:
        W = W * s["w_scale"][:, None]
    l = (x.reshape(-1, H) @ W.T).reshape(B, k + 1, V)
    of = s["ids"].long().clamp_min(0)
    u = torch.bmm(x, s["A"][of].float().transpose(1, 2)) * torch.where(s["ids"] >= 0, s["scale"][of], 0.0)[:, None, None]
    l += torch.bmm(u, s["Bup"][of].float().transpose(1, 2))
    m = l.amax(dim=2, keepdim=True)
    d = l - m
    e = torch.exp(d)
    z = e.sum(dim=2)
    return {"logits": l, "logZ": m[..., 0] + torch.log(z), "entropy": torch.log(z) - (e * d).sum(dim=2) / z}


def _adapt_own(s):
    out = s["ctx"].hola_lm_head_adapters(s["hidden"], s["W"], s["bank"], s["ids"], want_logits=True, w_scale=s["w_scale"])
    return {"logits": out.logits, "logZ": out.logZ, "entropy": out.entropy}


def run(state):
    if state["case"]["op"] == "score":
        return _score_own(state) if own else _score_plain(state)
    return _adapt_own(state) if own else _adapt_plain(state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "score":
        rows, V, k = case["rows"], case["V"], case["emitted_k"]
        size = 4 if case["dtype"] == "f32" else 2
        read = rows if k < 0 else rows // (k + 1) * (k / 2 + 1)           # rows that hold a token
        passes = k < 0 or case["n_top"] > 0 or case["rank"]               # (else the tokens' own entries alone)
        n = read * V * size if passes else read * size
        n += rows * (case["tokens"] * (8 + 4 * case["rank"]) + 8 * case["n_top"] + 8)
        return {"bytes": n, "flops": 5 * read * V if k < 0 else 0}
    B, k, H, V, R = (case[n] for n in ("B", "k", "H", "V", "rank"))
    M = B * (k + 1)
    used = min(case["active"], B - case["bare"])
    adapted = (B - case["bare"]) * (k + 1)
    n = V * H * (1 if case["weights"] == "int8" else 2) + (V * 4 if case["weights"] == "int8" else 0)
    n += M * H * 2 + M * V * 4 + M * 8 + B * 4 + used * R * (H + V) * 2
    return {"bytes": n, "flops": 2 * M * V * H + 2 * adapted * R * (H + V)}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _score_exact(case, s):
    """Row by row in blocks: every entry gets a whole number that orders it (the logit first, then the id)."""
    V, n_top, k = case["V"], case["n_top"], case["emitted_k"]
    rows, T = case["rows"], case["tokens"]
    logits = s["logits"].reshape(rows, V)
    if k >= 0:
        B = rows // (k + 1)
        tok = torch.full((B, k + 1), -1, dtype=torch.int64, device=logits.device)
        for b, n in enumerate(s["accept_len"].tolist()):
            tok[b, :n] = s["draft_tok"][b, :n].long()
            tok[b, n] = s["next_tok"][b].long()
        tok = tok.reshape(rows, 1)
    else:
        tok = s["tokens"].long()
    parts = []
    for r0 in range(0, rows, 128):
        x = logits[r0:r0 + 128].double()
        t = tok[r0:r0 + 128]
        absent = t < 0
        t = t.clamp_min(0)
        bits = (logits[r0:r0 + 128].float() + 0.0).view(torch.int32).long()              # (+ 0.0: one zero only)
        bits = torch.where(bits < 0, -1 - (bits & 0x7fffffff), bits)
        order = (bits << 20) - torch.arange(V, device=x.device)[None, :]
        p = {}
        if k >= 0:
            logZ = s["logZ"].reshape(-1)[r0:r0 + 128].double()
        else:
            p["logZ"] = logZ = torch.logsumexp(x, dim=1)
            lp = x - logZ[:, None]
            p["entropy"] = -torch.where(lp > -math.inf, torch.exp(lp) * lp, 0.0).sum(dim=1)
        p["logprob"] = torch.where(absent, 0.0, x.gather(1, t) - logZ[:, None])
        if case["rank"]:
            mine = order.gather(1, t)
            rank = torch.stack([(order > mine[:, j:j + 1]).sum(dim=1) for j in range(T)], dim=1)
            p["rank"] = torch.where(absent, -1, rank).int()
        if n_top:
            at = torch.topk(order, n_top, dim=1).indices
            gone = absent if k >= 0 else torch.zeros_like(absent[:, :1])
            p["top_ids"] = torch.where(gone, -1, at).int()
            p["top_logprobs"] = torch.where(gone, 0.0, x.gather(1, at) - logZ[:, None])
        parts.append(p)
    got = {n: torch.cat([p[n] for p in parts]) for n in parts[0]}
    if k >= 0:
        got = {n: t.reshape(B, k + 1, -1) if n.startswith("top") else t.reshape(B, k + 1) for n, t in got.items()}
    return got


def _adapt_exact(case, s):
    """The adapted heads one vocabulary block at a time: W + scale * B A for each adapter that is used."""
    B, k, H, V = (case[n] for n in ("B", "k", "H", "V"))
    x = s["hidden"].double()
    ids = s["ids"].long()
    l = torch.empty((B, k + 1, V), dtype=torch.float64, device=x.device)
    low = {a: s["scale"][a].double() * torch.matmul(x[ids == a], s["A"][a].double().T) for a in set(ids.tolist()) if a >= 0}
    for v0 in range(0, V, 8192):
        W = s["W"][v0:v0 + 8192].double()
        if s["w_scale"] is not None:
            W = W * s["w_scale"][v0:v0 + 8192, None].double()
        block = torch.matmul(x, W.T)
        for a, u in low.items():
            block[ids == a] += torch.matmul(u, s["Bup"][a, v0:v0 + 8192].double().T)
        l[:, :, v0:v0 + 8192] = block
    logZ = torch.logsumexp(l, dim=2)
    lp = l - logZ[..., None]
    return {"logits": l, "logZ": logZ, "entropy": -(torch.exp(lp) * lp).sum(dim=2)}


def exact(case, seed):
    if case["op"] == "score":
        return _score_exact(case, _score_inputs(case, seed))
    return _adapt_exact(case, _adapt_inputs(case, seed))
