"""Measured cases of the operators around the LM head that a decoder with beams and a learning draft table need, beside their plain
forms in elementary torch operations: the selection over beams and vocabulary, the reordering of the beams' states, the lookup of
token embeddings in any stored form of a table, and the gradient of a table by sorted tokens.

`listed()` names the cases, `draw()` gives more of the same ranges; `prepare()` makes what a decoding or training loop holds before a
call (inputs from a seed, resident tables and states), `run()` is one pass, `exact()` the same outputs in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False      # False: run() computes the plain form; True: it calls the framework

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32, "i64": torch.int64}
SIZES = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8, "int8": 1}
MOST_LOGITS = 64 * 6 * 128256                   # the dearest listed selection
MOST_MOVED = 1 << 30                            # bytes of the state that a drawn reordering holds at most
MOST_ROWS = 32768 * 4096                        # the dearest listed gradient


# ------------------------------------------------------------------------------------------------ cases
def _select(name, B, W, V, n, dtype, pad=0, inputs="spread", finished=0.0, weight=False, keep=False, first=False):
    """B sequences of W beams; `n` candidates are kept; `finished`: share of ended beams; `weight`: length-normalised keys; `keep`:
    children of a surviving beam stay in its slot; `first`: one beam of each sequence is alive, as behind a prompt."""
    return {"name": name, "op": "select", "B": B, "W": W, "V": V, "n": n, "dtype": dtype, "pad": pad, "inputs": inputs,
            "finished": finished, "weight": weight, "keep": keep, "first": first}


def _reorder(name, B, W, kind, form, survivors, steps, layers=1, heads=1, width=1, dtype="f32"):
    """`kind` "rows": a history of `steps` tokens, a vector of `width` per beam, a table of steps / 16 pages; "cache": keys and values
    of `layers` x `heads`, `steps` positions of `width` each, of which a sequence has filled some.  `form`: "inplace" (children in
    their parents' slots) or "copy" (from one buffer into another, parents in any order)."""
    return {"name": name, "op": "reorder", "B": B, "W": W, "kind": kind, "form": form, "survivors": survivors, "steps": steps,
            "layers": layers, "heads": heads, "width": width, "dtype": dtype}


def _embed(name, N, V, H, table, out, ids, tokens="zipf", scale=1.0, add=False, absent=0.0):
    """`absent`: share of places that hold no token (-1), as in a padded batch."""
    return {"name": name, "op": "embed", "N": N, "V": V, "H": H, "table": table, "out": out, "ids": ids, "tokens": tokens,
            "scale": scale, "add": add, "absent": absent}


def _grad(name, N, V, H, grad, form, ids, tokens="zipf", scale=1.0, out="f32", absent=0.0):
    """`form` "rows": the distinct tokens and their rows; "dense": the gradient of the whole table."""
    return {"name": name, "op": "grad", "N": N, "V": V, "H": H, "grad": grad, "form": form, "ids": ids, "tokens": tokens,
            "scale": scale, "out": out, "absent": absent}


def listed():
    return [
        # one user, four beams, one step: all latency
        _select("select_one_user", 1, 4, 32000, 4, "f32", keep=True),
        # a serving batch behind the LM head; twice the beams are kept, so that ended ones can be set aside by the caller
        _select("select_batch", 64, 6, 32000, 12, "f32"),
        # large vocabulary, ended beams compete with length-normalised keys
        _select("select_large_vocab", 64, 6, 128256, 6, "f32", finished=0.15, weight=True, keep=True),
        # constrained decoding: most entries masked, 16-bit logits, odd sizes, rows on no 16-byte boundary
        _select("select_constrained", 23, 3, 50003, 6, "f16", pad=6, inputs="masked"),
        # token history, trunk state and page table of one user, into the other of two buffers
        _reorder("reorder_one_user", 1, 4, "rows", "copy", 3, 512, width=4096),
        # keys and values of a serving batch, in place: half of the beams die in a step
        _reorder("reorder_cache", 16, 4, "cache", "inplace", 2, 1024, layers=8, heads=8, width=128, dtype="bf16"),
        # the tokens of one verify round
        _embed("embed_round", 5, 32000, 4096, "bf16", "bf16", "i32", tokens="uniform"),
        # prompts of a serving batch, padded; embeddings scaled by the root of the width
        _embed("embed_prompts", 16384, 128256, 4096, "bf16", "bf16", "i64", scale=64.0, absent=0.1),
        # the head's own 8-bit form serves as the table (tied weights); added to what is there
        _embed("embed_tied_int8", 2304, 32000, 4096, "int8", "f32", "i32", add=True),
        # distillation of a draft's table in a serving loop: one round's positions, distinct tokens only
        _grad("grad_round", 320, 32000, 4096, "f32", "rows", "i32"),
        # a training batch over a large vocabulary; frequent tokens occur thousands of times
        _grad("grad_batch_rows", 32768, 128256, 4096, "bf16", "rows", "i64"),
        # the whole table's gradient, as an optimiser without sparse updates wants it
        _grad("grad_batch_dense", 8192, 32000, 4096, "bf16", "dense", "i32", scale=64.0, absent=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["select", "reorder", "embed", "grad"])
    if op == "select":
        while True:
            B, W, V = _log_int(rng, 1, 256), rng.choice([1, 2, 3, 4, 4, 5, 6, 8, 8, 12, 16, 32]), _log_int(rng, 1000, 128256)
            if B * W * V <= MOST_LOGITS:
                break
        keep = rng.random() < 0.4
        n = W if keep else rng.choice([W, min(2 * W, 32), rng.randint(1, 32)])
        c = _select("", B, W, V, n, rng.choice(["f32", "f32", "bf16", "f16"]), rng.choice([0, 0, 1, 6, 64]),
                    rng.choice(["spread", "spread", "masked"]), rng.choice([0.0, 0.0, 0.2]), rng.random() < 0.3, keep,
                    rng.random() < 0.2)
    elif op == "reorder":
        W = rng.choice([2, 3, 4, 4, 5, 6, 8, 12, 16, 32])
        if rng.random() < 0.5:
            c = _reorder("", _log_int(rng, 1, 256), W, "rows", rng.choice(["copy", "inplace"]), rng.randint(1, W),
                         _log_int(rng, 16, 4096), width=_log_int(rng, 64, 8192), dtype=rng.choice(["f32", "bf16"]))
        else:
            while True:
                B, layers, heads, steps = _log_int(rng, 1, 64), _log_int(rng, 1, 32), rng.choice([1, 2, 8]), _log_int(rng, 16, 8192)
                width = rng.choice([64, 80, 128])
                if 2 * B * W * layers * heads * steps * width * 2 <= MOST_MOVED:
                    break
            c = _reorder("", B, W, "cache", rng.choice(["copy", "inplace"]), rng.randint(1, W), steps, layers, heads, width,
                         rng.choice(["bf16", "f16"]))
    else:
        while True:
            N, V, H = _log_int(rng, 1, 65536), _log_int(rng, 1000, 128256), _log_int(rng, 64, 8192)
            H = H if rng.random() < 0.2 else max(8, H // 8 * 8)
            if N * H <= MOST_ROWS and V * H <= 128256 * 4096:
                break
        ids, tokens, absent = rng.choice(["i32", "i64"]), rng.choice(["zipf", "zipf", "uniform"]), rng.choice([0.0, 0.0, 0.1])
        scale = rng.choice([1.0, 1.0, round(math.sqrt(H), 3)])
        if op == "embed":
            table = rng.choice(["f32", "bf16", "bf16", "f16", "int8"])
            c = _embed("", N, V, H, table, rng.choice(["f32", "bf16", table if table != "int8" else "bf16"]), ids, tokens, scale,
                       rng.random() < 0.3, absent)
        else:
            form = "dense" if V * H <= 32000 * 4096 and rng.random() < 0.4 else "rows"
            c = _grad("", N, V, H, rng.choice(["f32", "bf16", "bf16", "f16"]), form, ids, tokens, scale,
                      rng.choice(["f32", "f32", "bf16"]), absent)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _select_inputs(case, seed):
    B, W, V = case["B"], case["W"], case["V"]
    g = _generator(seed)
    rows, pitch = B * W, V + case["pad"]
    full = torch.empty((rows, pitch), dtype=DTYPES[case["dtype"]], device="cuda")
    logZ = torch.empty((rows,), device="cuda")
    # a spread of its own for each row, from flat to peaked
    spread = torch.exp(torch.empty((rows, 1), device="cuda").uniform_(math.log(0.7), math.log(4.0), generator=g))
    step = max(1, (1 << 27) // pitch)
    for r0 in range(0, rows, step):
        l = torch.randn((min(step, rows - r0), pitch), generator=g, device="cuda") * spread[r0:r0 + step]
        if case["inputs"] == "masked":
            share = torch.exp(torch.empty((l.shape[0], 1), device="cuda").uniform_(math.log(2.0 / V), 0.0, generator=g))
            keep = torch.rand(l.shape, generator=g, device="cuda") < share
            keep.scatter_(1, torch.randint(0, V, (l.shape[0], 1), generator=g, device="cuda"), True)
            l = torch.where(keep, l, -math.inf)
        l = l.to(full.dtype)
        full[r0:r0 + step] = l
        for r in range(0, l.shape[0], 64):
            logZ[r0 + r:r0 + r + 64] = torch.logsumexp(l[r:r + 64, :V].double(), dim=1).float()
    # beams that compete: within a few nats of each other after some tens of steps
    score = -20.0 - 30.0 * torch.rand((B, 1), generator=g, device="cuda") - torch.rand((B, W), generator=g, device="cuda") * 4.0
    if case["first"]:
        score[:, 1:] = -math.inf
    s = {"logits": full.view(B, W, pitch)[:, :, :V], "logZ": logZ.view(B, W), "score": score.contiguous(), "finished": None, "weight": None}
    if case["finished"] > 0:
        s["finished"] = torch.rand((B, W), generator=g, device="cuda") < case["finished"]
    if case["weight"]:
        # 1 / length ^ 0.6; ended beams are shorter
        length = torch.randint(20, 60, (B, 1), generator=g, device="cuda").expand(B, W).float()
        if s["finished"] is not None:
            length = torch.where(s["finished"], (length - torch.randint(0, 15, (B, W), generator=g, device="cuda")), length)
        s["weight"] = (length ** -0.6).contiguous()
    return s


def _parents(case, g):
    """int32 [B, W]: `survivors` beams have children, the others have none.  In place: every survivor's first child is in its slot."""
    B, W, n = case["B"], case["W"], case["survivors"]
    order = torch.argsort(torch.rand((B, W), generator=g, device="cuda"), dim=1)      # the survivors come first
    child = torch.arange(W, device="cuda") % n
    parent = torch.empty((B, W), dtype=torch.int64, device="cuda")
    slots = order if case["form"] == "inplace" else torch.argsort(torch.rand((B, W), generator=g, device="cuda"), dim=1)
    parent.scatter_(1, slots, order[:, child])
    return parent.to(torch.int32)


def _used(case, g):
    """int32 [B]: positions filled, evenly spread over the upper half of the steps, dealt out by chance."""
    T, B = case["steps"], case["B"]
    n = T // 2 + (T - T // 2) * torch.arange(1, B + 1, device="cuda") // B
    return n[torch.randperm(B, generator=g, device="cuda")].to(torch.int32)


def _reorder_inputs(case, seed):
    B, W, T, D = case["B"], case["W"], case["steps"], case["width"]
    g = _generator(seed)
    t = DTYPES[case["dtype"]]
    if case["kind"] == "rows":
        states = [torch.randint(0, 128000, (B, W, T), generator=g, device="cuda"), torch.randn((B, W, D), generator=g, device="cuda").to(t),
                  torch.randint(0, 1 << 20, (B, W, -(-T // 16)), generator=g, device="cuda", dtype=torch.int32)]
        axes, positions = [0, 0, 0], [2, None, None]
    else:
        shape = (case["layers"], B, W, case["heads"], T, D)
        states = [torch.empty(shape, dtype=t, device="cuda").normal_(generator=g) for _ in range(2)]
        axes, positions = [1, 1], [4, 4]
    s = {"states": states, "axes": axes, "positions": positions, "parent": _parents(case, g), "used": _used(case, g)}
    s["into"] = [torch.zeros_like(x) for x in states] if case["form"] == "copy" else states
    return s


def _tokens(case, g):
    """Token ids by falling frequency, p(id) about 1 / (id + 1) ("zipf"), or all alike; -1 where there is none."""
    N, V = case["N"], case["V"]
    u = torch.rand((N,), generator=g, device="cuda", dtype=torch.float64)
    t = torch.exp(u * math.log(V + 1.0)) - 1.0 if case["tokens"] == "zipf" else u * V
    t = t.long().clamp_(0, V - 1)
    if case["absent"] > 0:
        t = torch.where(torch.rand((N,), generator=g, device="cuda") < case["absent"], -1, t)
    return t.to(DTYPES[case["ids"]])


def _normal(shape, dtype, g, std=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for part in out.view(-1, shape[-1]).split(max(1, (1 << 26) // shape[-1])):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * std)
    return out


def _embed_inputs(case, seed):
    N, V, H = case["N"], case["V"], case["H"]
    g = _generator(seed)
    s = {"tokens": _tokens(case, g), "w_scale": None, "add": None}
    if case["table"] == "int8":
        s["table"] = torch.randint(-127, 128, (V, H), generator=g, device="cuda", dtype=torch.int8)
        s["w_scale"] = torch.empty((V,), device="cuda").uniform_(0.01, 0.03, generator=g)
    else:
        s["table"] = _normal((V, H), DTYPES[case["table"]], g)
    if case["add"]:
        s["add"] = _normal((N, H), DTYPES[case["out"]], g)
    return s


def _grad_inputs(case, seed):
    g = _generator(seed)
    return {"tokens": _tokens(case, g), "grad": _normal((case["N"], case["H"]), DTYPES[case["grad"]], g)}


INPUTS = {"select": _select_inputs, "reorder": _reorder_inputs, "embed": _embed_inputs, "grad": _grad_inputs}
END = 2                                          # the token that ends a text


def prepare(case, seed):
    s = INPUTS[case["op"]](case, seed)
    s["case"] = case
    if case["op"] == "grad" and case["form"] == "rows":
        # buffers of a loop: as many rows as there are tokens, what lies behind the distinct ones is not touched
        s["ids"] = torch.full((case["N"],), -1, dtype=torch.int32, device="cuda")
        s["rows"] = torch.zeros((case["N"], case["H"]), dtype=DTYPES[case["out"]], device="cuda")
        s["count"] = torch.zeros((1,), dtype=torch.int32, device="cuda")
    if own:
        from paper_2506_18952_b200 import binding
        s["binding"] = binding
        if case["op"] == "reorder":
            s["handle"] = binding.BeamStates(s["states"], axes=s["axes"], positions=s["positions"],
                                             into=s["into"] if case["form"] == "copy" else None)
        elif case["op"] == "grad" and case["form"] == "rows":
            s["buffers"] = binding.TokenRows(s["ids"], s["rows"], s["count"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _select_plain(s):
    case = s["case"]
    B, W, V, n = (case[x] for x in ("B", "W", "V", "n"))
    few = min(n, V)
    v, i = torch.sort(s["logits"].float(), dim=2, descending=True, stable=True)
    v, token = v[:, :, :few].double(), i[:, :, :few].clone()
    del i
    c = (s["score"].double() - s["logZ"].double())[:, :, None] + v
    ended = s["finished"]
    if ended is not None:
        c = torch.where(ended[:, :, None], -math.inf, c)
        c[:, :, 0] = torch.where(ended, s["score"].double(), c[:, :, 0])
        token[:, :, 0] = torch.where(ended, END, token[:, :, 0])
    key = c if s["weight"] is None else c * s["weight"].double()[:, :, None]
    parent = torch.arange(W, device=c.device)[None, :, None].expand(B, W, few)
    c, token, parent, key = (x.reshape(B, W * few) for x in (c, token, parent, key))
    place = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :n]
    c, token, parent = (x.gather(1, place) for x in (c, token, parent))
    if c.shape[1] < n:                                          # (fewer entries than asked for)
        more = n - c.shape[1]
        c, token, parent = (torch.nn.functional.pad(x, (0, more), value=p) for x, p in ((c, -math.inf), (token, -1), (parent, -1)))
    none = c == -math.inf
    token, parent = torch.where(none, -1, token), torch.where(none, -1, parent)
    if case["keep"]:
        # the first child of a beam goes to its slot, the others fill what is free, in order
        slot = torch.full((B, n), -1, dtype=torch.int64, device=c.device)
        taken = torch.zeros((B, W), dtype=torch.bool, device=c.device)
        for j in range(n):
            p = parent[:, j:j + 1].clamp_min(0)
            stays = (parent[:, j:j + 1] >= 0) & ~taken.gather(1, p)
            slot[:, j:j + 1] = torch.where(stays, p, -1)
            taken.scatter_(1, p, taken.gather(1, p) | stays)
        free = torch.sort(taken.int(), dim=1, stable=True).indices
        waits = slot < 0
        slot = torch.where(waits, free.gather(1, (torch.cumsum(waits.int(), 1) - 1).clamp_min(0)), slot)
        c, token, parent = (torch.empty_like(x).scatter_(1, slot, x) for x in (c, token, parent))
    got = {"score": c.float(), "parent": parent.int(), "token": token.int()}
    if ended is not None:
        got["finished"] = (parent >= 0) & (ended.gather(1, parent.clamp_min(0)) | (token == END))
    return got


def _select_own(s):
    case = s["case"]
    out = s["binding"].hola_beam_select(s["logits"], s["logZ"], s["score"], case["n"], finished=s["finished"],
                                        end_token=END if s["finished"] is not None else -1, weight=s["weight"], keep_slots=case["keep"])
    got = {"score": out.score, "parent": out.parent, "token": out.token}
    if s["finished"] is not None:
        got["finished"] = out.finished
    return got


def _reorder_plain(s):
    for x, to, axis, at in zip(s["states"], s["into"], s["axes"], s["positions"]):
        index = s["parent"].long().reshape([1] * axis + list(s["parent"].shape) + [1] * (x.dim() - axis - 2))
        new = x.gather(axis + 1, index.expand(x.shape))
        if at is None:
            to.copy_(new)
            continue
        here = torch.arange(x.shape[at], device=x.device).reshape([-1] + [1] * (x.dim() - at - 1))
        filled = here < s["used"].reshape([-1] + [1] * (x.dim() - axis - 1))
        to.copy_(torch.where(filled, new, to))
    return s["into"]


def _reorder_own(s):
    s["binding"].hola_beam_reorder(s["handle"], s["parent"], used=s["used"])
    return s["into"]


def _embed_plain(s):
    case = s["case"]
    t = s["tokens"].long()
    x = s["table"][t.clamp_min(0)].float()
    if s["w_scale"] is not None:
        x = x * s["w_scale"][t.clamp_min(0)][:, None]
    x = torch.where((t >= 0)[:, None], x * case["scale"], 0.0)
    if s["add"] is not None:
        x = x + s["add"].float()
    return x.to(DTYPES[case["out"]])


def _embed_own(s):
    case = s["case"]
    return s["binding"].hola_embed(s["tokens"], s["table"], scale=case["scale"], add=s["add"], w_scale=s["w_scale"], dtype=DTYPES[case["out"]])


def _grad_plain(s):
    case = s["case"]
    N, V, H = case["N"], case["V"], case["H"]
    t = s["tokens"].long()
    g = s["grad"].float() * case["scale"]
    if case["form"] == "dense":
        got = torch.zeros((V, H), device=g.device)
        got.index_add_(0, t.clamp_min(0), torch.where((t >= 0)[:, None], g, 0.0))
        return got.to(DTYPES[case["out"]])
    t, order = torch.sort(torch.where(t < 0, V, t), stable=True)
    new = torch.ones_like(t, dtype=torch.bool)
    new[1:] = t[1:] != t[:-1]
    place = torch.cumsum(new, 0) - 1
    have = t < V
    rows = torch.zeros((N, H), device=g.device)
    rows.index_add_(0, place, torch.where(have[:, None], g[order], 0.0))
    ids = torch.full((N,), -1, dtype=torch.int64, device=g.device)
    ids.scatter_(0, place, torch.where(have, t, -1))
    return {"ids": ids.int(), "rows": rows.to(DTYPES[case["out"]]), "count": (new & have).sum().int().reshape(1)}


def _grad_own(s):
    case = s["case"]
    if case["form"] == "dense":
        return s["binding"].hola_embed_grad(s["tokens"], s["grad"], case["V"], scale=case["scale"], dtype=DTYPES[case["out"]])
    got = s["binding"].hola_embed_grad_rows(s["tokens"], s["grad"], case["V"], scale=case["scale"], out=s["buffers"])
    return {"ids": got.ids, "rows": got.rows, "count": got.count}


PLAIN = {"select": _select_plain, "reorder": _reorder_plain, "embed": _embed_plain, "grad": _grad_plain}
OWN = {"select": _select_own, "reorder": _reorder_own, "embed": _embed_own, "grad": _grad_own}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def _distinct(case):
    """Expected number of distinct tokens."""
    V, n = case["V"], case["N"] * (1.0 - case["absent"])
    if case["tokens"] == "uniform":
        return V * -math.expm1(n * math.log1p(-1.0 / V)) if V > 1 else 1.0
    i = np.arange(V, dtype=np.float64)
    p = (np.log(i + 2.0) - np.log(i + 1.0)) / math.log(V + 1.0)
    return float(-np.expm1(n * np.log1p(-np.minimum(p, 1.0 - 1e-12))).sum())


def work(case):
    op = case["op"]
    if op == "select":
        rows = case["B"] * (1 if case["first"] else case["W"]) * (1.0 - case["finished"])
        return {"bytes": rows * case["V"] * SIZES[case["dtype"]] + case["B"] * (case["W"] * 8 + case["n"] * 12), "flops": 0}
    if op == "reorder":
        B, W, T, alive = case["B"], case["W"], case["steps"], case["survivors"]
        at = T // 2
        filled = sum(at + (T - at) * (b + 1) // B for b in range(B))          # positions, over all sequences
        if case["kind"] == "rows":
            beam = 8 * filled + B * (case["width"] * SIZES[case["dtype"]] + -(-T // 16) * 4)
        else:
            beam = 2 * filled * case["layers"] * case["heads"] * case["width"] * SIZES[case["dtype"]]
        moved = alive + W if case["form"] == "copy" else min(alive, W - alive) + W - alive
        return {"bytes": beam * moved + B * W * 4 + B * 4, "flops": 0}
    N, H, distinct = case["N"], case["H"], _distinct(case)
    n = N * SIZES[case["ids"]]
    if op == "embed":
        n += distinct * H * SIZES[case["table"]] + N * H * SIZES[case["out"]] * (2 if case["add"] else 1)
        return {"bytes": n, "flops": 0}
    n += N * (1.0 - case["absent"]) * H * SIZES[case["grad"]]
    n += (distinct * (H * SIZES[case["out"]] + 4) if case["form"] == "rows" else case["V"] * H * SIZES[case["out"]])
    return {"bytes": n, "flops": N * H}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _select_exact(case, s):
    """Sequence by sequence: the first entries of every live beam by whole numbers that order them (the logit, then the id), the
    candidates of all beams sorted on the host as (key, beam, place in its row)."""
    B, W, V, n = (case[x] for x in ("B", "W", "V", "n"))
    score, logZ = s["score"].double().tolist(), s["logZ"].double().tolist()
    ended = s["finished"].tolist() if s["finished"] is not None else [[False] * W] * B
    weight = s["weight"].double().tolist() if s["weight"] is not None else [[1.0] * W] * B
    few = min(n, V)
    got_c, got_p, got_t, got_f = [], [], [], []
    ids = torch.arange(V, device="cuda")
    for b in range(B):
        bits = (s["logits"][b].float() + 0.0).view(torch.int32).long()              # (+ 0.0: one zero only)
        bits = torch.where(bits < 0, -1 - (bits & 0x7fffffff), bits)
        at = torch.topk((bits << 20) - ids, few, dim=1).indices
        top, at = s["logits"][b].gather(1, at).double().tolist(), at.tolist()
        found = []
        for w in range(W):
            if ended[b][w]:
                found.append((-(score[b][w] * weight[b][w]), w, 0, score[b][w], END))
                continue
            for j in range(few):
                c = (score[b][w] - logZ[b][w]) + top[w][j]
                if c > -math.inf:
                    found.append((-(c * weight[b][w]), w, j, c, at[w][j]))
        found = [(c, w, t) for _, w, _, c, t in sorted(found)[:n] if c > -math.inf]
        found += [(-math.inf, -1, -1)] * (n - len(found))
        if case["keep"]:
            slots = [None] * n
            later = []
            for f in found:
                if f[1] >= 0 and slots[f[1]] is None:
                    slots[f[1]] = f
                else:
                    later.append(f)
            it = iter(later)
            found = [f if f is not None else next(it) for f in slots]
        got_c.append([f[0] for f in found])
        got_p.append([f[1] for f in found])
        got_t.append([f[2] for f in found])
        got_f.append([f[1] >= 0 and (ended[b][f[1]] or f[2] == END) for f in found])
    dev = s["score"].device
    got = {"score": torch.tensor(got_c, dtype=torch.float64, device=dev), "parent": torch.tensor(got_p, dtype=torch.int32, device=dev),
           "token": torch.tensor(got_t, dtype=torch.int32, device=dev)}
    if s["finished"] is not None:
        got["finished"] = torch.tensor(got_f, device=dev)
    return got


def _reorder_exact(case, s):
    """Beam by beam, from a copy of what was there."""
    parent, used = s["parent"].tolist(), s["used"].tolist()
    got = []
    for x, to, axis, at in zip(s["states"], s["into"], s["axes"], s["positions"]):
        new = to.clone()
        for b, row in enumerate(parent):
            for i, p in enumerate(row):
                a, c = x.select(axis, b).select(axis, p), new.select(axis, b).select(axis, i)
                if at is not None:
                    a, c = a.narrow(at - 2, 0, used[b]), c.narrow(at - 2, 0, used[b])
                c.copy_(a)
        got.append(new)
    return got


def _embed_exact(case, s):
    out = torch.zeros((case["N"], case["H"]), dtype=torch.float64, device="cuda")
    have = torch.nonzero(s["tokens"] >= 0)[:, 0]
    for part in have.split(8192):
        t = s["tokens"][part].long()
        x = s["table"].index_select(0, t).double()
        if s["w_scale"] is not None:
            x = x * s["w_scale"].index_select(0, t).double()[:, None]
        out[part] = x * case["scale"]
    return out if s["add"] is None else out + s["add"].double()


def _grad_exact(case, s):
    V, H = case["V"], case["H"]
    t = s["tokens"].long()
    have = torch.nonzero(t >= 0)[:, 0]
    ids, place = torch.unique(t[have], return_inverse=True)
    rows = torch.zeros((ids.numel(), H), dtype=torch.float64, device="cuda")
    for part in torch.arange(have.numel(), device="cuda").split(8192):
        rows.index_add_(0, place[part], s["grad"][have[part]].double() * case["scale"])
    if case["form"] == "dense":
        return torch.zeros((V, H), dtype=torch.float64, device="cuda").index_copy_(0, ids, rows)
    n, more = ids.numel(), case["N"] - ids.numel()
    return {"ids": torch.nn.functional.pad(ids, (0, more), value=-1).int(), "rows": torch.nn.functional.pad(rows, (0, 0, 0, more)),
            "count": torch.tensor([n], dtype=torch.int32, device="cuda")}


def exact(case, seed):
    s = INPUTS[case["op"]](case, seed)
    return {"select": _select_exact, "reorder": _reorder_exact, "embed": _embed_exact, "grad": _grad_exact}[case["op"]](case, s)
