"""Low-rank adapters beside the LM head: logits, statistics and the whole step against the definition in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import compare, ref
from paper_2506_18952_b200 import binding, workloads

gpu = pytest.mark.gpu
U = 2.0 ** -24                          # half a unit in the last place of fp32, relative


# ------------------------------------------------------------------------------------------------ inputs and reference
def make(B, k, H, V, slots, rank, seed=0, weights="bf16"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")                     # noqa: E731
    hidden = rnd(B, k + 1, H).to(torch.bfloat16)
    W = (rnd(V, H) * 1.28 / H ** 0.5).to(torch.bfloat16)
    A = (rnd(slots, rank, H) / H ** 0.5).to(torch.bfloat16)
    Bup = (rnd(slots, V, rank) * 0.5 / rank ** 0.5).to(torch.bfloat16)
    scale = torch.rand((slots,), generator=g, device="cuda") * 1.5 + 0.25
    ids = torch.randint(-1, slots, (B,), generator=g, device="cuda", dtype=torch.int32)
    w_scale, a8 = None, False
    if weights == "mixed":
        widths = [(4, 8, 16)[i % 3] for i in range(-(-V // 256))]
        W = binding.hola_quantize_mixed(W, widths)
    elif weights != "bf16":
        W, w_scale = binding.hola_quantize_w8(W)
        a8 = {"int8": False, "w8a8": True, "w8a16": "a16"}[weights]
    return dict(hidden=hidden, W=W, A=A, Bup=Bup, scale=scale, ids=ids, w_scale=w_scale, a8=a8)


def delta64(d):
    """The adapters' part of the logits in 64 bits, and what bounds its fp32 evaluation.  A tensor-core step of 16 products adds no
    more than 2^-22 of its operands' absolute sum (products are exact, terms are cut off at the largest one's last place); u passes
    through H / 16 such steps and 16 additions, the second product through 3 rank / 16; u itself enters it as two bf16 planes at
    least, which leave 2^-18 of it; the scale is one more rounding."""
    H, rank = d["hidden"].shape[-1], d["A"].shape[1]
    x, ids = d["hidden"].double(), d["ids"].long()
    B, k1, _ = x.shape
    out = torch.zeros((B, k1, d["Bup"].shape[1]), dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    for b in range(B):
        a = int(ids[b])
        if 0 <= a < d["A"].shape[0]:
            A, Bu, s = d["A"][a].double(), d["Bup"][a].double(), d["scale"][a].double()
            u, u_abs = s * (x[b] @ A.T), s * (x[b].abs() @ A.abs().T)
            out[b] = u @ Bu.T
            e_u = u_abs * ((-(-H // 16)) * 2.0 ** -22 + 17 * U) + u.abs() * (2.0 ** -18 + U)
            bound[b] = e_u @ Bu.abs().T + (u.abs() @ Bu.abs().T) * (3 * -(-rank // 16) + 3) * 2.0 ** -22
    return out, bound


def check_stats(out, V, logits=None):
    """entropy and logZ are those of the logits that came with them: fp32 sums of V terms in pieces (V / 1000 + 40 roundings deep
    at most, 2^-22 per exponential), H = ln s - t / s with |t / s| <= ln V."""
    l = (out.logits if logits is None else logits).double()
    logZ = torch.logsumexp(l, dim=-1)
    lp = l - logZ[..., None]
    H = -(lp.exp() * lp).sum(-1)
    E = (V / 1000 + 40) * U + 2.0 ** -22 + 4 * U * float(l.abs().max())
    assert (out.logZ.double() - logZ).abs().max() <= E + 2 * U * float(l.abs().max())
    assert (out.entropy.double() - H).abs().max() <= E * (1 + 3 * np.log(V + 1)) + 4 * U * np.log(V + 1)


def check_logits(got, base, d):
    """Against the bare head's own logits, plus the adapters' part.  Where both products are accumulated together the running sum
    is rounded once per step: 2^-22 of it for each of 2 x slots x rank / 16 steps."""
    want, bound = delta64(d)
    want = want + base.double()
    steps = 2 * -(-d["A"].shape[0] * (-(-d["A"].shape[1] // 8) * 8) // 64) * 4 + 4
    tol = bound + steps * 2.0 ** -22 * (base.double().abs() + want.abs() + want.abs().amax(dim=-1, keepdim=True) * 0.25)
    assert ((got.double() - want).abs() <= tol).all(), float(((got.double() - want).abs() - tol).max())


SHAPES = [  # B, k, H, V, slots, rank
    (1, 4, 64, 1000, 1, 8), (1, 0, 64, 33, 2, 8), (2, 3, 128, 8, 3, 16), (5, 1, 72, 1001, 4, 24), (3, 4, 256, 5003, 2, 16),
    (1, 4, 4096, 32000, 4, 16), (7, 20, 512, 3001, 5, 8), (2, 40, 264, 2000, 2, 40), (23, 3, 1032, 50003, 8, 24), (64, 5, 512, 32000, 16, 16),
    (9, 5, 1024, 4099, 3, 128), (40, 7, 256, 6000, 64, 8), (100, 5, 256, 2000, 7, 16), (32, 0, 1024, 128256, 16, 32), (300, 8, 64, 700, 9, 16),
    (17, 2, 640, 9001, 64, 16), (12, 5, 256, 3003, 5, 32), (12, 5, 256, 3003, 5, 64), (12, 5, 256, 3004, 5, 64), (33, 0, 128, 4001, 3, 16)]


@gpu
@pytest.mark.parametrize("B,k,H,V,slots,rank", SHAPES)
def test_logits_and_statistics(B, k, H, V, slots, rank):
    d = make(B, k, H, V, slots, rank, seed=B + V)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        base = ctx.hola_lm_head_entropy(d["hidden"], d["W"], want_logits=True)
        out = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"])
        assert out.status.item() == 0
        check_logits(out.logits, base.logits, d)
        check_stats(out, V)
        kept = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"], want_logits=False)     # logits in the context's scratch
        check_stats(kept, V, out.logits)
        # a sequence without an adapter gets what the bare head gives it
        d["ids"].fill_(-1)
        none = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"])
        assert torch.equal(none.logits, base.logits)
        check_stats(none, V)


@gpu
@pytest.mark.parametrize("B,k,H,V,slots,rank", [(23, 3, 128, 5003, 8, 24), (17, 2, 256, 9000, 64, 16), (12, 5, 64, 3004, 5, 64), (9, 5, 128, 4099, 3, 128),
                                                (6, 2, 64, 2001, 4, 8), (12, 5, 256, 3003, 5, 32)])
def test_logits_within_the_two_products_own_bounds(B, k, H, V, slots, rank):
    """The second product is made apart from the head's and added once, in fp32: what bounds a logit's error are the steps of its own
    sequence's two products (delta64's, but for u, which enters with all its bits) and that addition, however many slots there are."""
    d = make(B, k, H, V, slots, rank, seed=B + V + 1)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        base = ctx.hola_lm_head_entropy(d["hidden"], d["W"], want_logits=True).logits.double()
        got = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"]).logits.double()
    delta, _ = delta64(d)
    for b in range(B):
        a = int(d["ids"][b])
        if a < 0:
            continue
        x, A, Bu, s = d["hidden"][b].double(), d["A"][a].double(), d["Bup"][a].double(), d["scale"][a].double()
        u, u_abs = s * (x @ A.T), s * (x.abs() @ A.abs().T)
        e_u = u_abs * (-(-H // 16) * 2.0 ** -22 + 17 * U) + u.abs() * U
        tol = e_u @ Bu.abs().T + (u.abs() @ Bu.abs().T) * (3 * -(-rank // 16) + 3) * 2.0 ** -22 + U * (base[b] + delta[b]).abs()
        assert ((got[b] - base[b] - delta[b]).abs() <= tol).all()


@gpu
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 64, 128])
@pytest.mark.parametrize("V", [1000, 1003])
def test_u_enters_the_second_product_with_all_its_bits(rank, V):
    """u = scale exactly (one channel of x and of A is 1, the others 0), every entry of the vocabulary has one rank, with a power of two,
    and W = 0: a logit is that power times a number of 24 bits.  The tensor cores add the planes smallest first and cut a sum off at the
    larger operand's last place.  Where the largest plane lies below the next power of two above u that is u's own last place and
    nothing is lost; where u rounds up to that power (u from 2 - 2^-8 on, say), less than 2^-22 beside 2 is: 2^-23 of u and a little.
    (Without the third plane up to 2^-17 would be.)"""
    n = 48
    g = torch.Generator(device="cuda").manual_seed(rank)
    scale = 1 + torch.randint(0, 2 ** 23, (n,), generator=g, device="cuda").float() * 2.0 ** -23           # (exact)
    scale[:6] = torch.tensor([2 - 2.0 ** -23, 1 + 2.0 ** -23, 1 + 2.0 ** -8 + 2.0 ** -23, 2 - 2.0 ** -8 - 2.0 ** -23, 1 + 2.0 ** -9 + 2.0 ** -17 + 2.0 ** -23,
                              2 - 2.0 ** -16 - 2.0 ** -23])
    scale[::3] *= -1
    scale[1::4] *= 2.0 ** -20
    hidden = torch.zeros((n, 1, 64), dtype=torch.bfloat16, device="cuda")
    hidden[:, :, 0] = 1.0
    A = torch.zeros((n, rank, 64), dtype=torch.bfloat16, device="cuda")
    A[:, :, 0] = 1.0
    at = torch.arange(V, device="cuda")
    power = 2.0 ** ((at % 7) - 3).float() * (1 - 2 * (at // 7 % 2)).float()
    Bup = torch.zeros((n, V, rank), dtype=torch.bfloat16, device="cuda")
    Bup[:, at, at % rank] = power.bfloat16()
    with binding.HolaVerify(n, 0, 64, V) as ctx:
        W = torch.zeros((V, 64), dtype=torch.bfloat16, device="cuda")
        out = ctx.hola_lm_head_adapters(hidden, W, binding.AdapterBank(A, Bup, scale), torch.arange(n, dtype=torch.int32, device="cuda"))
    want = scale.double()[:, None] * power.double()
    up = (scale.abs().bfloat16().float() >= 2.0 ** (scale.abs().log2().floor() + 1))[:, None]              # (u rounds up to a power of two)
    assert up.any() and not up.all()
    err = (out.logits[:, 0].double() - want).abs()
    assert (err[~up.expand_as(err)] == 0).all()
    assert (err <= 2.0 ** -23 * (1 + 2.0 ** -7) * want.abs()).all()


@gpu
@pytest.mark.parametrize("V", [1000, 9003])
def test_statistics_of_logits_far_from_zero(V):
    """A logit's distance to the maximum counts, not where the maximum is.  Sums of differences, which are rounded once: relative to
    e^d |d| <= 0.37 per unit, like each merge's."""
    sizes = [1e3, 1e5, 1e7, 1e9, 1e10, 3e12, 1e20, 1e30]
    d = make(2 * len(sizes), 3, 256, V, len(sizes), 8, seed=V)
    for i, big in enumerate(sizes):
        d["Bup"][i, :, 0] = big                              # all of a row's logits by the same
    d["ids"] = torch.arange(2 * len(sizes), device="cuda", dtype=torch.int32) // 2
    with binding.HolaVerify(2 * len(sizes), 3, 256, V) as ctx:
        out = ctx.hola_lm_head_adapters(d["hidden"], d["W"], binding.AdapterBank(d["A"], d["Bup"], d["scale"]), d["ids"])
    l = out.logits.double()
    m = l.amax(dim=-1)
    logZ = torch.logsumexp(l - m[..., None], dim=-1)
    lp = l - m[..., None] - logZ[..., None]
    H = -(lp.exp() * lp).sum(-1)
    E = (V / 1000 + 80) * U + 2.0 ** -22
    assert ((out.logZ.double() - m - logZ).abs() <= E + 2 * U * m.abs()).all()
    assert ((out.entropy.double() - H).abs() <= E * (1 + 3 * np.log(V + 1)) + 4 * U * np.log(V + 1)).all()


@gpu
@pytest.mark.parametrize("weights", ["int8", "w8a8", "w8a16", "mixed"])
@pytest.mark.parametrize("B,k,H,V,slots,rank", [(1, 4, 256, 3001, 3, 16), (16, 5, 1024, 8000, 4, 8), (64, 5, 512, 9000, 8, 24),
                                                (90, 5, 256, 5000, 64, 16)])
def test_every_storage_form_of_the_head(weights, B, k, H, V, slots, rank):
    d = make(B, k, H, V, slots, rank, seed=3, weights=weights)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    kw = dict(w_scale=d["w_scale"], a8=d["a8"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        base = ctx.hola_lm_head_entropy(d["hidden"], d["W"], want_logits=True, **kw)
        out = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"], **kw)
        check_logits(out.logits, base.logits, d)
        check_stats(out, V)
        bare = (d["ids"] < 0).nonzero()[:, 0]
        assert torch.equal(out.logits[bare], base.logits[bare])


@gpu
def test_against_the_whole_definition():
    """W x + s B A x in 64 bits throughout."""
    B, k, H, V = 6, 3, 1024, 7001
    d = make(B, k, H, V, 4, 16, seed=8)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        out = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"])
    want, bound = delta64(d)
    x, W = d["hidden"].double(), d["W"].double()
    want += x @ W.T
    bound += (x.abs() @ W.abs().T) * (H // 16 + 8) * 2.0 ** -22 + 8 * 2.0 ** -22 * want.abs()
    assert ((out.logits.double() - want).abs() <= bound).all()


def _verify_inputs(B, k, H, V, slots, rank, seed, q_dtype=torch.bfloat16):
    w = workloads.gaussian_head("adapters", B, k, H, V, seed=seed, device="cuda", w_std=2.0 / H ** 0.5, sigma=0.5, tau=2.0,
                                sigma_far=1.5, q_dtype=q_dtype)
    d = make(B, k, H, V, slots, rank, seed)
    d["hidden"], d["W"] = w.hidden, w.W_lm
    return w, d


@gpu
@pytest.mark.parametrize("gate,fallback", [(0, 0), (1, 0), (0, 1), (1, 1)])
@pytest.mark.parametrize("B,k,H,V", [(1, 4, 512, 6000), (24, 5, 256, 5000), (70, 4, 256, 3001), (5, 0, 64, 1000)])
def test_whole_step(B, k, H, V, gate, fallback):
    if k == 0 and gate == 1:
        pytest.skip("no draft rows")
    w, d = _verify_inputs(B, k, H, V, 5, 16, seed=21 + B)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        out = ctx.hola_verify_adapters(w.hidden, w.W_lm, w.draft_tok, w.draft_q, w.uniforms, w.tau, bank, d["ids"], want_logits=True,
                                       gate_source=gate, fallback=fallback)
        again = ctx.hola_verify_adapters(w.hidden, w.W_lm, w.draft_tok, w.draft_q, w.uniforms, w.tau, bank, d["ids"],
                                         gate_source=gate, fallback=fallback)            # logits in the context's scratch
        torch.cuda.synchronize()
    want, _ = delta64(d)
    want += w.hidden.double() @ w.W_lm.double().T
    n = compare.torch_to_numpy
    orc = ref.verify_from_logits(want.cpu().numpy(), n(w.draft_tok), n(w.draft_q), n(w.uniforms), w.tau, gate, fallback)
    rep = compare.compare(orc, n(w.draft_q), n(w.uniforms), n(out.accept_len), n(out.next_tok), n(out.entropy), n(out.logZ),
                          n(out.logits))
    assert rep.ok, rep.summary()
    assert out.status.item() == 0
    for f in ("accept_len", "next_tok", "entropy", "logZ"):
        assert torch.equal(getattr(out, f), getattr(again, f))


@gpu
def test_adapters_then_scores_of_what_was_emitted():
    """The run of them as a server makes it: adapted verify step, then the log probabilities of the tokens that it emitted."""
    B, k, H, V = 12, 4, 256, 5003
    w, d = _verify_inputs(B, k, H, V, 3, 16, seed=5)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        out = ctx.hola_verify_adapters(w.hidden, w.W_lm, w.draft_tok, w.draft_q, w.uniforms, w.tau, bank, d["ids"], want_logits=True)
        lp = binding.hola_token_logprobs(out.logits, n_top=5, logZ=out.logZ, emitted=(w.draft_tok, out.accept_len, out.next_tok))
    l = delta64(d)[0] + w.hidden.double() @ w.W_lm.double().T
    want = torch.log_softmax(l, dim=-1)
    for b in range(B):
        n = int(out.accept_len[b])
        for j in range(k + 1):
            if j > n:
                assert lp.logprob[b, j] == 0 and lp.rank[b, j] == -1 and (lp.top_ids[b, j] == -1).all()
                continue
            x = int(w.draft_tok[b, j] if j < n else out.next_tok[b])
            assert abs(float(lp.logprob[b, j] - want[b, j, x])) <= compare.ENTROPY_ATOL
            row = out.logits[b, j]
            before = int(((row > row[x]) | ((row == row[x]) & (torch.arange(V, device="cuda") < x))).sum())
            assert int(lp.rank[b, j]) == before
            assert int(lp.top_ids[b, j, 0]) == int((row == row.max()).nonzero()[0])


@gpu
@pytest.mark.parametrize("B", [2048, 2100])
def test_more_sequences_than_are_sorted(B):
    k, H, V = 1, 64, 300
    d = make(B, k, H, V, 40, 8, seed=6)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        base = ctx.hola_lm_head_entropy(d["hidden"], d["W"], want_logits=True)
        out = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"])
        check_logits(out.logits, base.logits, d)
        check_stats(out, V)


@gpu
def test_what_is_not_finite_stays_in_its_requests():
    """A slot of NaN and infinities spoils the sequences that use it, and no others; one that nobody uses spoils nothing."""
    B, k, H, V = 9, 3, 128, 2050
    d = make(B, k, H, V, 4, 16, seed=17)
    d["ids"].copy_(torch.tensor([0, 1, 2, -1, 0, 1, 2, 2, 1]))
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        want = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"])
        bank.A[3], bank.B[3], bank.scale[3] = float("nan"), float("inf"), float("nan")
        bank.A[1, 0, 0], bank.B[1, 5, 3] = float("nan"), float("-inf")
        got = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"])
        clean = (d["ids"] != 1).nonzero()[:, 0]
        for f in ("logits", "logZ", "entropy"):
            assert torch.equal(getattr(got, f)[clean], getattr(want, f)[clean])
        assert got.logZ[d["ids"] == 1].isnan().all()


@gpu
@pytest.mark.parametrize("V", [2052, 2051, 9000])
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 64, 104])
def test_infinite_factors(rank, V):
    """An infinite factor makes of its entries what the formula says: infinities (-inf: an entry of probability 0) or, with a factor of
    zero or another infinity, NaN.  The other entries are bounded as everywhere: the product's own bound and one addition in fp32."""
    B, k, H, inf = 12, 2, 128, float("inf")
    d = make(B, k, H, V, 6, rank, seed=rank + V)
    d["ids"].copy_(torch.tensor([0, 1, 2, 3, 4, -1, 0, 1, 2, 5, 5, 0]))
    d["hidden"][:, :, 0] = 1.0
    for s in (0, 5):                                          # u[0] is positive: masks
        d["A"][s, 0], d["A"][s, 0, 0] = 0.0, 1.0
    d["Bup"][0, 5::3, 0] = -inf
    d["Bup"][5, : V - 7, rank - 1 if rank > 8 else 0] = -inf  # (of either sign where the rank is not u[0])
    d["Bup"][5, V - 3, 0] = -inf
    d["Bup"][1, 7, 2], d["Bup"][1, V - 1, 3] = inf, -inf
    d["Bup"][2, 11, 1], d["Bup"][2, 11, 5], d["Bup"][2, 64:80, 4] = inf, -inf, -inf
    d["A"][3, 1] = 0.0                                        # u[1] is zero
    d["Bup"][3, 300, 1] = -inf
    d["A"][4, 0, 0] = inf                                     # u[0] is infinite
    d["Bup"][4, 100, 0] = 0.0
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        base = ctx.hola_lm_head_entropy(d["hidden"], d["W"])
        out = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"])
        one = [t[:, :1].contiguous() for t in (d["hidden"], torch.rand((B, 1), device="cuda"))]
        greedy = ctx.hola_verify_adapters(one[0], d["W"], None, None, one[1], 1.5, bank, d["ids"], want_logits=True, fallback=1)
        for f in ("logits", "logZ", "entropy"):
            assert torch.equal(getattr(out, f)[5], getattr(base, f)[5])
    delta, bound = delta64(d)
    want = base.logits.double() + delta
    fine = want.isfinite()
    got = out.logits.double()
    assert torch.equal(got.isfinite(), fine) and torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got[want.isinf()], want[want.isinf()])
    assert ((got - want).abs() <= bound + 2 * U * (base.logits.double().abs() + want.abs()))[fine].all()
    # rows without NaN and +inf have a distribution
    row = (got < inf).all(dim=-1)
    assert row[[0, 5, 6, 11]].all() and not row[4].any()
    assert out.logZ[~row].isnan().all()
    m = got[row].amax(dim=-1, keepdim=True)
    ln_s = (got[row] - m).exp().sum(dim=-1).log()
    lp = got[row] - m - ln_s[:, None]
    want_H = -torch.where(lp > -inf, lp.exp() * lp, 0.0).sum(dim=-1)
    E = (V / 1000 + 40) * U + 2.0 ** -22 + 4 * U * float(got[row].abs().nan_to_num(posinf=0.0).max())
    assert ((out.logZ[row].double() - m[:, 0] - ln_s).abs() <= E + 2 * U * m[:, 0].abs()).all()
    assert ((out.entropy[row].double() - want_H).abs() <= E * (1 + 3 * np.log(V + 1)) + 4 * U * np.log(V + 1)).all()
    assert torch.equal(greedy.next_tok[row[:, 0]].long(), greedy.logits[row[:, 0], 0].argmax(dim=-1))


@gpu
def test_an_empty_batch():
    bank = binding.AdapterBank.empty(2, 8, 64, 500, "cuda")
    with binding.HolaVerify(2, 1, 64, 500) as ctx:
        hidden, W = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((500, 64), dtype=torch.bfloat16, device="cuda")
        out = ctx.hola_lm_head_adapters(hidden, W, bank, torch.zeros((0,), dtype=torch.int32, device="cuda"))
        assert out.logits.shape == (0, 2, 500) and out.status.item() == 0


@gpu
def test_indices_that_no_slot_has():
    B, k, H, V = 6, 2, 128, 999
    d = make(B, k, H, V, 2, 8, seed=4)
    d["ids"].copy_(torch.tensor([0, 1, -1, 2, -2, 2 ** 31 - 1]))
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        base = ctx.hola_lm_head_entropy(d["hidden"], d["W"], want_logits=True)
        out = ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"])
        assert out.status.item() == binding.FLAG_BAD_ADAPTER
        assert torch.equal(out.logits[2:], base.logits[2:])
        check_logits(out.logits, base.logits, d)
        check_stats(out, V)
        out.status.fill_(binding.FLAG_R_ZERO)                 # the caller's word: bits are added
        ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"], out=out)
        assert out.status.item() == binding.FLAG_BAD_ADAPTER | binding.FLAG_R_ZERO


@gpu
def test_ranks_are_filled_up_and_slots_are_replaced():
    B, k, H, V = 8, 3, 256, 3000
    d = make(B, k, H, V, 4, 13, seed=9)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    assert bank.rank == 16 and bank.B.shape == (4, V, 16)
    with binding.HolaVerify(B, k, H, V) as ctx:
        base = ctx.hola_lm_head_entropy(d["hidden"], d["W"], want_logits=True)
        check_logits(ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"]).logits, base.logits, d)
        e = make(B, k, H, V, 4, 4, seed=10)                   # rank 4 takes a slot's place
        other = binding.AdapterBank.empty(4, 13, H, V)
        for s in (3, 0, 2, 1):
            other.set(s, d["A"][s], d["Bup"][s], float(d["scale"][s]))
        other.set(2, e["A"][2], e["Bup"][2], e["scale"][2])
        d["A"][2], d["Bup"][2] = 0, 0
        d["A"][2, :4], d["Bup"][2, :, :4], d["scale"][2] = e["A"][2], e["Bup"][2], e["scale"][2]
        check_logits(ctx.hola_lm_head_adapters(d["hidden"], d["W"], other, d["ids"]).logits, base.logits, d)
        ones = binding.AdapterBank(d["A"], d["Bup"])
        d["scale"].fill_(1.0)
        check_logits(ctx.hola_lm_head_adapters(d["hidden"], d["W"], ones, d["ids"]).logits, base.logits, d)


@gpu
def test_graphs_streams_and_changing_batches():
    """A captured call follows its inputs: the hidden rows and the adapters of the batch change between replays."""
    B, k, H, V = 20, 4, 512, 8000
    d = make(B, k, H, V, 6, 16, seed=12)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as ctx:
        src, ids = d["hidden"].clone(), d["ids"].clone()
        out = ctx.hola_lm_head_adapters(src, d["W"], bank, ids)
        ctx.hola_lm_head_adapters(src, d["W"], bank, ids, out=out)
        torch.cuda.synchronize()
        hid = torch.empty_like(src)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            torch.mul(src, 1, out=hid)                        # written right in front of the call
            ctx.hola_lm_head_adapters(hid, d["W"], bank, ids, out=out)
        for r in range(3):
            src.copy_(d["hidden"].roll(r, 0))
            ids.copy_(d["ids"].roll(2 * r, 0))
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (out.logits, out.logZ, out.entropy)]
            want = ctx.hola_lm_head_adapters(src, d["W"], bank, ids)
            assert all(torch.equal(x, y) for x, y in zip(got, (want.logits, want.logZ, want.entropy)))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        aside = ctx.hola_lm_head_adapters(src, d["W"], bank, ids, stream=side)
        side.synchronize()
        assert torch.equal(aside.logits, want.logits)


@gpu
def test_the_whole_run_in_two_graphs_of_one_context():
    """Adapted verify step and scores of what it emitted, captured twice on one context (they share its workspace) and replayed in
    turn; every input is written by kernels right in front of the call."""
    B, k, H, V = 12, 4, 256, 6000
    w, d = _verify_inputs(B, k, H, V, 3, 16, seed=41)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    src = [w.hidden, w.draft_tok, w.draft_q, w.uniforms, d["ids"]]
    with binding.HolaVerify(B, k, H, V) as ctx:
        def run(x, out=None):
            out = ctx.hola_verify_adapters(x[0], w.W_lm, x[1], x[2], x[3], w.tau, bank, x[4], want_logits=True, out=out)
            lp = binding.hola_token_logprobs(out.logits, n_top=7, logZ=out.logZ, emitted=(x[1], out.accept_len, out.next_tok))
            return [out.accept_len, out.next_tok, out.entropy, out.logZ, out.logits, lp.logprob, lp.rank, lp.top_ids, lp.top_logprobs]
        graphs = []
        for _ in range(2):
            host = [t.clone() for t in src]
            run(host)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                x = [t.roll(0, 0) if t.dtype != torch.bfloat16 else t * 1 for t in host]
                got = run(x)
            graphs.append((graph, host, x, got))
        for r in range(4):
            graph, host, x, got = graphs[r % 2]
            for h, t in zip(host, src):
                h.copy_(t.roll(r, 0))
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in got]
            want = run([t.roll(r, 0) for t in src])
            for a, b in zip(got, want):
                assert torch.equal(a, b)


@gpu
def test_rows_behind_the_batch_and_calls_in_between_keep_their_results():
    """A context made for more: nothing beyond the batch's rows is written, and bare calls before and after give the same bits."""
    B, k, H, V = 3, 2, 128, 1003
    d = make(B, k, H, V, 2, 8, seed=14)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(10, 6, H, V) as ctx:
        before = ctx.hola_lm_head_entropy(d["hidden"], d["W"], want_logits=True)
        room = torch.full((B * (k + 1) * V + 2 * V,), 7.5, device="cuda")
        stats = torch.full((2, B * (k + 1) + 32), 7.5, device="cuda")
        out = ctx.alloc_outputs(B, k)
        out.logits = room[V:-V].view(B, k + 1, V)
        out.entropy, out.logZ = (stats[i, 16:-16].view(B, k + 1) for i in range(2))
        ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"], out=out)
        check_logits(out.logits, before.logits, d)
        assert (room[:V] == 7.5).all() and (room[-V:] == 7.5).all()
        assert (stats[:, :16] == 7.5).all() and (stats[:, -16:] == 7.5).all()
        after = ctx.hola_lm_head_entropy(d["hidden"], d["W"], want_logits=True)
        for f in ("logits", "entropy", "logZ"):
            assert torch.equal(getattr(before, f), getattr(after, f))


# ------------------------------------------------------------------------------------------------ refusals
def _adapters(**kw):
    a = binding.hola_adapters()
    for n, v in dict(dict(A=4096, B=4096, scale=4096, ids=4096, slots=3, rank=8), **kw).items():
        setattr(a, n, v)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(A=None), 1), (dict(B=None), 1), (dict(ids=None), 1), (dict(slots=0), 1), (dict(slots=-1), 1), (dict(rank=0), 1), (dict(rank=-8), 1),
    (dict(A=4104), 1), (dict(B=4104), 1), (dict(rank=4), 2), (dict(rank=136), 2), (dict(rank=12), 2), ({}, 1), (dict(B=None, ids=None), 1)])
def test_refused_by_the_library(change, status):
    """(The last one: adapters that are in order, and no context.)"""
    lib = binding.load_library()
    ad, a = _adapters(**change), binding.hola_verify_args()
    a.B = 1
    for fn in (lib.hola_lm_head_adapters, lib.hola_verify_adapters):
        assert fn(None, ctypes.byref(a), ctypes.byref(ad), None) == status
        assert fn(None, ctypes.byref(a), None, None) == 1


@gpu
def test_two_contexts_on_two_streams_at_once():
    B, k, H, V = 16, 3, 256, 20000
    d = make(B, k, H, V, 4, 16, seed=31)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(B, k, H, V) as one, binding.HolaVerify(B, k, H, V) as two:
        want = one.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"])
        other = d["ids"].roll(1)
        want2 = two.hola_lm_head_adapters(d["hidden"], d["W"], bank, other)
        torch.cuda.synchronize()
        s, t = torch.cuda.Stream(), torch.cuda.Stream()
        for _ in range(5):
            a = one.hola_lm_head_adapters(d["hidden"], d["W"], bank, d["ids"], stream=s)
            b = two.hola_lm_head_adapters(d["hidden"], d["W"], bank, other, stream=t)
            torch.cuda.synchronize()
            for f in ("logits", "logZ", "entropy"):
                assert torch.equal(getattr(a, f), getattr(want, f)) and torch.equal(getattr(b, f), getattr(want2, f))


def test_struct_layout():
    assert ctypes.sizeof(binding.hola_adapters) == 4 * 8 + 2 * 4


def test_bank_layout_and_refusals_need_no_device():
    A, Bup = torch.randn(3, 5, 16).bfloat16(), torch.randn(3, 40, 5).bfloat16()
    bank = binding.AdapterBank(A, Bup, torch.tensor([1.0, 2.0, 3.0]))
    assert (bank.slots, bank.rank, bank.H, bank.V) == (3, 8, 16, 40)
    for s in range(3):
        assert torch.equal(bank.A[s, :5], A[s]) and (bank.A[s, 5:] == 0).all()
        assert torch.equal(bank.B[s, :, :5], Bup[s]) and (bank.B[s, :, 5:] == 0).all()
    assert bank.scale.tolist() == [1.0, 2.0, 3.0]
    bank.set(1, A[0, :2], Bup[0][:, :2], 0.5)
    assert (bank.A[1, 2:] == 0).all() and (bank.B[1, :, 2:] == 0).all() and bank.scale[1] == 0.5
    for bad in (lambda: binding.AdapterBank(A, Bup[:2]), lambda: binding.AdapterBank(A, Bup.transpose(1, 2)), lambda: binding.AdapterBank(A[0], Bup),
                lambda: binding.AdapterBank(A, Bup, torch.ones(2)), lambda: binding.AdapterBank(A.float(), Bup),
                lambda: binding.AdapterBank.empty(0, 8, 16, 40, "cpu"), lambda: binding.AdapterBank.empty(1, 129, 16, 40, "cpu"),
                lambda: bank.set(3, A[0], Bup[0]), lambda: bank.set(-1, A[0], Bup[0]), lambda: bank.set(0, A[0][:, :8], Bup[0]),
                lambda: bank.set(0, A[0], Bup[0][:, :4]), lambda: bank.set(0, A[0].float(), Bup[0])):
        with pytest.raises(binding.HolaError):
            bad()


@gpu
def test_refused_by_the_binding():
    d = make(2, 1, 64, 500, 2, 8)
    bank = binding.AdapterBank(d["A"], d["Bup"], d["scale"])
    with binding.HolaVerify(2, 1, 64, 500) as ctx:
        for ids in (d["ids"].long(), d["ids"].cpu(), d["ids"][:1], d["ids"].repeat(2)[::2]):
            with pytest.raises(binding.HolaError):
                ctx.hola_lm_head_adapters(d["hidden"], d["W"], bank, ids)
        for other in (binding.AdapterBank.empty(2, 8, 128, 500), binding.AdapterBank.empty(2, 8, 64, 501), binding.AdapterBank.empty(2, 8, 64, 500, "cpu")):
            with pytest.raises(binding.HolaError):
                ctx.hola_lm_head_adapters(d["hidden"], d["W"], other, d["ids"])
        with pytest.raises(binding.HolaError):
            ctx.hola_verify_adapters(d["hidden"], d["W"], None, None, None, 1.0, bank, d["ids"])


class _NoDevice(binding.HolaVerify):
    """A context that is never asked for anything on a device."""

    def __init__(self, H, V):
        self.H, self.V, self.device, self._dev, self._ctx = H, V, 0, torch.device("cpu"), ctypes.c_void_p()
        self.lib = binding.load_library()

    def close(self):
        pass


@pytest.mark.parametrize("adapters,ids", [(None, True), ("bank", None), ("bank", [0, 1]), ("struct", True), (object(), True), (None, None)])
def test_what_is_no_bank_is_refused_before_anything_native_is_called(monkeypatch, adapters, ids):
    """The library's functions for adapters take one argument more than the others: none of them may be called without a bank."""
    calls = []
    ctx = _NoDevice(64, 40)
    monkeypatch.setattr(binding, "_host", type("Host", (), {"call": staticmethod(lambda *a: calls.append(a) or 1),
                                                            "outputs": staticmethod(lambda *a: calls.append(a))}))
    bank = binding.AdapterBank.empty(2, 8, 64, 40, "cpu")
    adapters = {"bank": bank, "struct": bank.struct}.get(adapters, adapters) if isinstance(adapters, str) else adapters
    ids = torch.zeros(2, dtype=torch.int32) if ids is True else ids
    hidden, W = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(40, 64, dtype=torch.bfloat16)
    out = ctx.alloc_outputs(2, 3, device="cpu")
    q, u, t = torch.zeros(2, 3, 40), torch.zeros(2, 4), torch.zeros(2, 3, dtype=torch.int32)
    stream = type("Stream", (), {"cuda_stream": 4096})()
    for o in (out, None):
        with pytest.raises(binding.HolaError):
            ctx.hola_lm_head_adapters(hidden, W, adapters, ids, out=o, stream=stream)
        with pytest.raises(binding.HolaError):
            ctx.hola_verify_adapters(hidden, W, t, q, u, 1.5, adapters, ids, out=o, stream=stream)
    assert not calls
    for entry in ("hola_lm_head_adapters", "hola_verify_adapters"):      # (nor by the short way itself)
        assert ctx._native(entry, hidden, W, t, q, u, 1.5, out, 1, 0, 0, 0, None, False, stream, None, ids) is None
    assert not calls


@gpu
def test_decode_loop_with_adapters_and_scores():
    """The driver's loop on adapted heads: log probabilities as the records' logits have them, tokens as a bare loop's without adapters."""
    from paper_2506_18952_b200 import driver
    B, k, H, V, rounds = 6, 3, 256, 2000, 4
    dev = torch.device("cuda", torch.cuda.current_device())
    models = driver.SyntheticPair(V, H, 5, dev)
    prompt = torch.randint(0, V, (B, 2), device=dev, generator=torch.Generator(device=dev).manual_seed(1))
    bank = driver.seeded_adapters(models, 3, 4, 9)
    ids = torch.tensor([0, 1, 2, -1, 0, 2], dtype=torch.int32, device=dev)
    with binding.HolaVerify(B, k, H, V) as ctx:
        run = lambda **kw: driver.hsd_decode(ctx, models, prompt, k, 1.5, rounds, 3, keep_records=True, **kw)     # noqa: E731
        bare, none = run(), run(adapters=bank, adapter_ids=torch.full_like(ids, -1), score=True)
        assert torch.equal(bare.tokens, none.tokens) and bare.logprob is None
        res = run(adapters=bank, adapter_ids=ids, score=True)
    want = torch.zeros(B, dtype=torch.float64)
    for rec in res.records:
        d = dict(hidden=rec.hidden, ids=ids, A=bank.A, Bup=bank.B, scale=bank.scale)
        lp = torch.log_softmax(delta64(d)[0] + rec.hidden.double() @ models.W_lm.double().T, dim=-1)
        for b in range(B):
            n = int(rec.out.accept_len[b])
            for j in range(n + 1):
                want[b] += float(lp[b, j, rec.draft_tok[b, j] if j < n else rec.out.next_tok[b]])
    assert (res.logprob.cpu() - want).abs().max() <= rounds * (k + 1) * 1e-4
    assert not torch.equal(res.tokens, bare.tokens)
