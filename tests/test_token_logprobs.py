"""Log probabilities of given tokens, ranks, entropy and top alternatives against the definition in 64 bits."""
import ctypes
import math

import pytest
import torch

from paper_2506_18952_b200 import binding

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
gpu = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ reference
def reference(logits, tokens, n_top):
    """Everything in 64 bits from the logits [rows, V] as stored; ids by a stable sort (descending, equal ones by id)."""
    l = logits.cpu().double()
    rows, V = l.shape
    bad = ~(l < math.inf).all(dim=1)
    m = l.amax(dim=1, keepdim=True)
    ln_s = (l - m).exp().sum(dim=1).log()                    # (about the maximum: m + ln s loses ln s where m is 1e38)
    logZ = m[:, 0] + ln_s
    lp = (l - m) - ln_s[:, None]
    H = -torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(dim=1)
    empty = (m == -math.inf)[:, 0] & ~bad
    logZ[empty], H[empty] = -math.inf, 0.0
    lp[empty] = -math.inf
    logZ[bad], H[bad], lp[bad] = math.nan, math.nan, math.nan
    order = torch.argsort(l + 0.0, dim=1, descending=True, stable=True)
    place = torch.empty_like(order).scatter_(1, order, torch.arange(V).expand(rows, V))
    got = {"logZ": logZ, "entropy": H, "top_ids": order[:, :n_top].clone(), "top_logprobs": lp.gather(1, order[:, :n_top])}
    got["top_ids"][bad] = -1
    if tokens is not None:
        t = tokens.cpu().long()
        inside = (t >= 0) & (t < V)
        at = t.clamp(0, V - 1)
        got["logprob"] = torch.where(inside, lp.gather(1, at), torch.where(t == -1, 0.0, math.nan))
        got["rank"] = torch.where(inside & ~bad[:, None], place.gather(1, at), -1)
    return got


def slack(logits, V):
    """Bound on |error| of a fp32 log-sum-exp of this kernel, per row.  A thread adds at most ceil(V / (8 * 256)) groups of eight
    entries, pairwise inside a group (4 additions in either half, 1 across), and 5 + 3 + 7 merges follow: that many roundings of
    2^-24 relative to the sum; each exponential is off by 2^-22 (ex2.approx: 2 units in the last place) and by the rounding of
    its argument, d log2 e, twice 2^-24 |d|, which counts with weight e^d |d| <= 0.37 per unit of the largest term and with
    |d| e^d summed, at most the entropy, over all (<= ln V); then ln s and m + ln s are rounded."""
    n = -(-V // 2048) + 20
    E = n * 2.0 ** -24 + 2.0 ** -22 + 2 * 2.0 ** -24 * math.log(V + 1)
    big = torch.where(logits.isfinite(), logits.double().abs(), 0.0).amax(dim=1).cpu() + math.log(V + 1)
    return E, big


def check(out, ref, logits, V, tokens=None, n_top=0, sums=True):
    E, big = slack(logits, V)
    flat = lambda t, *s: t.reshape(-1, *s).cpu()             # noqa: E731

    def close(got, want, tol):
        got = got.double()
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got.isinf(), want.isinf())
        fine = want.isfinite()
        assert (got[~fine & ~want.isnan()] == want[~fine & ~want.isnan()]).all()
        err = (got - want).abs()
        tol = tol.expand_as(err) if torch.is_tensor(tol) else torch.full_like(err, tol)
        worst = float((err - tol)[fine].max()) if fine.any() else -1.0
        assert worst <= 0, worst

    # logZ = m + ln s: E, and two roundings relative to the result; so (l - m) - ln s for a log probability
    tol = E + 2 * 2.0 ** -24 * big
    if sums:
        close(flat(out.logZ), ref["logZ"], tol)
        # H = ln s - t / s: s and t are off by E relative (t by its own weights |d| e^d as well: 2 E), |t / s| <= ln V
        close(flat(out.entropy), ref["entropy"], E * (1 + 3 * math.log(V + 1)) + 4 * 2.0 ** -24 * math.log(V + 1))
    if tokens is not None:
        T = ref["logprob"].shape[1]
        close(flat(out.logprob).reshape(-1, T), ref["logprob"], (tol + 2.0 ** -24 * big)[:, None])
        if out.rank is not None:
            assert torch.equal(flat(out.rank).reshape(-1, T).long(), ref["rank"])
    if n_top:
        assert torch.equal(flat(out.top_ids, n_top).long(), ref["top_ids"])
        close(flat(out.top_logprobs, n_top), ref["top_logprobs"], (tol + 2.0 ** -24 * big)[:, None])


def same_but_for_rounding(given, own, logits):
    """l - logZ under a given logZ = m + ln s against (l - m) - ln s: two roundings each, none of a number above
    max |l| + |logZ| <= 2 max |l| + ln V."""
    big = 2 * float(logits.double().abs().max()) + math.log(logits.shape[1])
    return bool(((given - own).abs().nan_to_num(0.0) <= 4 * 2.0 ** -24 * big).all())


def make(rows, V, dtype, seed, pad=0, spread=2.5, lead=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((rows * (V + pad) + lead,), math.nan, dtype=dtype, device="cuda")
    view = buf[lead:].view(rows, V + pad)
    view[:, :V] = (torch.randn((rows, V), generator=g, device="cuda") * spread).to(dtype)
    return view[:, :V]                                       # (what lies between the rows is NaN)


def some_tokens(logits, T, seed):
    rows, V = logits.shape
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(0, V, (rows, T), generator=g, device="cuda", dtype=torch.int32)
    if T > 1:
        t[:, 0] = logits.float().argmax(dim=1)
        t[::3, T - 1] = -1
    return t


# ------------------------------------------------------------------------------------------------ results
@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 2), (5, 7), (2, 8), (7, 9), (4, 33), (9, 255), (6, 2048), (3, 2049), (5, 4097),
                                    (2, 16384), (130, 1000), (700, 513), (5, 32000), (33, 50003), (2, 128256), (3, 600001)])
def test_rows_of_all_sizes(rows, V, dtype):
    n = min(V, 32)
    for pad, lead, n_top, T in ((0, 0, n, 1), (3, 1, min(5, n), 3), (1, 5, 0, 2), (8, 0, 1, 0)):
        l = make(rows, V, dtype, rows * 1000 + V, pad, lead=lead)
        t = some_tokens(l, T, V) if T else None
        out = binding.hola_token_logprobs(l, t, n_top=n_top)
        check(out, reference(l, t, n_top), l, V, t, n_top)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n_top", [1, 2, 8, 20, 31, 32])
def test_ties_go_to_the_lowest_id(dtype, n_top):
    V, rows = 9001, 12
    g = torch.Generator(device="cuda").manual_seed(n_top)
    l = torch.randint(-3, 4, (rows, V), generator=g, device="cuda").to(dtype)      # thousands of equal entries
    l[1] = 2.0                                                # one value throughout
    l[2] = -math.inf
    l[3] = -0.0
    l[3, ::2] = 0.0                                           # one zero only
    l[4] = torch.arange(V, device="cuda").to(dtype)           # rising: the best all in the last groups
    l[5] = -torch.arange(V, device="cuda").to(dtype)
    l[6, :] = -5.0
    l[6, 4096:4160] = 1.0                                     # the best all in neighbouring groups
    l[7] = torch.finfo(dtype).min                             # a mask of the lowest value throughout
    l[8, 5:] = torch.finfo(dtype).min
    l[9, 3:] = -math.inf                                      # fewer left than asked for
    l[10] = -5.0
    l[10, 17::2048] = torch.arange(len(range(17, V, 2048)), device="cuda").to(dtype)   # many in one thread's groups
    t = some_tokens(l, 4, 5)
    t[2, 1], t[9, 0], t[9, 1] = 77, 2, 6
    out = binding.hola_token_logprobs(l, t, n_top=n_top)
    ref = reference(l, t, n_top)
    check(out, ref, l, V, t, n_top)
    mine = out.rank[:, 0].cpu()
    assert (mine >= 0).all()
    for r in range(rows):
        if 0 <= mine[r] < n_top:
            assert out.top_ids[r, mine[r]] == t[r, 0]


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 3000, 70001])
def test_masks_of_any_depth_and_logits_of_any_size(dtype, V):
    """Masks of -1e4 .. -1e38 in single entries, in whole groups and throughout, and logits far from zero: sums are of differences."""
    sizes = [1e4, 4e5, 6e5, 1e7, 1e9, 1e12, 1e20, 1e30, 9e36, 2e37, 2e38]
    l = make(5 * len(sizes), V, dtype, V)
    for i, big in enumerate(sizes):
        l[5 * i, 1::2] = -big
        l[5 * i + 1, V // 3:] = -big
        l[5 * i + 2] = -big                                   # all of it
        l[5 * i + 3] = l[5 * i + 3] + big                     # (where the type has it: a handful of steps)
        l[5 * i + 4] = -big
        l[5 * i + 4, V // 2] = big
    t = some_tokens(l, 2, 3)
    out = binding.hola_token_logprobs(l, t, n_top=9)
    ref = reference(l, t, 9)
    for name in ("logprob", "top_logprobs"):    # -4e38 (2e38 below a maximum of 2e38) has no fp32 of its own: it rounds to -inf
        ref[name] = torch.where(ref[name] < -torch.finfo(torch.float32).max, -torch.inf, ref[name])
    check(out, ref, l, V, t, 9)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 3000, 70001])
def test_entries_beside_masks_of_any_depth_keep_their_precision(dtype, V):
    """How deep a mask is puts nothing on the entries beside it.  A log probability is (l - m) - ln s: ln s is off by s's relative error E,
    by 2^-22 for each exponential that a thread's sums pass through afterwards (to its own maximum, the warp's, the CTA's, the row's) and
    by logf's 2 x 2^-24 of itself (<= ln V); two more roundings are relative to the result, which is no smaller than either operand
    but for ln s.  logZ = m + ln s: one rounding of the result."""
    U = 2.0 ** -24
    sizes = [0.0, 1e4, 4e5, 1e7, 1e9, 1e20, 1e38, torch.finfo(torch.float32).max, math.inf]
    if dtype == torch.float16:
        sizes = [0.0, 300.0, 1e4, 65504.0, math.inf]
    l = make(4 * len(sizes), V, dtype, V + 1)
    for i, big in enumerate(sizes):
        big = min(big, torch.finfo(dtype).max) if big < math.inf else big
        if big:
            l[4 * i, 1::2] = -big
            l[4 * i + 1, V // 3:] = -big
            l[4 * i + 2, torch.arange(V, device="cuda") % 16 != 5] = -big          # one entry in a group or two
            l[4 * i + 3, :V - 3] = -big                                            # three entries left
    t = some_tokens(l, 3, 4)
    out, ref = binding.hola_token_logprobs(l, t, n_top=min(20, V)), reference(l, t, min(20, V))
    ln_V = math.log(V + 1)
    E = slack(l, V)[0] + 4 * 2.0 ** -22 + 2 * U * ln_V
    big = torch.finfo(torch.float32).max
    for name in ("logZ", "logprob", "top_logprobs"):
        got, want = getattr(out, name).double().cpu().reshape(ref[name].shape), ref[name]
        want = torch.where(want < -big, -math.inf, want)
        fine = want.isfinite()
        assert torch.equal(got[~fine], want[~fine])
        assert ((got - want).abs() <= E + (1 if name == "logZ" else 2) * U * (want.abs() + ln_V))[fine].all(), name
    assert torch.equal(out.rank.cpu().long(), ref["rank"]) and torch.equal(out.top_ids.cpu().long(), ref["top_ids"])


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [62, 3001, 70001])
@pytest.mark.parametrize("kept", [1.0, 0.99, 0.5])
def test_masked_entries_among_logits_far_from_zero(dtype, V, kept):
    """Groups that hold a masked entry, or a row's end, add up with those that hold none, about one and the same point."""
    centre = torch.tensor([-4e5, -1e5, -1e4, -300.0, 300.0, 1e4, 4e4, 1e5, 4e5], device="cuda")[:, None]
    centre = centre.clamp(-6e4, 6e4) if dtype == torch.float16 else centre
    g = torch.Generator(device="cuda").manual_seed(V)
    l = (centre + 3 * torch.randn((len(centre), V), generator=g, device="cuda")).to(dtype)
    l[torch.rand(l.shape, generator=g, device="cuda") > kept] = -torch.inf
    t = some_tokens(l, 2, 8)
    check(binding.hola_token_logprobs(l, t, n_top=5), reference(l, t, 5), l, V, t, 5)


@gpu
@pytest.mark.parametrize("span", [12.0, 40.0, 2e5, 2e6])
def test_a_maximum_that_rises_through_large_numbers(span):
    """Rows that climb, a little in every group of a thread, from below a large number (of either sign) to above it."""
    rows, V = 230, 66000
    g = torch.Generator(device="cuda").manual_seed(7)
    ramp = torch.arange(V, device="cuda") / V - 0.5
    centre = 5e5 + (torch.rand((rows, 1), generator=g, device="cuda") - 0.5) * 10
    centre[::2] *= -1
    l = centre + span * ramp + torch.randn((rows, V), generator=g, device="cuda")
    check(binding.hola_token_logprobs(l, some_tokens(l, 1, 5), n_top=5), reference(l, some_tokens(l, 1, 5), 5), l, V, some_tokens(l, 1, 5), 5)


@gpu
@pytest.mark.parametrize("rows", [6, 230])          # a cluster per row; one CTA, long rows of which are taken two groups at a time
@pytest.mark.parametrize("dtype", DTYPES)
def test_best_entries_gathered_in_few_threads(dtype, rows):
    """The best entries all lie in one thread's groups, in one warp's, in one CTA's part: lists fill up and are merged."""
    V, n_top = (70000, 32) if rows == 6 else (66000, 20)
    l = make(rows, V, dtype, 3, spread=0.5)
    at = torch.arange(V, device="cuda")
    l[0, (at // 8) % 256 == 37] += 20
    l[1, ((at // 8) % 256) // 32 == 6] += 20
    l[2, at > V - 300] += 20
    l[3, (at // 8) % 256 < 40] += 20
    l[4] = (at.float() / 7).to(dtype) if dtype != torch.float16 else (at.float() / 70).to(dtype)
    l[5, 12345] += 30
    t = some_tokens(l, 2, 9)
    out = binding.hola_token_logprobs(l, t, n_top=n_top)
    some = slice(0, 8)                                        # (the others: as the first ones' kind, less to compare)
    assert all(torch.equal(a, b) for a, b in zip((out.top_ids[some], out.rank[some]),
                                                 (lambda o: (o.top_ids, o.rank))(binding.hola_token_logprobs(l[some], t[some], n_top=n_top))))
    ref = reference(l[some], t[some], n_top)
    part = binding.TokenLogprobs(**{f: getattr(out, f)[some] for f in ("logprob", "rank", "entropy", "logZ", "top_ids", "top_logprobs")})
    check(part, ref, l[some], V, t[some], n_top)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_without_a_distribution(dtype):
    V, rows, n_top = 5003, 6, 6
    l = make(rows, V, dtype, 11)
    l[1, 4000] = math.nan
    l[2, 0] = math.inf
    l[3, V - 1] = -math.nan
    l[4] = -math.inf
    l[5, 17] = math.nan
    l[5, 18] = math.inf
    t = some_tokens(l, 3, 4)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = binding.hola_token_logprobs(l, t, n_top=n_top, status=status)
    check(out, reference(l, t, n_top), l, V, t, n_top)
    assert status.item() == binding.FLAG_BAD_LOGIT
    logZ = torch.full((rows,), 3.0, device="cuda")
    given = binding.hola_token_logprobs(l, t, n_top=n_top, logZ=logZ)
    assert given.entropy is None and given.logZ is None
    assert (given.top_ids[[1, 2, 3, 5]] == -1).all() and (given.rank[[1, 2, 3, 5]] == -1).all()
    assert (given.rank[0] == out.rank[0]).all() and (given.top_ids[[0, 4]] == out.top_ids[[0, 4]]).all()


@gpu
def test_tokens_that_are_none_and_tokens_that_cannot_be():
    V = 1000
    l = make(4, V, torch.float32, 1)
    t = torch.tensor([[0, -1], [V - 1, V], [-2, 5], [2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device="cuda")
    for want_rank in (True, False):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = binding.hola_token_logprobs(l, t, want_rank=want_rank, status=status)
        check(out, reference(l, t, 0), l, V, t)
        assert status.item() == binding.FLAG_BAD_TOKEN
        status.zero_()
        given = binding.hola_token_logprobs(l, t, logZ=out.logZ, want_rank=want_rank, status=status)
        assert torch.equal(given.logprob.isnan(), out.logprob.isnan())
        assert same_but_for_rounding(given.logprob, out.logprob, l) and status.item() == binding.FLAG_BAD_TOKEN
    status.zero_()
    binding.hola_token_logprobs(l, t[:1].expand(4, 2).contiguous(), status=status)
    assert status.item() == 0


@gpu
@pytest.mark.parametrize("T", [4, 5, 9, 40])
@pytest.mark.parametrize("want_rank", [True, False])
def test_many_tokens_per_row(T, want_rank):
    l = make(21, 6007, torch.bfloat16, T)
    t = some_tokens(l, T, T)
    out = binding.hola_token_logprobs(l, t, n_top=4, want_rank=want_rank)
    assert (out.rank is not None) == want_rank
    check(out, reference(l, t, 4), l, 6007, t, 4)
    logZ = out.logZ.clone()
    again = binding.hola_token_logprobs(l, t, logZ=logZ, want_rank=want_rank)
    assert same_but_for_rounding(again.logprob, out.logprob, l) and (not want_rank or torch.equal(again.rank, out.rank))


@gpu
@pytest.mark.parametrize("k", [0, 1, 5])
@pytest.mark.parametrize("n_top,want_rank", [(0, False), (0, True), (7, False), (7, True)])
def test_emitted_tokens_of_a_verify_call(k, n_top, want_rank):
    B, V = 13, 4099
    l = make(B * (k + 1), V, torch.float32, k)
    g = torch.Generator(device="cuda").manual_seed(k + 5)
    draft = torch.randint(0, V, (B, k), generator=g, device="cuda", dtype=torch.int32)
    nxt = torch.randint(0, V, (B,), generator=g, device="cuda", dtype=torch.int32)
    n = torch.randint(0, k + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    at = torch.arange(k + 1, device="cuda")[None]
    tok = torch.cat([draft, nxt[:, None]], 1)
    tok = torch.where(at == n[:, None], nxt[:, None], tok)
    tok = torch.where(at <= n[:, None], tok, -1).to(torch.int32)
    ref = reference(l, tok.reshape(-1, 1), n_top)
    logZ = ref["logZ"].float().cuda().reshape(B, k + 1)
    gone = (tok.reshape(-1) < 0).cpu()
    ref["top_ids"][gone] = -1
    ref["top_logprobs"][gone] = 0.0
    out = binding.hola_token_logprobs(l.view(B, k + 1, V), n_top=n_top, logZ=logZ, emitted=(draft, n, nxt), want_rank=want_rank)
    assert out.logprob.shape == (B, k + 1) and out.entropy is None
    check(out, ref, l, V, tok, n_top, sums=False)
    # an accept length that cannot be spoils its sequence, and says so
    n2 = n.clone()
    n2[3], n2[4] = k + 1, -1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    worse = binding.hola_token_logprobs(l.view(B, k + 1, V), n_top=n_top, logZ=logZ, emitted=(draft, n2, nxt), want_rank=want_rank,
                                        status=status)
    assert status.item() == binding.FLAG_BAD_TOKEN and worse.logprob[3:5].isnan().all()
    keep = [b for b in range(B) if b not in (3, 4)]
    assert torch.equal(worse.logprob[keep], out.logprob[keep])
    if n_top:
        assert (worse.top_ids[3:5] == -1).all() and worse.top_logprobs[3:5].isnan().all()


@gpu
def test_shapes_strides_and_outputs_of_the_caller():
    V, k1, B = 777, 3, 5
    buf = make(2 * B * k1, V, torch.float16, 2, pad=7)
    every_other = buf[::2].unflatten(0, (B, k1))              # [B, k1, V], rows 2 (V + 7) apart
    t = some_tokens(buf[::2].contiguous(), 1, 3).view(B, k1)
    out = binding.hola_token_logprobs(every_other, t, n_top=3)
    assert out.logprob.shape == (B, k1) and out.top_ids.shape == (B, k1, 3)
    check(out, reference(buf[::2], t.view(-1, 1), 3), buf[::2], V, t, 3)
    last = buf[::2][-1]
    one = binding.hola_token_logprobs(last, t[-1, -1].reshape(()), n_top=3)           # a single row
    assert one.logprob.shape == () and torch.equal(one.top_ids, out.top_ids[-1, -1])
    same = binding.hola_token_logprobs(last.expand(6, V), n_top=3)                    # a broadcast row
    assert torch.equal(same.top_ids, out.top_ids[-1, -1].expand(6, 3))
    for f in (out.logprob, out.rank, out.top_ids, out.top_logprobs, out.entropy, out.logZ):
        f.zero_()
    again = binding.hola_token_logprobs(every_other, t, n_top=3, out=out)
    assert again.logprob.data_ptr() == out.logprob.data_ptr()
    check(out, reference(buf[::2], t.view(-1, 1), 3), buf[::2], V, t, 3)
    none = binding.hola_token_logprobs(buf[:0], torch.zeros((0,), dtype=torch.int32, device="cuda"), n_top=2)
    assert none.logprob.shape == (0,) and none.top_ids.shape == (0, 2)


@gpu
def test_offsets_beyond_32_bits():
    V = 3001
    buf = torch.zeros(3 * 1_200_000_000 + V, dtype=torch.bfloat16, device="cuda")
    rows = buf.as_strided((4, V), (1_200_000_000, 1))
    src = make(4, V, torch.bfloat16, 8)
    rows.copy_(src)
    t = some_tokens(src, 2, 1)
    check(binding.hola_token_logprobs(rows, t, n_top=9), reference(src, t, 9), src, V, t, 9)


@gpu
def test_counts_beyond_32_bits_are_refused():
    """(2^32 + 4 rows or entries are not 4.)"""
    many = 2 ** 32 + 4
    for l, t in ((torch.zeros((1, 9), device="cuda").expand(many, 9), torch.zeros(1, dtype=torch.int32, device="cuda").expand(many)),
                 (torch.zeros(many, dtype=torch.bfloat16, device="cuda"), torch.zeros((), dtype=torch.int32, device="cuda")),
                 (torch.zeros((2 ** 31, 1), dtype=torch.bfloat16, device="cuda"), None)):
        with pytest.raises(binding.HolaError, match="32 bits"):
            binding.hola_token_logprobs(l, t)


@gpu
def test_nothing_outside_the_outputs_is_written():
    rows, V, n = 9, 3001, 5
    l = make(rows, V, torch.float32, 5)
    t = some_tokens(l, 1, 5)
    want = binding.hola_token_logprobs(l, t, n_top=n)
    room = {}
    for name in ("logprob", "rank", "entropy", "logZ", "top_ids", "top_logprobs"):
        w = getattr(want, name)
        buf = torch.full((w.numel() + 64,), 12345, dtype=w.dtype, device="cuda")
        room[name] = (buf, buf[32:32 + w.numel()].view(w.shape))
    binding.hola_token_logprobs(l, t, n_top=n, out=binding.TokenLogprobs(**{k: v for k, (_, v) in room.items()}))
    for name, (buf, v) in room.items():
        assert torch.equal(v, getattr(want, name))
        assert (buf[:32] == 12345).all() and (buf[32 + v.numel():] == 12345).all()


@gpu
def test_streams_graphs_and_repeated_calls():
    l = make(40, 32000, torch.bfloat16, 1)
    t = some_tokens(l, 1, 1)
    want = binding.hola_token_logprobs(l, t, n_top=20)
    fields = ("logprob", "rank", "entropy", "logZ", "top_ids", "top_logprobs")
    same = lambda a, b: all(torch.equal(getattr(a, f), getattr(b, f)) for f in fields)     # noqa: E731
    assert same(want, binding.hola_token_logprobs(l, t, n_top=20))                        # the same bits every time
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [binding.hola_token_logprobs(l, t, n_top=20, stream=s) for s in (side, None, side, None)]   # two at once
    torch.cuda.synchronize()
    assert all(same(want, o) for o in outs)
    src = l.contiguous().clone()
    out = binding.hola_token_logprobs(src, t, n_top=20)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        src2 = src * 1                                        # a kernel right in front, whose results are read
        binding.hola_token_logprobs(src2, t, n_top=20, out=out)
    for r in range(3):
        src.copy_(l.roll(r, dims=0))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.top_ids, want.top_ids.roll(r, dims=0)) and torch.equal(out.logZ, want.logZ.roll(r, dims=0))


# ------------------------------------------------------------------------------------------------ refusals
def _args(**kw):
    a = binding.hola_logprobs_args()
    base = dict(rows=2, V=100, T=1, n_top=3, logits=4096, row_stride=100, l_dtype=0, tokens=4096, logprob=4096, top_ids=4096,
                top_logprobs=4096)
    base.update(kw)
    for k, v in base.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 1), (dict(V=0), 1), (dict(T=-1), 1), (dict(n_top=-1), 1), (dict(row_stride=-1), 1), (dict(l_dtype=3), 1),
    (dict(l_dtype=-1), 1), (dict(n_top=33), 2), (dict(V=2, row_stride=2), 2), (dict(logits=None), 1), (dict(logits=4097), 1),
    (dict(logits=4098), 1), (dict(logits=4097, l_dtype=1), 1), (dict(tokens=None), 1), (dict(logprob=None), 1), (dict(T=0), 1),
    (dict(top_ids=None), 1), (dict(top_logprobs=None), 1), (dict(n_top=0), 1), (dict(logZ_in=4096, logZ=4096), 1),
    (dict(logZ_in=4096, entropy=4096), 1), (dict(T=0, logprob=None, n_top=0, top_ids=None, top_logprobs=None), 1),
    (dict(T=0, logprob=None, rank=4096), 1), (dict(rows=2 ** 31 - 1), 2), (dict(V=2 ** 31 - 1), 2),
    # the emitted form
    (dict(accept_len=4096, next_tok=4096, logZ_in=4096), 1), (dict(tokens=None, accept_len=4096, next_tok=4096), 1),
    (dict(tokens=None, next_tok=4096, logZ_in=4096), 1), (dict(tokens=None, accept_len=4096, logZ_in=4096), 1),
    (dict(tokens=None, accept_len=4096, next_tok=4096, logZ_in=4096, k=2, draft_tok=4096), 1),
    (dict(tokens=None, accept_len=4096, next_tok=4096, logZ_in=4096, k=1), 1),
    (dict(tokens=None, accept_len=4096, next_tok=4096, logZ_in=4096, k=-1), 1),
    (dict(tokens=None, accept_len=4096, next_tok=4096, logZ_in=4096, T=2), 1),
    (dict(tokens=None, draft_tok=4096, logZ_in=4096), 1)])
def test_refused_by_the_library(change, status):
    lib = binding.load_library()
    assert lib.hola_token_logprobs(ctypes.byref(_args(**change)), None) == status


def test_no_rows_is_no_work_and_no_device_needed():
    lib = binding.load_library()
    assert lib.hola_token_logprobs(ctypes.byref(_args(rows=0)), None) == 0
    assert lib.hola_token_logprobs(None, None) == 1
    assert ctypes.sizeof(binding.hola_logprobs_args) == 16 + 8 + 8 + 8 + 12 * 8


@gpu
def test_refused_by_the_binding():
    l = torch.zeros((2, 3, 50), device="cuda")
    t = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    call = binding.hola_token_logprobs
    for args, kw in [((l.double(), t), {}), ((l.cpu(), t), {}), ((l, t.long()), {}), ((l, t.cpu()), {}), ((l, t[:1]), {}),
                     ((l, t[:, :, None, None]), {}), ((l, t), {"n_top": 33}), ((l, t), {"n_top": 51}), ((l, t), {"n_top": -1}),
                     ((l.transpose(1, 2), None), {"n_top": 1}), ((l.transpose(0, 1), t.T), {}), ((l[:, :, ::2], t), {}),
                     ((l, t), {"logZ": torch.zeros(6, device="cuda")}), ((l, t.T.contiguous().T), {}),
                     ((l, t), {"emitted": (t[:, :2], t[:, 0], t[:, 0])}), ((l,), {"emitted": (t[:, :2], t[:, 0], t[:, 0])}),
                     ((l, t), {"out": binding.TokenLogprobs(None, None, None, None, None, None)}),
                     ((l, t), {"status": torch.zeros(2, dtype=torch.int32, device="cuda")})]:
        with pytest.raises(binding.HolaError):
            call(*args, **kw)
