"""A beam search's step: the selection against the definition in 64 bits, equal to the bit, and the reordering of states."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2506_18952_b200 import binding

gpu = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


# ------------------------------------------------------------------------------------------------ selection: reference
def reference(logits, logZ, score, n, finished=None, end_token=-1, weight=None, keep_slots=False):
    """score, parent, token, finished of every sequence, candidate by candidate in 64 bits."""
    B, W, V = logits.shape
    l, z, s = logits.cpu().double().numpy(), logZ.cpu().double().numpy(), score.cpu().double().numpy()
    f = finished.cpu().numpy() if finished is not None else np.zeros((B, W), bool)
    wt = weight.cpu().double().numpy() if weight is not None else np.ones((B, W))
    out = []
    for b in range(B):
        keys, cs, beams, ls, ids = [], [], [], [], []
        for w in range(W):
            if not s[b, w] < math.inf or s[b, w] == -math.inf or not (0 < wt[b, w] < math.inf):
                continue
            if f[b, w]:
                c, x, v = np.array([s[b, w]]), np.zeros(1), np.array([end_token])
            else:
                if not z[b, w] < math.inf or z[b, w] == -math.inf or not (l[b, w] < math.inf).all():
                    continue
                v = np.nonzero(l[b, w] > -math.inf)[0]
                x = l[b, w][v]
                c = (s[b, w] - z[b, w]) + x
            keys.append(c * wt[b, w]); cs.append(c); beams.append(np.full(len(v), w)); ls.append(x); ids.append(v)
        cat = lambda t, kind: np.concatenate(t).astype(kind) if t else np.zeros(0, kind)          # noqa: E731
        key, c, beam, x, v = cat(keys, float), cat(cs, float), cat(beams, int), cat(ls, float), cat(ids, int)
        order = np.lexsort((v, -x, beam, -key))[:n]
        got = [(float(c[i]), int(beam[i]), int(v[i])) for i in order] + [(-math.inf, -1, -1)] * (n - len(order))
        if keep_slots:
            slots, later = [None] * n, []
            for g in got:
                if g[1] >= 0 and slots[g[1]] is None:
                    slots[g[1]] = g
                else:
                    later.append(g)
            it = iter(later)
            got = [g if g is not None else next(it) for g in slots]
        out.append(got)
    t = lambda k, kind: torch.tensor([[g[k] for g in row] for row in out], dtype=kind).reshape(B, n)          # noqa: E731
    parent, token = t(1, torch.int32), t(2, torch.int32)
    ended = torch.tensor([[g[1] >= 0 and (bool(f[b, g[1]]) or (end_token >= 0 and g[2] == end_token)) for g in row] for b, row in enumerate(out)],
                         dtype=torch.bool).reshape(B, n)
    return t(0, torch.float64).float(), parent, token, ended


def same(out, ref):
    assert torch.equal(out.parent.cpu(), ref[1]), (out.parent.cpu() - ref[1]).nonzero()[:4]
    assert torch.equal(out.token.cpu(), ref[2])
    assert torch.equal(out.score.cpu(), ref[0])
    if out.finished is not None:
        assert torch.equal(out.finished.cpu(), ref[3])


def make(B, W, V, dtype, seed, pad=0, lead=0, spread=2.5):
    """Logits whose rows lie `pad` entries apart and `lead` from the start of the buffer (NaN in between), logZ, scores."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((B * W * (V + pad) + lead,), math.nan, dtype=dtype, device="cuda")
    view = buf[lead:].view(B, W, V + pad)[:, :, :V]
    view.copy_((torch.randn((B, W, V), generator=g, device="cuda") * spread).to(dtype))
    return view, *beams(view, g)


def beams(logits, g=None):
    g = g or torch.Generator(device="cuda").manual_seed(1)
    B, W, _ = logits.shape
    logZ = torch.logsumexp(logits.double(), dim=2).float()
    return logZ, -10.0 - 3.0 * torch.rand((B, W), generator=g, device="cuda")


# ------------------------------------------------------------------------------------------------ selection: results
@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,W,V", [(1, 1, 1), (2, 3, 2), (1, 2, 7), (3, 1, 8), (2, 4, 9), (5, 2, 33), (1, 32, 17), (4, 7, 255), (3, 5, 2048),
                                   (2, 3, 2049), (150, 2, 300), (70, 4, 1000), (1, 4, 32000), (8, 6, 5001), (2, 2, 50003), (1, 3, 128256), (1, 1, 600001)])
def test_sequences_of_all_sizes(B, W, V, dtype):
    for pad, lead, n in ((0, 0, W), (3, 1, min(2 * W, 32)), (8, 5, 32), (1, 0, 1)):
        l, z, s = make(B, W, V, dtype, 100 * W + V, pad, lead)
        same(binding.hola_beam_select(l, z, s, n), reference(l, z, s, n))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 4, 9, 20, 21, 32])
def test_equal_candidates_go_by_beam_logit_and_id(dtype, n):
    W, V, B = 4, 9001, 12
    g = torch.Generator(device="cuda").manual_seed(n)
    l = torch.randint(-3, 4, (B, W, V), generator=g, device="cuda").to(dtype)      # thousands of equal entries
    l[1] = 2.0                                                # one value throughout
    l[2] = torch.arange(V, device="cuda").to(dtype)           # rising: the best all in the last groups
    l[3] = -torch.arange(V, device="cuda").to(dtype)
    l[4] = -5.0
    l[4, :, 4096:4160] = 1.0                                  # the best all in neighbouring groups
    l[5] = -0.0
    l[5, :, ::2] = 0.0                                        # one zero only
    l[6] = -5.0
    l[6, 2, 17::2048] = torch.arange(len(range(17, V, 2048)), device="cuda").to(dtype)     # many in one thread's groups
    l[7] = torch.finfo(dtype).min                             # a mask of the lowest value throughout
    l[8, :, 5:] = torch.finfo(dtype).min
    l[9, 1:] = l[9, :1]                                       # the beams are alike
    z, s = beams(l)
    z[7:9], s[7:9] = 3.0, -7.0                                # (no log-sum-exp of their own worth the name)
    s[9], z[9] = -4.0, 1.5
    s[10], z[10] = -1.0, 0.0
    for keep in ([False, True] if n == W else [False]):
        same(binding.hola_beam_select(l, z, s, n, keep_slots=keep), reference(l, z, s, n, keep_slots=keep))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 3000, 50003])
def test_masks_dead_beams_and_rows_without_entries(dtype, V):
    W, n = 5, 10
    l, z, s = make(10, W, V, dtype, V, pad=2)
    l[0, :, 3:] = -math.inf                                   # three entries a beam
    l[1, 1:] = -math.inf                                      # rows that have none
    l[2] = -math.inf                                          # nor the sequence
    l[3, :, torch.arange(V, device="cuda") % 16 != 5] = -math.inf
    l[4, :, ::2] = torch.finfo(dtype).min
    l[5, :, : V - 2] = -math.inf
    l[6, 2, 7:] = -math.inf
    z = torch.logsumexp(l.double(), dim=2).float()
    s[6] = -math.inf                                          # one live beam, as behind a prompt
    s[6, 2] = 0.0
    s[7] = -math.inf                                          # none
    s[8, ::2] = -math.inf
    s[9, 1] = -math.inf
    l[9, 1] = math.nan                                        # (not read)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = binding.hola_beam_select(l, z, s, n, status=status)
    same(out, reference(l, z, s, n))
    assert (out.parent[2] == -1).all() and (out.parent[7] == -1).all() and (out.score[7] == -math.inf).all()
    assert status.item() == 0


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [9, 4000, 60001])
def test_beams_without_a_distribution_are_set_aside_and_reported(dtype, V):
    """What a bad row holds reaches neither the other beams of its sequence nor other sequences."""
    W, n = 6, 12
    clean, z, s = make(9, W, V, dtype, V + 5)
    for where in (0, V // 2, V - 1):
        l, zz, ss = clean.clone(), z.clone(), s.clone()
        l[1, 2] += 8.0                                        # (its entries would come first)
        l[1, 2, where] = math.nan
        l[2, 0, where] = math.inf
        l[3, 1:5, where] = math.nan
        l[4, :, where] = math.inf
        zz[5, 3] = math.nan
        zz[6, 1] = math.inf
        ss[7, 4] = math.nan
        ss[8, 0] = math.inf
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        same(binding.hola_beam_select(l, zz, ss, n, status=status), reference(l, zz, ss, n))
        assert status.item() == binding.FLAG_BAD_LOGIT


@gpu
def test_logits_and_scores_of_any_size():
    """Offsets and masks up to the ends of fp32; keys are compared in 64 bits, so the order is the definition's there too."""
    W, V, n = 4, 2000, 8
    sizes = [1e4, 1e7, 1e12, 1e20, 1e29, 1e31, 1e36, 2e38]
    l, z, s = make(4 * len(sizes), W, V, torch.float32, 3)
    for i, big in enumerate(sizes):
        l[4 * i, :, 1::2] = -big
        l[4 * i + 1] += big
        s[4 * i + 2] -= big
        z[4 * i + 3] = torch.tensor([big, -big, 1.0, 0.0])
    same(binding.hola_beam_select(l, z, s, n), reference(l, z, s, n))
    w = torch.full_like(s, 0.5)
    w[:, 1] = 3.0
    w[:, 2] = 1e-30
    w[:, 3] = 1e30
    same(binding.hola_beam_select(l, z, s, n, weight=w), reference(l, z, s, n, weight=w))


@gpu
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("V", [50, 7000])
def test_ended_beams_and_normalised_keys(V, keep):
    W, B = 6, 40
    n = W if keep else 11
    l, z, s = make(B, W, V, torch.float32, V + 7)
    g = torch.Generator(device="cuda").manual_seed(4)
    f = torch.rand((B, W), generator=g, device="cuda") < 0.4
    f[0], f[1] = True, False
    l[f] = math.nan                                           # (rows of ended beams are not read)
    z[f] = math.nan
    l[2:8, :, 3] += 9.0                                       # the end token comes up
    z = torch.where(f, z, torch.logsumexp(l.double(), dim=2).float())
    s[3] = s[3, :1]
    w = torch.rand((B, W), generator=g, device="cuda") + 0.2
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for weight in (None, w):
        out = binding.hola_beam_select(l, z, s, n, finished=f, end_token=3, weight=weight, keep_slots=keep, status=status)
        same(out, reference(l, z, s, n, f, 3, weight, keep))
        assert out.finished.any() and not out.finished.all()
    assert status.item() == 0
    w[5, 1], w[6, 0], w[7, 2], w[8, 3] = 0.0, -1.0, math.nan, math.inf
    same(binding.hola_beam_select(l, z, s, n, finished=f, end_token=3, weight=w, keep_slots=keep, status=status), reference(l, z, s, n, f, 3, w, keep))
    assert status.item() == binding.FLAG_BAD_LOGIT
    none = torch.zeros_like(f)
    same(binding.hola_beam_select(l[1:3], z[1:3], s[1:3], n, end_token=3, keep_slots=keep), reference(l[1:3], z[1:3], s[1:3], n, none[1:3], 3, None, keep))


@gpu
@pytest.mark.parametrize("keep", [False, True])
def test_children_stay_in_their_parents_places(keep):
    B, W, V = 64, 8, 400
    l, z, s = make(B, W, V, torch.float32, 5, spread=6.0)
    out = binding.hola_beam_select(l, z, s, keep_slots=keep)
    same(out, reference(l, z, s, W, keep_slots=keep))
    p = out.parent.cpu()
    stays = sum(int(p[b, i]) == i for b in range(B) for i in range(W))
    distinct = sum(len(set(p[b].tolist())) for b in range(B))
    assert stays == distinct if keep else stays < distinct    # every survivor, and only they


@gpu
def test_strides_and_entries_far_into_a_buffer():
    """Rows of [W, B, V] read as [B, W, V]; a sequence that begins more than 2^32 bytes into its buffer."""
    l, z, s = make(3, 4, 700, torch.float32, 8)
    turned = l.transpose(0, 1).contiguous().transpose(0, 1)
    same(binding.hola_beam_select(turned, z, s, 6), reference(l, z, s, 6))
    one = l[:, :1].expand(3, 4, 700)                          # the beams share a row
    z1 = z[:, :1].expand(3, 4).contiguous()
    same(binding.hola_beam_select(one, z1, s, 6), reference(one, z1, s, 6))
    apart, V = 2 ** 31 + 8, 1000
    buf = torch.empty(apart + 2 * V, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(buf, (2, 2, V), (apart, V, 1))
    far.copy_(l[:2, :2, :1].float() + torch.randn((2, 2, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) * 3)
    same(binding.hola_beam_select(far, *beams(far), 7), reference(far, *beams(far), 7))


# ------------------------------------------------------------------------------------------------ reordering: reference
def reordered(tensors, into, axes, positions, parent, used=None):
    got = []
    for x, to, axis, at in zip(tensors, into, axes, positions):
        x, new = x.cpu(), to.cpu().clone()
        for b, row in enumerate(parent.cpu().tolist()):
            for i, p in enumerate(row):
                if 0 <= p < x.shape[axis + 1]:
                    a, c = x.select(axis, b).select(axis, p), new.select(axis, b).select(axis, i)
                    if at is not None and used is not None:
                        d = at if at < axis else at - 2
                        m = min(max(int(used[b]), 0), a.shape[d])
                        a, c = a.narrow(d, 0, m), c.narrow(d, 0, m)
                    c.copy_(a)
        got.append(new)
    return got


def anything(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = math.prod(shape) * torch.empty(0, dtype=dtype).element_size()
    return torch.randint(0, 256, (n,), generator=g, device="cuda", dtype=torch.uint8).view(dtype).view(shape)


def some_parents(B, W, n, seed):
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(-1, W, (B, n), generator=g, dtype=torch.int32)
    if B > 2 and n == W:
        p[0] = torch.arange(W)                                # all stay
        p[1] = torch.arange(W).flip(0)                        # all swap
        p[2] = W - 1                                          # one survivor
    return p.cuda()


def equal(xs, ys):
    return all(torch.equal(x.cpu().contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(xs, ys, strict=True))


# ------------------------------------------------------------------------------------------------ reordering: results
@gpu
@pytest.mark.parametrize("W", [1, 2, 3, 4, 5, 8, 9, 16, 17, 32])
def test_states_in_the_order_of_their_parents(W):
    B = 5
    shapes = [((B, W), torch.int64, 0, None), ((B, W, 1), torch.uint8, 0, None), ((B, W, 7), torch.uint8, 0, 2), ((B, W, 40), torch.int64, 0, 2),
              ((B, W, 4096), torch.float32, 0, None), ((2, B, W, 3, 30, 16), torch.bfloat16, 1, 4), ((3, B, W, 21, 5), torch.float16, 1, 3),
              ((B, W, 2500, 6), torch.int32, 0, 2), ((2, 2, B, W, 9), torch.bool, 2, 4)]
    for into in (False, True):
        for used in (None, torch.tensor([0, 3, 100000, -4, 20], dtype=torch.int32, device="cuda")):
            xs = [anything(s, t, i) if t != torch.bool else anything(s, torch.uint8, i) > 127 for i, (s, t, _, _) in enumerate(shapes)]
            axes, positions = [s[2] for s in shapes], [s[3] for s in shapes]
            to = [torch.zeros_like(x) for x in xs] if into else xs
            parent = some_parents(B, W, W, W)
            want = reordered(xs, to, axes, positions, parent, used)
            states = binding.BeamStates(xs, axes, positions, to if into else None)
            binding.hola_beam_reorder(states, parent, used)
            assert equal(to, want)
            if not into:                                      # once more, from where they are now
                parent = some_parents(B, W, W, W + 40)
                want = reordered(xs, xs, axes, positions, parent, used)
                binding.hola_beam_reorder(states, parent, used)
                assert equal(xs, want)


@gpu
def test_other_numbers_of_beams_columns_and_layouts():
    B = 4
    x = anything((2, B, 1, 50, 8), torch.bfloat16, 1)         # from a prompt's one beam to six
    y = torch.zeros((2, B, 6, 50, 8), dtype=torch.bfloat16, device="cuda")
    parent = torch.zeros((B, 6), dtype=torch.int32, device="cuda")
    parent[1, 3] = -1
    used = torch.tensor([50, 1, 0, 17], dtype=torch.int32, device="cuda")
    want = reordered([x], [y], [1], [3], parent, used)
    binding.hola_beam_reorder(binding.BeamStates([x], 1, [3], [y]), parent, used)
    assert equal([y], want)
    # the first columns of a wider selection, in place
    wide = some_parents(B, 3, 6, 9)
    x = anything((B, 3, 33), torch.int32, 2)
    want = reordered([x], [x], [0], [None], wide[:, :3])
    binding.hola_beam_reorder(binding.BeamStates([x]), wide[:, :3])
    assert equal([x], want)
    # time-major, heads behind the positions, a slice of a larger buffer, rows on odd bytes
    big = anything((60, B, 3, 10), torch.uint8, 3)
    cases = [(anything((60, B, 3), torch.int32, 4), 1, None), (big[:, :, :, 1:8], 1, None), (anything((B, 3, 64, 20), torch.float16, 5)[:, :, :50], 0, 2),
             (anything((7, B, 3, 4, 6, 5), torch.float16, 6)[..., :4], 1, None), (anything((B + 1, 3, 31), torch.uint8, 7)[1:], 0, 2)]
    parent = some_parents(B, 3, 3, 10)
    used = torch.tensor([5, 31, 2, 50], dtype=torch.int32, device="cuda")
    for x, axis, at in cases[:3] + cases[4:]:
        want = reordered([x], [x], [axis], [at], parent, used)
        behind = big.clone()
        binding.hola_beam_reorder(binding.BeamStates([x], axis, [at]), parent, used)
        assert equal([x], want)
        if x.data_ptr() == big.data_ptr() + 1:
            assert torch.equal(big[..., [0, 8, 9]], behind[..., [0, 8, 9]])
    with pytest.raises(binding.HolaError, match="more than two axes"):
        binding.BeamStates([cases[3][0].transpose(0, 4)], 1)


@gpu
def test_many_states_in_one_call():
    B, W = 3, 4
    xs = [anything((B, W, 3 + 5 * i), torch.int32 if i % 2 else torch.uint8, i) for i in range(60)]
    parent = some_parents(B, W, W, 3)
    want = reordered(xs, xs, [0] * 60, [None] * 60, parent)
    binding.hola_beam_reorder(binding.BeamStates(xs), parent)
    assert equal(xs, want)


@gpu
def test_parents_that_there_are_not_are_reported_and_leave_their_places():
    x = anything((2, 4, 100), torch.int32, 1)
    keep = x.clone()
    parent = torch.tensor([[1, 4, -2, 0], [-1, 2 ** 31 - 1, 2, -2 ** 31]], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.hola_beam_reorder(binding.BeamStates([x]), parent, status=status)
    assert status.item() == binding.FLAG_BAD_BEAM
    assert torch.equal(x[1], keep[1]) and torch.equal(x[0], keep[0][[1, 1, 2, 0]])
    status.zero_()
    binding.hola_beam_reorder(binding.BeamStates([x]), torch.full_like(parent, -1), status=status)
    assert status.item() == 0


@gpu
def test_states_beyond_32_bits():
    """A run of more than 2^31 bytes, and beams more than 2^32 bytes apart."""
    run = 2 ** 31 + 2 ** 20 + 16
    x = torch.zeros((1, 3, run), dtype=torch.uint8, device="cuda")
    for w in range(3):
        x[0, w, :1000] = w + 1
        x[0, w, -1000:] = w + 11
        x[0, w, run // 2:run // 2 + 1000] = w + 21
    binding.hola_beam_reorder(binding.BeamStates([x]), torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda"))
    for w, p in enumerate((2, 0, 1)):
        assert (x[0, w, :1000] == p + 1).all() and (x[0, w, -1000:] == p + 11).all() and (x[0, w, run // 2:run // 2 + 1000] == p + 21).all()
        assert int(x[0, w].count_nonzero()) == 3000


# ------------------------------------------------------------------------------------------------ calls
@gpu
def test_outputs_are_filled_again_and_streams_and_graphs_work():
    B, W, V = 6, 4, 20000
    one, two = make(B, W, V, torch.float32, 1), make(B, W, V, torch.float32, 2)
    want = [reference(*x, W, keep_slots=True) for x in (one, two)]
    out = binding.hola_beam_select(*one, keep_slots=True)
    again = binding.hola_beam_select(*two, keep_slots=True, out=out)
    assert again is out
    same(out, want[1])
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):                                       # two calls at once
        got[0].append(binding.hola_beam_select(*one, keep_slots=True, stream=side))
        got[1].append(binding.hola_beam_select(*two, keep_slots=True, stream=other))
    torch.cuda.synchronize()
    for which in (0, 1):
        for o in got[which]:
            same(o, want[which])
    # captured: one selection and the states behind it
    static = [x.clone() for x in one]
    x = anything((B, W, 300), torch.int32, 5)
    keep = x.clone()
    states = binding.BeamStates([x])
    sel = binding.hola_beam_select(*static, keep_slots=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.hola_beam_select(*static, keep_slots=True, out=sel)
        binding.hola_beam_reorder(states, sel.parent)
    for which, inputs in ((0, one), (1, two), (0, one)):
        for t, v in zip(static, inputs):
            t.copy_(v)
        x.copy_(keep)
        graph.replay()
        torch.cuda.synchronize()
        same(sel, want[which])
        assert equal([x], reordered([keep], [keep], [0], [None], want[which][1]))


@gpu
def test_a_search_step_by_step():
    """Head, selection, reordering, embedding as a decoder runs them, against the same search by hand."""
    B, W, H, V, steps = 3, 4, 128, 1000, 6
    g = torch.Generator(device="cuda").manual_seed(3)
    head = (torch.randn((V, H), generator=g, device="cuda") * 0.3).bfloat16()
    table = torch.randn((V, H), generator=g, device="cuda").bfloat16()
    tok = torch.randint(0, V, (B, 1), generator=g, device="cuda", dtype=torch.int32).expand(B, W).contiguous()
    score = torch.full((B, W), -math.inf, device="cuda")
    score[:, 0] = 0.0
    history = torch.full((B, W, steps), -1, dtype=torch.int32, device="cuda")
    trunk = torch.zeros((B, W, H), device="cuda")
    states = binding.BeamStates([history, trunk], positions=[2, None])
    hand = [[(0.0, [], torch.zeros(H, dtype=torch.float64), int(tok[b, 0]))] for b in range(B)]
    with binding.HolaVerify(B, W - 1, H, V) as ctx:
        for t in range(steps):
            trunk.copy_(binding.hola_embed(tok, table, scale=0.5, add=trunk * 0.5))
            out = ctx.hola_lm_head_entropy(trunk.bfloat16(), head)
            want = reference(out.logits, out.logZ, score, W, keep_slots=True)
            sel = binding.hola_beam_select(out.logits, out.logZ, score, keep_slots=True)
            same(sel, want)
            for b in range(B):                                # the same by hand, in 64 bits, on the head's own logits
                new = []
                for s, path, state, last in hand[b]:
                    x = 0.5 * table[last].double().cpu() + 0.5 * state
                    lp = torch.log_softmax(x.float().bfloat16().double() @ head.double().cpu().T, dim=0)
                    top = torch.topk(lp, W)
                    new += [(s + float(v), path + [int(i)], x, int(i)) for v, i in zip(top.values, top.indices)]
                hand[b] = sorted(new, key=lambda c: -c[0])[:W]
            binding.hola_beam_reorder(states, sel.parent, used=torch.full((B,), t, dtype=torch.int32, device="cuda"))
            history[:, :, t] = sel.token
            tok, score = sel.token, sel.score
    for b in range(B):
        order = torch.argsort(score[b], descending=True)
        # the head's logits are those of bf16 rows, with the tensor cores' accumulation: 1e-5 of their size each, over `steps`
        for r, (s, path, _, _) in enumerate(hand[b]):
            assert abs(float(score[b, order[r]]) - s) <= steps * 1e-3
        assert history[b, order[0]].tolist() == hand[b][0][1]


# ------------------------------------------------------------------------------------------------ refusals
def _args(**kw):
    a = binding.hola_beam_args()
    a.B, a.W, a.V, a.n, a.end_token = 2, 4, 100, 4, -1
    a.seq_stride, a.beam_stride = 400, 100
    for i, name in enumerate(("logits", "logZ", "score", "score_out", "parent", "token")):
        setattr(a, name, 4096 * (20 + i))
    for name, v in kw.items():
        setattr(a, name, v)
    return a


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), 1), (dict(W=0), 1), (dict(V=0), 1), (dict(n=0), 1), (dict(l_dtype=3), 1), (dict(l_dtype=-1), 1), (dict(seq_stride=-1), 1),
    (dict(W=33, n=4), 2), (dict(n=33), 2), (dict(V=2 ** 27 + 1), 2), (dict(B=2 ** 31 - 1), 2), (dict(keep_slots=1, n=5), 1), (dict(end_token=100), 1),
    (dict(end_token=-2), 1), (dict(finished=4096), 1), (dict(logits=None), 1), (dict(logZ=None), 1), (dict(score=None), 1), (dict(parent=None), 1),
    (dict(token=None), 1), (dict(score_out=None), 1), (dict(logits=4098), 1), (dict(B=0), 0), (dict(B=0, logits=None), 0),
    (dict(score=8192, score_out=8192 + 16), 1), (dict(score=8192, score_out=8192, n=3), 1), (dict(score=8192, score_out=16384, token=8192 + 28), 1),
    (dict(score=8192, score_out=16384, logZ=16384), 1), (dict(finished=8192, end_token=3, finished_out=8196), 1)])
def test_selections_that_are_refused(kw, status):
    lib = binding.load_library()
    assert lib.hola_beam_select(ctypes.byref(_args(**kw)), None) == status
    assert lib.hola_beam_select(None, None) == 1


def _state(**kw):
    s = binding.hola_beam_state()
    s.src = s.dst = 4096
    s.seq_stride = s.dst_seq_stride = 400
    s.beam_stride = s.dst_beam_stride = s.run = 100
    s.outer[0] = s.outer[1] = 1
    for name, v in kw.items():
        setattr(s, name, v)
    return s


@pytest.mark.parametrize("kw,args,status", [
    (dict(), dict(B=-1), 1), (dict(), dict(W=0), 1), (dict(), dict(n=0), 1), (dict(), dict(n=5), 1), (dict(), dict(W=33), 2), (dict(), dict(n=33), 2),
    (dict(), dict(parent=None), 1), (dict(), dict(states=None), 1), (dict(), dict(parent_stride=-1), 1), (dict(run=-1), {}, 1), (dict(position=-1), {}, 1),
    (dict(src=None), {}, 1), (dict(beam_stride=99, dst_beam_stride=99), {}, 1), (dict(dst_seq_stride=500), {}, 1), (dict(seq_stride=-400), {}, 1),
    (dict(run=2 ** 60, beam_stride=2 ** 60, dst_beam_stride=2 ** 60), {}, 2), (dict(), dict(B=0), 0), (dict(), dict(count=0), 0), (dict(run=0), {}, 0)])
def test_reorderings_that_are_refused(kw, args, status):
    lib = binding.load_library()
    s = (binding.hola_beam_state * 1)(_state(**kw))
    a = binding.hola_reorder_args()
    a.B, a.W, a.n, a.count, a.states, a.parent, a.parent_stride = 2, 4, 4, 1, ctypes.addressof(s), 4096, 4
    for name, v in args.items():
        setattr(a, name, v)
    assert lib.hola_beam_reorder(ctypes.byref(a), None) == status
    assert lib.hola_beam_reorder(None, None) == 1
    both = (binding.hola_beam_state * 2)(_state(), _state(dst=8192))          # in place, and not
    a.states, a.count, a.B, a.W, a.n, a.parent, a.parent_stride = ctypes.addressof(both), 2, 2, 4, 4, 4096, 4
    assert lib.hola_beam_reorder(ctypes.byref(a), None) == 1


def test_layout_of_the_structs():
    assert ctypes.sizeof(binding.hola_beam_args) == 16 + 3 * 8 + 8 + 4 * 8 + 8 + 5 * 8
    assert ctypes.sizeof(binding.hola_beam_state) == 14 * 8 and ctypes.sizeof(binding.hola_reorder_args) == 16 + 5 * 8


def test_states_that_are_refused():
    x = torch.zeros((3, 2, 4, 10))
    for bad in (lambda: binding.BeamStates([]), lambda: binding.BeamStates([x], axes=3), lambda: binding.BeamStates([x, x], axes=[1, 0]),
                lambda: binding.BeamStates([x[0]], into=[x[0]]), lambda: binding.BeamStates([x], 1, into=[x.double()]),
                lambda: binding.BeamStates([x], 1, [0]), lambda: binding.BeamStates([x], 1, [1]), lambda: binding.BeamStates([x], 1, [4]),
                lambda: binding.BeamStates([x[:, :, :1].expand(3, 2, 4, 10)], 1), lambda: binding.BeamStates([x.transpose(1, 3)], 1, [3]),
                lambda: binding.BeamStates([torch.zeros(2, 33, 4)]), lambda: binding.BeamStates([x], 1, into=[x, x]), lambda: binding.BeamStates(["x"]),
                lambda: binding.hola_beam_reorder([x], torch.zeros((2, 4), dtype=torch.int32)),
                lambda: binding.hola_beam_reorder(binding.BeamStates([x], 1), torch.zeros((2, 4), dtype=torch.int32)),
                lambda: binding.hola_beam_select(x[0], torch.zeros(2, 4), torch.zeros(2, 4))):
        with pytest.raises(binding.HolaError):
            bad()


@gpu
def test_operands_that_are_refused():
    l, z, s = make(2, 4, 100, torch.float32, 1)
    ok = dict(logits=l, logZ=z, score=s)
    f = torch.zeros((2, 4), dtype=torch.bool, device="cuda")
    for kw in (dict(logits=l[0]), dict(logits=l.double()), dict(logits=l.transpose(1, 2)), dict(logZ=z[:, :3]), dict(logZ=z.cpu()), dict(score=s.double()),
               dict(n=0), dict(n=33), dict(n=5, keep_slots=True), dict(finished=f), dict(finished=f.int(), end_token=1), dict(end_token=100),
               dict(weight=z.half()), dict(status=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(out=binding.hola_beam_select(l, z, s, 3)),
               dict(out=binding.hola_beam_select(l, z, s), end_token=1)):
        with pytest.raises(binding.HolaError):
            binding.hola_beam_select(**{**ok, **kw})
    x = torch.zeros((2, 4, 10), device="cuda")
    states = binding.BeamStates([x])
    p = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    for parent, used in ((p.long(), None), (p[:1], None), (p.cpu(), None), (torch.zeros((2, 5), dtype=torch.int32, device="cuda"), None),
                         (p.t().contiguous().t(), None), (p, p[0]), (p, torch.zeros(2, device="cuda"))):
        with pytest.raises(binding.HolaError):
            binding.hola_beam_reorder(states, parent, used)


@gpu
def test_calls_through_the_native_helper_and_without_it(monkeypatch):
    """The same results and the same refusals either way."""
    l, z, s = make(3, 4, 500, torch.float16, 6, pad=3)
    f = torch.zeros((3, 4), dtype=torch.bool, device="cuda")
    f[1, 2] = True
    w = torch.rand((3, 4), device="cuda") + 0.5
    calls = [lambda: binding.hola_beam_select(l, z, s), lambda: binding.hola_beam_select(l, z, s, 7, f, 9, w),
             lambda: binding.hola_beam_select(l, z, s, 4, f, 9, keep_slots=True), lambda: binding.hola_beam_select(l[:0], z[:0], s[:0], 3),
             lambda: binding.hola_beam_select(l, z.half(), s), lambda: binding.hola_beam_select(l, z, s, 33), lambda: binding.hola_beam_select(l, z, s, 5, f)]

    def run():
        got = []
        for call in calls:
            try:
                o = call()
                got.append((o.score.cpu(), o.parent.cpu(), o.token.cpu(), None if o.finished is None else o.finished.cpu()))
            except binding.HolaError as e:
                got.append(str(e))
        x = anything((3, 4, 50), torch.int32, 1)
        binding.hola_beam_reorder(binding.BeamStates([x]), got[0][1].cuda())
        return [*got, (x.cpu(),)]

    assert binding._host is not None
    with_it = run()
    monkeypatch.setattr(binding, "_host", None)
    for a, b in zip(with_it, run(), strict=True):
        assert a == b if isinstance(a, str) else all((x is None and y is None) or torch.equal(x, y) for x, y in zip(a, b, strict=True))


@gpu
def test_the_drivers_beam_search():
    """Scores are the log probabilities of the emitted tokens; one beam is the greedy decoder; more beams never score less than the
    prefix of fewer would allow at the last step, and ended beams keep what they have."""
    from paper_2506_18952_b200 import driver
    B, H, V, steps, W = 4, 256, 2000, 7, 5
    models = driver.SyntheticPair(V, H, 5, torch.device("cuda", torch.cuda.current_device()))
    prompt = torch.randint(0, V, (B, 2), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))

    def logprobs(tokens):                                     # of every position behind the prompt, in 64 bits from the head's bf16 rows
        c1, c2 = tokens[..., 1:-1].long(), tokens[..., :-2].long()
        h = models._norm(models.E1[c1] + 0.35 * models.E2[c2], c1).bfloat16().double()
        lp = torch.log_softmax(h @ models.W_lm.double().T, dim=-1)
        return lp.gather(-1, tokens[..., 2:].long()[..., None])[..., 0], lp

    with binding.HolaVerify(B, W - 1, H, V) as ctx:
        res = driver.beam_decode(ctx, models, prompt, W, steps)
        lp, _ = logprobs(res.tokens)
        # logits to 1e-5 of their size (tens), sums of `steps` of them in fp32
        assert (res.score.double() - lp.sum(-1)).abs().max() <= steps * 1e-3
        assert (res.score[:, :-1] >= res.score[:, 1:]).all()
        assert len({tuple(t.tolist()) for t in res.tokens.reshape(-1, 2 + steps)}) == B * W
        one = driver.beam_decode(ctx, models, prompt, 1, steps)
        lp, every = logprobs(one.tokens)
        assert (every.amax(-1)[:, 0] - lp[:, 0]).max() <= 1e-3
        end = int(res.tokens[0, 0, 4])                        # a token that comes up
        ended = driver.beam_decode(ctx, models, prompt, W, steps, end_token=end)
        lp, _ = logprobs(ended.tokens)
        for b in range(B):
            for w in range(W):
                where = (ended.tokens[b, w, 2:] == end).nonzero()
                n = int(where[0]) + 1 if len(where) else steps
                assert abs(float(ended.score[b, w]) - float(lp[b, w, :n].sum())) <= steps * 1e-3
                assert (ended.tokens[b, w, 2 + n:] == end).all()
        assert (ended.tokens[0, :, 2:] == end).any()


@gpu
@pytest.mark.parametrize("B", [1, 200])
def test_scores_that_are_written_over(B):
    """A loop that keeps its scores in place: many CTAs a sequence, and one."""
    W, V = 4, 30000 if B == 1 else 900
    l, z, s = make(B, W, V, torch.float32, 9)
    f = torch.zeros((B, W), dtype=torch.bool, device="cuda")
    f[:, 1] = True
    want = reference(l, z, s, W, f, 5)
    out = binding.BeamSelection(s, torch.empty((B, W), dtype=torch.int32, device="cuda"), torch.empty((B, W), dtype=torch.int32, device="cuda"), f)
    binding.hola_beam_select(l, z, s, W, f, 5, out=out)
    same(out, want)


def test_outputs_on_one_another_and_states_twice_are_refused():
    lib = binding.load_library()
    a = binding.hola_beam_args()
    a.B, a.W, a.V, a.n, a.seq_stride, a.beam_stride, a.end_token = 2, 4, 100, 4, 400, 100, 7
    a.logits, a.logZ, a.score, a.score_out, a.parent, a.token, a.finished_out = 1 << 20, 4096, 8192, 12288, 16384, 20480, 24576
    for name, at in (("parent", 12288), ("token", 16384), ("token", 20480 - 4096 + 28), ("finished_out", 12288 + 31), ("parent", 20480 + 28)):
        kept = getattr(a, name)
        setattr(a, name, at)
        assert lib.hola_beam_select(ctypes.byref(a), None) == 1, name
        setattr(a, name, kept)
    x, y = torch.zeros((2, 4, 6)), torch.zeros((2, 4, 6))
    for twice in (lambda: binding.BeamStates([x, x]), lambda: binding.BeamStates([x, x.view(2, 4, 3, 2)]),
                  lambda: binding.BeamStates([x, x.clone()], into=[y, y])):
        with pytest.raises(binding.HolaError):
            twice()
    kv = torch.zeros((2, 4, 2, 6))
    binding.BeamStates(list(kv.unbind(2)) + [kv[:, :, :0], kv[:, :, :0]])            # (side by side in one buffer; nothing at all)
    binding.BeamStates([x, x], into=[y, y.clone()])


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,seen", [(4096, 3), (4096, 9), (8192, 5), (3000, 2), (30000, 3)])
def test_masks_of_both_kinds_beside_offsets_beyond_fp32(V, seen, dtype):
    """A few entries at the lowest value of fp32 and -inf behind them: the logZ is that low too, and an offset times a weight above 1 is more
    than fp32 holds.  (Only entries that are there count, and each of them once.)"""
    low = torch.finfo(torch.float32).min
    for W, n in ((1, 4), (3, 7), (2, 32)):
        l = torch.full((4, W, V), -math.inf, device="cuda", dtype=dtype)
        l[..., :seen] = torch.finfo(dtype).min
        l[1, ..., V // 2:V // 2 + seen] = 0.5 * torch.finfo(dtype).min
        l[2, ..., ::8] = torch.finfo(dtype).min
        z = torch.full((4, W), low, device="cuda")
        s = torch.full((4, W), -3.0, device="cuda")
        z[3] = -low                                           # (and far above what is there)
        for weight in (1.0, 1.5, 3.0, 1e30):
            w = torch.full((4, W), weight, device="cuda")
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            same(binding.hola_beam_select(l, z, s, n, weight=w, status=status), reference(l, z, s, n, weight=w))
            assert status.item() == 0


def test_states_that_share_bytes_are_refused():
    """Parts of one buffer: side by side they are states of their own, in place and from one half into the other; with a byte in common they
    are not."""
    buf = torch.zeros((3, 4, 2, 12))
    x, y = buf[:, :, 0], buf[:, :, 1]
    binding.BeamStates([x], into=[y])                         # (interleaved)
    binding.BeamStates([buf[..., :6], buf[..., 6:]])
    binding.BeamStates([x, y])
    binding.BeamStates([buf[:, :, 0, :4], buf[:, :, 1, 6:]], into=[buf[:, :, 0, 4:8], buf[:, :, 1, :6]])
    halves = torch.zeros((3, 8, 12))
    binding.BeamStates([halves[:, :4]], into=[halves[:, 4:]])
    turns = torch.zeros((2, 12, 3, 4))                        # layers first, time-major
    binding.BeamStates([torch.zeros(99).as_strided((3, 4, 2, 2), (4, 12, 2, 1))])       # (4 b + 12 w: a fourth sequence would be on the next beam)
    binding.BeamStates([turns[0], turns[1]], axes=1)
    binding.BeamStates([turns[0]], axes=1, into=[turns[1]])
    for bad in (lambda: binding.BeamStates([buf[:, :, 0, :4], buf[:, :, 1, 4:]], into=[buf[:, :, 0, 4:8], buf[:, :, 1, :8]]),       # (4 .. 7 of the second)
                lambda: binding.BeamStates([buf[..., :8], buf[..., 4:]]), lambda: binding.BeamStates([x, buf[:, :, 0, 11:]]),
                lambda: binding.BeamStates([x, y.clone()], into=[x.clone(), x]), lambda: binding.BeamStates([x], into=[buf.view(3, 4, 24)[..., 11:23]]),
                lambda: binding.BeamStates([x, y], into=[torch.zeros_like(x), x]), lambda: binding.BeamStates([x, y], into=[y, torch.zeros_like(x)]),
                lambda: binding.BeamStates([x.clone(), y.clone()], into=[buf[..., 0, :8], buf[..., 0, 4:]]),
                lambda: binding.BeamStates([halves[:, :4]], into=[halves[:, 3:7]]), lambda: binding.BeamStates([torch.zeros(99).unfold(0, 12, 1)[:12].view(3, 4, 12)]),
                lambda: binding.BeamStates([torch.zeros(99).as_strided((4, 4, 2, 2), (4, 12, 2, 1))])):
        with pytest.raises(binding.HolaError):
            bad()


def test_calls_on_states_that_share_bytes_are_refused():
    """The C entry: a state's own two sides, its own sequences, and what the call reads besides."""
    lib = binding.load_library()
    a = binding.hola_reorder_args()
    a.B, a.W, a.n, a.count, a.parent, a.parent_stride, a.used = 2, 4, 4, 1, 1 << 20, 4, 1 << 21

    def status(check=False, parent=1 << 20, used=1 << 21, **kw):
        s = (binding.hola_beam_state * 1)(_state(**{"src": 1 << 24, "dst": 1 << 25, **kw}))
        a.states, a.parent, a.used = ctypes.addressof(s), parent, used
        return lib.hola_beam_states_check(ctypes.byref(a)) if check else lib.hola_beam_reorder(ctypes.byref(a), None)

    src = 1 << 24
    for kw in (dict(dst=src + 100), dict(dst=src + 99), dict(dst=src - 1), dict(dst=src + 799), dict(dst=src + 50, beam_stride=200, seq_stride=800),
               dict(dst=src, dst_seq_stride=500), dict(dst_seq_stride=399), dict(dst=src, seq_stride=399, dst_seq_stride=399)):
        assert status(**kw) == 1 and status(True, **kw) == 1, kw
    for kw in (dict(parent=1 << 25), dict(parent=(1 << 25) + 799), dict(parent=(1 << 25) - 31), dict(used=(1 << 25) + 796), dict(used=(1 << 25) - 4)):
        assert status(**kw) == 1, kw
    fine = [dict(), dict(dst=src), dict(dst=src + 800), dict(dst=src - 800), dict(parent=(1 << 25) + 800), dict(used=(1 << 25) - 8),
            dict(dst=src + 100, beam_stride=200, seq_stride=800, dst_beam_stride=200, dst_seq_stride=800)]
    for kw in fine:
        if "parent" not in kw and "used" not in kw:
            assert status(True, **kw) == 0, kw
        if not torch.cuda.is_available():                     # (no device here: nothing runs)
            assert status(**kw) not in (0, 1), kw
    both = (binding.hola_beam_state * 2)(_state(src=src, dst=src), _state(src=src + 800, dst=src + 800))
    a.states, a.count = ctypes.addressof(both), 2
    assert lib.hola_beam_states_check(ctypes.byref(a)) == 0
    both[1].src = both[1].dst = src + 799
    assert lib.hola_beam_states_check(ctypes.byref(a)) == 1
    assert lib.hola_beam_states_check(None) == 1


@gpu
def test_states_side_by_side_in_one_buffer():
    B, W, T = 3, 5, 37
    for used in (None, torch.tensor([4, 37, 0], dtype=torch.int32, device="cuda")):
        buf = anything((B, W, 2, T, 3), torch.float16, 1)
        parent = some_parents(B, W, W, 2)
        want = reordered([buf[:, :, 0]], [buf[:, :, 1]], [0], [2], parent, used)
        kept = buf[:, :, 0].clone()
        binding.hola_beam_reorder(binding.BeamStates([buf[:, :, 0]], 0, [2], [buf[:, :, 1]]), parent, used)
        assert equal([buf[:, :, 1]], want) and equal([buf[:, :, 0]], [kept.cpu()])
        xs = [buf[..., :1], buf[..., 1:]]                     # (channels)
        want = reordered(xs, xs, [0, 0], [None, None], parent)
        binding.hola_beam_reorder(binding.BeamStates(xs), parent)
        assert equal(xs, want)


def test_selections_into_their_logits_are_refused():
    """Results on an entry of any row; behind the rows and between them there is room."""
    lib = binding.load_library()
    base = 1 << 24
    for l_dtype, e in ((binding.HOLA_L_F32, 4), (binding.HOLA_L_BF16, 2), (binding.HOLA_L_F16, 2)):
        a = _args(logits=base, l_dtype=l_dtype, seq_stride=800, beam_stride=200, end_token=5, finished_out=1 << 22)      # rows of 100 entries, 200 apart
        row = 100 * e
        for name, length in (("score_out", 32), ("parent", 32), ("token", 32), ("finished_out", 8)):
            kept = getattr(a, name)
            for at in (base, base + row - length, base + 2 * row, base + 7 * 2 * row + row - 4, base - length + 4, base + 4 * 2 * row - length + 4):
                setattr(a, name, at)
                assert lib.hola_beam_select(ctypes.byref(a), None) == 1, (l_dtype, name, at - base)
            for at in (base + row, base + 2 * row - length, base + 7 * 2 * row + row, base - length):
                setattr(a, name, at)
                if not torch.cuda.is_available():             # (no device here: nothing runs)
                    assert lib.hola_beam_select(ctypes.byref(a), None) not in (0, 1), (l_dtype, name, at - base)
            setattr(a, name, kept)


@gpu
def test_results_of_a_call_with_ends_filled_again_without():
    """What an earlier call has left in out.finished does not stay there."""
    l, z, s = make(3, 4, 200, torch.float32, 11)
    f = torch.ones((3, 4), dtype=torch.bool, device="cuda")
    out = binding.hola_beam_select(l, z, s, finished=f, end_token=7)
    assert out.finished.all()
    for keep in (False, True):
        out.finished.fill_(True)
        binding.hola_beam_select(l, z, s, keep_slots=keep, out=out)
        same(out, reference(l, z, s, 4, keep_slots=keep))
        assert not out.finished.any()


def test_operands_on_no_address_of_their_type_are_refused():
    lib = binding.load_library()
    ok = dict(finished=1 << 20, finished_out=1 << 21, weight=1 << 22, status_word=1 << 23, end_token=3)
    for name in ("logZ", "score", "weight", "score_out", "parent", "token", "status_word"):
        for off in (1, 2, 3):
            a = _args(**ok)
            setattr(a, name, getattr(a, name) + off)
            assert lib.hola_beam_select(ctypes.byref(a), None) == 1, (name, off)
    s = (binding.hola_beam_state * 1)(_state())
    for name in ("parent", "used", "status_word"):
        for off in (0, 1, 2, 3):
            a = binding.hola_reorder_args()
            a.B, a.W, a.n, a.count, a.states, a.parent, a.parent_stride, a.used, a.status_word = 2, 4, 4, 1, ctypes.addressof(s), 1 << 20, 4, 1 << 21, 1 << 22
            setattr(a, name, getattr(a, name) + off)
            if off or not torch.cuda.is_available():          # (no device here: nothing runs)
                assert (lib.hola_beam_reorder(ctypes.byref(a), None) == 1) == (off > 0), (name, off)
    if not torch.cuda.is_available():                         # flags of one byte and logits lie anywhere
        assert lib.hola_beam_select(ctypes.byref(_args(**{**ok, "finished": (1 << 20) + 1, "finished_out": (1 << 21) + 3})), None) not in (0, 1)


@gpu
@pytest.mark.parametrize("V", [30, 9000])
def test_what_is_no_beam_is_not_reported(V):
    """A score of -inf beside a logZ, a weight and logits that are nothing; rows without entries beside others."""
    W, n = 4, 6
    l, z, s = make(6, W, V, torch.float32, 12)
    w = torch.rand((6, W), device="cuda") + 0.5
    s[:, 2] = -math.inf
    l[:, 2] = math.nan
    for b, x in enumerate((math.nan, math.inf, -math.inf, 0.0)):
        z[b, 2] = x
        w[b, 2] = (math.nan, -1.0, 0.0, math.inf)[b]
    l[4, 1], z[4, 1] = -math.inf, -math.inf
    s[5], z[5], w[5] = -math.inf, math.nan, math.nan
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for weight in (None, w):
        same(binding.hola_beam_select(l, z, s, n, weight=weight, status=status), reference(l, z, s, n, weight=weight))
        assert status.item() == 0


@gpu
@pytest.mark.parametrize("lead", [0, 1])
def test_the_longest_rows(lead):
    """2^27 entries a row: the best at its ends, some equal ones among them."""
    W, V, n = 3, 2 ** 27, 12
    buf = torch.full((W * V + lead,), -9.0, dtype=torch.bfloat16, device="cuda")
    l = buf[lead:].view(1, W, V)
    s, z = torch.tensor([[-1.0, -1.25, -1.0]], device="cuda"), torch.full((1, W), 2.0, device="cuda")
    want = []
    for w, marks in enumerate(({0: 3.0, V - 1: 3.0, V // 2: 1.0}, {V - 1: 4.0, V - 2: 3.25, 7: 0.5}, {V - 1: 3.0, 1: 2.0, V - 17: 2.0})):
        for v, x in marks.items():
            l[0, w, v] = x
            want.append((float(s[0, w]) - 2.0 + x, w, v))
    want.sort(key=lambda c: (-c[0], c[1], c[2]))
    want += [(-1.0 - 2.0 - 9.0, 0, v) for v in (1, 2, 3)]
    out = binding.hola_beam_select(l, z, s, n)
    assert list(zip(out.score[0].tolist(), out.parent[0].tolist(), out.token[0].tolist())) == want
