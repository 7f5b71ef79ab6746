"""Rows of a table by token, equal to the bit with the same operations in fp32, and the gradient of the table against 64 bits."""
import ctypes
import math

import pytest
import torch

from paper_2506_18952_b200 import binding

gpu = pytest.mark.gpu
FLOATS = [torch.float32, torch.bfloat16, torch.float16]


def rnd(shape, dtype, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * std).to(dtype)


def some_tokens(N, V, seed, dtype=torch.int32, absent=0.1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.exp(torch.rand((N,), generator=g, device="cuda", dtype=torch.float64) * math.log(V + 1.0)) - 1.0
    t = torch.where(torch.rand((N,), generator=g, device="cuda") < absent, -1, t.long().clamp_(0, V - 1))
    return t.to(dtype)


def looked_up(tokens, rows32, scale, add, dtype):
    """rows32: the table in fp32.  One rounding for the product, one for the sum, one for the result's type."""
    t = tokens.long()
    inside = (t >= 0) & (t < rows32.shape[0])
    y = torch.where(inside[..., None], rows32[t.clamp(0, rows32.shape[0] - 1)] * scale, 0.0)
    return (y if add is None else add.float() + y).to(dtype)


# ------------------------------------------------------------------------------------------------ lookup
@gpu
@pytest.mark.parametrize("table_dtype", [*FLOATS, torch.int8])
@pytest.mark.parametrize("N,V,H", [(1, 1, 1), (1, 5, 8), (3, 7, 5), (2, 100, 64), (5, 1000, 4096), (17, 33, 1000), (130, 500, 2056), (9, 50, 8200),
                                   (4000, 3000, 128), (2500, 100, 2048)])
def test_rows_of_every_type(N, V, H, table_dtype):
    t32 = some_tokens(N, V, N)
    scale = rnd((V,), torch.float32, 1).abs() * 0.01 if table_dtype == torch.int8 else None
    table = rnd((V, H), torch.float32, 2, 30.0).to(table_dtype) if scale is not None else rnd((V, H), table_dtype, 2)
    rows32 = table.float() * scale[:, None] if scale is not None else table.float()
    for dtype in FLOATS:
        for s, with_add, wide in ((1.0, False, False), (math.sqrt(H), False, True), (0.35, True, False)):
            tokens = t32.long() if wide else t32
            add = rnd((N, H), dtype, 3) if with_add else None
            got = binding.hola_embed(tokens, table, scale=s, add=add, w_scale=scale, dtype=dtype)
            assert got.dtype == dtype and torch.equal(got, looked_up(tokens, rows32, s, add, dtype))


@gpu
@pytest.mark.parametrize("V,H", [(256, 128), (700, 256), (3000, 1024)])
def test_rows_of_a_head_of_mixed_widths(V, H):
    W = rnd((V, H), torch.bfloat16, 4)
    groups = -(-V // 256)
    for widths in ([(4, 8, 16)[i % 3] for i in range(groups)], [4] * groups, [8] * groups, [16] * groups):
        head = binding.hola_quantize_mixed(W, widths)
        codes = torch.empty((V, H), device="cuda")
        at = {4: 0, 8: 0, 16: 0}
        for g, width in enumerate(widths):
            n = min(256, V - 256 * g)
            r = slice(at[width], at[width] + n)
            if width == 16:
                part = head.W16[r].float()
            elif width == 8:
                part = head.W8[r].float()
            else:
                b = head.W4[r].int()
                both = torch.stack([(b << 28) >> 28, (b << 24) >> 28], dim=2).reshape(n, H)
                part = (both << head.shift4[:, r].t().int().repeat_interleave(128, dim=1)).float()
            codes[256 * g:256 * g + n] = part
            at[width] += n
        rows32 = codes * head.w_scale[:, None]
        tokens = torch.arange(-1, V, device="cuda", dtype=torch.int32)
        assert torch.equal(binding.hola_embed(tokens, head, scale=1.7), looked_up(tokens, rows32, 1.7, None, torch.bfloat16))
        # rows on odd addresses: channel by channel
        out = torch.zeros((V + 1, H + 1), device="cuda")
        binding.hola_embed(tokens, head, scale=0.3, out=out[:, 1:])
        assert torch.equal(out[:, 1:], looked_up(tokens, rows32, 0.3, None, torch.float32)) and (out[:, 0] == 0).all()
    # and those that the LM head itself multiplies with: W8 is the quantiser's
    q, scale = binding.hola_quantize_w8(W)
    tokens = torch.arange(V, device="cuda", dtype=torch.int32)
    assert torch.equal(binding.hola_embed(tokens, q, w_scale=scale), binding.hola_embed(tokens, binding.hola_quantize_mixed(W, [8] * groups)))


@gpu
@pytest.mark.parametrize("H", [7, 64, 1000])
def test_strides_shapes_and_results_in_place(H):
    V = 90
    table = rnd((V, H + 3), torch.float32, 1)[:, :H]          # rows further apart
    tokens = some_tokens(24, V, 2).view(2, 3, 4)
    want = looked_up(tokens, table, 2.0, None, torch.float32)
    assert torch.equal(binding.hola_embed(tokens, table, 2.0), want)
    buf = torch.full((2, 3, 4, H + 5), math.nan, device="cuda")
    got = binding.hola_embed(tokens, table, 2.0, out=buf[..., :H])
    assert got.data_ptr() == buf.data_ptr() and torch.equal(buf[..., :H], want) and buf[..., H:].isnan().all()
    x = rnd((2, 3, 4, H), torch.float32, 5)
    want = looked_up(tokens, table, 2.0, x, torch.float32)
    binding.hola_embed(tokens, table, 2.0, add=x, out=x)      # onto what is there
    assert torch.equal(x, want)
    row = rnd((1, 1, 1, H), torch.float32, 6).expand(2, 3, 4, H)                  # one row for all
    assert torch.equal(binding.hola_embed(tokens, table, 2.0, add=row), looked_up(tokens, table, 2.0, row, torch.float32))
    assert binding.hola_embed(tokens[:0], table).shape == (0, 3, 4, H)
    assert binding.hola_embed(tokens[0, 0, 0], table).shape == (H,)


@gpu
def test_tokens_that_there_are_not():
    V, H = 50, 40
    table = rnd((V, H), torch.float32, 1)
    for dtype in (torch.int32, torch.int64):
        t = torch.tensor([0, -1, 49, 50, -2, 2 ** 31 - 1, -2 ** 31, 7], device="cuda").to(dtype)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = binding.hola_embed(t, table, status=status)
        assert torch.equal(got, looked_up(t, table, 1.0, None, torch.float32)) and (got[[1, 3, 4, 5, 6]] == 0).all()
        assert status.item() == binding.FLAG_BAD_TOKEN
        status.zero_()
        binding.hola_embed(t[:3].contiguous(), table, status=status)
        assert status.item() == 0
        status.zero_()
        got = binding.hola_embed_grad(t, torch.ones((8, H), device="cuda"), V, status=status)
        assert status.item() == binding.FLAG_BAD_TOKEN and got.sum().item() == 3 * H and (got[[0, 49, 7]] == 1).all()
    big = torch.tensor([2 ** 32, 2 ** 32 + 3, 2 ** 40 - 1], device="cuda")        # not 0, 3, -1 cut off
    status.zero_()
    assert (binding.hola_embed(big, table, status=status) == 0).all() and status.item() == binding.FLAG_BAD_TOKEN
    assert (binding.hola_embed_grad(big, torch.ones((3, H), device="cuda"), V) == 0).all()


@gpu
def test_parts_of_a_vocabulary_add_up():
    V, H, cuts = 1000, 72, [0, 130, 131, 600, 1000]
    table = rnd((V, H), torch.bfloat16, 3)
    tokens = some_tokens(300, V, 4)
    grad = rnd((300, H), torch.float32, 5)
    whole, dense = binding.hola_embed(tokens, table, 3.0), binding.hola_embed_grad(tokens, grad, V, 3.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = torch.zeros((300, H), dtype=torch.bfloat16, device="cuda")
    ids = []
    for a, b in zip(cuts, cuts[1:]):
        got = binding.hola_embed(tokens, table[a:b], 3.0, add=got, v_offset=a, V_global=V, status=status)
        assert torch.equal(binding.hola_embed_grad(tokens, grad, b - a, 3.0, v_offset=a, V_global=V, status=status), dense[a:b])
        rows = binding.hola_embed_grad_rows(tokens, grad, b - a, 3.0, v_offset=a, V_global=V, status=status)
        n = rows.count.item()
        ids += rows.ids[:n].tolist()
        assert torch.equal(rows.rows[:n], dense[rows.ids[:n].long()])
    assert torch.equal(got, whole) and status.item() == 0
    assert ids == sorted(set(tokens.tolist()) - {-1})


# ------------------------------------------------------------------------------------------------ gradient
def check_grad(tokens, grad, V, scale, got, before=None, rows=None):
    """|error| <= (c + 2) 2^-24 scale sum |g| for c rows: at most c additions in fp32 (the pieces' own ones among them) and the product;
    with what was there before, one more rounding of the sum; and half a step of the result's type."""
    t, H = tokens.reshape(-1).long(), grad.shape[-1]
    g = grad.reshape(-1, H).double()
    inside = (t >= 0) & (t < V)
    t, g = t[inside], g[inside]
    want = torch.zeros((V, H), dtype=torch.float64, device="cuda").index_add_(0, t, g) * scale
    size = torch.zeros((V, H), dtype=torch.float64, device="cuda").index_add_(0, t, g.abs()) * abs(scale)
    count = torch.bincount(t, minlength=V).double()[:, None]
    tol = (count + 2) * 2.0 ** -24 * size
    if before is not None:
        want = want + before.double()
        tol = tol + 2.0 ** -24 * (want.abs() + size)
    if rows is not None:
        want, tol = want[rows], tol[rows]
    eps = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * eps       # (steps below the smallest normal number)
    over = (got.double() - want).abs() - (tol * (1 + eps) + eps * want.abs() + (tiny if got.dtype != torch.float32 else 0))
    assert float(over.max()) <= 0, float(over.max())
    if before is None and rows is None:
        assert (got[count[:, 0] == 0] == 0).all()


SIZES = [(1, 1, 1), (1, 300, 8), (2, 5, 7), (33, 4, 64), (65, 2, 1000), (320, 5000, 4096), (200, 7, 1032), (1000, 1000, 72), (5000, 40, 128), (3000, 128256, 256),
         (20000, 3, 16), (70000, 500, 8)]


@gpu
@pytest.mark.parametrize("g_dtype", FLOATS)
@pytest.mark.parametrize("N,V,H", SIZES)
def test_gradients_of_all_sizes(N, V, H, g_dtype):
    tokens, grad = some_tokens(N, V, N + V), rnd((N, H), g_dtype, H)
    for dtype, scale, wide in ((torch.float32, 1.0, False), (torch.bfloat16, math.sqrt(H), True), (torch.float16, 0.01, False)):
        t = tokens.long() if wide else tokens
        got = binding.hola_embed_grad(t, grad, V, scale, dtype=dtype)
        check_grad(t, grad, V, scale, got)
        assert torch.equal(got, binding.hola_embed_grad(t, grad, V, scale, dtype=dtype))          # the same bits
        base = rnd((V, H), dtype, 9)
        more = base.clone()
        binding.hola_embed_grad(t, grad, V, scale, out=more, accumulate=True)
        check_grad(t, grad, V, scale, more, before=base)
        untouched = torch.ones(V, dtype=torch.bool, device="cuda")
        untouched[tokens[tokens >= 0].long()] = False
        assert torch.equal(more[untouched], base[untouched])
        mark = binding.TokenRows(torch.full((N,), -7, dtype=torch.int32, device="cuda"), torch.full((N, H), -7.0, dtype=dtype, device="cuda"),
                                 torch.full((1,), -7, dtype=torch.int32, device="cuda"))
        rows = binding.hola_embed_grad_rows(t, grad, V, scale, out=mark)
        n = rows.count.item()
        want = sorted(set(tokens.tolist()) - {-1})
        assert rows.ids[:n].tolist() == want and (rows.ids[n:] == -7).all() and (rows.rows[n:] == -7).all()
        assert torch.equal(rows.rows[:n], got[rows.ids[:n].long()])


@gpu
@pytest.mark.parametrize("kind", ["one", "two", "all", "none", "last", "runs"])
def test_tokens_that_occur_never_once_and_always(kind):
    """One token throughout (many pieces, the last CTA adds them up), tokens at the borders of ranges and pieces."""
    N, V, H = 40000, 3001, 40
    g = torch.Generator(device="cuda").manual_seed(1)
    t = {"one": lambda: torch.full((N,), 1234), "two": lambda: torch.arange(N) % 2 * 3000, "all": lambda: torch.arange(N) % V,
         "none": lambda: torch.full((N,), -1), "last": lambda: torch.where(torch.arange(N) < N - 1, -1, 3000),
         "runs": lambda: torch.repeat_interleave(torch.arange(V), torch.randint(0, 27, (V,), generator=torch.Generator().manual_seed(2)))[:N]}[kind]()
    t = t.cuda().to(torch.int32)
    grad = torch.randn((t.numel(), H), generator=g, device="cuda")
    got = binding.hola_embed_grad(t, grad, V)
    check_grad(t, grad, V, 1.0, got)
    rows = binding.hola_embed_grad_rows(t, grad, V)
    n = rows.count.item()
    assert rows.ids[:n].tolist() == sorted(set(t.tolist()) - {-1})
    assert torch.equal(rows.rows[:n], got[rows.ids[:n].long()])


@gpu
def test_pieces_of_every_length():
    """Runs of 1 .. 300 equal tokens, so that pieces end inside and at the ends of windows; whole numbers: exact sums."""
    V, H = 300, 24
    t = torch.repeat_interleave(torch.arange(V), torch.arange(1, V + 1)).cuda().to(torch.int32)
    t = t[torch.randperm(t.numel(), generator=torch.Generator().manual_seed(3)).cuda()]
    grad = torch.randint(-8, 9, (t.numel(), H), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).float()
    want = torch.zeros((V, H), dtype=torch.float64, device="cuda").index_add_(0, t.long(), grad.double()).float()
    assert torch.equal(binding.hola_embed_grad(t, grad, V), want)
    assert torch.equal(binding.hola_embed_grad(t, grad.bfloat16(), V), want)


@gpu
def test_vocabularies_of_any_size():
    for V in (1, 2, 147, 148, 149, 1536 * 148, 1536 * 148 + 1, 3000001):
        t = torch.tensor([0, V - 1, V // 2, V - 1, 0, max(0, V - 2)], device="cuda")
        grad = torch.arange(12.0, device="cuda").view(6, 2)
        rows = binding.hola_embed_grad_rows(t, grad, V)
        n = rows.count.item()
        want = sorted(set(t.tolist()))
        assert rows.ids[:n].tolist() == want
        for i, v in enumerate(want):
            assert torch.equal(rows.rows[i], grad[t == v].sum(dim=0))
        if V < 10 ** 6:
            assert torch.equal(binding.hola_embed_grad(t, grad, V), torch.zeros((V, 2), device="cuda").index_add_(0, t, grad))


@gpu
def test_strides_of_gradients():
    N, V = 100, 30
    t = some_tokens(N, V, 1).view(4, 25)
    for H in (8, 9, 1024):
        wide = rnd((4, 25, H + 8), torch.bfloat16, 2)
        for grad in (wide[..., :H], wide[..., 1:H + 1], wide[:1, :1, :H].expand(4, 25, H)):       # (a broadcast one)
            got = binding.hola_embed_grad(t, grad, V)
            check_grad(t, grad, V, 1.0, got)
            out = torch.full((V, H + 3), 7.0, device="cuda")
            binding.hola_embed_grad(t, grad, V, out=out[:, 1:H + 1])
            assert torch.equal(out[:, 1:H + 1], got) and (out[:, 0] == 7).all() and (out[:, H + 1:] == 7).all()
    for N in (0, 1):
        t, grad = torch.zeros(N, dtype=torch.int32, device="cuda"), torch.ones((N, 16), device="cuda")
        assert binding.hola_embed_grad(t, grad, 5).sum().item() == 16 * N
        assert binding.hola_embed_grad_rows(t, grad, 5).count.item() == N


@gpu
@pytest.mark.parametrize("H", [24, 25])
def test_gradient_against_differences(H):
    """f(W) = sum r * sin(lookup): its derivative along D, from the gradient and from (f(W + h D) - f(W - h D)) / 2 h with lookups in fp32,
    everything behind them in 64.  The difference's own error is h^2 / 6 sum |r D^3| (the third derivative of sin is at most 1), the
    lookups' roundings 2^-24 (|scale W| + h |scale D|) |r| / h, the gradient's 2^-24 (c + 3) of the sum of its terms."""
    N, V, scale, h = 400, 60, 1.5, 2.0 ** -8
    t, W, D = some_tokens(N, V, 1), rnd((V, H), torch.float32, 2), rnd((V, H), torch.float32, 3)
    r = rnd((N, H), torch.float64, 4)
    f = lambda w: float((r * torch.sin(binding.hola_embed(t, w.float(), scale).double())).sum())          # noqa: E731
    x = binding.hola_embed(t, W, scale).double()
    g = (r * torch.cos(x)).float()
    got = float((binding.hola_embed_grad(t, g, V, scale).double() * D.double()).sum())
    want = (f(W.double() + h * D.double()) - f(W.double() - h * D.double())) / (2 * h)
    d = scale * D[t.long().clamp_min(0)].double().abs() * (t >= 0)[:, None]
    w = scale * W[t.long().clamp_min(0)].double().abs()
    tol = h * h / 6 * (r.abs() * d ** 3).sum() + 2 * 2.0 ** -24 / h * (r.abs() * (w + h * d)).sum() + 2.0 ** -24 * (N + 3) * (r.abs() * d).sum()
    assert abs(got - want) <= float(tol) and abs(want) > 4 * float(tol)


@gpu
def test_streams_graphs_and_two_calls_at_once():
    N, V, H = 5000, 700, 256
    tokens = [some_tokens(N, V, i) for i in (1, 2)]
    grads = [rnd((N, H), torch.bfloat16, i) for i in (3, 4)]
    table = rnd((V, H), torch.bfloat16, 5)
    want = [(binding.hola_embed_grad(t, g, V), binding.hola_embed(t, table)) for t, g in zip(tokens, grads)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [(i, binding.hola_embed_grad(tokens[i], grads[i], V, stream=streams[i]), binding.hola_embed(tokens[i], table, stream=streams[i]))
           for _ in range(10) for i in (0, 1)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[i][0]) and torch.equal(b, want[i][1]) for i, a, b in got)
    # two graphs of the same kind, replayed by turns and together
    graphs = []
    for i in (0, 1):
        t, g, out = tokens[i].clone(), grads[i].clone(), torch.zeros((V, H), device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.hola_embed_grad(t, g, V, out=out)
        graphs.append((graph, t, g, out))
    for swap in (0, 1):
        for i, (graph, t, g, out) in enumerate(graphs):
            t.copy_(tokens[i ^ swap])
            g.copy_(grads[i ^ swap])
        torch.cuda.synchronize()
        for (graph, _, _, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out, want[i ^ swap][0]) for i, (_, _, _, out) in enumerate(graphs))


@gpu
def test_tables_and_gradients_beyond_32_bits():
    """Rows that begin more than 2^32 bytes into a table or a gradient."""
    V, H = 300001, 8192
    table = torch.empty((V, H), dtype=torch.bfloat16, device="cuda")
    t = torch.tensor([0, V - 1, 262144, 131072, V // 2], device="cuda")
    table[t] = rnd((5, H), torch.bfloat16, 1)
    assert torch.equal(binding.hola_embed(t, table), table[t])
    grad = torch.as_strided(table, (5, H), (75000 * H, 1))                        # rows 0, 75000 .. 300000 of the same memory
    grad.copy_(rnd((5, H), torch.bfloat16, 2))
    rows = binding.hola_embed_grad_rows(t, grad, V)
    order = torch.argsort(t)
    assert rows.ids.tolist() == t[order].tolist() and torch.equal(rows.rows, grad[order].float())
    del rows
    out = binding.hola_embed_grad(t, grad, V, dtype=torch.bfloat16)
    assert torch.equal(out[t], grad) and int(out.count_nonzero()) == int(grad.count_nonzero())


# ------------------------------------------------------------------------------------------------ refusals
def _embed_args(**kw):
    a = binding.hola_embed_args()
    a.N, a.V, a.H, a.row_stride, a.out_stride = 4, 10, 16, 16, 16
    a.tokens = a.table = a.out = 4096
    for name, v in kw.items():
        setattr(a, name, v)
    return a


@pytest.mark.parametrize("kw,status", [
    (dict(N=-1), 1), (dict(V=0), 1), (dict(H=0), 1), (dict(t_dtype=5), 1), (dict(out_dtype=3), 1), (dict(row_stride=-1), 1), (dict(out_stride=15), 1),
    (dict(tokens=None), 1), (dict(table=None), 1), (dict(out=None), 1), (dict(t_dtype=3), 1), (dict(w_scale=4096), 1), (dict(t_dtype=4, w_scale=4096), 2),
    (dict(t_dtype=4, w_scale=4096, H=128, out_stride=128), 1), (dict(v_offset=1), 1), (dict(v_offset=1, V_global=10), 1), (dict(v_offset=-1, V_global=20), 1),
    (dict(tokens=4098), 1), (dict(tokens=4100, wide_tokens=1), 1), (dict(out=4098), 1), (dict(add=4097), 1), (dict(N=2 ** 31), 2), (dict(N=0), 0)])
def test_lookups_that_are_refused(kw, status):
    lib = binding.load_library()
    assert lib.hola_embed(ctypes.byref(_embed_args(**kw)), None) == status
    assert lib.hola_embed(None, None) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(N=-1), 1), (dict(V=0), 1), (dict(H=0), 1), (dict(g_dtype=3), 1), (dict(out_dtype=3), 1), (dict(out_stride=15), 1), (dict(tokens=None), 1),
    (dict(grad=None), 1), (dict(out=None), 1), (dict(workspace=None), 1), (dict(workspace=4097), 1), (dict(workspace_bytes=100), 1), (dict(ids_out=4096), 1),
    (dict(count_out=4096), 1), (dict(ids_out=4096, count_out=4096, accumulate=1), 1), (dict(N=2 ** 31 - 1), 2), (dict(N=2 ** 25 + 1), 2), (dict(V=2 ** 30 + 1), 2), (dict(V=2 ** 31 - 1), 2), (dict(grad=4098), 1),
    (dict(v_offset=1), 1), (dict(v_offset=5, V_global=12), 1)])
def test_gradients_that_are_refused(kw, status):
    lib = binding.load_library()
    a = binding.hola_embed_grad_args()
    a.N, a.V, a.H, a.grad_stride, a.out_stride, a.workspace_bytes = 4, 10, 16, 16, 16, lib.hola_embed_grad_workspace_bytes(4, 10, 16)
    a.tokens = a.grad = a.out = a.workspace = 4096
    for name, v in kw.items():
        setattr(a, name, v)
    assert lib.hola_embed_grad(ctypes.byref(a), None) == status
    assert lib.hola_embed_grad(None, None) == 1
    assert lib.hola_embed_grad_workspace_bytes(-1, 10, 16) == 0 and lib.hola_embed_grad_workspace_bytes(4, 0, 16) == 0


def test_layout_of_the_structs():
    assert ctypes.sizeof(binding.hola_embed_args) == 8 + 16 + 8 + 8 + 4 * 8 + 8 + 5 * 8
    assert ctypes.sizeof(binding.hola_embed_grad_args) == 8 + 16 + 8 + 8 + 2 * 8 + 8 + 2 * 8 + 8 + 5 * 8


def test_tensors_without_a_device_are_refused():
    t, w = torch.zeros(3, dtype=torch.int32), torch.zeros((5, 8))
    for call in (lambda: binding.hola_embed(t, w), lambda: binding.hola_embed_grad(t, torch.zeros((3, 8)), 5),
                 lambda: binding.hola_embed_grad_rows(t, torch.zeros((3, 8)), 5), lambda: binding.hola_embed([1, 2], w)):
        with pytest.raises(binding.HolaError):
            call()


@gpu
def test_operands_that_are_refused():
    t, w = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((5, 8), device="cuda")
    g = torch.zeros((3, 8), device="cuda")
    s = torch.ones(5, device="cuda")
    for kw in (dict(tokens=t.short()), dict(tokens=t.cpu()), dict(tokens=torch.zeros(6, dtype=torch.int32, device="cuda")[::2]), dict(table=w.double()),
               dict(table=w[0]), dict(table=w.cpu()), dict(table=w.t()), dict(w_scale=s), dict(table=w.to(torch.int8)), dict(table=w.to(torch.int8), w_scale=s[:4]),
               dict(add=g[:2]), dict(add=g.half(), dtype=torch.float32), dict(out=g[:, :7]), dict(out=g.t().contiguous().t()), dict(dtype=torch.int32),
               dict(v_offset=1), dict(v_offset=2, V_global=6), dict(status=torch.zeros(1, device="cuda")), dict(add=g.cpu())):
        with pytest.raises(binding.HolaError):
            binding.hola_embed(**{"tokens": t, "table": w, **kw})
    for kw in (dict(tokens=t.cpu()), dict(grad=g.double()), dict(grad=g[:2]), dict(grad=g[:, :1].expand(3, 8)), dict(V=0), dict(accumulate=True), dict(out=w[:4]),
               dict(out=w.to(torch.int32)), dict(out=w.cpu()), dict(dtype=torch.int64), dict(out=w[:1].expand(5, 8))):
        with pytest.raises(binding.HolaError):
            binding.hola_embed_grad(**{"tokens": t, "grad": g, "V": 5, **kw})
    ids, rows, count = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((3, 8), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for out in (binding.TokenRows(ids[:2], rows, count), binding.TokenRows(ids, rows[:2], count), binding.TokenRows(ids, rows, ids),
                binding.TokenRows(ids.long(), rows, count), binding.TokenRows(ids, rows.cpu(), count)):
        with pytest.raises(binding.HolaError):
            binding.hola_embed_grad_rows(t, g, 5, out=out)


@gpu
def test_calls_through_the_native_helper_and_without_it(monkeypatch):
    """The same results and the same refusals either way."""
    V, H = 300, 128
    t = some_tokens(40, V, 1).view(5, 8)
    W, add, g = rnd((V, H), torch.bfloat16, 2), rnd((5, 8, H), torch.float32, 3), rnd((5, 8, H), torch.float16, 4)
    q, scale = binding.hola_quantize_w8(W)
    head = binding.hola_quantize_mixed(W, [4, 8])
    rows = lambda r: (lambda n: [r.ids[:n], r.rows[:n], r.count])(r.count.item())          # noqa: E731
    calls = [lambda: binding.hola_embed(t, W), lambda: binding.hola_embed(t.long(), W, 2, add=add), lambda: binding.hola_embed(t, q, 0.5, w_scale=scale),
             lambda: binding.hola_embed(t, head, dtype=torch.float32), lambda: binding.hola_embed(t, head, 3.0, add=add), lambda: binding.hola_embed(t[:0], W),
             lambda: binding.hola_embed(t, W[5:], v_offset=5, V_global=V), lambda: binding.hola_embed(t, W.float().t()),
             lambda: binding.hola_embed(t, W, add=add, dtype=torch.bfloat16), lambda: binding.hola_embed(t, W, dtype=torch.int32),
             lambda: binding.hola_embed(t, W, v_offset=5), lambda: binding.hola_embed_grad(t, g, V, 2.0), lambda: binding.hola_embed_grad(t, g, V, dtype=torch.bfloat16),
             lambda: binding.hola_embed_grad(t[:0], g[:0], V), lambda: binding.hola_embed_grad(t, g[:2], V), lambda: rows(binding.hola_embed_grad_rows(t, g, V)),
             lambda: rows(binding.hola_embed_grad_rows(t, g, 50, v_offset=10, V_global=V, dtype=torch.float16)), lambda: binding.hola_embed_grad_rows(t, g, 0)]

    def run():
        got = []
        for call in calls:
            try:
                o = call()
                got.append([x.cpu() for x in (o if isinstance(o, list) else [o])])
            except binding.HolaError as e:
                got.append(str(e))
        return got

    assert binding._host is not None
    with_it = run()
    monkeypatch.setattr(binding, "_host", None)
    for a, b in zip(with_it, run(), strict=True):
        assert a == b if isinstance(a, str) else all(x.dtype == y.dtype and torch.equal(x, y) for x, y in zip(a, b, strict=True))


@gpu
def test_outputs_on_another_stream_are_not_written_over():
    """Results of a call on another stream, dropped while the current one has still to read them, and the other way round."""
    N, V, H = 3000, 400, 512
    table = rnd((V, H), torch.float32, 1)
    tokens, grads = [some_tokens(N, V, i) for i in (2, 3)], [rnd((N, H), torch.float32, i) for i in (4, 5)]
    scores = [rnd((4, 3, 3000), torch.float32, i) for i in (6, 7)]
    logZ, score = [torch.logsumexp(x, 2) for x in scores], torch.zeros((4, 3), device="cuda")
    here, side = torch.cuda.current_stream(), torch.cuda.Stream()
    calls = [lambda i, s: [binding.hola_embed(tokens[i], table, stream=s)], lambda i, s: [binding.hola_embed_grad(tokens[i], grads[i], V, stream=s)],
             lambda i, s: [binding.hola_embed_grad_rows(tokens[i], grads[i], V, stream=s).count],
             lambda i, s: list(vars(binding.hola_beam_select(scores[i], logZ[i], score, stream=s)).values())[:3]]

    def busy(stream):
        with torch.cuda.stream(stream):
            torch.cuda._sleep(40_000_000)
    for call in calls:
        want = [[t.clone() for t in call(i, None)] for i in (0, 1)]
        torch.cuda.synchronize()
        got = call(0, side)
        here.wait_stream(side)
        busy(here)
        kept = [t.clone() for t in got]
        del got
        other = call(1, side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want[0])) and all(torch.equal(a, b) for a, b in zip(other, want[1]))
        busy(side)
        call(0, side)                                         # dropped at once
        fresh = [torch.full_like(t, 7) for t in want[0]]
        torch.cuda.synchronize()
        assert all((t == 7).all() for t in fresh)
        del kept, other, fresh


@gpu
def test_distillation_of_the_drivers_draft():
    """The gradient of KL(verifier || draft) by the draft's table against differences in 64 bits; the decode loop runs with it."""
    from paper_2506_18952_b200 import driver
    B, k, H, V, rounds = 4, 3, 64, 400, 3
    dev = torch.device("cuda", torch.cuda.current_device())
    models = driver.SyntheticPair(V, H, 7, dev, sharpness=0.5)
    t = torch.tensor([3, 9, 3, 399, 0, 9, 3, 12], device="cuda")
    p = torch.softmax(rnd((8, V), torch.float32, 1), dim=-1)
    got = models.draft_grad(t, models.E1, p)
    n = got.count.item()
    assert got.ids[:n].tolist() == [0, 3, 9, 12, 399]

    def loss(E):
        e = E[t]
        h = e / e.norm(dim=-1, keepdim=True) * models.gain[t].double()[:, None]
        return float(-(p.double() * torch.log_softmax(h @ models.W_lm.double().T, dim=-1)).sum() / 8)

    E, D, eps = models.E1.double(), rnd((V, H), torch.float64, 2), 1e-4
    want = (loss(E + eps * D) - loss(E - eps * D)) / (2 * eps)
    mine = float((got.rows[:n].double() * D[got.ids[:n].long()]).sum())
    # the draft's rows h are rounded to bf16 (2^-8 of each), which moves q by up to 2^-8 |h W| of itself, logits of about 0.5 here: some
    # 2^-9 of the gradient's terms, whose sizes are those of |dE D|
    size = float((got.rows[:n].double().abs() * D[got.ids[:n].long()].abs()).sum())
    assert abs(mine - want) <= 2.0 ** -8 * size and abs(want) > 2.0 ** -6 * size
    prompt = torch.randint(0, V, (B, 2), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    with binding.HolaVerify(B, k, H, V) as ctx:
        bare = driver.hsd_decode(ctx, models, prompt, k, 1.5, rounds, 3, keep_records=True)
        res = driver.hsd_decode(ctx, models, prompt, k, 1.5, rounds, 3, keep_records=True, distill=0.5)
    # (a round's q depends on the table through the rows of its own tokens alone, so what has moved shows in the table)
    assert torch.equal(res.records[0].draft_q, bare.records[0].draft_q) and bare.draft_table is None
    last = [prompt[:, 1], *(r.out.next_tok.long() for r in res.records)]
    used = {v for i, r in enumerate(res.records) for v in (*last[i].tolist(), *r.draft_tok[:, :k - 1].flatten().tolist())}
    assert set((res.draft_table != models.E1).any(dim=1).nonzero()[:, 0].tolist()) == used
    assert all(torch.isfinite(r.draft_q.float()).all() for r in res.records)


@gpu
def test_the_drivers_lookups_are_those_of_the_tables():
    from paper_2506_18952_b200 import driver
    models = driver.SyntheticPair(500, 96, 3, torch.device("cuda", torch.cuda.current_device()))
    a, b = some_tokens(60, 500, 1, torch.int64, 0.0).view(20, 3), some_tokens(60, 500, 2, torch.int64, 0.0).view(20, 3)
    assert torch.equal(models.target_hidden(a, b), models._norm(models.E1[a] + 0.35 * models.E2[b], a).to(torch.bfloat16))
    h = models._norm(models.E1[a], a).to(torch.bfloat16).float()
    assert torch.equal(models.draft_probs(a), torch.softmax(h @ models.W_lm.float().T, dim=-1))


@gpu
def test_what_absent_tokens_hold_is_not_read():
    """NaN and infinities in gradients of places without a token; in a table's rows that nobody names; in a row, for its own token alone."""
    N, V, H = 500, 90, 64
    t = some_tokens(N, V, 1, absent=0.3)
    grad = rnd((N, H), torch.float32, 2)
    want = binding.hola_embed_grad(t, grad, V)
    dirty = grad.clone()
    dirty[t < 0] = math.nan
    assert torch.equal(binding.hola_embed_grad(t, dirty, V), want)
    one = int(t[t >= 0][7])
    dirty[t == one] = math.inf
    got = binding.hola_embed_grad(t, dirty, V)
    assert (got[one] == math.inf).all()
    got[one] = want[one]
    assert torch.equal(got, want)
    table = rnd((V, H), torch.float32, 3)
    clean = binding.hola_embed(t, table, 2.0)
    table[[v for v in range(V) if v not in set(t.tolist())]] = math.nan
    assert torch.equal(binding.hola_embed(t, table, 2.0), clean)


@gpu
def test_the_most_tokens_of_a_call():
    """2^25 of them, whole numbers: every sum is exact."""
    N, V, H = 2 ** 25, 1000, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    t = torch.randint(-1, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    t[N - 5:] = 7
    grad = torch.randint(-1, 2, (N, H), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    want = torch.zeros((V + 1, H), dtype=torch.float64, device="cuda")
    for a in range(0, N, 1 << 22):
        want.index_add_(0, t[a:a + (1 << 22)].long() + 1, grad[a:a + (1 << 22)].double())
    assert torch.equal(binding.hola_embed_grad(t, grad, V).double(), want[1:])
    with pytest.raises(binding.HolaError):
        binding.hola_embed_grad(torch.zeros(N + 1, dtype=torch.int32, device="cuda"), grad[:1].expand(N + 1, H), V)


@gpu
@pytest.mark.parametrize("table_dtype", [*FLOATS, torch.int8])
@pytest.mark.parametrize("H", [1, 3, 15, 17, 333, 1001, 2050])
def test_rows_that_start_anywhere(H, table_dtype):
    """Tables, results and what is added on every address of their type, first and last rows of their buffers among them."""
    V, N = 41, 83
    tokens = some_tokens(N, V, H)
    tokens[:3] = torch.tensor([0, V - 1, 0], dtype=torch.int32)
    scale = rnd((V,), torch.float32, 1).abs() if table_dtype == torch.int8 else None
    for lead in range(0, 9):
        wide = H + lead % 3
        buf = rnd((lead + V * wide,), torch.float32, lead, 20.0).to(table_dtype)[lead:]
        table = buf.view(V, wide)[:, :H]
        rows32 = table.float() * scale[:, None] if scale is not None else table.float()
        for dtype in FLOATS:
            out = torch.full((N * (H + 1) + 9,), -3.0, dtype=dtype, device="cuda")
            view = out[lead:lead + N * (H + 1)].view(N, H + 1)[:, :H]
            add = rnd((N * H + lead,), dtype, 5)[lead:].view(N, H) if lead % 2 else None
            binding.hola_embed(tokens, table, 1.25, add=add, w_scale=scale, out=view)
            assert torch.equal(view, looked_up(tokens, rows32, 1.25, add, dtype))
            view.fill_(-3.0)
            assert (out == -3.0).all()                        # (nothing beside the rows has been written)


@gpu
@pytest.mark.parametrize("g_dtype", FLOATS)
@pytest.mark.parametrize("H", [1, 3, 15, 17, 333, 1001, 2050])
def test_gradients_that_start_anywhere(H, g_dtype):
    V, N = 60, 700
    tokens = some_tokens(N, V, H)
    for lead in (0, 1, 2, 5, 8):
        grad = rnd((N * (H + lead % 3) + lead,), g_dtype, lead)[lead:].view(N, -1)[:, :H]
        out = torch.full((V * (H + 1) + 9,), -3.0, device="cuda")
        view = out[lead:lead + V * (H + 1)].view(V, H + 1)[:, :H]
        binding.hola_embed_grad(tokens, grad, V, 0.5, out=view)
        check_grad(tokens, grad, V, 0.5, view)
        view.fill_(-3.0)
        assert (out == -3.0).all()


def test_results_on_what_is_read_are_refused():
    """Rows that share a byte with the table, the addend, the gradient or the tokens; views side by side in one buffer do not."""
    lib = binding.load_library()
    e = dict(table=1 << 20, tokens=1 << 16, out=1 << 24, out_stride=40, add_stride=40)
    for kw in (dict(out=1 << 20, out_stride=16), dict(out=(1 << 20) - 4), dict(out=(1 << 20) + 9 * 64 + 60), dict(tokens=(1 << 24) + 64 - 4),
               dict(add=(1 << 24) + 60), dict(add=(1 << 24) - 60), dict(add=(1 << 24) + 160 - 60), dict(add=1 << 24, add_stride=0),
               dict(add=1 << 24, add_stride=16), dict(add=(1 << 24) + 160 + 60)):
        assert lib.hola_embed(ctypes.byref(_embed_args(**{**e, **kw})), None) == 1, kw
    beside = lib.hola_embed(ctypes.byref(_embed_args(**{**e, "add": (1 << 24) + 64})), None) if not torch.cuda.is_available() else 5
    assert beside != 1                                        # (no device here: nothing runs)
    a = binding.hola_embed_grad_args()
    a.N, a.V, a.H, a.grad_stride, a.out_stride, a.workspace_bytes = 4, 10, 16, 16, 16, lib.hola_embed_grad_workspace_bytes(4, 10, 16)
    a.tokens, a.grad, a.out, a.workspace = 1 << 16, 1 << 20, 1 << 24, 1 << 26
    for kw in (dict(out=1 << 20), dict(out=(1 << 20) + 3 * 64 + 60), dict(out=(1 << 20) - 9 * 64 - 60), dict(tokens=(1 << 24) + 636), dict(out=(1 << 16) + 12)):
        kept = {name: getattr(a, name) for name in kw}
        for name, at in kw.items():
            setattr(a, name, at)
        assert lib.hola_embed_grad(ctypes.byref(a), None) == 1, kw
        for name, at in kept.items():
            setattr(a, name, at)


@gpu
def test_results_beside_what_is_read():
    """Both halves of the rows of one buffer: the addend in one, the result in the other; and the addend itself."""
    g = torch.Generator(device="cuda").manual_seed(8)
    for H in (64, 33):
        table = torch.randn((50, H), generator=g, device="cuda")
        t = torch.randint(50, (37,), generator=g, device="cuda")
        buf = torch.randn((37, 2 * H), generator=g, device="cuda")
        kept = buf.clone()
        binding.hola_embed(t, table, 0.5, add=buf[:, H:], out=buf[:, :H])
        assert torch.equal(buf[:, :H], kept[:, H:] + 0.5 * table[t]) and torch.equal(buf[:, H:], kept[:, H:])
        binding.hola_embed(t, table, add=buf[:, H:], out=buf[:, H:])
        assert torch.equal(buf[:, H:], kept[:, H:] + table[t])
        with pytest.raises(binding.HolaError):
            binding.hola_embed(t, table, add=buf[:, H:], out=buf[:, H - 1:-1])
        with pytest.raises(binding.HolaError):
            binding.hola_embed(t, table, out=table[:37])
        with pytest.raises(binding.HolaError):
            binding.hola_embed_grad(t[:20], buf[:20, :H], 37, out=buf[:, 1:H + 1])


@gpu
@pytest.mark.parametrize("g_dtype", FLOATS)
@pytest.mark.parametrize("N", [0, 1, 17, 511, 512, 513, 700])
def test_gradients_of_few_tokens_and_of_some_more(N, g_dtype):
    """Ids with 15, 16, 17 and with most of the rows, absent and wrong tokens, results that lie apart, all forms of the result."""
    V, wrong = 90, 3 if N > 17 else 0
    for H in (5, 64, 72, 257, 2056):
        t = torch.arange(N) % 5 * 18
        for i, n in enumerate((15, 16, 17, 1, 2, 63, 64, 65)):
            if N > 400:
                t[sum((15, 16, 17, 1, 2, 63, 64, 65)[:i]):][:n] = 80 + i
        t[N // 2:N // 2 + N // 7] = -1
        if wrong:
            t[:wrong] = torch.tensor([V, -2, 2 ** 31 - 1])
        t = t[torch.randperm(N, generator=torch.Generator().manual_seed(N + H))].cuda()
        t = t if H == 64 else t.int()
        wide = rnd((N, H + 11), g_dtype, H)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        for grad in (wide[:, :H].contiguous(), wide[:, :H], wide[:, 3:H + 3]):
            got = binding.hola_embed_grad(t, grad, V, 0.7, status=status)
            check_grad(t, grad, V, 0.7, got)
            base = rnd((V, H + 5), torch.float32, 6)
            for lead in (0, 1):
                out = base.clone()
                binding.hola_embed_grad(t, grad, V, 0.7, out=out[:, lead:lead + H])
                assert torch.equal(out[:, lead:lead + H], got)
                out[:, lead:lead + H] = base[:, lead:lead + H]
                assert torch.equal(out, base)
                binding.hola_embed_grad(t, grad, V, 0.7, out=out[:, lead:lead + H], accumulate=True)
                check_grad(t, grad, V, 0.7, out[:, lead:lead + H], before=base[:, lead:lead + H])
            rows = binding.TokenRows(torch.full((N,), -7, dtype=torch.int32, device="cuda"), torch.full((N, H), -7.0, device="cuda"),
                                     torch.full((1,), -7, dtype=torch.int32, device="cuda"))
            binding.hola_embed_grad_rows(t, grad, V, 0.7, out=rows)
            ids = sorted({v for v in t.tolist() if 0 <= v < V})
            n = rows.count.item()
            assert rows.ids[:n].tolist() == ids and (rows.ids[n:] == -7).all() and (rows.rows[n:] == -7).all()
            assert torch.equal(rows.rows[:n], got[rows.ids[:n].long()])
        assert status.item() == (binding.FLAG_BAD_TOKEN if wrong else 0)


@gpu
@pytest.mark.parametrize("N", [300, 600])
def test_ids_of_few_tokens_that_share_places_of_the_table(N):
    """Ids at equal distances of 2^20 and the largest ones, each some times, in a falling order."""
    V = 2 ** 30
    t = torch.cat([torch.arange(N // 3) * 2 ** 20, V - 1 - torch.arange(N // 3), torch.arange(N // 3) * 2 ** 20]).flip(0).cuda() % V
    grad = torch.randint(-8, 9, (t.numel(), 8), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).float()
    rows = binding.hola_embed_grad_rows(t, grad, V)
    ids, which = torch.unique(t, return_inverse=True)
    n = rows.count.item()
    assert torch.equal(rows.ids[:n].long(), ids)
    assert torch.equal(rows.rows[:n], torch.zeros((n, 8), dtype=torch.float64, device="cuda").index_add_(0, which, grad.double()).float())


def test_gradients_by_rows_on_what_is_read_or_on_one_another_are_refused():
    """CTAs read the tokens and the gradient while others write ids, rows and their number."""
    lib = binding.load_library()
    a = binding.hola_embed_grad_args()
    for N in (4, 600):                                        # (one launch, and two)
        need = lib.hola_embed_grad_workspace_bytes(N, 10, 16)
        a.N, a.V, a.H, a.grad_stride, a.out_stride, a.workspace_bytes = N, 10, 16, 16, 20, need
        ok = dict(tokens=1 << 16, grad=1 << 20, out=1 << 24, ids_out=1 << 28, count_out=1 << 29, workspace=1 << 30)
        for name, at in ok.items():
            setattr(a, name, at)
        row, last = 4 * N, (1 << 24) + 80 * (N - 1)
        for kw in (dict(ids_out=1 << 16), dict(ids_out=(1 << 16) + row - 4), dict(ids_out=(1 << 16) - row + 4), dict(ids_out=1 << 20),
                   dict(ids_out=(1 << 20) + 64 * N - 4), dict(ids_out=1 << 24), dict(count_out=1 << 16), dict(count_out=(1 << 16) + row - 4),
                   dict(count_out=(1 << 20) + 60), dict(count_out=last + 60), dict(count_out=1 << 28), dict(count_out=(1 << 28) + row - 4),
                   dict(workspace=1 << 16), dict(workspace=1 << 20), dict(workspace=1 << 24), dict(workspace=1 << 28), dict(tokens=(1 << 30) + need - 4),
                   dict(count_out=(1 << 30) + 8), dict(grad=(1 << 30) + need - 4), dict(out=(1 << 30) - last + (1 << 24) - 60)):
            for name, at in kw.items():
                setattr(a, name, at)
            assert lib.hola_embed_grad(ctypes.byref(a), None) == 1, (N, kw)
            for name in kw:
                setattr(a, name, ok[name])
        if not torch.cuda.is_available():                     # (no device here: nothing runs)
            for kw in ({}, dict(count_out=last + 64), dict(ids_out=(1 << 16) + row), dict(count_out=(1 << 28) + row)):
                for name, at in kw.items():
                    setattr(a, name, at)
                assert lib.hola_embed_grad(ctypes.byref(a), None) not in (0, 1), (N, kw)
                for name in kw:
                    setattr(a, name, ok[name])


@gpu
@pytest.mark.parametrize("N", [300, 600])
def test_ids_in_the_tokens_place_are_refused(N, monkeypatch):
    t, grad = some_tokens(N, 50, 1), rnd((N, 16), torch.float32, 2)
    kept = t.clone()
    rows, count = torch.zeros((N, 16), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(2):                                        # through the native helper and without it
        for out in (binding.TokenRows(t, rows, count), binding.TokenRows(torch.zeros_like(t), grad, count), binding.TokenRows(torch.zeros_like(t), rows, t[:1])):
            with pytest.raises(binding.HolaError):
                binding.hola_embed_grad_rows(t, grad, 50, out=out)
        monkeypatch.setattr(binding, "_host", None)
    assert torch.equal(t, kept)


def test_channels_that_32_bits_do_not_step_over_are_refused():
    """Every type of the table, rows on aligned addresses and on others."""
    lib = binding.load_library()
    for H, refused in ((2 ** 31 - 65537, True), (2 ** 31 - 65536, True), (2010000000, True), (2 ** 30 + 128, True), (2 ** 30, False), (2 ** 30 - 1, False)):
        for t_dtype, lead in ((0, 0), (1, 0), (2, 4), (3, 0), (3, 1)):
            a = _embed_args(N=1, V=2, H=H, t_dtype=t_dtype, row_stride=H, out_stride=H, table=(1 << 20) + lead, out=1 << 44, w_scale=1 << 45 if t_dtype == 3 else None)
            if refused:
                assert lib.hola_embed(ctypes.byref(a), None) == 2, (H, t_dtype)
            elif not torch.cuda.is_available():               # (no device here: nothing runs)
                assert lib.hola_embed(ctypes.byref(a), None) not in (0, 1, 2), (H, t_dtype)


@gpu
@pytest.mark.parametrize("H,lead", [(2 ** 27 + 24, 0), (2 ** 26 + 1001, 1)])
def test_rows_of_more_channels_than_slices_of_a_launch(H, lead):
    table = torch.randint(-20000, 20000, (2 * H + lead,), device="cuda", dtype=torch.int16, generator=torch.Generator(device="cuda").manual_seed(1))
    table = table.view(torch.bfloat16)[lead:].view(2, H)
    out = torch.zeros((3, H), dtype=torch.bfloat16, device="cuda")
    binding.hola_embed(torch.tensor([1, -1, 0], device="cuda"), table, out=out)
    # (the bits of -127 .. -1 are NaN, which comes out as a NaN, perhaps another one; everything else bit by bit)
    for got, want in ((out[0], table[1]), (out[2], table[0])):
        nan = want.isnan()
        assert bool((got.isnan() == nan).all()) and bool(((got.view(torch.int16) == want.view(torch.int16)) | nan).all())
    assert int(out[1].count_nonzero()) == 0


@pytest.mark.parametrize("V,H", [(1, 1), (300, 16), (32000, 4096), (128256, 256), (128256, 257), (2 ** 30, 64)])
def test_a_workspace_for_many_tokens_serves_fewer(V, H):
    """The size that is asked for rises with the number of tokens, across all borders of the plan, and the call takes the size for more."""
    lib = binding.load_library()
    borders = [1, 512, 1024, 65535, *(512 * 32 * 2 ** i for i in range(6)), 2 ** 25 - 1]
    counts = sorted({n for b in borders for n in (b - 1, b, b + 1, b + 40)} | {int(1.03 ** i) for i in range(1, 586)})
    sizes = [lib.hola_embed_grad_workspace_bytes(n, V, H) for n in counts if n <= 2 ** 25]
    assert sizes == sorted(sizes) and min(sizes) > 0
    a = binding.hola_embed_grad_args()
    a.V, a.H, a.grad_stride, a.out_stride, a.tokens, a.grad, a.out, a.workspace = V, H, 0, H, 1 << 40, 1 << 41, 1 << 50, 1 << 45
    a.ids_out, a.count_out = 1 << 42, 1 << 43
    for n, more in zip(counts, sizes[1:]):
        a.N, a.workspace_bytes = n, more
        if not torch.cuda.is_available():                     # (no device here: nothing runs)
            assert lib.hola_embed_grad(ctypes.byref(a), None) not in (0, 1), n


def test_the_drivers_models_on_the_host():
    """Hidden rows and draft probabilities of models that lie on the CPU, from the tables as they are."""
    from paper_2506_18952_b200 import driver
    models = driver.SyntheticPair(300, 32, 3, torch.device("cpu"))
    g = torch.Generator().manual_seed(1)
    a, b = torch.randint(0, 300, (2, 5, 6), generator=g).unbind(0)
    want = models._norm(models.E1[a] + 0.35 * models.E2[b], a).to(torch.bfloat16)
    assert torch.equal(models.target_hidden(a, b), want) and torch.equal(models.target_hidden(a.t(), b.t()), want.transpose(0, 1))
    h = models._norm(models.E1[a], a).to(torch.bfloat16).float()
    assert torch.equal(models.draft_probs(a), torch.softmax(h @ models.W_lm.float().T, dim=-1))


def test_results_on_scales_codes_and_their_tables_are_refused():
    """What a lookup in the quantised forms reads beside the table: one byte of it in one row of the result."""
    lib = binding.load_library()
    out, N, V, H = 1 << 30, 3, 600, 128
    last = out + 2 * 160 * 4 + 4 * H                          # (rows of fp32, 160 entries apart)
    a = _embed_args(N=N, V=V, H=H, t_dtype=3, row_stride=H, out=out, out_stride=160, w_scale=1 << 24, table=1 << 20)
    for at, status in ((out, 1), (last - 4, 1), (out - 4 * V + 4, 1), (last, 0), (out - 4 * V, 0)):
        a.w_scale = at
        if status or not torch.cuda.is_available():           # (no device here: nothing runs)
            assert (lib.hola_embed(ctypes.byref(a), None) == 1) == bool(status), at
    mix = binding.hola_wmix()
    sizes = dict(W16=88 * H * 2, W8=256 * H, W4=256 * H // 2, shift4=256, group_width=3, group_row=12)
    for i, name in enumerate(sizes):
        setattr(mix, name, (2 + i) << 32)
    mix.rows16, mix.rows8, mix.rows4 = 88, 256, 256
    a.t_dtype, a.w_scale, a.wmix, a.table = 4, 1 << 24, ctypes.addressof(mix), None
    for name, size in sizes.items():
        kept = getattr(mix, name)
        step = {"W16": 2, "group_row": 4}.get(name, 1)
        for at, status in ((out, 1), (last - step, 1), (out - size + step, 1), (last, 0), (out - size, 0)):
            setattr(mix, name, at)
            if status or not torch.cuda.is_available():
                assert (lib.hola_embed(ctypes.byref(a), None) == 1) == bool(status), (name, at)
        setattr(mix, name, kept)


def test_large_vocabularies_by_rows_and_added_to_are_not_refused_for_zeros_that_nobody_writes():
    lib = binding.load_library()
    a = binding.hola_embed_grad_args()
    N, V, H = 600, 2 ** 30, 2 ** 18
    a.N, a.V, a.H, a.grad_stride, a.out_stride, a.workspace_bytes = N, V, H, 0, H, lib.hola_embed_grad_workspace_bytes(N, V, H)
    a.tokens, a.grad, a.out, a.workspace = 1 << 16, 1 << 20, 1 << 56, 1 << 40
    assert lib.hola_embed_grad(ctypes.byref(a), None) == 2    # (the whole table: 2^24 x 256 CTAs of zeros and more)
    if not torch.cuda.is_available():                         # (no device here: nothing runs)
        a.accumulate = 1
        assert lib.hola_embed_grad(ctypes.byref(a), None) not in (0, 1, 2)
        a.accumulate, a.ids_out, a.count_out = 0, 1 << 17, 1 << 18
        assert lib.hola_embed_grad(ctypes.byref(a), None) not in (0, 1, 2)


@gpu
def test_sizes_that_are_not_served_are_refused_before_anything_is_made(monkeypatch):
    """2^30 + 1 rows of the whole table would be more memory than there is."""
    t, grad = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros((4, 4096), device="cuda")
    many = torch.zeros(2 ** 25 + 1, dtype=torch.int32, device="cuda")
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    for _ in range(2):                                        # through the native helper and without it
        for call in (lambda: binding.hola_embed_grad(t, grad, 2 ** 30 + 1), lambda: binding.hola_embed_grad_rows(t, grad, 2 ** 30 + 1),
                     lambda: binding.hola_embed_grad_rows(many, grad[:1, :8].expand(2 ** 25 + 1, 8), 100)):
            with pytest.raises(binding.HolaError, match="at most"):
                call()
        monkeypatch.setattr(binding, "_host", None)
    assert torch.cuda.max_memory_allocated() == before


def test_operands_on_no_address_of_their_type_are_refused():
    lib = binding.load_library()
    a = _embed_args(t_dtype=3, w_scale=1 << 24, out=1 << 28, status_word=1 << 29)
    mix = binding.hola_wmix()
    mix.W16, mix.group_width, mix.group_row, mix.rows16 = 1 << 32, 1 << 33, 1 << 34, 10
    b = _embed_args(t_dtype=4, H=128, out_stride=128, out=1 << 28, w_scale=1 << 24, wmix=ctypes.addressof(mix))
    g = binding.hola_embed_grad_args()
    g.N, g.V, g.H, g.grad_stride, g.out_stride, g.workspace_bytes = 4, 10, 16, 16, 16, 256
    g.tokens, g.grad, g.out, g.workspace, g.ids_out, g.count_out, g.status_word = (1 << (16 + i) for i in range(7))
    for call, args, of, name in ((lib.hola_embed, a, a, "w_scale"), (lib.hola_embed, a, a, "status_word"), (lib.hola_embed, b, b, "w_scale"),
                                 (lib.hola_embed, b, mix, "W16"), (lib.hola_embed, b, mix, "group_row"), (lib.hola_embed_grad, g, g, "ids_out"),
                                 (lib.hola_embed_grad, g, g, "count_out"), (lib.hola_embed_grad, g, g, "status_word")):
        kept = getattr(of, name)
        for off in (0, 1, 3) if name == "W16" else (0, 1, 2, 3):
            setattr(of, name, kept + off)
            if off or not torch.cuda.is_available():          # (no device here: nothing runs)
                assert (call(ctypes.byref(args), None) == 1) == (off > 0), (name, off)
        setattr(of, name, kept)


# ------------------------------------------------------------------------------------------------ one launch and two
# Up to 512 tokens are served by one kernel, more by a sort (of 16 warps, of more from 1025 tokens on, with wide counters from 65536) and the
# sums behind it: what every call is promised, on all sides of these borders.
BOTH = [300, 513, 1025, 66000]


def spread_over(t, N, seed):
    """The tokens of `t`, each at some places of N, in some order; -1 elsewhere."""
    g = torch.Generator().manual_seed(seed)
    out = torch.full((N,), -1, dtype=torch.int64)
    at = torch.randperm(N, generator=g)
    times = max(1, N // (2 * t.numel()))
    out[at[:t.numel() * times]] = t.cpu().long().repeat(times)
    return out.cuda()


@gpu
@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("N", BOTH)
def test_gradients_of_parts_of_a_vocabulary(N, dtype):
    V, H, cuts = 1000, 72, [0, 130, 131, 600, 1000]
    tokens, grad = some_tokens(N, V, 4, dtype), rnd((N, H), torch.float32, 5)
    dense = binding.hola_embed_grad(tokens, grad, V, 3.0)
    check_grad(tokens, grad, V, 3.0, dense)
    status, ids = torch.zeros(1, dtype=torch.int32, device="cuda"), []
    for a, b in zip(cuts, cuts[1:]):
        for whole in (V, 2 ** 31 - 1):                        # (the same part of a larger vocabulary)
            assert torch.equal(binding.hola_embed_grad(tokens, grad, b - a, 3.0, v_offset=a, V_global=whole, status=status), dense[a:b])
            rows = binding.hola_embed_grad_rows(tokens, grad, b - a, 3.0, v_offset=a, V_global=whole, status=status)
            n = rows.count.item()
            assert torch.equal(rows.rows[:n], dense[rows.ids[:n].long()])
        ids += rows.ids[:n].tolist()
    assert status.item() == 0 and ids == sorted(set(tokens.tolist()) - {-1})
    # the last part of the largest vocabulary: ids up to 2^31 - 2
    shift = 2 ** 31 - 1 - V
    far = torch.where(tokens >= 0, tokens + shift, -1)
    assert torch.equal(binding.hola_embed_grad(far, grad, V, 3.0, v_offset=shift, V_global=2 ** 31 - 1, status=status), dense)
    rows = binding.hola_embed_grad_rows(far, grad, V, 3.0, v_offset=shift, V_global=2 ** 31 - 1, status=status)
    n = rows.count.item()
    assert rows.ids[:n].tolist() == [v + shift for v in ids] and torch.equal(rows.rows[:n], dense[(rows.ids[:n] - shift).long()])
    assert status.item() == 0
    binding.hola_embed_grad(tokens, grad, 130, v_offset=0, V_global=999, status=status)
    assert status.item() == (binding.FLAG_BAD_TOKEN if bool((tokens == 999).any()) else 0)


@gpu
@pytest.mark.parametrize("N", BOTH)
def test_gradients_of_tokens_that_there_are_not(N):
    V, H = 50, 40
    some = torch.tensor([0, 49, 50, -2, 2 ** 31 - 1, -2 ** 31, 7])
    big = torch.tensor([2 ** 32, 2 ** 32 + 3, 2 ** 40 - 1, -2 ** 32 + 5, 2 ** 63 - 1, -2 ** 63, 2 ** 32 - 1])          # not 0, 3, -1, 5, -1, 0, -1 cut off
    for t in (some.int(), some, big):
        tokens = spread_over(t, N, 1).to(t.dtype)
        grad = rnd((N, H), torch.float32, 2)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = binding.hola_embed_grad(tokens, grad, V, status=status)
        assert status.item() == binding.FLAG_BAD_TOKEN
        check_grad(tokens, grad, V, 1.0, got)
        assert set(got.count_nonzero(dim=1).nonzero()[:, 0].tolist()) == ({0, 7, 49} if t is not big else set())
        rows = binding.hola_embed_grad_rows(tokens, grad, V)
        assert rows.ids[:rows.count.item()].tolist() == ([0, 7, 49] if t is not big else [])
        status.zero_()
        fine = torch.where((tokens >= 0) & (tokens < V), tokens, -1)
        assert torch.equal(binding.hola_embed_grad(fine, grad, V, status=status), got) and status.item() == 0


@gpu
@pytest.mark.parametrize("N", BOTH)
def test_gradients_of_vocabularies_of_any_size(N):
    """Whole numbers: exact sums.  (Where the marks of the sort's ranges coincide.)"""
    for V in (1, 2, 3, 73, 74, 75, 147, 148, 149, 1536 * 148, 1536 * 148 + 1, 3000001):
        few = torch.tensor(sorted({0, V - 1, V // 2, max(0, V - 2), min(1, V - 1), V // 3}))
        t = spread_over(few, N, V)
        grad = torch.randint(-8, 9, (N, 8), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).float()
        rows = binding.hola_embed_grad_rows(t, grad, V)
        n = rows.count.item()
        assert rows.ids[:n].tolist() == few.tolist()
        for i, v in enumerate(few.tolist()):
            assert torch.equal(rows.rows[i], grad[t == v].double().sum(dim=0).float())
        if V < 10 ** 6:
            assert torch.equal(binding.hola_embed_grad(t, grad, V)[few.cuda()], rows.rows[:n])


@gpu
@pytest.mark.parametrize("N", BOTH)
def test_strides_of_gradients_of_few_and_of_many_tokens(N):
    """Rows further apart, on any address, one row for all; results in a part of a wider buffer."""
    V = 30
    t = some_tokens(N, V, 1)
    for H in (8, 9, 256, 264) if N > 2000 else (8, 9, 264, 1024):
        wide = rnd((N, H + 8), torch.bfloat16, 2)
        for grad in (wide[:, :H], wide[:, 1:H + 1], wide[:1, :H].expand(N, H), wide[:1, 3:H + 3].expand(N, H)):
            got = binding.hola_embed_grad(t, grad, V)
            check_grad(t, grad, V, 1.0, got)
            for lead in (0, 1):
                out = torch.full((V, H + 3), 7.0, device="cuda")
                binding.hola_embed_grad(t, grad, V, out=out[:, lead:lead + H])
                assert torch.equal(out[:, lead:lead + H], got)
                out[:, lead:lead + H] = 7.0
                assert (out == 7.0).all()
            rows = binding.hola_embed_grad_rows(t, grad, V)
            n = rows.count.item()
            assert torch.equal(rows.rows[:n], got[rows.ids[:n].long()])


@gpu
@pytest.mark.parametrize("N", [300, 600])
def test_gradients_beyond_32_bits(N):
    """Rows that begin more than 2^32 bytes into a gradient, and into its result."""
    V, H = 300001, 8192
    buf = torch.empty((V, H), dtype=torch.bfloat16, device="cuda")
    grad = torch.as_strided(buf, (N, H), (300000 // N * H, 1))
    grad.copy_(rnd((N, H), torch.bfloat16, 2))
    t = torch.full((N,), -1, dtype=torch.int64, device="cuda")
    at = torch.tensor([0, N - 1, N // 2, N - 2, 5], device="cuda")
    t[at] = torch.tensor([V - 1, 0, 262144, 131072, V // 2], device="cuda")
    rows = binding.hola_embed_grad_rows(t, grad, V)
    order = torch.argsort(t[at])
    assert rows.count.item() == 5 and torch.equal(rows.ids[:5].long(), t[at][order]) and torch.equal(rows.rows[:5], grad[at][order].float())
    out = binding.hola_embed_grad(t, grad, V, dtype=torch.bfloat16)
    assert torch.equal(out[t[at]], grad[at]) and int(out.count_nonzero()) == int(grad[at].count_nonzero())


@gpu
@pytest.mark.parametrize("N", BOTH)
def test_gradients_of_absent_tokens_and_of_rows_that_are_not_finite(N):
    V, H = 90, 64
    t = some_tokens(N, V, 1, absent=0.3)
    grad = rnd((N, H), torch.float32, 2)
    want = binding.hola_embed_grad(t, grad, V)
    dirty = grad.clone()
    dirty[t < 0] = math.nan
    assert torch.equal(binding.hola_embed_grad(t, dirty, V), want)
    one = int(t[t >= 0][7])
    dirty[t == one] = math.inf
    got = binding.hola_embed_grad(t, dirty, V)
    assert (got[one] == math.inf).all()
    got[one] = want[one]
    assert torch.equal(got, want)


@gpu
@pytest.mark.parametrize("N", BOTH)
def test_gradients_through_the_native_helper_and_without_it(N, monkeypatch):
    V, H = 300, 128
    t, g = some_tokens(N, V, 1), rnd((N, H), torch.float16, 4)

    def run():
        got = [binding.hola_embed_grad(t, g, V, 2.0), binding.hola_embed_grad(t.long(), g, V, dtype=torch.bfloat16),
               binding.hola_embed_grad(t, g, 100, v_offset=200, V_global=V)]
        for rows in (binding.hola_embed_grad_rows(t, g, V), binding.hola_embed_grad_rows(t, g, 50, v_offset=10, V_global=V, dtype=torch.float16)):
            n = rows.count.item()
            got += [rows.ids[:n], rows.rows[:n]]
        return got

    assert binding._host is not None
    with_it = run()
    monkeypatch.setattr(binding, "_host", None)
    assert all(x.dtype == y.dtype and torch.equal(x, y) for x, y in zip(with_it, run(), strict=True))


@gpu
@pytest.mark.parametrize("N", BOTH)
def test_captured_gradients_two_at_once(N):
    """Two graphs of a lookup and both forms of its gradient, replayed by turns, together and with other inputs."""
    V, H = 700, 256
    tokens, grads = [some_tokens(N, V, i) for i in (1, 2)], [rnd((N, H), torch.bfloat16, i) for i in (3, 4)]
    table = rnd((V, H), torch.bfloat16, 5)
    want = [(binding.hola_embed(t, table), binding.hola_embed_grad(t, g, V), binding.hola_embed_grad_rows(t, g, V)) for t, g in zip(tokens, grads)]
    graphs = []
    for i in (0, 1):
        t, g = tokens[i].clone(), grads[i].clone()
        out = [torch.zeros((N, H), dtype=torch.bfloat16, device="cuda"), torch.zeros((V, H), device="cuda"),
               binding.TokenRows(torch.zeros_like(want[i][2].ids), torch.zeros((N, H), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.hola_embed(t, table, out=out[0])
            binding.hola_embed_grad(t, g, V, out=out[1])
            binding.hola_embed_grad_rows(t, g, V, out=out[2])
        graphs.append((graph, t, g, out))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for swap in (0, 1, 0):
        for i, (_, t, g, _) in enumerate(graphs):
            t.copy_(tokens[i ^ swap])
            g.copy_(grads[i ^ swap])
        torch.cuda.synchronize()
        for _ in range(5):
            for (graph, *_), s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    graph.replay()
        torch.cuda.synchronize()
        for i, (*_, out) in enumerate(graphs):
            e, d, r = want[i ^ swap]
            n = r.count.item()
            assert torch.equal(out[0], e) and torch.equal(out[1], d) and out[2].count.item() == n
            assert torch.equal(out[2].ids[:n], r.ids[:n]) and torch.equal(out[2].rows[:n], r.rows[:n])


@gpu
@pytest.mark.parametrize("N", [700, 1500])
def test_gradient_of_many_tokens_against_differences(N):
    """As test_gradient_against_differences, where a sort comes first; the same bounds."""
    H, V, scale, h = 25, 60, 1.5, 2.0 ** -8
    t, W, D = some_tokens(N, V, 1), rnd((V, H), torch.float32, 2), rnd((V, H), torch.float32, 3)
    r = rnd((N, H), torch.float64, 4)
    f = lambda w: float((r * torch.sin(binding.hola_embed(t, w.float(), scale).double())).sum())          # noqa: E731
    g = (r * torch.cos(binding.hola_embed(t, W, scale).double())).float()
    got = float((binding.hola_embed_grad(t, g, V, scale).double() * D.double()).sum())
    want = (f(W.double() + h * D.double()) - f(W.double() - h * D.double())) / (2 * h)
    d = scale * D[t.long().clamp_min(0)].double().abs() * (t >= 0)[:, None]
    w = scale * W[t.long().clamp_min(0)].double().abs()
    tol = h * h / 6 * (r.abs() * d ** 3).sum() + 2 * 2.0 ** -24 / h * (r.abs() * (w + h * d)).sum() + 2.0 ** -24 * (N + 3) * (r.abs() * d).sum()
    assert abs(got - want) <= float(tol)
