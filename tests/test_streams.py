"""Memory of a call's own outputs when the call runs on another stream than the current one."""
import pytest
import torch

from paper_2506_18952_b200 import binding, workloads

gpu = pytest.mark.gpu
B, K, H, V = 4, 3, 256, 9000


def _runs(ctx):
    """name -> run(i, stream): a call on inputs i (0 or 1) that makes its own outputs, as a list of them."""
    x = [workloads.gaussian_head("streams", B, K, H, V, seed=60 + i, device="cuda", w_std=2.0 / H ** 0.5, sigma=0.5, tau=2.0, sigma_far=1.5,
                                 q_dtype=torch.bfloat16) for i in (0, 1)]
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")                     # noqa: E731
    bank = binding.AdapterBank((rnd(2, 8, H) / H ** 0.5).bfloat16(), rnd(2, V, 8).bfloat16())
    ids = torch.tensor([0, 1, -1, 1], dtype=torch.int32, device="cuda")
    tokens = torch.full((B, K + 1), 5, dtype=torch.int32, device="cuda")           # (every input is there before a call is queued)
    heads = [ctx.hola_lm_head_entropy(w.hidden, w.W_lm) for w in x]
    tensors = lambda o: [t for t in vars(o).values() if isinstance(t, torch.Tensor)]        # noqa: E731
    verify = lambda w: (w.hidden, w.W_lm, w.draft_tok, w.draft_q, w.uniforms, w.tau)        # noqa: E731

    def accept_sample(i, s):
        w, h = x[i], heads[i]
        out = ctx.hola_accept_sample(h.logits, h.entropy, h.logZ, w.draft_tok, w.draft_q, w.uniforms, w.tau, stream=s)
        return [out.accept_len, out.next_tok, out.entropy, out.logZ]

    return {
        "lm_head": lambda i, s: tensors(ctx.hola_lm_head_entropy(x[i].hidden, x[i].W_lm, stream=s)),
        "lm_head_adapters": lambda i, s: tensors(ctx.hola_lm_head_adapters(x[i].hidden, x[i].W_lm, bank, ids, stream=s)),
        "verify": lambda i, s: tensors(ctx.hola_verify(*verify(x[i]), want_logits=True, stream=s)),
        "verify_adapters": lambda i, s: tensors(ctx.hola_verify_adapters(*verify(x[i]), bank, ids, want_logits=True, stream=s)),
        "accept_sample": accept_sample,
        "token_logprobs": lambda i, s: tensors(binding.hola_token_logprobs(heads[i].logits, tokens, n_top=20, stream=s)),
        "quantize_w8": lambda i, s: list(binding.hola_quantize_w8(x[i].W_lm, stream=s)),
    }


def _busy(stream):
    """Some 30 ms of work ahead of what is queued next."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(60_000_000)


NAMES = ["lm_head", "lm_head_adapters", "verify", "verify_adapters", "accept_sample", "token_logprobs", "quantize_w8"]


@gpu
@pytest.mark.parametrize("external", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_outputs_of_a_call_on_another_stream(name, external):
    here, side = torch.cuda.current_stream(), torch.cuda.Stream()
    given = type("Stream", (), {"cuda_stream": side.cuda_stream})() if external else side
    with binding.HolaVerify(B, K, H, V) as ctx:
        run = _runs(ctx)[name]
        want = [[t.clone() for t in run(i, None)] for i in (0, 1)]
        same = lambda got, i: all(torch.equal(a, b) for a, b in zip(got, want[i], strict=True))       # noqa: E731
        torch.cuda.synchronize()
        got = run(0, given)
        torch.cuda.synchronize()
        assert same(got, 0) and not same(got, 1)
        del got

        # what the current stream has still to read is not written over, although its tensors are gone
        got = run(0, None)
        torch.cuda.synchronize()
        _busy(here)
        kept = [t.clone() for t in got]
        del got
        other = run(1, given)
        torch.cuda.synchronize()
        assert same(kept, 0) and same(other, 1)
        del other, kept

        # a result that is dropped at once is not handed out again while the other stream has yet to write it
        _busy(side)
        run(0, given)
        fresh = [torch.full_like(t, 7) for t in want[0]]
        torch.cuda.synchronize()
        assert all((t == 7).all() for t in fresh)
        del fresh

        # one that the current stream has still to read is not written over by the other stream's next call
        got = run(0, given)
        here.wait_stream(side)
        _busy(here)
        kept = [t.clone() for t in got]
        del got
        other = run(1, given)
        torch.cuda.synchronize()
        assert same(kept, 0) and same(other, 1)


@gpu
def test_self_tests_on_another_stream():
    """Their counters are cleared in order with the kernel that counts."""
    side = torch.cuda.Stream()
    with binding.HolaVerify(1, 1, 64, 1000) as ctx:
        want = ctx.hola_selftest_bounded_wait(), ctx.hola_selftest_staged_wait(), ctx.hola_selftest_mass_wait()
        t, s = torch.rand(1000, device="cuda"), torch.rand(1000, device="cuda") + 1
        q = ctx.hola_selftest_quotient(t, s)
        torch.cuda.synchronize()
        _busy(torch.cuda.current_stream())                    # (a clearing that is queued here comes too late)
        got = ctx.hola_selftest_bounded_wait(stream=side), ctx.hola_selftest_staged_wait(stream=side), ctx.hola_selftest_mass_wait(stream=side)
        q2, words = ctx.hola_selftest_quotient(t, s, stream=side), ctx.hola_selftest_pace(stream=side)
        torch.cuda.synchronize()
        assert got == want and torch.equal(q, q2) and (words == 0).all()
