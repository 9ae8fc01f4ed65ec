"""The operators together: steps of the example against the same target run over the whole sequence at once."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests,drafts,steps", [(5, 4, 5), (1, 0, 3), (70, 2, 3)])
def test_steps_leave_the_cache_of_the_accepted_tokens(requests, drafts, steps):
    import torch
    from paper_2603_12617_amd import serving_step as S
    tokens, lengths, server = S.serve(requests, drafts, steps, prompt=23, vocab=1000, seed=requests)
    assert all(len(row) == 1 + sum(n[b] + 1 for n in lengths) for b, row in enumerate(tokens))
    assert drafts == 0 or sum(map(sum, lengths)) > 0
    pages, length, nfree = (server.now[k].cpu() for k in ("pages", "length", "nfree"))
    held = [int(x) for x in pages]
    # no page is held twice, none is lost
    used = [int(x) for b in range(requests) for x in server.table[b, :held[b]].cpu()] + [int(x) for x in server.free[:int(nfree)].cpu()]
    assert sorted(used) == list(range(server.free.numel()))
    # valid tokens before the last step's chunk: the prompt and what the steps before emitted
    want = [23 + sum(n[b] + 1 for n in lengths[:-1]) for b in range(requests)]
    assert length.tolist() == want
    # the cache holds the projections of exactly these tokens, in order
    t = server.t
    g = torch.Generator(device="cuda:0").manual_seed(requests + 1)
    prompt = torch.randint(0, 1000, (requests, 23), generator=g, device="cuda:0", dtype=torch.int32)
    for b in range(0, requests, 3):
        seq = torch.cat([prompt[b], torch.tensor(tokens[b], dtype=torch.int32, device="cuda:0")])[:want[b]].long()
        qkv = (t.embed[seq].float() @ t.qkv.float()).view(len(seq), -1, t.D)
        j = torch.arange(len(seq), device="cuda:0")
        at = server.table[b].long()[j // server.page]
        for c, first in ((server.k, t.Hq), (server.v, t.Hq + t.Hkv)):
            got = c[at, j % server.page].float()
            assert float((got - qkv[:, first:first + t.Hkv]).abs().max()) < 0.05


def _record(monkeypatch, S):
    """Notes what goes into and comes out of the target's passes and the verifications."""
    import torch
    passes, checks = [], []
    forward, verify = S.Server.forward, S.Server.verify

    def noted_forward(self, tokens, add, accepted):
        hidden = forward(self, tokens, add, accepted)
        passes.append([x.clone() for x in (tokens, add, hidden, self.cu, self.kv, self.now["length"])])
        return hidden

    def noted_verify(self, p, q, tok, r, noise, tau):
        n, nxt = verify(self, p, q, tok, r, noise, tau)
        checks.append([x if x is None else x.clone() for x in (p, q, tok, r, noise, tau, self.cu, n, nxt)])
        return n, nxt

    monkeypatch.setattr(S.Server, "forward", noted_forward)
    monkeypatch.setattr(S.Server, "verify", noted_verify)
    return passes, checks


def _hidden(t, tokens):
    """The target's hidden rows of a whole sequence, on the host: dense causal attention in float64."""
    import torch
    x = t.embed[tokens].double().cpu()
    qkv = (x @ t.qkv.double().cpu()).to(torch.bfloat16).double().view(len(x), -1, t.D)
    G, n = t.Hq // t.Hkv, len(x)
    later = torch.ones((n, n), dtype=torch.bool).triu(1)
    out = torch.empty((n, t.Hq, t.D), dtype=torch.float64)
    for h in range(t.Hq):
        s = (qkv[:, h] @ qkv[:, t.Hq + h // G].t()) * t.D ** -0.5
        out[:, h] = torch.softmax(s.masked_fill(later, -float("inf")), 1) @ qkv[:, t.Hq + t.Hkv + h // G]
    return x, x + out.view(n, -1) @ t.proj.double().cpu()


@pytest.mark.parametrize("requests,drafts,steps,prompt", [(5, 4, 5, 23), (2, 0, 3, 1), (66, 3, 2, 40), (3, 3, 8, 1011)])
def test_steps_are_those_of_the_whole_sequence(monkeypatch, requests, drafts, steps, prompt):
    """Every pass against dense attention over the tokens that stand and the chunk, every verification against the plain reference, and
    the emitted tokens against both.  (3, 3, 8, 1011): tables of 1024 tokens, so that requests are refused in the end."""
    import numpy as np
    import torch
    from oracle import serve_oracle as SO
    from paper_2603_12617_amd import serving_step as S
    passes, checks = _record(monkeypatch, S)
    tokens, lengths, server = S.serve(requests, drafts, steps, prompt=prompt, vocab=1000, seed=requests)
    assert len(passes) == len(checks) == steps + 1
    stand = [[] for _ in range(requests)]                    # tokens in the cache
    emitted, sure, all_refused = [[] for _ in range(requests)], 0, 0
    for step, ((tok, add, hidden, cu, kv, length), (p, q, drafted, r, noise, tau, vcu, n, nxt)) in enumerate(zip(passes, checks)):
        tok, add, cu, kv, length = (x.tolist() for x in (tok, add, cu, kv, length))
        refused = [kv[b] == length[b] and add[b] > 0 for b in range(requests)]
        all_refused += sum(refused)
        host = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
        want_n, want_next, close = SO.verify_logits(host(p), host(q), drafted.cpu().numpy(), host(r), host(noise), host(tau), vcu.cpu().numpy())
        n, nxt = n.cpu().numpy(), nxt.cpu().numpy()
        ok = close > 4e-5                                    # (the bound of the operator's own tests)
        sure += int(ok.sum())
        assert np.array_equal(n[ok], want_n[ok]) and np.array_equal(nxt[ok], want_next[ok])
        for b in range(requests):
            chunk = tok[cu[b]:cu[b + 1]]
            assert len(chunk) == add[b] and length[b] == len(stand[b]), (step, b)
            if step:
                assert drafted[b * drafts:(b + 1) * drafts].tolist() == chunk[1:]
                assert lengths[step - 1][b] == (-1 if refused[b] else n[b]), (step, b)
            if refused[b]:
                continue
            if b % 7 == 0 or requests < 7:
                x, want = _hidden(server.t, stand[b] + chunk)
                got = hidden[cu[b]:cu[b + 1]].double().cpu()
                # (bfloat16: projections of size 5 rounded to 2^-8, through an average and a projection, and the result's own rounding)
                assert float((got - want[-len(chunk):]).abs().max()) < 0.05, (step, b)
                # attention is more than that: of n values of size 1 with weights e^N(0, 1) a mean of size sqrt(e / n), 512 of them a row
                assert float((want - x)[-len(chunk):].abs().max()) > 2 * min(1.0, 2.718 / len(x)) ** 0.5
            kept = chunk if step == 0 else chunk[:n[b] + 1]
            stand[b] += kept
            emitted[b] += [int(nxt[b])] if step == 0 else kept[1:] + [int(nxt[b])]
    assert emitted == tokens
    assert sure > 0.9 * requests * (steps + 1)
    assert (all_refused > 0) == (prompt > 1000)


def test_prompts_that_do_not_fit_are_refused():
    from paper_2603_12617_amd import serving_step as S
    with pytest.raises(ValueError):
        S.serve(2, 2, 1, prompt=1025, vocab=1000)
