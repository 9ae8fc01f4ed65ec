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
