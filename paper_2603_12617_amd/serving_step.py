"""Verification steps of a served target model, with the library's operators as a serving program calls them:

    python -m paper_2603_12617_amd.serving_step [--requests 8] [--drafts 4] [--steps 6]

The target is one attention layer with random weights between an embedding and an output projection, the draft a noisy copy of its
output projection that looks at the last token alone.  Each step drafts k tokens per request, builds the block tables on the GPU (``sd_pages``), runs the chunk of
last token and drafts through the target (``sd_cache_store``, ``sd_attend``), verifies the drafts from both models' logits (``sd_verify_logits``) and
goes on from the accepted lengths.  Prompts enter the same way, as longer chunks without drafts.  Nothing is read back between the steps: the
tokens are the program's result, at its end.  A request whose table is full is refused from then on and emits no more.
"""
import argparse

import torch

from . import binding as B


class Target:
    """Embedding, one attention layer, output projection; random weights, bfloat16."""

    def __init__(self, vocab, heads_q, heads_kv, D, device, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        width = heads_q * D
        w = lambda *s: (torch.randn(s, generator=g, device=device) / s[0] ** 0.5).to(torch.bfloat16)  # noqa: E731
        self.embed = torch.randn((vocab, width), generator=g, device=device).to(torch.bfloat16)
        self.qkv, self.proj, self.head = w(width, (heads_q + 2 * heads_kv) * D), w(width, width), 4 * w(width, vocab)
        self.draft_head = self.head + 0.3 * w(width, vocab)
        self.Hq, self.Hkv, self.D, self.vocab = heads_q, heads_kv, D, vocab


class Server:
    """The state of B requests: tables, lengths and the cache; and one step of it."""

    def __init__(self, target, requests, page=16, pages_each=64, device="cuda:0"):
        self.t, self.Bn, self.page, self.dev = target, requests, page, torch.device(device)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=self.dev)  # noqa: E731
        pool = requests * pages_each
        self.table, self.free = i32(requests, pages_each), torch.arange(pool, dtype=torch.int32, device=self.dev)
        # what a step reads and what it writes change places
        self.now = dict(pages=i32(requests), length=i32(requests), nfree=torch.full((1,), pool, dtype=torch.int32, device=self.dev))
        self.then = dict(pages=i32(requests), length=i32(requests), nfree=i32(1))
        shape = (pool, page, target.Hkv, target.D)
        self.k, self.v = (torch.empty(shape, dtype=torch.bfloat16, device=self.dev) for _ in range(2))
        self.kv, self.cu = i32(requests), i32(requests + 1)
        self.refused = torch.zeros(requests, dtype=torch.bool, device=self.dev)
        self.ws = torch.empty(16, dtype=torch.uint8, device=self.dev)

    def _workspace(self, n):
        if n > self.ws.numel():
            self.ws = torch.empty(n, dtype=torch.uint8, device=self.dev)
        return self.ws

    def forward(self, tokens, add, accepted):
        """The target's hidden rows behind a batch of chunks: `tokens` of all requests, add[b] of request b.  Those of a request that
        is refused for want of pages mean nothing: none of its chunk is in the cache, and its accepted length is -1 in the next step."""
        t, T = self.t, tokens.numel()
        slot, pos = (torch.empty(T, dtype=torch.int32, device=self.dev) for _ in range(2))
        a, b = self.now, self.then
        B.sd_pages(a["pages"], a["length"], add, self.table, self.free, a["nfree"], self.page, b["pages"], b["length"], self.kv, b["nfree"], self.cu, slot, pos,
                   accepted=accepted)
        self.now, self.then = b, a
        self.refused = (self.kv == b["length"]) & (add > 0)
        x = t.embed[tokens.long()]
        qkv = (x @ t.qkv).view(T, t.Hq + 2 * t.Hkv, t.D)
        q, k, v = qkv[:, :t.Hq], qkv[:, t.Hq:t.Hq + t.Hkv], qkv[:, t.Hq + t.Hkv:]
        B.sd_cache_store(k, v, slot, self.k, self.v)
        out = torch.empty((T, t.Hq, t.D), dtype=torch.bfloat16, device=self.dev)
        B.sd_attend(q, self.k, self.v, self.cu, self.kv, self.table, out, t.D ** -0.5, ws=self._workspace(B.sd_attend_workspace_bytes(q, self.k, self.table)))
        return x + out.view(T, -1) @ t.proj

    def verify(self, p, q, tok, r, noise, tau):
        n, nxt = (torch.empty(self.Bn, dtype=torch.int32, device=self.dev) for _ in range(2))
        B.sd_verify_logits(p, q, tok, r, noise, tau, self.cu, n, nxt, self._workspace(B.sd_verify_logits_workspace_bytes(p, q, tau)))
        return n, nxt


def serve(requests=8, drafts=4, steps=6, prompt=50, vocab=32000, tau=0.8, seed=0, device="cuda:0"):
    """Tokens of every request, and the accepted lengths of the steps [steps][requests] (both lists; -1: refused in that step)."""
    dev = torch.device(device)
    g = torch.Generator(device=dev).manual_seed(seed + 1)
    target = Target(vocab, 8, 2, 64, dev, seed)
    server = Server(target, requests, device=device)
    if not 0 < prompt <= server.table.shape[1] * server.page:
        raise ValueError("prompts of 1 to %d tokens are wanted: got %d" % (server.table.shape[1] * server.page, prompt))
    temp = torch.full((requests,), tau, device=dev)
    rand = lambda *s: torch.rand(s, generator=g, device=dev)  # noqa: E731
    race = lambda: torch.empty((requests, vocab), device=dev).exponential_(generator=g)  # noqa: E731
    tokens = torch.randint(0, vocab, (requests, prompt), generator=g, device=dev, dtype=torch.int32)
    hidden = server.forward(tokens.flatten(), torch.full((requests,), prompt, dtype=torch.int32, device=dev), None)
    last = hidden.view(requests, prompt, -1)[:, -1]
    # (the first token: a verification without drafts, one row a request)
    cu, server.cu = server.cu, torch.arange(requests + 1, dtype=torch.int32, device=dev)
    empty = torch.empty(0, dtype=torch.int32, device=dev)
    _, nxt = server.verify(last @ target.head, None, empty, empty.float(), race(), temp)
    server.cu = cu
    accepted = torch.full((requests,), prompt - 1, dtype=torch.int32, device=dev)    # the whole prompt stands
    emitted, lengths = [nxt[:, None]], []
    add = torch.full((requests,), drafts + 1, dtype=torch.int32, device=dev)
    for _ in range(steps):
        chunk, logits = [nxt], []
        for _ in range(drafts):                                                       # the draft looks at the last token alone
            logits.append(target.embed[chunk[-1].long()] @ target.draft_head)
            chunk.append((logits[-1].float() / tau - race().log()).argmax(1).to(torch.int32))
        tok = torch.stack(chunk, 1)
        hidden = server.forward(tok.flatten(), add, accepted)
        q = torch.stack(logits, 1).view(requests * drafts, vocab) if drafts else None
        accepted, nxt = server.verify(hidden @ target.head, q, tok[:, 1:].flatten(), rand(requests * drafts), race(), temp)
        accepted, nxt = torch.where(server.refused, -1, accepted), torch.where(server.refused, tok[:, 0], nxt)     # (where it was)
        step = torch.cat([tok[:, 1:], nxt[:, None]], 1)
        at = torch.arange(drafts + 1, device=dev)
        step = torch.where(at < accepted[:, None], step, torch.where(at == accepted[:, None], nxt[:, None], -1))
        emitted.append(step)
        lengths.append(accepted)
    out = torch.cat(emitted, 1).cpu()
    return [[int(x) for x in row if x >= 0] for row in out], torch.stack(lengths).cpu().tolist() if lengths else [], server


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--steps", type=int, default=6)
    a = ap.parse_args()
    tokens, lengths, _ = serve(a.requests, a.drafts, a.steps)
    for b, row in enumerate(tokens):
        print("request %d: %d tokens, accepted %s: %s" % (b, len(row), [n[b] for n in lengths], row[:12]))


if __name__ == "__main__":
    main()
