"""Streams that share a system prompt, served by one small decoder layer with drafted tokens.

The system prompt is computed once; the streams' page tables name its pages.  Every step a stream adds its next token and a few drafts,
looked up in what was said before.  On the layer that is: keys and queries normed head by head, rotated and appended to the
paged cache in one pass, attention that shares the lines of the prompt among the streams (read once for all where the tables can hold
enough for that to pay), the routed experts, and the drafts verified
against the target's probabilities, with a token after the last that was taken.  Lines of drafts that were not taken are written over by the next
step.  Weights are random; projections are plain torch.  ``python examples/draft_step.py`` prints the tokens and how many drafts were
taken, and compares the logits of the last step with those of one pass over the whole sequences.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import serve_step as base  # noqa: E402

mf = base.mf
DRAFTS = 3


class Server(base.Server):
    """The layer with weights of the queries' and keys' norms, and streams that begin alike."""

    def __init__(self, streams, max_tokens, max_len, seed=0):
        super().__init__(streams, max_tokens, max_len, seed)
        g = torch.Generator("cuda").manual_seed(seed + 7)
        self.norm = mf.qk_norm(*((1 + 0.2 * torch.randn(base.DIM, device="cuda", generator=g)).bfloat16() for _ in range(2)), 1e-6)
        mf.mf_attn_share(self.attn, 1)
        self.group = torch.tensor([0, streams], dtype=torch.int32, device="cuda")

    def rows(self, tokens, new, total, shared=0, streams=None):
        """The logits after every new token (`tokens` are all streams' new ones, new[i] of stream i, which then holds total[i] lines), the
        first `shared` lines of all streams being the same."""
        n = self.streams if streams is None else streams
        start = [0]
        for x in new:
            start.append(start[-1] + x)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.start = torch.tensor(start, **i32)
        step = mf.step(self.start, torch.tensor(total, **i32), self.pages[:n].contiguous(), start[-1], max(new))
        x = self.embed[tokens]
        heads, kv, dim = base.HEADS, base.KV_HEADS, base.DIM
        q, k, v = (t.unflatten(1, (-1, dim)) for t in (base.norm(x) @ self.wqkv).bfloat16().split((heads * dim, kv * dim, kv * dim), 1))
        mf.mf_kv_append_norm(self.attn, self.cache, step, self.norm, k, v, q, q, self.rope)
        out = torch.empty(start[-1], heads, dim, dtype=torch.bfloat16, device="cuda")
        if shared:
            groups = mf.shared(self.group, torch.tensor([shared], **i32))
            mf.mf_attn_forward_shared(self.attn, self.cache, step, groups, q, out, scale=dim ** -0.5)
        else:
            mf.mf_attn_forward(self.attn, self.cache, step, q, out, scale=dim ** -0.5)
        x = x + out.flatten(1).float() @ self.wo
        y = torch.empty_like(x)
        mf.mf_moe_forward(self.ctx, 0, base.norm(x).contiguous(), self.router, None, start[-1], y)
        return base.norm(x + base.norm(y)) @ self.head


def look_up(said):
    """Up to DRAFTS tokens that followed the last one's latest occurrence before."""
    for i in range(len(said) - 2, -1, -1):
        if said[i] == said[-1]:
            return said[i + 1:i + 1 + DRAFTS]
    return []


def serve(system, questions, steps, seed=0, temperature=0.8):
    """What each stream says after its question, how many drafts were taken of how many, the last step's logits and those of one pass
    over the whole sequences."""
    n = len(questions)
    held = [list(system) + list(q) for q in questions]
    longest = max(map(len, held)) + steps * (DRAFTS + 1)
    server = Server(n, n * longest, longest, seed)
    shared = len(system) // base.PAGE * base.PAGE
    server.pages[1:, :shared // base.PAGE] = server.pages[0, :shared // base.PAGE]
    if shared:  # the system prompt's whole pages, once
        server.rows(torch.tensor(system[:shared], device="cuda"), [shared], [shared], streams=1)
    g = torch.Generator("cuda").manual_seed(seed + 1)
    cuts = mf.cuts(torch.full((n,), temperature, device="cuda"), torch.full((n,), 50, dtype=torch.int32, device="cuda"),
                   torch.full((n,), 0.95, device="cuda"))
    fresh, cached, drafts = [h[shared:] for h in held], [shared] * n, [[] for _ in range(n)]
    taken = offered = 0
    for _ in range(steps):
        rows = [f + d for f, d in zip(fresh, drafts)]
        total = [c + len(r) for c, r in zip(cached, rows)]
        tokens = torch.tensor(sum(rows, []), device="cuda")
        logits = server.rows(tokens, [len(r) for r in rows], total, shared)
        # the rows that decide: of each stream's last token and of its drafts
        ends = server.start[1:].tolist()
        keep = torch.cat([torch.arange(e - len(d) - 1, e) for e, d in zip(ends, drafts)]).cuda()
        start = [0]
        for d in drafts:
            start.append(start[-1] + len(d) + 1)
        R, i32 = start[-1], dict(dtype=torch.int32, device="cuda")
        u = torch.rand(R, device="cuda", generator=g)
        noise = -torch.log(-torch.log(torch.rand(n, base.VOCAB, device="cuda", generator=g).clamp_(1e-10, 1 - 1e-7)))
        token, accepted = torch.empty(R, **i32), torch.empty(n, **i32)
        work = torch.empty(mf.mf_verify_bytes(n, R, base.VOCAB), dtype=torch.uint8, device="cuda")
        last, before = logits[keep], [h[:] for h in held]
        mf.mf_verify(last, torch.tensor(start, **i32), tokens[keep].int(), u, noise, token, accepted, work, cuts=cuts)
        said, took = token.tolist(), accepted.tolist()
        offered += sum(map(len, drafts))
        taken += sum(took)
        for i in range(n):
            more = said[start[i]:start[i] + took[i] + 1]
            assert more[:-1] == drafts[i][:took[i]]
            held[i] += more
            cached[i], fresh[i] = len(held[i]) - 1, held[i][-1:]
            before[i] += drafts[i]
            drafts[i] = look_up(held[i])
    again = server.rows(torch.tensor(sum(before, []), device="cuda"), [len(b) for b in before], [len(b) for b in before])
    ends, was = server.start[1:].tolist(), [b - a for a, b in zip(start, start[1:])]
    again = torch.cat([again[e - w:e] for e, w in zip(ends, was)])
    status = mf.mf_attn_check(server.attn), mf.mf_check(server.ctx)
    server.close()
    assert status == (0, 0), status
    return [h[len(system) + len(q):] for h, q in zip(held, questions)], (taken, offered), last, again


def main():
    system = [(11 * i) % 97 for i in range(150)]
    questions = [[(7 * i + 13 * s) % base.VOCAB for i in range(n)] for s, n in enumerate((5, 40, 1, 23))]
    said, (taken, offered), last, again = serve(system, questions, 12)
    for i, t in enumerate(said):
        print(f"stream {i}: {len(questions[i])} tokens of question, then", *t)
    print(f"{taken} of {offered} drafts taken")
    print("largest difference of the last logits from one pass over the whole sequences:", float((last - again).abs().max()))


if __name__ == "__main__":
    main()
