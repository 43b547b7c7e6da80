"""A few streams served by one small decoder layer: prompts of different lengths, then tokens one by one.

Every step runs what a serving loop runs on a layer: the new tokens' keys and values appended to a paged cache with the
rotation by position, attention over that cache, the routed experts, and at the end a token sampled from the logits
of each stream.  The cache's bytes are the K(n) of the static plan.  Weights are random; projections and norms are plain
torch.  ``python examples/serve_step.py`` prints the tokens and compares the logits of the last step with those of one
pass over the whole sequences.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_09686_gb300 as mf  # noqa: E402
import synth  # noqa: E402

CFG = synth.CONFIGS["tiny"]  # hidden 256, 8 experts, top-2, intermediate 512, Q8_0
HEADS, KV_HEADS, DIM, PAGE, VOCAB = 8, 2, 64, 16, 1000


def norm(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)


class Server:
    """The layer's weights, the experts' context, the cache and its pages."""

    def __init__(self, streams, max_tokens, max_len, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        h = CFG.hidden
        self.streams, self.max_len = streams, max_len
        shape = mf.AttnShape(HEADS, KV_HEADS, DIM, mf.MF_BF16)
        model = mf.Model(CFG.n_layers, h, CFG.n_experts, CFG.top_k, CFG.inter, CFG.qtype)
        kv = streams * mf.mf_kv_bytes(shape, CFG.n_layers, max_len, PAGE)
        plan = mf.mf_plan(model, mf.PlanReq(100.0, 1 << 33, 0, kv, max_tokens, 0))
        assert plan.accepted
        self.ctx = mf.mf_create(model, plan, 0)
        for e in range(CFG.n_experts):
            mf.mf_pack_put(self.ctx, 0, e, synth.payload(CFG.model_seed, 0, e, h, CFG.inter, CFG.qtype))
        self.attn = mf.mf_attn_create(shape, streams, max_tokens, 0)

        def weight(*s):
            return torch.randn(*s, device="cuda", generator=g) / math.sqrt(s[0])

        self.embed = torch.randn(VOCAB, h, device="cuda", generator=g)
        self.wqkv, self.wo = weight(h, (HEADS + 2 * KV_HEADS) * DIM), weight(HEADS * DIM, h)
        self.router = torch.from_numpy(synth.router_weights(CFG.model_seed, 0, CFG.n_experts, h)).cuda()
        self.head = weight(h, VOCAB)
        pages = -(-max_len // PAGE)
        k, v = (torch.empty(streams * pages, PAGE, KV_HEADS, DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.cache = mf.kv_cache(k, v)
        self.pages = torch.randperm(streams * pages, generator=g, device="cuda").int().view(streams, pages)
        angle = torch.arange(max_len, device="cuda").double()[:, None] * 1e4 ** (-torch.arange(DIM // 2, device="cuda").double() / (DIM // 2))
        self.rope = mf.rope(angle.cos().float(), angle.sin().float())

    def close(self):
        mf.mf_attn_destroy(self.attn)
        mf.mf_destroy(self.ctx)

    def step(self, tokens, new, total):
        """The logits after each stream's last token: `tokens` are all streams' new ones, new[i] of stream i, which then holds
        total[i] in the cache."""
        start = [0]
        for n in new:
            start.append(start[-1] + n)
        i32 = dict(dtype=torch.int32, device="cuda")
        step = mf.step(torch.tensor(start, **i32), torch.tensor(total, **i32), self.pages, start[-1], max(new))
        x = self.embed[tokens]
        qkv = (norm(x) @ self.wqkv).bfloat16()
        q, k, v = (t.unflatten(1, (-1, DIM)) for t in qkv.split((HEADS * DIM, KV_HEADS * DIM, KV_HEADS * DIM), 1))
        mf.mf_kv_append(self.attn, self.cache, step, k, v, q, q, self.rope)
        out = torch.empty(start[-1], HEADS, DIM, dtype=torch.bfloat16, device="cuda")
        mf.mf_attn_forward(self.attn, self.cache, step, q, out, scale=DIM ** -0.5)
        x = x + out.flatten(1).float() @ self.wo
        y = torch.empty_like(x)
        mf.mf_moe_forward(self.ctx, 0, norm(x).contiguous(), self.router, None, start[-1], y)
        x = x + norm(y)
        last = torch.tensor(start[1:], device="cuda") - 1
        return norm(x[last]) @ self.head


def serve(prompts, steps, seed=0):
    """Tokens sampled after each prompt, the last step's logits, and those of one pass over everything before them."""
    n, longest = len(prompts), max(map(len, prompts)) + steps
    server = Server(n, n * longest, longest, seed)
    g = torch.Generator("cuda").manual_seed(seed + 1)
    token, logprob = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    settings = dict(temperature=torch.full((n,), 0.8, device="cuda"), top_k=torch.full((n,), 50, dtype=torch.int32, device="cuda"),
                    top_p=torch.full((n,), 0.95, device="cuda"), min_p=torch.full((n,), 0.02, device="cuda"))
    held = [list(p) for p in prompts]
    fresh, new = torch.tensor(sum(held, []), device="cuda"), [len(p) for p in prompts]
    for _ in range(steps):
        logits = server.step(fresh, new, [len(p) for p in held])
        u = torch.rand(n, VOCAB, device="cuda", generator=g).clamp_(1e-10, 1 - 1e-7)
        mf.mf_sample(logits, -torch.log(-torch.log(u)), token, logprob, **settings)
        before = [list(p) for p in held]
        for p, t in zip(held, token.tolist()):
            p.append(t)
        fresh, new = token.long(), [1] * n
    again = server.step(torch.tensor(sum(before, []), device="cuda"), [len(p) for p in before], [len(p) for p in before])
    status = mf.mf_attn_check(server.attn), mf.mf_check(server.ctx)
    server.close()
    assert status == (0, 0), status
    return [p[len(q):] for p, q in zip(held, prompts)], logits, again


def main():
    prompts = [[(7 * i + 13 * s) % VOCAB for i in range(n)] for s, n in enumerate((5, 40, 1, 23))]
    tokens, logits, again = serve(prompts, 12)
    for i, t in enumerate(tokens):
        print(f"stream {i}: {len(prompts[i])} tokens of prompt, then", *t)
    print("largest difference of the last logits from one pass over the whole sequences:", float((logits - again).abs().max()))


if __name__ == "__main__":
    main()
