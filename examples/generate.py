"""Token-generating experts on one GPU: a collaboration of small decoder-only transformers with random weights, each request
answered by the expert it is routed to, all of them in shared steps.

    python examples/generate.py --experts 4 --requests 24 --prompt 300 --new 32

A step serves prompt chunks and single tokens together.  Requests are regrouped by expert (coe_regroup_static), so an expert's
tokens are one stretch of the step's token order; blocks and slots come from coe_kv_plan; every layer's coe_kv_append and
coe_kv_attention are one call for all experts, whose projections run on their own stretch; coe_sample_tokens draws for every
request whose prompt is through.  The projections are plain matrix products and left to torch.
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2503_02354_amd import binding as B


class Experts:
    """Decoder-only transformers of one shape: learned positions, grouped heads, RMS norms without gains, GELU feed-forward."""

    def __init__(self, n, layers=2, width=256, heads=8, kv_heads=2, head_dim=32, vocab=1000, max_len=1024, seed=0):
        self.n, self.layers, self.width, self.heads, self.kv_heads, self.head_dim, self.vocab, self.max_len = (
            n, layers, width, heads, kv_heads, head_dim, vocab, max_len)
        g = torch.Generator().manual_seed(seed)
        w = lambda rows, cols, gain=1.0: (gain * rows ** -0.5 * torch.randn(n, rows, cols, generator=g)).bfloat16().cuda()
        self.embedding, self.position = w(vocab, width, vocab ** 0.5), w(max_len, width, 0.5 * max_len ** 0.5)
        self.qkv = [w(width, (heads + 2 * kv_heads) * head_dim) for _ in range(layers)]
        self.o = [w(heads * head_dim, width) for _ in range(layers)]
        self.up, self.down = [w(width, 4 * width) for _ in range(layers)], [w(4 * width, width) for _ in range(layers)]
        self.head = w(width, vocab)


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5)).bfloat16()


class Server:
    """Requests of the experts over one paged cache of n_blocks blocks; at most token_cap tokens a step."""

    def __init__(self, experts, n_blocks=1024, block_size=16, token_cap=512):
        self.e, self.n_blocks, self.block_size, self.token_cap = experts, n_blocks, block_size, token_cap
        self.max_blocks = -(-experts.max_len // block_size)
        # a layer's keys and values: [block][key, value][row in the block][head][channel]
        self.pool = [torch.empty(n_blocks, 2, block_size, experts.kv_heads, experts.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(experts.layers)]
        self.cache = [B.coe_kv_cache(B.COE_DT_BF16, n_blocks, block_size, experts.kv_heads, experts.head_dim, p[:, 0].data_ptr(), p[:, 1].data_ptr(),
                                     *p.stride()[0:1], *p.stride()[2:4]) for p in self.pool]

    def _matmul(self, x, weights, stretch):
        """Every expert's own weights on its stretch of the tokens."""
        out = torch.empty(len(x), weights.shape[2], dtype=x.dtype, device="cuda")
        for e, (lo, hi) in enumerate(stretch):
            if hi > lo:
                torch.matmul(x[lo:hi], weights[e], out=out[lo:hi])
        return out

    def generate(self, prompts, route, new, temperature=0.0, top_k=0, top_p=1.0, seed=0):
        """prompts: lists of token ids; route[i]: the expert of prompt i.  Returns per prompt the `new` drawn tokens and their
        log-probabilities, and the number of steps."""
        e, n, stream = self.e, len(prompts), torch.cuda.current_stream().cuda_stream
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
        dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")

        # requests by expert
        cur, cnt, off, perm, inv = dev(route), i32(e.n), i32(e.n + 1), i32(n), i32(n)
        B.coe_regroup_static(n, cur.data_ptr(), e.n, cnt.data_ptr(), off.data_ptr(), perm.data_ptr(), inv.data_ptr(), stream)
        order, group = perm.tolist(), off.tolist()
        known = [list(prompts[i]) for i in order]      # prompt, then what was drawn
        goal = [len(k) + new for k in known]
        logprobs = [[] for _ in known]
        assert all(0 < len(p) for p in prompts) and max(goal) <= e.max_len, "a request does not fit"

        ring, state, next_state = torch.arange(self.n_blocks, dtype=torch.int32, device="cuda"), dev([0, self.n_blocks]), i32(4)
        table, q_off, slot, position = i32(n, self.max_blocks), i32(n + 1), i32(self.token_cap), i32(self.token_cap)
        have, length = i32(n), i32(n)
        t, k, p = (torch.full((n,), v, dtype=d, device="cuda") for v, d in ((temperature, torch.float32), (top_k, torch.int32), (top_p, torch.float32)))
        token, logprob = i32(n), torch.empty(n, device="cuda")
        generator = torch.Generator(device="cuda").manual_seed(seed)
        cached, done, steps = [0] * n, [False] * n, 0
        while not all(done):
            # what every request is to add: its tokens that are not cached yet, as far as the step reaches; -1 gives a finished one's
            # blocks back
            add, left = [], self.token_cap
            for r in range(n):
                add.append(-1 if len(known[r]) == goal[r] and not done[r] else min(len(known[r]) - cached[r], left) if not done[r] else 0)
                left -= max(add[r], 0)
            B.coe_kv_plan(n, self.block_size, self.n_blocks, self.max_blocks, self.token_cap, have.data_ptr(), dev(add).data_ptr(), ring.data_ptr(),
                          state.data_ptr(), table.data_ptr(), length.data_ptr(), q_off.data_ptr(), slot.data_ptr(), position.data_ptr(),
                          next_state.data_ptr(), stream)
            first = q_off.tolist()
            done = [d or a < 0 for d, a in zip(done, add)]
            have, length = length, have
            state, next_state = next_state, torch.empty_like(next_state)
            tokens, steps = first[n], steps + 1
            if tokens == 0:
                if not all(done) and all(a >= 0 for a in add):
                    raise RuntimeError("the cache is too small for the next request")
                continue
            took = [first[r + 1] - first[r] for r in range(n)]
            ids = [i for r in range(n) for i in known[r][cached[r]:cached[r] + took[r]]]
            cached = [c + m for c, m in zip(cached, took)]
            stretch = [(first[group[x]], first[group[x + 1]]) for x in range(e.n)]

            owner = torch.repeat_interleave(torch.arange(e.n, device="cuda"), dev([hi - lo for lo, hi in stretch]))
            x = (e.embedding[owner, dev(ids).long()] + e.position[owner, position[:tokens].long()]).float()
            for layer in range(e.layers):
                qkv = self._matmul(norm(x), e.qkv[layer], stretch).view(tokens, -1, e.head_dim)
                q, key, value = qkv.split([e.heads, e.kv_heads, e.kv_heads], 1)
                B.coe_kv_append(self.cache[layer], tokens, key.data_ptr(), *key.stride()[:2], value.data_ptr(), *value.stride()[:2], slot.data_ptr(), stream)
                out = torch.empty(tokens, e.heads, e.head_dim, dtype=torch.bfloat16, device="cuda")
                need = B.coe_kv_attention_workspace(n, tokens, max(took), e.heads, e.kv_heads, e.head_dim)
                work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
                B.coe_kv_attention(self.cache[layer], n, tokens, max(took), e.heads, 0, e.head_dim ** -0.5, q.data_ptr(), *q.stride()[:2], q_off.data_ptr(),
                                   have.data_ptr(), table.data_ptr(), self.max_blocks, out.data_ptr(), *out.stride()[:2], 0, work.data_ptr(), need, stream)
                x = x + self._matmul(out.view(tokens, -1), e.o[layer], stretch)
                x = x + self._matmul(torch.nn.functional.gelu(self._matmul(norm(x), e.up[layer], stretch)), e.down[layer], stretch)

            # a token for every request that has all its known ones cached
            ready = [r for r in range(n) if took[r] and cached[r] == len(known[r])]
            if not ready:
                continue
            last = norm(x[dev([first[r + 1] - 1 for r in ready]).long()])
            rows = [0] * (e.n + 1)
            for r in ready:
                rows[next(g for g in range(e.n) if group[g] <= r < group[g + 1]) + 1] += 1
            for g in range(e.n):
                rows[g + 1] += rows[g]
            logits = self._matmul(last, e.head, list(zip(rows, rows[1:])))
            noise = torch.empty(logits.shape, device="cuda").exponential_(generator=generator)
            need = B.coe_sample_workspace(len(ready), e.vocab)
            work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
            B.coe_sample_tokens(len(ready), e.vocab, B.COE_DT_BF16, logits.data_ptr(), logits.stride(0), t.data_ptr(), k.data_ptr(), p.data_ptr(), 0,
                                noise.data_ptr(), noise.stride(0), token.data_ptr(), logprob.data_ptr(), work.data_ptr(), need, stream)
            for r, i, lp in zip(ready, token.tolist(), logprob.tolist()):
                known[r].append(i)
                logprobs[r].append(lp)
        back = inv.tolist()
        return [known[back[i]][len(prompts[i]):] for i in range(n)], [logprobs[back[i]] for i in range(n)], steps


def main():
    parser = argparse.ArgumentParser(description="Generate tokens with several random experts over one paged cache.")
    for name, value in (("experts", 4), ("requests", 24), ("prompt", 300), ("new", 32)):
        parser.add_argument("--" + name, type=int, default=value)
    parser.add_argument("--temperature", type=float, default=0.8)
    parser.add_argument("--top-p", type=float, default=0.95)
    a = parser.parse_args()
    g = torch.Generator().manual_seed(1)
    experts = Experts(a.experts, max_len=max(1024, a.prompt + a.new))
    prompts = [torch.randint(experts.vocab, (int(m),), generator=g).tolist() for m in torch.randint(1, a.prompt + 1, (a.requests,), generator=g)]
    route = torch.randint(a.experts, (a.requests,), generator=g).tolist()
    server = Server(experts)
    server.generate(prompts[:2], route[:2], 2)
    start = time.perf_counter()
    tokens, logprobs, steps = server.generate(prompts, route, a.new, a.temperature, 0, a.top_p)
    seconds = time.perf_counter() - start
    for i in range(min(4, a.requests)):
        print(f"request {i}: expert {route[i]}, prompt of {len(prompts[i])}, {tokens[i][:8]} ... mean log-probability {sum(logprobs[i]) / a.new:.2f}")
    print(f"{sum(map(len, prompts))} prompt tokens and {a.requests * a.new} drawn ones in {steps} steps, {seconds * 1e3:.0f} ms")


if __name__ == "__main__":
    main()
