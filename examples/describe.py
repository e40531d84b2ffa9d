"""An expert that writes about what an encoder has seen, on one GPU: a small decoder with random weights that rotates positions into its keys and
queries, looks at an encoder's states in every layer and is searched with beams.

    python examples/describe.py --requests 6 --beams 4 --rows 197 --new 16

A request's beams are consecutive rows of the paged cache.  A step plans (coe_kv_plan), appends and rotates the new tokens' keys
(coe_kv_append_rotated), attends to the cache (coe_kv_attention) and to the request's states (coe_cross_attention) in every layer, chooses among all
continuations (coe_beam_select) and lets the rows' caches follow their parents' (coe_kv_fork, coe_kv_copy).  Nothing of it is read on the host
before the end.  The projections are plain matrix products and left to torch.
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2503_02354_amd import binding as B


class Decoder:
    """A decoder of one shape: grouped heads, RMS norms without gains, GELU feed-forward; states have the decoder's width."""

    def __init__(self, layers=2, width=256, heads=8, kv_heads=2, head_dim=32, vocab=1000, rotated=32, base=10000.0, seed=0):
        self.layers, self.width, self.heads, self.kv_heads, self.head_dim, self.vocab, self.rotated = layers, width, heads, kv_heads, head_dim, vocab, rotated
        g = torch.Generator().manual_seed(seed)
        w = lambda rows, cols, gain=1.0: (gain * rows ** -0.5 * torch.randn(rows, cols, generator=g)).bfloat16().cuda()
        self.embedding = w(vocab, width, vocab ** 0.5)
        self.qkv = [w(width, (heads + 2 * kv_heads) * head_dim) for _ in range(layers)]
        self.o, self.cross_o = ([w(heads * head_dim, width) for _ in range(layers)] for _ in range(2))
        self.cross_q, self.cross_kv = [w(width, heads * head_dim) for _ in range(layers)], [w(width, 2 * kv_heads * head_dim) for _ in range(layers)]
        self.up, self.down = [w(width, 4 * width) for _ in range(layers)], [w(4 * width, width) for _ in range(layers)]
        self.head = w(width, vocab)
        self.frequency = torch.tensor([base ** (-2 * i / rotated) for i in range(rotated // 2)], dtype=torch.float32, device="cuda")


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5)).bfloat16()


class Writer:
    """Searches over one paged cache of n_blocks blocks; a row holds at most max_len tokens."""

    def __init__(self, decoder, n_blocks=1024, block_size=16, max_len=256):
        d = self.d = decoder
        self.n_blocks, self.block_size, self.max_blocks = n_blocks, block_size, -(-max_len // block_size)
        self.pool = [torch.empty(n_blocks, 2, block_size, d.kv_heads, d.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(d.layers)]
        self.cache = (B.coe_kv_cache * d.layers)(*(
            B.coe_kv_cache(B.COE_DT_BF16, n_blocks, block_size, d.kv_heads, d.head_dim, p[:, 0].data_ptr(), p[:, 1].data_ptr(), p.stride(0), *p.stride()[2:4])
            for p in self.pool))
        self.ring, self.state = torch.arange(n_blocks, dtype=torch.int32, device="cuda"), torch.tensor([0, n_blocks, 0, 0], dtype=torch.int32, device="cuda")

    def write(self, states, prompts, beams=4, new=16, end=1):
        """states: [rows][width] per request; prompts: lists of token ids.  Returns per request its beams, best first: (tokens, sum of their
        log-probabilities); tokens end with `end`, or are `new` long."""
        d, n_requests, stream = self.d, len(prompts), torch.cuda.current_stream().cuda_stream
        n = n_requests * beams
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
        dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        p = lambda t: t.data_ptr()

        # what the encoder left, for every layer: all sources' rows behind each other
        length = [len(s) for s in states]
        first, longest, seen = dev([sum(length[:i]) for i in range(n_requests)]), max(length), torch.cat(states)
        lengths, kv = dev(length), []
        for layer in range(d.layers):
            both = (seen @ d.cross_kv[layer]).view(len(seen), 2 * d.kv_heads, d.head_dim)
            kv.append((both, B.coe_states(B.COE_DT_BF16, len(seen), d.kv_heads, d.head_dim, p(both), p(both[:, d.kv_heads:]), *both.stride()[:2], *both.stride()[:2], 0)))

        table, next_table, have, length_now, next_len = i32(n, self.max_blocks), i32(n, self.max_blocks), i32(n), i32(n), i32(n)
        plan_state, fork_state, copy = i32(4), i32(4), i32(n, 2)
        # a request begins with its prompt in its first row, the others are not there yet
        score = torch.full((n_requests, beams), float("-inf"), device="cuda")
        score[:, 0] = 0
        ended, next_score, next_ended = i32(n_requests, beams), torch.empty_like(score), i32(n_requests, beams)
        parent, token = i32(n_requests, beams), i32(n_requests, beams)
        history = torch.full((n, new), end, dtype=torch.int32, device="cuda")
        add = i32(n)
        add[::beams] = dev([len(x) for x in prompts])
        ids, fine = dev([t for x in prompts for t in x]), torch.ones((), dtype=torch.bool, device="cuda")
        most_new, most_beams = max(len(x) for x in prompts), max(len(x) for x in prompts)          # tokens of a row, and of a source, in a step
        work, need = {}, {}

        def room(name, bytes_needed):
            if name not in work or work[name].numel() < bytes_needed:
                work[name] = torch.empty(max(bytes_needed, 16), dtype=torch.uint8, device="cuda")
            need[name] = bytes_needed
            return p(work[name]), bytes_needed

        for step in range(new):
            cap = len(ids)                                                # tokens that the step may have
            q_off, slot, position = i32(n + 1), i32(cap), i32(cap)
            B.coe_kv_plan(n, self.block_size, self.n_blocks, self.max_blocks, cap, p(have), p(add), p(self.ring), p(self.state), p(table), p(length_now), p(q_off), p(slot),
                          p(position), p(plan_state), stream)
            fine &= plan_state[2] == n
            x = d.embedding[ids.long()].float()
            for layer in range(d.layers):
                qkv = (norm(x) @ d.qkv[layer]).view(cap, -1, d.head_dim)
                q, k, v = qkv.split([d.heads, d.kv_heads, d.kv_heads], 1)
                B.coe_kv_append_rotated(self.cache[layer], cap, d.heads, p(q), *q.stride()[:2], p(q), *q.stride()[:2], p(k), *k.stride()[:2], p(v), *v.stride()[:2], p(slot),
                                        p(position), p(d.frequency), d.rotated, B.COE_PAIR_HALVES, stream)
                out = torch.zeros(cap, d.heads, d.head_dim, dtype=torch.bfloat16, device="cuda")
                B.coe_kv_attention(self.cache[layer], n, cap, most_new, d.heads, 0, d.head_dim ** -0.5, p(q), *q.stride()[:2], p(q_off), p(length_now), p(table),
                                   self.max_blocks, p(out), *out.stride()[:2], 0,
                                   *room("self", B.coe_kv_attention_workspace(n, cap, most_new, d.heads, d.kv_heads, d.head_dim)), stream)
                x = x + out.view(cap, -1) @ d.o[layer]
                q = (norm(x) @ d.cross_q[layer]).view(cap, d.heads, d.head_dim)
                out = torch.zeros_like(q)
                B.coe_cross_attention(kv[layer][1], n_requests, cap, beams, most_beams, longest, d.heads, d.head_dim ** -0.5, p(q), *q.stride()[:2], p(q_off), p(first),
                                      p(lengths), p(out), *out.stride()[:2], 0,
                                      *room("cross", B.coe_cross_attention_workspace(n_requests, cap, most_beams, longest, d.heads, d.kv_heads, d.head_dim)), stream)
                x = x + out.view(cap, -1) @ d.cross_o[layer]
                x = x + torch.nn.functional.gelu(norm(x) @ d.up[layer]) @ d.down[layer]
            last = (q_off[1:].long() - 1).clamp(0, cap - 1)               # of rows without a new token: any, their logits are not read
            logits = norm(x[last]) @ d.head
            B.coe_beam_select(n_requests, beams, beams, d.vocab, B.COE_DT_BF16, p(logits), logits.stride(0), p(score), p(ended), end, p(next_score), p(parent), p(token),
                              p(next_ended), *room("beams", B.coe_beam_workspace(n_requests, beams, beams, d.vocab)), stream)
            B.coe_kv_fork(n_requests, beams, self.block_size, self.n_blocks, self.max_blocks, p(parent), p(length_now), p(table), p(self.ring), p(plan_state), p(next_table),
                          p(next_len), p(copy), p(fork_state), *room("fork", B.coe_kv_fork_workspace(n_requests, beams)), stream)
            B.coe_kv_copy(self.cache, n, p(copy), p(next_len), stream)
            fine &= fork_state[2] == n_requests
            row = parent.view(-1).long().clamp(min=0)
            history = history[row]
            history[:, step] = torch.where(ended.view(-1)[row] != 0, end, token.view(-1))
            score, next_score, ended, next_ended = next_score, score, next_ended, ended
            table, next_table, have, next_len = next_table, table, next_len, have
            self.state = fork_state.clone()
            # every row that has not ended goes on with its token; the step's tokens are in row order
            add = ((ended.view(-1) == 0) & (parent.view(-1) >= 0)).int()
            ids = torch.zeros(n, dtype=torch.int32, device="cuda").scatter_add_(0, (torch.cumsum(add, 0) - 1).clamp(min=0), token.view(-1) * add)
            most_new, most_beams = 1, beams
        # every block goes back
        B.coe_kv_fork(n_requests, beams, self.block_size, self.n_blocks, self.max_blocks, p(torch.full((n,), -1, dtype=torch.int32, device="cuda")), p(have), p(table),
                      p(self.ring), p(self.state), p(next_table), p(next_len), p(copy), p(fork_state), p(work["fork"]), need["fork"], stream)
        self.state = fork_state.clone()
        if not bool(fine):
            raise RuntimeError("the cache is too small")
        out = []
        for r in range(n_requests):
            found = []
            for b in range(beams):
                if float(score[r, b]) == float("-inf"):
                    continue
                tokens = history[r * beams + b].tolist()
                found.append((tokens[:tokens.index(end) + 1] if end in tokens else tokens, float(score[r, b])))
            out.append(found)
        return out


def main():
    parser = argparse.ArgumentParser(description="Search for what a random decoder would write about random states.")
    for name, value in (("requests", 6), ("beams", 4), ("rows", 197), ("new", 16)):
        parser.add_argument("--" + name, type=int, default=value)
    a = parser.parse_args()
    g = torch.Generator().manual_seed(1)
    decoder = Decoder()
    states = [torch.randn(int(m), decoder.width, generator=g).bfloat16().cuda() for m in torch.randint(1, a.rows + 1, (a.requests,), generator=g)]
    prompts = [torch.randint(2, decoder.vocab, (int(m),), generator=g).tolist() for m in torch.randint(1, 9, (a.requests,), generator=g)]
    writer = Writer(decoder)
    writer.write(states[:1], prompts[:1], a.beams, 2)
    start = time.perf_counter()
    found = writer.write(states, prompts, a.beams, a.new)
    seconds = time.perf_counter() - start
    for r, beams in enumerate(found[:4]):
        print(f"request {r}: {len(states[r])} rows, prompt of {len(prompts[r])}, best {beams[0][0][:8]} ... with ln p = {beams[0][1]:.2f}, {len(beams)} beams")
    print(f"{a.requests} requests of {a.beams} beams, {a.new} steps, {seconds * 1e3:.0f} ms")


if __name__ == "__main__":
    main()
