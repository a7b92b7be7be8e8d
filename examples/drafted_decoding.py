"""Decoding with drafted tokens: each round a drafter proposes a tree of tokens for every request, a small decoder takes all of them in
one step over its paged 8-bit cache, samples behind each, and keeps the path that its own choices confirm.

  python examples/drafted_decoding.py [--prompt 200] [--rounds 12] [--seqs 3] [--temperature 0.0]

Weights are random, but for a head that continues most tokens in a way that the drafter partly knows.  Nothing is read back
within a round: the whole of it is captured into a graph, which is replayed.  Prints how many tokens a round gives, and how far the cache that the rounds leave
is from the one that the same tokens give as a prompt.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2605_20315_amd as mq  # noqa: E402

LAYERS, HIDDEN, HQ, HKV, D, P, VOCAB = 2, 512, 8, 2, 64, 16, 1000
EPS, SCALE = 1e-6, D ** -0.5
# token 0 is the last one that was kept; two candidates behind it, two behind the first of those, then chains
PARENTS = [-1, 0, 0, 1, 1, 2, 3, 4, 6]
RANKS = [0, 0, 1, 0, 1, 0, 0, 0, 0]  # which of the drafter's guesses a token is


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Decoder:
    """Weights, caches and the state of `seqs` requests of up to `longest` tokens."""

    def __init__(self, seqs, longest, gen):
        normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
        bf16 = lambda x: x.to(torch.bfloat16)  # noqa: E731
        self.seqs, self.nodes = seqs, len(PARENTS)
        # the head likes, behind token t, the token after[t]; the drafter's first guess is right for four of five
        after = torch.randperm(VOCAB, device="cuda", generator=gen)
        self.guesses = torch.stack([torch.where(torch.arange(VOCAB, device="cuda") % 5 > 0, after, (after + 1) % VOCAB), after], 1)
        self.after = after
        self.embed = bf16(normal(VOCAB, HIDDEN))
        self.head = torch.empty_like(self.embed)
        self.head[after] = bf16(self.embed.float() * HIDDEN ** -0.5)
        self.qkv = [bf16(normal((HQ + 2 * HKV) * D, HIDDEN) * HIDDEN ** -0.5) for _ in range(LAYERS)]
        self.out = [bf16(normal(HIDDEN, HQ * D) * 0.1 * (HQ * D) ** -0.5) for _ in range(LAYERS)]
        self.table = mq.mq_rope_table(longest, D, 10000.0)
        width = -(-longest // P)
        self.page_table = torch.randperm(seqs * width, device="cuda", generator=gen).to(torch.int32).view(seqs, width)
        self.caches = [self.empty_cache() for _ in range(LAYERS)]
        self.workspace = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        # a round's constants
        self.words = -(-self.nodes // 32)
        self.parents = ints(PARENTS * seqs)
        self.cu_q = ints([self.nodes * b for b in range(seqs + 1)])
        # what rounds hand on: kept tokens in the caches, and the token to go on from, which is not there yet
        self.lens, self.last = ints([0] * seqs), ints([0] * seqs)
        self.uniform = torch.zeros(seqs * self.nodes, device="cuda")
        self.temperature = torch.zeros(seqs * self.nodes, device="cuda")

    def empty_cache(self):
        pages = self.page_table.numel()
        return [x for _ in "kv" for x in (torch.zeros(pages, HKV, P, D, dtype=torch.uint8, device="cuda"), torch.zeros(pages, HKV, dtype=torch.uint8, device="cuda"))]

    def forward(self, tokens, cu_q, kv_lens, caches, tree=None, positions=None):
        """Logits behind every token."""
        x = self.embed[tokens.long()]
        for qkv, out, cache in zip(self.qkv, self.out, caches):
            h = x.float()
            h = (h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)).to(torch.bfloat16)
            p = mq.bf16_gemm_ws(h, qkv, self.workspace).view(len(x), HQ + 2 * HKV, D)
            q = mq.kv8_append(p[:, :HQ], p[:, HQ : HQ + HKV], p[:, HQ + HKV :], *cache, self.page_table, cu_q, kv_lens, self.table, positions)
            if tree is None:
                a = mq.kv8_attention(q, *cache, self.page_table, cu_q, kv_lens, SCALE, workspace=self.workspace)
            else:
                a = mq.kv8_tree_attention(q, *cache, self.page_table, cu_q, kv_lens, tree, SCALE, positions=positions, workspace=self.workspace)
            x = x + mq.bf16_gemm_ws(a.view(len(x), HQ * D), out, self.workspace)
        return mq.bf16_gemm_ws(x, self.head, self.workspace)

    def prompt(self, lens, tokens):
        """Prompts of lens[b] tokens, all but the last of each into the cache."""
        kept = [t[:-1] for t in tokens.split(lens)]
        self.lens.copy_(ints([len(t) for t in kept]))
        cu_q = ints([sum(len(t) for t in kept[:b]) for b in range(self.seqs + 1)])
        self.forward(torch.cat(kept), cu_q, self.lens, self.caches)
        self.last.copy_(torch.stack([t[-1] for t in tokens.split(lens)]))

    def draft(self):
        rows = [self.last.long()]
        for parent, rank in zip(PARENTS[1:], RANKS[1:]):
            rows.append(self.guesses[rows[parent], rank])
        return torch.stack(rows, 1).reshape(-1).to(torch.int32)

    def round(self):
        """(drafted tokens, path, counts, next): sequence b's kept tokens are those that path names, and next[b] goes on from them."""
        tokens, kv_lens = self.draft(), self.lens + self.nodes
        tree, positions = mq.mq_draft_tree(self.parents, self.cu_q, kv_lens, self.words)
        logits = self.forward(tokens, self.cu_q, kv_lens, self.caches, tree, positions)
        sampled = mq.mq_sample(logits, self.uniform, self.temperature)
        path, counts, ends, lens = mq.mq_draft_accept(self.parents, tokens, sampled, self.cu_q, kv_lens)
        for cache in self.caches:
            mq.kv8_compact(*cache, self.page_table, self.cu_q, kv_lens, path, counts)
        self.lens.copy_(lens)
        self.last.copy_(ends)
        return tokens, path, counts, ends

    def kept(self, tokens, path, counts, ends):
        """The tokens that a round adds to each request's cache, as lists."""
        tokens, path = tokens.view(self.seqs, -1).tolist(), path.view(self.seqs, -1).tolist()
        return [[tokens[b][i] for i in path[b][:n]] for b, n in enumerate(counts.tolist())]

    def values(self, cache):
        """Keys and values of each request's kept tokens in 32 bits, [2][seqs] of [tokens, HKV, D]."""
        out = []
        for i in (0, 2):
            x = torch.ldexp(cache[i].view(torch.float8_e4m3fn).float(), cache[i + 1].int()[..., None, None] - 127)
            out.append([x[self.page_table[b].long()].transpose(1, 2).reshape(-1, HKV, D)[:n] for b, n in enumerate(self.lens.tolist())])
        return out


def start(prompt, rounds, seqs, temperature, seed):
    """A decoder behind its prompts, the tokens in its caches, and each round's uniform numbers."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dec = Decoder(seqs, prompt + (rounds + 1) * len(PARENTS) + 1, gen)
    lens = [max(2, prompt - 37 * b) for b in range(seqs)]
    tokens = torch.randint(VOCAB, (sum(lens),), device="cuda", generator=gen).to(torch.int32)
    dec.temperature.fill_(temperature)
    dec.prompt(lens, tokens)
    draws = torch.rand(rounds, len(dec.uniform), device="cuda", generator=gen)
    return dec, [t[:-1].tolist() for t in tokens.split(lens)], draws


def run(prompt=200, rounds=12, seqs=3, temperature=0.0, seed=0):
    """(tokens a round, largest distance of a cache from a prompt's relative to its norm)."""
    dec, texts, draws = start(prompt, rounds, seqs, temperature, seed)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dec.uniform.copy_(draws[0])
        steps = [dec.round()]  # the first as it is, which also readies what a capture must not
        for text, new in zip(texts, dec.kept(*steps[0])):
            text += new
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            captured = dec.round()
    torch.cuda.current_stream().wait_stream(side)
    for u in draws[1:]:
        dec.uniform.copy_(u)
        graph.replay()
        for text, new in zip(texts, dec.kept(*captured)):
            text += new
    made = sum(len(t) for t in texts) - sum(max(2, prompt - 37 * b) - 1 for b in range(seqs))
    # the same tokens as prompts
    plain = [dec.empty_cache() for _ in range(LAYERS)]
    cu_q = ints([sum(len(t) for t in texts[:b]) for b in range(seqs + 1)])
    dec.forward(ints([t for text in texts for t in text]), cu_q, ints([len(t) for t in texts]), plain)
    worst = 0.0
    for one, two in zip(dec.caches, plain):
        for a, b in zip(dec.values(one), dec.values(two)):
            worst = max([worst] + [float((x - y).norm() / y.norm()) for x, y in zip(a, b)])
    return made / (rounds * seqs), worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, kind, default in (("prompt", int, 200), ("rounds", int, 12), ("seqs", int, 3), ("temperature", float, 0.0)):
        ap.add_argument("--" + name, type=kind, default=default)
    args = ap.parse_args()
    tokens, distance = run(args.prompt, args.rounds, args.seqs, args.temperature)
    print(f"{args.seqs} requests behind prompts of up to {args.prompt} tokens, {args.rounds} rounds of {len(PARENTS)} drafted tokens each: "
          f"{tokens:.2f} tokens a round, caches {distance:.2e} from those of prompts")
