"""The attention block of one decoder layer as a server runs it: a prompt through the NVFP4 W4A4 path into the 8-bit paged cache,
then tokens one at a time for a batch of requests, with the same NVFP4 weights and BF16 activations.

  python examples/attention_block.py [--prompt 1000] [--steps 8] [--seqs 3]

Weights and activations are random, of the shape of an 8B-class layer.  Prints how far the block is from a plain evaluation in
32 bits with the same dequantized weights and cache.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2605_20315_amd as mq  # noqa: E402

HIDDEN, HQ, HKV, D, P = 4096, 32, 8, 128, 64
EPS, SCALE = 1e-6, D ** -0.5


class Block:
    """Weights, rotation table, cache and workspaces of one layer, for up to `seqs` sequences of `longest` tokens."""

    def __init__(self, seqs, longest, gen):
        normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
        self.norm = (1.0 + 0.1 * normal(HIDDEN)).to(torch.bfloat16)
        self.qkv_bf16 = (normal((HQ + 2 * HKV) * D, HIDDEN) * HIDDEN ** -0.5).to(torch.bfloat16)
        self.o_bf16 = (normal(HIDDEN, HQ * D) * HIDDEN ** -0.5).to(torch.bfloat16)
        self.qkv, self.o = self._quantize(self.qkv_bf16), self._quantize(self.o_bf16)
        self.alpha_in = torch.tensor([8.0 / 2688.0], device="cuda")   # calibrated scales of the two activations
        self.alpha_out = torch.tensor([4.0 / 2688.0], device="cuda")
        self.table = mq.mq_rope_table(longest, D, 500000.0, mq.MQ_ROPE_YARN, 4.0, max(longest // 4, 1))
        width = -(-longest // P)
        self.page_table = torch.randperm(seqs * width, device="cuda", generator=gen).to(torch.int32).view(seqs, width)
        self.cache = []
        for _ in "kv":
            self.cache += [torch.empty(seqs * width, HKV, P, D, dtype=torch.uint8, device="cuda"), torch.empty(seqs * width, HKV, dtype=torch.uint8, device="cuda")]
        self.workspace = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    @staticmethod
    def _quantize(w):
        alpha = mq.nvfp4_global_scale(w)
        return mq.nvfp4_quantize(w, alpha, layout=mq.MQ_LAYOUT_KTILE) + (alpha,)

    def __call__(self, x, cu_q, kv_lens, prefill):
        """x [T, HIDDEN]: the new tokens of the sequences, kv_lens with them counted.  Returns (block's output, attention's)."""
        if prefill:
            c, s = mq.nvfp4_quantize_rmsnorm(x, self.norm, EPS, self.alpha_in, layout=mq.MQ_LAYOUT_KTILE)
            qkv = mq.nvfp4_gemm_ws(c, s, self.alpha_in, *self.qkv, self.workspace, layout=mq.MQ_LAYOUT_KTILE)
        else:
            h = mq.nvfp4_quantize_rmsnorm(x, self.norm, EPS, self.alpha_in, return_bf16=True)[2]
            qkv = mq.nvfp4_matvec(h, *self.qkv, layout=mq.MQ_LAYOUT_KTILE, workspace=self.workspace)
        qkv = qkv.view(len(x), HQ + 2 * HKV, D)
        q = mq.kv8_append(qkv[:, :HQ], qkv[:, HQ : HQ + HKV], qkv[:, HQ + HKV :], *self.cache, self.page_table, cu_q, kv_lens, self.table)
        a = mq.kv8_attention(q, *self.cache, self.page_table, cu_q, kv_lens, SCALE, workspace=self.workspace)
        flat = a.view(len(x), HQ * D)
        if prefill:
            y = mq.nvfp4_linear(flat, self.alpha_out, *self.o, layout=mq.MQ_LAYOUT_KTILE, workspace=self.workspace)
        else:
            y = mq.nvfp4_matvec(flat, *self.o, layout=mq.MQ_LAYOUT_KTILE, workspace=self.workspace)
        return y, a

    def dequantized(self, name):
        """A weight matrix in 32 bits from its codes."""
        codes, scales, alpha = getattr(self, name)
        codes, scales = mq.nvfp4_relayout(codes, scales, mq.MQ_LAYOUT_KTILE, mq.MQ_LAYOUT_LINEAR)
        grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device="cuda")
        grid = torch.cat([grid, -grid])
        q = torch.stack([grid[(codes & 15).long()], grid[(codes >> 4).long()]], -1).view(codes.shape[0], -1, 16)
        return (q * scales.view(torch.float8_e4m3fn).float()[..., None]).view(codes.shape[0], -1) * alpha

    def step_in_32_bits(self, x, kv_lens):
        """One token a sequence, evaluated plainly on the weights' and the cache's values (which hold the new tokens)."""
        def turned(v, pos):
            row = self.table[pos]
            c, s = row[:, None, : D // 2], row[:, None, D // 2 :]
            lo, hi = v[..., : D // 2], v[..., D // 2 :]
            return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)

        h = x.float()
        h = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * self.norm.float()
        q = turned((h @ self.dequantized("qkv").t()).view(len(x), HQ + 2 * HKV, D)[:, :HQ], kv_lens.long() - 1)
        out = []
        for b, n in enumerate(kv_lens.tolist()):
            at = self.page_table[b, : -(-n // P)].long()
            k, v = (torch.ldexp(self.cache[i][at].view(torch.float8_e4m3fn).float(), self.cache[i + 1][at].int()[..., None, None] - 127)
                    .transpose(0, 1).reshape(HKV, -1, D)[:, :n].repeat_interleave(HQ // HKV, 0) for i in (0, 2))
            p = torch.softmax((k @ q[b][..., None])[..., 0] * SCALE, 1)
            out.append((p[:, None] @ v)[:, 0])
        a = torch.stack(out)
        return a.view(len(x), -1) @ self.dequantized("o").t(), a


def run(prompt=1000, steps=8, seqs=3, seed=0):
    """Largest relative error of (block's output, attention's output) over the decode steps."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    block = Block(seqs, prompt + steps + 1, gen)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    lens = [max(1, prompt - 37 * b) for b in range(seqs)]  # prompts of different lengths, in one batch
    x = torch.randn(sum(lens), HIDDEN, device="cuda", generator=gen).to(torch.bfloat16)
    block(x, ints([0] + [sum(lens[: b + 1]) for b in range(seqs)]), ints(lens), prefill=True)
    worst = [0.0, 0.0]
    for _ in range(steps):
        lens = [n + 1 for n in lens]
        x = torch.randn(seqs, HIDDEN, device="cuda", generator=gen).to(torch.bfloat16)
        got = block(x, ints(list(range(seqs + 1))), ints(lens), prefill=False)
        want = block.step_in_32_bits(x, ints(lens))
        for i, (g, w) in enumerate(zip(got, want)):
            worst[i] = max(worst[i], float((g.float().reshape(-1) - w.reshape(-1)).norm() / w.norm()))
    return tuple(worst)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("prompt", 1000), ("steps", 8), ("seqs", 3)):
        ap.add_argument("--" + name, type=int, default=default)
    args = ap.parse_args()
    block, attention = run(args.prompt, args.steps, args.seqs)
    print(f"{args.seqs} prompts of up to {args.prompt} tokens, {args.steps} decode steps: "
          f"attention {attention:.2e}, block {block:.2e} from a plain evaluation in 32 bits")
