"""A small state-space language model served with the block operators: prompts of uneven length in
one batch, then one token a sequence at a time, the token step replayed as a CUDA graph.

    python examples/state_space_lm.py [--layers 4] [--dim 1024] [--tokens 32] [--dtype bf16]

A block is: dense_q4 (gate z, channels x|B|C, time steps), causal_conv and StateSpace.scan for a
prompt or StateSpace.step for a token, the gated norm, dense_q4, and the sum into the fp32 residual
stream with the norms behind this block and before the next.  Weights are random.
"""
import argparse
import math
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2110_06037_gb300 as sn  # noqa: E402

WIDTH, GROUP = 4, 64


class Block:
    def __init__(self, dim, heads, head_dim, groups, state, gen):
        def rnd(*shape, scale=1.0):
            return scale * torch.randn(shape, device="cuda", generator=gen)

        def q4(n, k):
            return sn.Q4Weights(*sn.quantize_q4(rnd(n, k, scale=1 / math.sqrt(k)), GROUP), k, GROUP)

        self.inner, channels = heads * head_dim, heads * head_dim + 2 * groups * state
        self.cut = [self.inner, channels, heads]
        self.w_in, self.w_out = q4(sum(self.cut), dim), q4(dim, self.inner)
        self.conv_w, self.conv_b = rnd(channels, WIDTH, scale=0.5), rnd(channels, scale=0.1)
        self.ssm = sn.StateSpace(heads, head_dim, groups, state, a=-1 - 15 * torch.rand(heads, device="cuda", generator=gen),
                                 d=torch.ones(heads, device="cuda"), dt_bias=rnd(heads) - 4,
                                 conv_weight=self.conv_w, conv_bias=self.conv_b)
        ones = torch.ones
        self.gated = sn.BlockNorm(self.inner, post=ones(self.inner, device="cuda"), gate="silu", gate_at="before")
        self.after = sn.BlockNorm(dim, post=ones(dim, device="cuda"), scale=0.5 * ones(dim, device="cuda"),
                                  pre=ones(dim, device="cuda"))

    def cache(self, entries, dtype):
        s = self.ssm
        return (torch.zeros(entries, WIDTH, s.channels, dtype=dtype, device="cuda"),
                torch.zeros(entries, s.heads, s.head_dim, s.state, device="cuda"))

    def _out(self, y, z, r):
        return self.after(sn.dense_q4(self.gated(y, gate=z)[0], self.w_out), residual=r)

    def prompt(self, r, n, cache, offsets, max_len):
        z, xbc, dt = sn.dense_q4(n, self.w_in).split(self.cut, dim=1)
        c = sn.causal_conv(xbc, self.conv_w, self.conv_b, offsets=offsets, max_len=max_len, kept=cache[0])
        return self._out(self.ssm.scan(c, dt, offsets=offsets, max_len=max_len, state_out=cache[1]), z, r)

    def token(self, r, n, cache, pos):
        z, xbc, dt = sn.dense_q4(n, self.w_in).split(self.cut, dim=1)
        return self._out(self.ssm.step(xbc, dt, cache[0], cache[1], pos), z, r)


class Model:
    def __init__(self, layers=4, dim=1024, head_dim=64, groups=1, state=128, vocab=1000, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.dtype = dtype
        self.embed = torch.randn(vocab, dim, device="cuda", generator=gen)
        self.first = sn.BlockNorm(dim, pre=torch.ones(dim, device="cuda"))
        self.blocks = [Block(dim, 2 * dim // head_dim, head_dim, groups, state, gen) for _ in range(layers)]
        head = torch.randn(vocab, dim, device="cuda", generator=gen) / math.sqrt(dim)
        self.head = sn.Q4Weights(*sn.quantize_q4(head, GROUP), dim, GROUP)

    def caches(self, entries):
        return [b.cache(entries, self.dtype) for b in self.blocks]

    def _start(self, tokens):
        r = self.embed[tokens]
        return r, self.first(None, residual=r, dtype=self.dtype)[1]

    def prompt(self, tokens, caches, offsets, max_len):
        """Logits of every token row; the caches then stand behind the prompts."""
        r, n = self._start(tokens)
        for b, c in zip(self.blocks, caches):
            r, n = b.prompt(r, n, c, offsets, max_len)
        return sn.dense_q4(n, self.head)

    def token(self, tokens, caches, pos):
        """Logits of one token a sequence; pos int32: how many tokens each sequence has had."""
        r, n = self._start(tokens)
        for b, c in zip(self.blocks, caches):
            r, n = b.token(r, n, c, pos)
        return sn.dense_q4(n, self.head)


def generate(model, prompts, count):
    """Greedy continuation of each prompt by `count` tokens: [sequences, count]."""
    lens = [len(p) for p in prompts]
    offsets = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    caches = model.caches(len(prompts))
    logits = model.prompt(torch.cat(prompts), caches, offsets, max(lens))
    now = logits[offsets[1:].long() - 1].argmax(1)
    pos = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = [now.clone()]

    def step():
        now.copy_(model.token(now, caches, pos).argmax(1))
        pos.add_(1)

    graph = None
    for _ in range(count - 1):
        if graph is None:  # the first step as it is (first use of each kernel), the others replayed
            step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        else:
            graph.replay()
        out.append(now.clone())
    return torch.stack(out, dim=1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--dim", type=int, default=1024)
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--dtype", choices=("f32", "f16", "bf16"), default="bf16")
    a = ap.parse_args()
    dtype = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[a.dtype]
    model = Model(a.layers, a.dim, dtype=dtype)
    prompts = [torch.randint(0, 1000, (n,), device="cuda") for n in (1, 37, 700, 2000)]
    generate(model, prompts, 4)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    out = generate(model, prompts, a.tokens)
    torch.cuda.synchronize()
    sn.check_device()
    print(f"{len(prompts)} prompts of {[len(p) for p in prompts]} tokens, {a.tokens} tokens each: "
          f"{1e3 * (time.perf_counter() - t0):.1f} ms")
    print(out[:, :8].tolist())


if __name__ == "__main__":
    main()
