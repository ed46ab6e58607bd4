"""A small decoder served from a restored checkpoint: its weights go from a compressed difference to 4 bits without leaving the card, its
keys and values into a paged cache in 8 or 4 bits, and several drafted tokens a sequence are judged in one pass.

    python -m paper_2009_13003_amd.serve            # random weights; prints what it wrote and how long it took

The kernels are those behind lc_encode / lc_decode, lc_w4_* and lc_kv_*; torch does the rest (embedding, norms, the gate's SiLU, argmax).
"""
import argparse
import time

import torch

from . import lc


class Shape:
    def __init__(self, vocab=512, width=256, layers=2, heads=4, kv_heads=2, inner=512, context=1024):
        self.vocab, self.width, self.layers, self.heads, self.kv_heads, self.inner, self.context = vocab, width, layers, heads, kv_heads, inner, context
        self.dim = width // heads

    def matrices(self):
        """Names and sizes of the matrices, in the order in which they lie in the flat vector of parameters."""
        kv = self.kv_heads * self.dim
        yield "embed", (self.vocab, self.width)
        yield "position", (self.context, self.width)
        for i in range(self.layers):
            yield "qkv%d" % i, (self.width + 2 * kv, self.width)
            yield "out%d" % i, (self.width, self.width)
            yield "up%d" % i, (2 * self.inner, self.width)
            yield "down%d" % i, (self.width, self.inner)

    def numel(self):
        return sum(n * k for _, (n, k) in self.matrices())


def restored(base, blobs):
    """The parameters after `blobs`, each the compressed difference of one checkpoint to the one before."""
    flat = base.clone()
    lc.lc_decode_many(blobs, flat)
    return flat


class Decoder:
    """batch sequences of one model, each with `pages` pages of its own in the cache, and a chain of the last tokens' successors to draft from."""

    def __init__(self, shape, flat, batch, bits=8, group=64, dtype=torch.bfloat16, page_tokens=16):
        s = self.shape = shape
        self.dtype, self.batch = dtype, batch
        device, at, self.w = flat.device, 0, {}
        for name, (n, k) in s.matrices():
            m = flat[at:at + n * k].view(n, k)
            at += n * k
            self.w[name] = m.to(dtype) if name == "position" else lc.lc_w4_quantize(m, group)
        self.embed = lc.lc_w4_dequantize(self.w["embed"], dtype)     # rows are looked up here, and multiplied by as they lie in 4 bits
        per = -(-s.context // page_tokens)
        self.cache = [lc.new_kv_cache(batch * per, s.kv_heads, page_tokens, s.dim, bits, device) for _ in range(s.layers)]
        self.table = torch.randperm(batch * per, device=device, generator=torch.Generator(device).manual_seed(1)).to(torch.int32).view(batch, per)
        self.lens, self.count = torch.zeros(batch, dtype=torch.int32, device=device), [0] * batch      # tokens in the cache, on the card and here
        self.page_tokens, self.ws = page_tokens, {}

    def slots(self, at):
        """Where the tokens at positions `at` [batch][n] lie in the cache."""
        pages = torch.gather(self.table, 1, (at // self.page_tokens).long())
        return (pages.long() * self.page_tokens + at % self.page_tokens).view(-1)

    @staticmethod
    def norm(x):
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def step(self, tokens, depth=None, mask=None):
        """Logits [batch][n][vocab] of n new tokens a sequence, which are put into the cache behind its lens tokens and counted.  depth [n]: each
        one's place behind the last known token, and mask int64 [batch][n] which of them it sees (None: one after another)."""
        s, (batch, n) = self.shape, tokens.shape
        kv, device = s.kv_heads * s.dim, tokens.device
        if max(self.count) + n > s.context:
            raise ValueError("more tokens than the model's context")
        self.count = [c + n for c in self.count]
        at = self.lens.view(-1, 1) + torch.arange(n, device=device, dtype=torch.int32)
        place = at if depth is None else self.lens.view(-1, 1) + depth
        slots = self.slots(at)
        self.lens += n
        if n not in self.ws:
            self.ws[n] = lc.new_kv_workspace(self.cache[0], batch, n, s.heads)
        x = (self.embed[tokens] + self.w["position"][place.long()]).view(batch * n, s.width)
        for i in range(s.layers):
            qkv = lc.lc_w4_matmul(self.norm(x), self.w["qkv%d" % i])
            k, v = (qkv[:, s.width + j * kv:s.width + (j + 1) * kv].view(batch * n, s.kv_heads, s.dim) for j in range(2))
            lc.lc_kv_write(self.cache[i], k, v, slots)
            q = qkv[:, :s.width].contiguous().view(batch, n, s.heads, s.dim)
            o = lc.lc_kv_attend(self.cache[i], q, self.table, self.lens, mask=mask, ws=self.ws[n])
            x = x + lc.lc_w4_matmul(o.view(batch * n, s.width), self.w["out%d" % i])
            gate, up = lc.lc_w4_matmul(self.norm(x), self.w["up%d" % i]).chunk(2, 1)
            x = x + lc.lc_w4_matmul(torch.nn.functional.silu(gate) * up, self.w["down%d" % i])
        return lc.lc_w4_matmul(self.norm(x), self.w["embed"]).view(batch, n, s.vocab)

    def read_in(self, tokens, piece=64):
        """Puts a prompt [batch][n] into the cache; the logits behind its last token."""
        for i in range(0, tokens.shape[1], piece):
            logits = self.step(tokens[:, i:i + piece])
        return logits[:, -1]

    def keep(self, first, chosen):
        """Of the tokens drafted behind the first[b] of each sequence, keeps those numbered chosen[b], in this order; the rest is forgotten.  Keys and
        values move within the cache."""
        device, most = self.lens.device, max(map(len, chosen))
        self.count = [f + len(c) for f, c in zip(first, chosen)]
        self.lens = torch.tensor(self.count, dtype=torch.int32, device=device)
        if any(c != list(range(len(c))) for c in chosen):
            start = torch.tensor(first, dtype=torch.int32, device=device).view(-1, 1)
            number = torch.tensor([c + [-1] * (most - len(c)) for c in chosen], dtype=torch.int32, device=device)
            of = self.slots(start + number.clamp(min=0))
            to = torch.where(number.view(-1) >= 0, self.slots(start + torch.arange(most, dtype=torch.int32, device=device)), -1)
            for cache in self.cache:
                k, v = lc.lc_kv_read(cache, of)
                lc.lc_kv_write(cache, k, v, to)


def seen_before(b, known):
    """What followed the last token of known before, the latest first."""
    return list(dict.fromkeys(known[i + 1] for i in range(len(known) - 2, -1, -1) if known[i] == known[-1])) or known[-1:]


def write_on(model, prompt, count, drafts=2, guess=seen_before):
    """The `count` tokens a sequence that model writes behind prompt [batch][n], each the likeliest; and the number of passes it took.  With drafts,
    a pass judges the known next token and, below it, a tree: `drafts` of the tokens that guess(b, tokens of sequence b) lists to follow, and
    one below each, as long as the model's context has room for the tree."""
    batch, device = model.batch, prompt.device
    known = [p.tolist() for p in prompt]
    for b, t in enumerate(model.read_in(prompt).argmax(-1).tolist()):
        known[b].append(t)
    goal, passes = prompt.shape[1] + count, 1
    # the tree: 0, the known token; 1 .. drafts, below it; drafts + 1 .. 2 drafts, one below each of those
    above = [-1] + [0] * drafts + list(range(1, drafts + 1))
    depth = torch.tensor([0] + [1] * drafts + [2] * drafts, dtype=torch.int32, device=device)
    sees = []
    for i, a in enumerate(above):
        sees.append((sees[a] if a >= 0 else 0) | 1 << i)
    mask = torch.tensor([sees] * batch, dtype=torch.int64, device=device)
    while min(map(len, known)) < goal:
        if max(model.count) + len(above) > model.shape.context:              # no room for the tree any more: the known token alone
            drafts, above, depth, mask = 0, above[:1], depth[:1], mask[:, :1].contiguous()
        rows = []
        for b, k in enumerate(known):
            below = guess(b, k) if drafts else []
            below = (below + below[-1:] * drafts)[:drafts]
            rows.append([k[-1]] + below + [guess(b, k + [t])[0] for t in below])
        first = model.count
        best = model.step(torch.tensor(rows, device=device), depth, mask).argmax(-1).tolist()
        passes += 1
        chosen = []
        for b, k in enumerate(known):
            path = []
            at = 0 if len(k) < goal else None                # (a sequence that has all it needs waits for the others)
            while at is not None:
                path.append(at)
                k.append(best[b][at])
                at = next((i for i, a in enumerate(above) if a == at and rows[b][i] == k[-1]), None) if len(k) < goal else None
            chosen.append(path)
        model.keep(first, chosen)
    return [k[prompt.shape[1]:goal] for k in known], passes


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--batch", type=int, default=4)
    p.add_argument("--prompt", type=int, default=100)
    p.add_argument("--tokens", type=int, default=64)
    p.add_argument("--bits", type=int, default=8, choices=(8, 4))
    p.add_argument("--drafts", type=int, default=2)
    a = p.parse_args()
    shape = Shape()
    g = torch.Generator("cuda").manual_seed(0)
    base = 0.08 * torch.randn(shape.numel(), device="cuda", generator=g)
    live = base + 1e-3 * torch.randn(shape.numel(), device="cuda", generator=g)
    blob = lc.alloc_out(live.numel(), 3, "cuda")
    blob = blob[:lc.lc_encode(live, base, 3, blob)]
    model = Decoder(shape, restored(base, [blob]), a.batch, a.bits)
    prompt = torch.randint(shape.vocab, (a.batch, a.prompt), device="cuda", generator=g)
    t0 = time.time()
    tokens, passes = write_on(model, prompt, a.tokens, a.drafts)
    print("%d parameters from %d bytes; %d x %d tokens in %d passes, %.1f ms" % (live.numel(), blob.numel(), a.batch, a.tokens, passes, 1e3 * (time.time() - t0)))
    for t in tokens:
        print(" ".join(map(str, t)))


if __name__ == "__main__":
    main()
