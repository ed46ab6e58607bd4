"""A small decoder served from a restored checkpoint: its weights go from a compressed difference to 4 or 8 bits without leaving the card, its
keys and values into a paged cache in 8 or 4 bits, whose pages sequences may share, prompts of unlike lengths are read in together, and several drafted tokens
a sequence are judged in one pass, by the likeliest token or by given random numbers.

    python -m paper_2009_13003_amd.serve            # random weights; prints what it wrote and how long it took

    python -m paper_2009_13003_amd.serve --weights 8 --shared --sample

The kernels are those behind lc_encode / lc_decode, lc_w4_*, lc_i8_*, lc_kv_* and lc_draft_verify; torch does the rest (embedding, norms, the gate's SiLU, argmax,
softmax).
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
    """batch sequences of one model, each with room for the model's context in the cache, and a chain of the last tokens' successors to draft from.
    weights: 4 bits with a scale for `group` elements, or 8 with one a row.  shared: None, where every sequence has pages of its own, or how many pages
    all of them share: they are given out as tokens come and taken back when `keep` forgets some."""

    def __init__(self, shape, flat, batch, bits=8, group=64, dtype=torch.bfloat16, page_tokens=16, weights=4, shared=None):
        s = self.shape = shape
        self.dtype, self.batch, self.weights = dtype, batch, weights
        device, at, self.w = flat.device, 0, {}
        for name, (n, k) in s.matrices():
            m = flat[at:at + n * k].view(n, k)
            at += n * k
            self.w[name] = m.to(dtype) if name == "position" else lc.lc_w4_quantize(m, group) if weights == 4 else lc.lc_i8_quantize(m)
        # rows are looked up here, and multiplied by as they lie in 4 or 8 bits
        self.embed = (lc.lc_w4_dequantize if weights == 4 else lc.lc_i8_dequantize)(self.w["embed"], dtype)
        per = -(-s.context // page_tokens)
        total = batch * per if shared is None else shared
        self.cache = [lc.new_kv_cache(total, s.kv_heads, page_tokens, s.dim, bits, device) for _ in range(s.layers)]
        if shared is None:
            self.pages = None
            self.table = torch.randperm(total, device=device, generator=torch.Generator(device).manual_seed(1)).to(torch.int32).view(batch, per)
            self.lens = torch.zeros(batch, dtype=torch.int32, device=device)
        else:
            self.pages = lc.new_kv_pages(self.cache[0], batch, s.context)
            self.table, self.lens = self.pages.table, self.pages.lens
        self.count = [0] * batch                                     # tokens in the cache, on the card (lens) and here
        self.page_tokens, self.total, self.ws = page_tokens, total, {}

    def times(self, x, name):
        return lc.lc_w4_matmul(x, self.w[name]) if self.weights == 4 else lc.lc_i8_linear(x, self.w[name])

    def lacking(self, add):
        """What has no room for add[b] more tokens of each sequence, or None."""
        count = [c + n for c, n in zip(self.count, add)]
        if max(count) > self.shape.context:
            return "the model's context"
        if self.pages is not None and sum(-(-c // self.page_tokens) for c in count) > self.total:
            return "the shared pages hold"
        return None

    def room_for(self, add):
        """Counts add[b] more tokens of each sequence, if there is room for them."""
        lacking = self.lacking(add)
        if lacking:
            raise ValueError("more tokens than " + lacking)
        self.count = [c + n for c, n in zip(self.count, add)]

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
        device = tokens.device
        self.room_for([n] * batch)
        place = self.lens.view(-1, 1) + (torch.arange(n, device=device, dtype=torch.int32) if depth is None else depth)
        if self.pages is None:
            slots = self.slots(self.lens.view(-1, 1) + torch.arange(n, device=device, dtype=torch.int32))
            self.lens += n
        else:
            slots = lc.lc_kv_extend(self.pages, torch.full((batch,), n, dtype=torch.int32, device=device), batch * n)[1]
        if n not in self.ws:
            self.ws[n] = lc.new_kv_workspace(self.cache[0], batch, n, s.heads)

        def attend(cache, q):
            return lc.lc_kv_attend(cache, q.contiguous().view(batch, n, s.heads, s.dim), self.table, self.lens, mask=mask, ws=self.ws[n])
        return self.layers(tokens.reshape(-1), place.reshape(-1), slots, attend).view(batch, n, s.vocab)

    def layers(self, tokens, place, slots, attend, last=None):
        """Logits behind tokens [n] at these places, whose keys and values go to `slots`; attend(cache, q [n][width]) is what they see.  last: of these alone."""
        s, n = self.shape, tokens.shape[0]
        kv = s.kv_heads * s.dim
        x = self.embed[tokens] + self.w["position"][place.long()]
        for i in range(s.layers):
            qkv = self.times(self.norm(x), "qkv%d" % i)
            k, v = (qkv[:, s.width + j * kv:s.width + (j + 1) * kv].view(n, s.kv_heads, s.dim) for j in range(2))
            lc.lc_kv_write(self.cache[i], k, v, slots)
            x = x + self.times(attend(self.cache[i], qkv[:, :s.width]).view(n, s.width), "out%d" % i)
            gate, up = self.times(self.norm(x), "up%d" % i).chunk(2, 1)
            x = x + self.times(torch.nn.functional.silu(gate) * up, "down%d" % i)
        return self.times(self.norm(x if last is None else x[last]), "embed")

    def read_prompts(self, prompts):
        """Puts prompts of unlike lengths (a list of tokens a sequence, none of them empty) into the cache in one pass; the logits [batch][vocab] behind their last
        tokens.  The sequences share their pages."""
        if self.pages is None:
            raise ValueError("prompts of unlike lengths need a cache whose pages are shared")
        if len(prompts) != self.batch or not all(len(p) for p in prompts):
            raise ValueError("one prompt a sequence, of a token or more")
        s, device = self.shape, self.lens.device
        add = [len(p) for p in prompts]
        self.room_for(add)
        tokens = torch.tensor([t for p in prompts for t in p], device=device)
        starts, slots, places, _ = lc.lc_kv_extend(self.pages, torch.tensor(add, dtype=torch.int32, device=device), tokens.shape[0])
        ws = lc.new_prompt_workspace(self.cache[0], tokens.shape[0], self.batch, s.heads)

        def attend(cache, q):
            return lc.lc_kv_attend_prompt(cache, q.view(-1, s.heads, s.dim), starts, self.table, self.lens, ws=ws)
        return self.layers(tokens, places, slots, attend, last=starts[1:].long() - 1)

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
        lens = torch.tensor(self.count, dtype=torch.int32, device=device)
        if any(c != list(range(len(c))) for c in chosen):
            start = torch.tensor(first, dtype=torch.int32, device=device).view(-1, 1)
            number = torch.tensor([c + [-1] * (most - len(c)) for c in chosen], dtype=torch.int32, device=device)
            of = self.slots(start + number.clamp(min=0))
            to = torch.where(number.view(-1) >= 0, self.slots(start + torch.arange(most, dtype=torch.int32, device=device)), -1)
            for cache in self.cache:
                k, v = lc.lc_kv_read(cache, of)
                lc.lc_kv_write(cache, k, v, to)
        if self.pages is None:
            self.lens = lens
        else:
            lc.lc_kv_trim(self.pages, lens)


def seen_before(b, known):
    """What followed the last token of known before, the latest first."""
    return list(dict.fromkeys(known[i + 1] for i in range(len(known) - 2, -1, -1) if known[i] == known[-1])) or known[-1:]


def drawn(logits, tokens, sample, temperature, parent=None):
    """Paths through trees of guessed tokens [batch][nodes], and the tokens drawn behind them, by logits [batch][nodes][vocab] and random numbers of `sample`."""
    target = torch.softmax(logits.float() / temperature, -1)
    uniform = torch.rand(tokens.shape, device=tokens.device, generator=sample)
    got = lc.lc_draft_verify(target, tokens.to(torch.int32), uniform, parent=parent)
    return [p[:n] for p, n in zip(got["path"].tolist(), got["count"].tolist())], got["next"].tolist()


def write_on(model, prompt, count, drafts=2, guess=seen_before, sample=None, temperature=1.0):
    """The `count` tokens a sequence that model writes behind prompt ([batch][n], or a list of tokens a sequence), each the likeliest, or drawn with the random numbers of
    `sample`; and the number of passes it took.  With drafts, a pass judges the known next token and, below it, a tree: `drafts` of the tokens that guess(b, tokens of
    sequence b) lists to follow, and one below each, as long as the model's context and the shared pages have room for the tree."""
    if sample is not None and not temperature >= 1e-30:     # (logits divided by less might not be finite)
        raise ValueError("a temperature above zero")
    batch, device = model.batch, model.lens.device
    if torch.is_tensor(prompt):
        known, logits = [p.tolist() for p in prompt], model.read_in(prompt)
    else:
        known, logits = [list(p) for p in prompt], model.read_prompts(prompt)
    first_of = [len(k) for k in known]
    if sample is None:
        following = logits.argmax(-1).tolist()
    else:
        following = drawn(logits[:, None], torch.zeros(batch, 1, dtype=torch.int32, device=device), sample, temperature)[1]
    for b, t in enumerate(following):
        known[b].append(t)
    goal, passes = [n + count for n in first_of], 1
    # the tree: 0, the known token; 1 .. drafts, below it; drafts + 1 .. 2 drafts, one below each of those
    above = [-1] + [0] * drafts + list(range(1, drafts + 1))
    depth = torch.tensor([0] + [1] * drafts + [2] * drafts, dtype=torch.int32, device=device)
    sees = []
    for i, a in enumerate(above):
        sees.append((sees[a] if a >= 0 else 0) | 1 << i)
    mask = torch.tensor([sees] * batch, dtype=torch.int64, device=device)
    while any(len(k) < g for k, g in zip(known, goal)):
        if model.lacking([len(above)] * batch):              # no room for the tree any more: the known token alone
            drafts, above, depth, mask = 0, above[:1], depth[:1], mask[:, :1].contiguous()
        rows = []
        for b, k in enumerate(known):
            below = guess(b, k) if drafts else []
            below = (below + below[-1:] * drafts)[:drafts]
            rows.append([k[-1]] + below + [guess(b, k + [t])[0] for t in below])
        first, tokens = model.count, torch.tensor(rows, device=device)
        logits = model.step(tokens, depth, mask)
        passes += 1
        chosen = []
        if sample is None:
            best = logits.argmax(-1).tolist()
            for b, k in enumerate(known):
                path = []
                at = 0 if len(k) < goal[b] else None             # (a sequence that has all it needs waits for the others)
                while at is not None:
                    path.append(at)
                    k.append(best[b][at])
                    at = next((i for i, a in enumerate(above) if a == at and rows[b][i] == k[-1]), None) if len(k) < goal[b] else None
                chosen.append(path)
        else:
            parent = torch.tensor([above] * batch, dtype=torch.int32, device=device)
            paths, following = drawn(logits, tokens, sample, temperature, parent)
            for b, k in enumerate(known):
                path = paths[b][:max(0, goal[b] - len(k))]
                new = [rows[b][i] for i in paths[b][1:]] + [following[b]]
                k += new[:len(path)]
                chosen.append(path)
        model.keep(first, chosen)
    return [k[n:n + count] for k, n in zip(known, first_of)], passes


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--batch", type=int, default=4)
    p.add_argument("--prompt", type=int, default=100)
    p.add_argument("--tokens", type=int, default=64)
    p.add_argument("--bits", type=int, default=8, choices=(8, 4))
    p.add_argument("--drafts", type=int, default=2)
    p.add_argument("--weights", type=int, default=4, choices=(4, 8))
    p.add_argument("--shared", action="store_true", help="sequences share the cache's pages, and prompts are of unlike lengths")
    p.add_argument("--sample", action="store_true", help="tokens are drawn instead of the likeliest ones taken")
    p.add_argument("--temperature", type=float, default=1.0)
    a = p.parse_args()
    shape = Shape()
    g = torch.Generator("cuda").manual_seed(0)
    base = 0.08 * torch.randn(shape.numel(), device="cuda", generator=g)
    live = base + 1e-3 * torch.randn(shape.numel(), device="cuda", generator=g)
    blob = lc.alloc_out(live.numel(), 3, "cuda")
    blob = blob[:lc.lc_encode(live, base, 3, blob)]
    room = -(-(a.prompt + a.tokens + 1 + 2 * a.drafts) // 16)
    model = Decoder(shape, restored(base, [blob]), a.batch, a.bits, weights=a.weights, shared=a.batch * room if a.shared else None)
    prompt = torch.randint(shape.vocab, (a.batch, a.prompt), device="cuda", generator=g)
    if a.shared:
        prompt = [t[:max(1, a.prompt * (i + 1) // a.batch)] for i, t in enumerate(prompt.tolist())]
    t0 = time.time()
    tokens, passes = write_on(model, prompt, a.tokens, a.drafts, sample=g if a.sample else None, temperature=a.temperature)
    print("%d parameters from %d bytes; %d x %d tokens in %d passes, %.1f ms" % (live.numel(), blob.numel(), a.batch, a.tokens, passes, 1e3 * (time.time() - t0)))
    for t in tokens:
        print(" ".join(map(str, t)))


if __name__ == "__main__":
    main()
