"""The paged cache of keys and values in 8 or 4 bits (include/lc_serve.h): written and read back against the definition's own
arithmetic, bit for bit; the attention over it against 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module")
def lc():
    from paper_2009_13003_amd import lc as mod
    return mod


# ---------------------------------------------------------------- writing and reading
def by_definition(v, bits):
    """q and scales of float32 vectors [..., dim], in numpy's IEEE arithmetic."""
    most = np.float32(127 if bits == 8 else 7)
    with np.errstate(all="ignore"):
        top = np.abs(v).max(-1)
        s = (top * np.float32(1.0 / float(most))).astype(np.float32)
        dead, zero = ~np.isfinite(top), s < np.float32(2.0 ** -126)
        live = ~dead & ~zero
        inv = np.where(live, np.float32(1) / np.where(live, s, np.float32(1)), np.float32(0)).astype(np.float32)
        q = np.rint((v * inv[..., None]).astype(np.float32))
        q = np.where(live[..., None], np.clip(q, -most, most), 0)
    return q.astype(np.float32), np.where(dead, np.float32("nan"), np.where(zero, np.float32(0), s))


def held(cache):
    """What the cache holds, by slot: q [slots][heads][dim] for k and v, and their scales."""
    out = []
    for codes, scales in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        b = codes.permute(0, 2, 1, 3).reshape(-1, cache.heads, codes.shape[-1]).cpu().numpy()
        if cache.bits == 8:
            q = b.view(np.int8).astype(np.float32)
        else:
            q = np.stack((b & 15, b >> 4), -1).reshape(*b.shape[:-1], -1).astype(np.float32) - 8
        out += [q, scales.permute(0, 2, 1).reshape(-1, cache.heads).cpu().numpy()]
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 32, 8), (5, 3, 64, 16), (17, 7, 96, 8), (40, 2, 128, 64), (9, 5, 160, 32), (33, 1, 256, 16), (700, 4, 224, 1024)])
def test_write_and_read_are_the_definition(lc, dtype, bits, tokens, heads, dim, page):
    g = torch.Generator(device=DEV); g.manual_seed(tokens + dim)
    pages = -(-tokens // page) + 2
    cache = lc.new_kv_cache(pages, heads, page, dim, bits, DEV)
    empty = held(cache)
    wide = torch.randn(2, tokens, heads + 1, dim + 3, generator=g, device=DEV) * torch.exp(2 * torch.randn(2, tokens, heads + 1, 1, generator=g, device=DEV))
    wide = wide.to(dtype)
    k, v = wide[0, :, 1:, 1:dim + 1], wide[1, :, 1:, 1:dim + 1]                  # pitches and first elements off every alignment
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:tokens]
    given = slots.clone()
    if tokens > 4:
        given[1], given[2], given[3] = -1, pages * page, 1 << 40                 # passed over
    lc.lc_kv_write(cache, k, v, given)
    now = held(cache)
    keep = np.ones(pages * page, bool)
    live = [i for i in range(tokens) if 0 <= int(given[i]) < pages * page]
    at = given.cpu().numpy()[live]
    keep[at] = False
    for n, x in enumerate((k, v)):
        q, s = by_definition(x.float().cpu().numpy()[live], bits)
        assert np.array_equal(now[2 * n][at], q) and np.array_equal(now[2 * n + 1][at], s, equal_nan=True)
        assert np.array_equal(now[2 * n][keep], empty[2 * n][keep]) and np.array_equal(now[2 * n + 1][keep], empty[2 * n + 1][keep])
    got = lc.lc_kv_read(cache, given, dtype)
    store = torch.full((2, tokens + 1, heads + 2, dim + 5), 9.0, dtype=dtype, device=DEV)
    views = (store[0, 1:, 1:-1, 2:dim + 2], store[1, 1:, 1:-1, 2:dim + 2])
    lc.lc_kv_read(cache, given, out=views)
    for n in range(2):
        want = torch.zeros(tokens, heads, dim)
        want[live] = torch.from_numpy(now[2 * n][at] * now[2 * n + 1][at][..., None])
        want = want.to(dtype).float().numpy()
        assert np.array_equal(got[n].float().cpu().numpy(), want, equal_nan=True)
        assert np.array_equal(views[n].float().cpu().numpy(), want, equal_nan=True)
        store[n, 1:, 1:-1, 2:dim + 2] = 9.0
    assert (store == 9).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_write_extremes(lc, bits):
    top = float(np.finfo(np.float32).max)
    x = torch.zeros(9, 1, 64, device=DEV)
    x[0, 0, 3], x[1, 0, :] = top, -top
    x[2, 0, 5], x[3, 0, 60], x[4, 0, 1] = float("inf"), float("nan"), 1e-45
    x[5, 0, 1] = 127 * 2.0 ** -126
    x[6, 0, :7] = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -126.5])
    x[7, 0, :5] = torch.tensor([7.0, 0.5, 1.5, -0.5, -2.5])
    x[8, 0, :] = -0.0
    cache = lc.new_kv_cache(2, 1, 8, 64, bits, DEV)
    slots = torch.arange(9, device=DEV)
    lc.lc_kv_write(cache, x, x.flip(0).contiguous(), slots)
    now = held(cache)
    q, s = by_definition(x.cpu().numpy(), bits)
    assert np.array_equal(now[0][:9], q) and np.array_equal(now[1][:9], s, equal_nan=True)
    assert np.array_equal(now[2][:9], q[::-1]) and np.array_equal(now[3][:9], s[::-1], equal_nan=True)
    k, _ = lc.lc_kv_read(cache, slots)
    assert k[2].isnan().all() and k[3].isnan().all() and (k[4] == 0).all() and (k[8] == 0).all()


# ---------------------------------------------------------------- attention
class Case:
    """A cache with sequences in shuffled pages; what no query may see holds NaN scales and any codes."""

    def __init__(self, lc, seed, lens, nq, heads, kv, dim, page, bits, dtype, spread=1.5, wide=None):
        g = torch.Generator(device=DEV); g.manual_seed(seed)
        self.lens, self.nq, self.heads, self.kv, self.dim, self.page, self.bits, self.dtype = lens, nq, heads, kv, dim, page, bits, dtype
        need = [-(-n // page) for n in lens]
        pages = sum(need) + 3
        wide = max(need + [1]) if wide is None else wide
        c = torch.Generator(); c.manual_seed(seed)
        order, at = torch.randperm(pages, generator=c)[:sum(need)].tolist(), 0
        table = torch.randint(-5, 1 << 30, (len(lens), wide), generator=c, dtype=torch.int32)      # behind a sequence's pages: anything
        owner = torch.full((pages * page,), -1)
        for b, n in enumerate(need):
            table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            for i in range(lens[b]):
                owner[order[at + i // page] * page + i % page] = b
            at += n
        row = dim * bits // 8
        low = 1 if bits == 8 else 0
        k, v = (torch.randint(low, 256, (pages, kv, page, row), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2))
        most = 127 if bits == 8 else 7
        ks, vs = (torch.exp(0.3 * torch.randn(pages, kv, page, generator=g, device=DEV)) * (1.7 / most) for _ in range(2))
        lost = (owner < 0).view(pages, 1, page).expand(-1, kv, -1).to(DEV)
        ks[lost], vs[lost] = float("nan"), float("nan")
        self.cache = lc.KvCache(k, v, ks, vs, bits)
        self.table, self.lens_dev = table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.q = (spread * torch.randn(len(lens), nq, heads, dim, generator=g, device=DEV)).to(dtype)
        self.scale = dim ** -0.5

    def run(self, lc, mask=None, **kw):
        return lc.lc_kv_attend(self.cache, self.q, self.table, self.lens_dev, self.scale, mask, **kw)

    def values(self, b, n):
        t = torch.arange(n)
        slots = (self.table[b].cpu().long()[t // self.page] * self.page + t % self.page).numpy()
        k, ks, v, vs = self.held
        return k[slots].astype(np.float64), ks[slots].astype(np.float64), v[slots].astype(np.float64), vs[slots].astype(np.float64)

    def check(self, out, mask=None):
        self.held = held(self.cache)
        rels = []
        for b, n in enumerate(self.lens):
            seen = np.ones((self.nq, max(n, 0)), bool)
            for i in range(self.nq):
                for j in range(self.nq):
                    t = n - self.nq + j
                    if t >= 0:
                        seen[i, t] = j <= i if mask is None else bool(int(mask[b, i]) >> j & 1)
            got = out[b].double().cpu().numpy()
            if n == 0:
                assert (got == 0).all()
                continue
            k, ks, v, vs = self.values(b, n)
            q = self.q[b].double().cpu().numpy()
            g = self.heads // self.kv
            for h in range(self.heads):
                c = h // g
                score = self.scale * (q[:, h] @ (k[:, c] * ks[:, c, None]).T)                       # [nq, n]
                score = np.where(seen, score, -np.inf)
                some = seen.any(1)
                top = np.where(some, score.max(1, initial=-np.inf), 0.0)
                p = np.exp(score - top[:, None])
                total = p.sum(1, keepdims=True)
                p = np.divide(p, total, out=np.zeros_like(p), where=total > 0)
                value = v[:, c] * vs[:, c, None]
                want, weight = p @ value, p @ np.abs(value)
                # The score: dim products and the take-away of 24 (4 bits: codes below 32 and that, else below 128), each sum rounded
                # once, and three products; a maximum's exponential and its sum the same again.  Probabilities: exp2 to 2 ulp, 16 bits
                # of them (24 for fp32), as many sums as tokens, and a rescaling a tile of 32 and one a wavefront and split.
                size = np.abs(q[:, h]).sum(1)[:, None] * (ks[:, c] * (56 if self.bits == 4 else 128))[None] * self.scale
                size = np.where(seen, size, 0).max(1)
                logit = 2.0 ** -24 * (2 * self.dim + 8) * size + 2.0 ** -22 * np.where(some, np.abs(np.where(seen, score, 0)).max(1), 0)
                part = 2.0 ** -15 if self.dtype != torch.float32 else 2.0 ** -23
                share = 2 * logit + part + 2.0 ** -21 + 2.0 ** -24 * (n + n / 16 + 80)
                bound = weight * share[:, None] * (1 + 2.0 ** -8) + HALF_ULP[self.dtype] * np.abs(want) + LEAST[self.dtype] + 1e-44
                off = np.abs(got[:, h] - want) - bound
                assert off.max() <= 0, (b, h, off.max())
                assert (got[~some, h] == 0).all()
                rels.append((np.sum((got[:, h] - want) ** 2), np.sum(want ** 2)))
        d, s = map(sum, zip(*rels)) if rels else (0, 0)
        # all together no further off than results rounded to nearest may be, and 32 bits' worth of sums
        assert math.sqrt(d) <= (HALF_ULP[self.dtype] + 1e-5) * math.sqrt(s) + 1e-30, math.sqrt(d / s)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("lens,nq,heads,kv,dim,page", [
    ([1], 1, 1, 1, 32, 8), ([31, 32, 33], 1, 4, 2, 64, 16), ([0, 1, 127, 128], 1, 8, 8, 128, 16), ([257], 1, 7, 1, 96, 8), ([1000, 3], 1, 16, 2, 256, 32),
    ([65, 500], 1, 33, 1, 160, 128), ([2100], 1, 2, 2, 128, 1024), ([4097, 17, 4000], 1, 4, 4, 64, 64), ([3000], 2, 40, 2, 128, 16), ([130, 9], 5, 8, 2, 224, 8)])
def test_attention(lc, dtype, bits, lens, nq, heads, kv, dim, page):
    case = Case(lc, sum(lens) + dim, lens, nq, heads, kv, dim, page, bits, dtype)
    case.check(case.run(lc))


def tree(batch, nq, seed):
    """Masks of random trees: every token sees its ancestors and itself."""
    c = torch.Generator(); c.manual_seed(seed)
    rows = []
    for _ in range(batch):
        row = [1]
        for j in range(1, nq):
            row.append(row[int(torch.randint(0, j, (1,), generator=c))] | 1 << j)
        rows.append([r - (1 << 64) if r >> 63 else r for r in row])
    return torch.tensor(rows, dtype=torch.int64, device=DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("lens,nq,heads,kv,dim,page", [([70, 300, 12], 12, 4, 2, 64, 16), ([64, 65, 63, 10], 64, 2, 1, 128, 32), ([1500], 24, 32, 8, 128, 64),
                                                       ([333, 40], 33, 3, 3, 96, 8), ([40, 5], 7, 14, 2, 256, 16)])
def test_attention_of_trees(lc, dtype, bits, lens, nq, heads, kv, dim, page):
    case = Case(lc, sum(lens) + nq, lens, nq, heads, kv, dim, page, bits, dtype)
    mask = tree(len(lens), nq, nq)
    case.check(case.run(lc, mask), mask)
    case.check(case.run(lc))                                 # and one behind the other


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("lens,nq,heads,kv,dim,page", [([512], 1, 8, 8, 128, 16), ([513, 2], 1, 8, 8, 128, 16), ([513], 40, 4, 2, 64, 32), ([512, 500, 0], 40, 4, 2, 64, 32),
                                                       ([641, 640, 639], 7, 18, 9, 96, 8), ([256, 257], 3, 6, 3, 256, 16), ([256, 255], 3, 6, 3, 192, 16),
                                                       ([530], 64, 16, 8, 128, 8), ([1, 1025, 7], 20, 20, 10, 128, 64)])
def test_attention_split_or_not(lc, dtype, bits, lens, nq, heads, kv, dim, page):
    """Lengths at which sequences begin to be split, and at the ends of the parts: some rows see nothing of the last."""
    case = Case(lc, sum(lens) + nq + dim, lens, nq, heads, kv, dim, page, bits, dtype)
    mask = tree(len(lens), nq, nq)
    case.check(case.run(lc, mask), mask)


@pytest.mark.parametrize("bits", [8, 4])
def test_rows_that_see_nothing(lc, bits):
    case = Case(lc, 5, [6, 3, 0, 90], 6, 4, 2, 64, 16, bits, torch.float32)
    mask = torch.zeros(4, 6, dtype=torch.int64, device=DEV)
    mask[0, 2] = 0b100
    mask[1, 5] = 0b111111                                    # of which three tokens exist
    out = case.run(lc, mask)
    case.check(out, mask)
    assert (out[0, 0] == 0).all() and (out[0, 2] != 0).any() and (out[1, 0] == 0).all() and (out[2] == 0).all() and (out[3, 0] != 0).any()


def test_pages_outside_the_cache_and_lengths_outside_the_table(lc):
    case = Case(lc, 6, [40, 64], 1, 2, 2, 64, 8, 8, torch.float32)
    want = case.run(lc)
    whole = case.lens_dev.clone()
    case.lens_dev[1] = 1 << 30                               # held to the eight pages of the table
    assert torch.equal(case.run(lc), want)
    case.lens_dev[0] = -7
    out = case.run(lc)
    assert (out[0] == 0).all() and torch.equal(out[1], want[1])
    case.lens_dev.copy_(whole)
    bad = case.table.clone()
    bad[0, 1], bad[1, 0], bad[1, 3] = -1, case.cache.pages, 0x7FFFFFFF
    got = lc.lc_kv_attend(case.cache, case.q, bad, case.lens_dev, case.scale)
    # the same as a cache in which those tokens have no weight: compare with the sequences' other pages alone
    for b, gone in ((0, [1]), (1, [0, 3])):
        pages = [int(p) for i, p in enumerate(case.table[b, :-(-case.lens[b] // 8)]) if i not in gone]
        few = torch.tensor([pages], dtype=torch.int32, device=DEV)
        n = torch.tensor([8 * len(pages)], dtype=torch.int32, device=DEV)
        other = lc.lc_kv_attend(case.cache, case.q[b:b + 1], few, n, case.scale)
        assert torch.allclose(got[b:b + 1], other, rtol=1e-5, atol=1e-6)      # (32-bit sums in another order)


@pytest.mark.parametrize("bits", [8, 4])
def test_what_is_not_finite(lc, bits):
    """A key or value that was not finite when it was written reaches those that see it, and nobody else."""
    case = Case(lc, 8, [50, 50], 4, 2, 1, 64, 16, bits, torch.float32)
    t = 47                                                   # drafted token 1 of sequence 0
    slot = int(case.table[0, t // 16]) * 16 + t % 16
    case.cache.v_scale.view(-1)[slot] = float("nan")
    out = case.run(lc)
    assert not out[0, 0].isnan().any() and out[0, 1:].isnan().all() and not out[1].isnan().any()
    case.cache.v_scale.view(-1)[slot] = 1.0
    case.cache.k_scale.view(-1)[slot] = float("nan")
    out = case.run(lc)
    assert not out[0, 0].isnan().any() and out[0, 1:].isnan().all() and not out[1].isnan().any()
    case.cache.k_scale.view(-1)[slot] = 1.0
    case.q[1, 2, 1, 5] = float("nan")
    out = case.run(lc)
    assert out[1, 2, 1].isnan().all() and not out[1, 2, 0].isnan().any() and not out[1, :2].isnan().any() and not out[0].isnan().any()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", TYPES)
def test_sharp_and_flat(lc, bits, dtype):
    """Scores of hundreds (one token takes it all) and none at all (the mean of thousands)."""
    case = Case(lc, 11, [3333, 700], 1, 4, 2, 128, 16, bits, dtype, spread=60.0)
    case.check(case.run(lc))
    case.q.zero_()
    case.check(case.run(lc))


def test_offsets_beyond_32_bits(lc):
    """Pages whose codes and rows lie past 2^32 bytes."""
    pages, heads, page, dim = 1100, 32, 1024, 128            # 4.6 GB of codes each
    cache = lc.new_kv_cache(pages, heads, page, dim, 8, DEV)
    g = torch.Generator(device=DEV); g.manual_seed(4)
    k, v = torch.randn(2, 40, heads, dim, generator=g, device=DEV).unbind(0)
    slots = (pages - 1) * page + torch.arange(40, device=DEV)
    lc.lc_kv_write(cache, k, v, slots)
    got = lc.lc_kv_read(cache, slots)
    small = lc.new_kv_cache(2, heads, page, dim, 8, DEV)
    lc.lc_kv_write(small, k, v, slots - (pages - 2) * page)
    assert torch.equal(got[0], lc.lc_kv_read(small, slots - (pages - 2) * page)[0])
    q = torch.randn(1, 1, heads, dim, generator=g, device=DEV)
    n = torch.tensor([40], dtype=torch.int32, device=DEV)
    one = lc.lc_kv_attend(cache, q, torch.tensor([[pages - 1]], dtype=torch.int32, device=DEV), n)
    two = lc.lc_kv_attend(small, q, torch.tensor([[1]], dtype=torch.int32, device=DEV), n)
    assert torch.equal(one, two)


def test_streams_workspaces_and_graphs(lc):
    cases = [Case(lc, s, [900, 40], 1, 8, 2, 128, 16, 8, torch.bfloat16) for s in (1, 2)]
    want = [c.run(lc) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [c.run(lc, stream=s) for c, s in zip(cases, streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    c = cases[0]
    ws, out = lc.new_kv_workspace(c.cache, 2, 1, 8), torch.empty_like(c.q)
    ws.fill_(0xFF)                                           # NaN everywhere: its content need not be anything
    k, v = torch.randn(2, 2, 2, 128, device=DEV).to(torch.bfloat16).unbind(0)
    slots = torch.stack([c.table[b, (n - 1) // 16].long() * 16 + (n - 1) % 16 for b, n in enumerate(c.lens)])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lc.lc_kv_write(c.cache, k, v, slots)
        c.run(lc, ws=ws, out=out)
    for _ in range(3):
        k.copy_(torch.randn(2, 2, 128, device=DEV))
        c.q.copy_(torch.randn_like(c.q))
        graph.replay()
        torch.cuda.synchronize()
        lc.lc_kv_write(c.cache, k, v, slots)
        assert torch.equal(out, c.run(lc))


def test_refusals(lc):
    c = Case(lc, 1, [20], 1, 4, 2, 64, 16, 8, torch.float32)
    with pytest.raises(lc.LcError) as e:
        c.run(lc, ws=torch.empty(0, dtype=torch.uint8, device=DEV))
    assert e.value.status == lc.ERR_WORKSPACE
    for bad in (dict(q=c.q.double()), dict(lens=c.lens_dev.long()), dict(table=c.table.long()), dict(q=c.q[..., :32].contiguous())):
        args = dict(q=c.q, table=c.table, lens=c.lens_dev)
        args.update(bad)
        with pytest.raises(AssertionError):
            lc.lc_kv_attend(c.cache, **args)
    with pytest.raises(lc.LcError):
        lc.lc_kv_attend(c.cache, c.q[:, :, :3].contiguous(), c.table, c.lens_dev)      # heads no multiple of the cache's
    with pytest.raises(lc.LcError):
        lc.lc_kv_attend(c.cache, torch.zeros(1, 65, 4, 64, device=DEV), c.table, c.lens_dev)
    odd = lc.KvCache(torch.zeros(2, 1, 16, 48, dtype=torch.uint8, device=DEV), torch.zeros(2, 1, 16, 48, dtype=torch.uint8, device=DEV),
                     torch.zeros(2, 1, 16, device=DEV), torch.zeros(2, 1, 16, device=DEV), 8)
    with pytest.raises(lc.LcError):
        lc.lc_kv_write(odd, torch.zeros(1, 1, 48, device=DEV), torch.zeros(1, 1, 48, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV))
    assert lc.lc_kv_attend(c.cache, c.q[:0], c.table[:0], c.lens_dev[:0]).shape == (0, 1, 4, 64)
    lc.lc_kv_write(c.cache, torch.zeros(0, 2, 64, device=DEV), torch.zeros(0, 2, 64, device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV))
