"""The paged cache and attention over it on the GPU: books of the pages against
a plain list of pages, attention against its definition in 64 bits.

Tolerances of the attention, element by element. Probabilities are rounded to
bf16 (2^-8 of each at most) before the products that sum them, and results once
more; everything else is fp32 (2^-15 covers its sums and the exponents'). With
absolute values written |.|:
  out  2^-8 (|out| + P|V|) + 2^-15 P|V|      lse  2^-18 (1 + |lse|)"""
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

R = 2.0 ** -8 * (1 + 2.0 ** -6)


def db():
    from paper_2609_28568_amd import decode_binding
    return decode_binding


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def f64(t):
    return t.double().cpu().numpy()


# ---- books of the pages

class Model:
    """A cache of lists: every sequence's tokens, and its pages."""

    def __init__(self, n_pages, n_seq, max_pages, ps):
        self.ps, self.max_pages, self.n_pages = ps, max_pages, n_pages
        self.pages = [[] for _ in range(n_seq)]
        self.tokens = [[] for _ in range(n_seq)]

    def refs(self):
        r = [0] * self.n_pages
        for q in self.pages:
            for p in q:
                r[p] += 1
        return r

    def fork(self, src, keep=None):
        n = len(self.pages)
        old = [(list(t), list(p)) for t, p in zip(self.tokens, self.pages)]
        for s in range(n):
            t, p = old[src[s]] if 0 <= src[s] < n else ([], [])
            m = len(t) if keep is None else min(len(t), max(keep[s], 0))
            self.tokens[s], self.pages[s] = t[:m], p[:-(-m // self.ps)]

    def append(self, new):
        """new[s]: the tokens of sequence s. Pages missing: nothing changes."""
        refs, need, over = self.refs(), [], 0
        free = [p for p, r in enumerate(refs) if r == 0]
        for s, t in enumerate(new):
            m = len(self.tokens[s])
            copy = bool(t) and m % self.ps != 0 and refs[self.pages[s][m // self.ps]] > 1
            pages = -(-(m + len(t)) // self.ps)
            over += max(0, pages - self.max_pages)
            need.append((copy, pages - len(self.pages[s])))
        total = sum(c + n for c, n in need)
        missing = max(0, total - len(free)) + over
        if missing:
            return missing
        for s, (copy, n) in enumerate(need):
            if copy:
                self.pages[s][-1] = free.pop(0)
            self.pages[s] += [free.pop(0) for _ in range(n)]
            self.tokens[s] += new[s]
        return 0

    def compact(self):
        refs = self.refs()
        used = sum(r > 0 for r in refs)
        holes = [p for p in range(used) if not refs[p]]
        to = {p: holes.pop(0) for p in range(used, self.n_pages) if refs[p]}
        self.pages = [[to.get(p, p) for p in q] for q in self.pages]

    def table(self):
        return [p + [-1] * (self.max_pages - len(p)) for p in self.pages]


def agree(c, m, value):
    assert c.table.tolist() == m.table()
    assert c.lens.tolist() == [len(t) for t in m.tokens]
    assert c.refs.tolist() == m.refs()
    # every token's key and value, in every layer
    pages = c.pages.cpu()
    for t, p in zip(m.tokens, m.pages):
        if not t:
            continue
        got = pages[:, p].permute(0, 2, 3, 1, 4, 5).flatten(3, 4)[:, :, :, :len(t)]   # [L, 2, Hkv, tokens, hd]
        want = torch.stack([value[x] for x in t], 0)                                 # [tokens, L, 2, Hkv, hd]
        assert torch.equal(got.permute(3, 0, 1, 2, 4), want)


@pytest.mark.parametrize("layers,H,Hkv,hd,ps,n_seq,n_pages,seed", [
    (1, 1, 1, 64, 16, 1, 4, 0), (3, 4, 2, 128, 16, 5, 40, 1), (2, 6, 2, 64, 32, 9, 25, 2), (1, 3, 3, 64, 64, 4, 1300, 3),
    (2, 2, 1, 128, 128, 3, 12, 4), (1, 8, 8, 128, 256, 2, 9, 5), (2, 12, 12, 64, 16, 70, 2500, 6)])
def test_books_against_lists(layers, H, Hkv, hd, ps, n_seq, n_pages, seed):
    """Forks, truncations, frees, appends (some of them short of pages) and
    compactions in any order."""
    rng = random.Random(seed)
    max_pages = max(2, min(12, n_pages // 2 + 1))
    c = db().PagedCache.empty(layers, n_pages, Hkv, ps, hd, n_seq, max_pages)
    m = Model(n_pages, n_seq, max_pages, ps)
    value, width = {}, (H + 2 * Hkv) * hd
    gen = torch.Generator().manual_seed(seed)
    for step in range(30):
        what = rng.choice(("append", "append", "append", "fork", "compact"))
        print(f"step {step}: {what}", flush=True)
        if what == "append":
            hi = rng.choice((1, 3, 3 * ps))
            given = [rng.choice((0, rng.randint(0, hi))) for _ in range(n_seq)]
            starts = [0]
            for g in given:
                starts.append(starts[-1] + g)
            lead = rng.randint(0, 3)   # rows before the first sequence's
            x = torch.randn(layers, lead + starts[-1] + 2, width, generator=gen).bfloat16()
            counts = path = None
            max_new = max(max(given), 1)
            taken = [list(range(g)) for g in given]
            if rng.random() < 0.5:
                counts = [rng.randint(0, g) for g in given]
                taken = [list(range(k)) for k in counts]
                if rng.random() < 0.6:
                    max_new = max(max(counts), 1) + rng.randint(0, 2)
                    taken = [sorted(rng.sample(range(g), k)) for g, k in zip(given, counts)]
                    path = [t + [-1] * (max_new - len(t)) for t in taken]
            new = []
            for s, t in enumerate(taken):
                names = [(step, s, i) for i in t]
                for i, name in zip(t, names):
                    row = x[:, lead + starts[s] + i].view(layers, H + 2 * Hkv, hd)[:, H:]
                    value[name] = row.reshape(layers, 2, Hkv, hd)
                new.append(names)
            missing = m.append(new)
            c.append(x.cuda(), ints([lead + a for a in starts]), max_new,
                     counts=None if counts is None else ints(counts), path=None if path is None else ints(path))
            assert c.short.tolist() == [missing]
        elif what == "fork":
            src = [rng.choice((s, s, -1, rng.randint(0, n_seq - 1), n_seq, -7)) for s in range(n_seq)]
            keep = None if rng.random() < 0.4 else [rng.choice((10 ** 9, rng.randint(-2, 3 * ps), 0, ps)) for _ in src]
            m.fork(src, keep)
            c.fork(ints(src), None if keep is None else ints(keep))
        else:
            m.compact()
            c.compact()
        agree(c, m, value)


def test_append_without_pages_changes_nothing():
    c = db().PagedCache.empty(1, 3, 1, 16, 64, 2, 3)
    x = torch.randn(1, 64, 3 * 64, device="cuda").bfloat16()
    c.append(x, ints([0, 17, 33]), 32)
    before = [t.clone() for t in (c.pages, c.table, c.lens, c.refs)]
    c.append(x, ints([0, 16, 32]), 32)   # 1 + 1 pages, none free
    assert c.short.item() == 2
    for a, b in zip(before, (c.pages, c.table, c.lens, c.refs)):
        assert torch.equal(a.view(torch.int16) if a.dtype == torch.bfloat16 else a,
                           b.view(torch.int16) if b.dtype == torch.bfloat16 else b)
    c.fork(ints([0, -1]))
    c.append(x, ints([0, 40, 40]), 40)   # past the table's three pages, by one
    assert c.short.item() == 2           # (and one more than the pool has)
    c.append(x, ints([0, 31, 31]), 40)
    assert c.short.item() == 0 and c.lens.tolist() == [48, 0]


# ---- attention

CASES = {
    # H, Hkv, hd, page, lengths in the cache, new tokens, tree, max_new
    "one_token": (2, 1, 128, 16, [1], [1], False, 1),
    "nothing_cached": (4, 2, 64, 16, [0], [1], False, 1),
    "single_tokens": (4, 2, 128, 16, [60, 1, 0, 17, 64, 33], [1] * 6, False, 1),
    "single_tokens_hd64": (6, 2, 64, 32, [100, 5, 64, 65, 128], [1] * 5, False, 1),
    "some_without_rows": (4, 2, 128, 32, [50, 70, 0, 9], [0, 3, 0, 1], False, 5),
    "drafts": (4, 2, 128, 16, [200, 31, 0, 129], [7, 16, 1, 12], True, 16),
    "drafts_wide": (8, 1, 128, 64, [300, 64, 1], [24, 60, 33], True, 64),
    "drafts_hd64": (9, 3, 64, 128, [500, 0], [10, 5], True, 10),
    "drafts_hd64_wide": (12, 12, 64, 16, [77, 400], [64, 50], True, 64),
    "drafts_past_64": (2, 2, 64, 32, [40, 90], [200, 130], True, 200),
    "chain": (4, 2, 128, 64, [150, 0, 33], [90, 129, 64], False, 129),
    "chain_hd64": (6, 2, 64, 16, [63, 1000], [200, 1], False, 200),
    "long_single": (2, 1, 128, 16, [9000], [1], False, 1),
    "long_single_hd64": (3, 3, 64, 64, [7001, 12], [1, 1], False, 1),
    "long_drafts": (4, 1, 128, 32, [6000, 5, 900], [8, 3, 5], True, 8),
    "long_wide": (16, 2, 128, 128, [5000, 100], [40, 7], True, 40),
    "many": (4, 2, 128, 16, [(37 * i) % 211 for i in range(200)], [i % 3 for i in range(200)], False, 2),
    "many_wide": (8, 2, 64, 16, [(91 * i) % 301 for i in range(70)], [1 + i % 40 for i in range(70)], True, 40),
    "more_than_4096_rows": (2, 1, 64, 256, [600], [3000], False, 3000),
}


def build(name, seed=3, poison=False):
    """A cache with pages in no order, rows, starts, mask and what each row sees."""
    H, Hkv, hd, ps, lens, new, tree, max_new = CASES[name]
    rng, g = random.Random(seed), np.random.default_rng(seed)
    held = [-(-n // ps) for n in lens]
    n_pages, width = sum(held) + 3, max(held + [1]) + 1
    order = rng.sample(range(n_pages), sum(held))
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += h
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pages = torch.randn(2, n_pages, 2, Hkv, ps, hd, generator=gen, device="cuda").bfloat16()
    refs = np.bincount(order, minlength=n_pages).astype(np.int32)
    if poison:   # everything that belongs to no token
        there = torch.zeros(n_pages, ps, dtype=torch.bool)
        for s, n in enumerate(lens):
            for p in range(held[s]):
                there[table[s, p], :n - p * ps] = True
        pages[:, :, :, :, :, :] = torch.where(there.cuda()[None, :, None, None, :, None], pages, float("nan"))
    c = db().PagedCache(pages, torch.from_numpy(table).cuda(), ints(lens), torch.from_numpy(refs).cuda(), ints([0]))
    lead = 2   # rows before the first sequence's, and two behind the last one's
    starts = [lead]
    for k in new:
        starts.append(starts[-1] + k)
    x = torch.randn(starts[-1] + 2, (H + 2 * Hkv) * hd, generator=gen, device="cuda")
    x[:, :(H + Hkv) * hd] *= 1.4
    parents = [[int(g.integers(-1, i)) if i else -1 for i in range(k)] for k in new]
    mask = None
    if tree:
        m = db().tree_mask(parents)
        mask = torch.full((x.shape[0], m.shape[1]), -1, dtype=torch.int32, device="cuda")
        mask[lead:lead + m.shape[0]] = m
        sees = []
        for p in parents:
            a = np.zeros((len(p), len(p)), bool)
            for i, up in enumerate(p):
                a[i] = a[up] if up >= 0 else False
                a[i, i] = True
            sees.append(a)
    else:
        sees = [np.tri(k, dtype=bool) for k in new]
    return c, x.bfloat16(), starts, mask, sees


def reference(c, x, starts, lens, sees, H, Hkv, hd, layer):
    """[(out, lse, bound)] of every sequence, in float64."""
    pages, table, rows = f64(c.pages[layer]), c.table.cpu().numpy(), f64(x)
    ps, res = pages.shape[3], []
    for s, n in enumerate(lens):
        y = rows[starts[s]:starts[s + 1]].reshape(-1, H + 2 * Hkv, hd)
        kv = pages[table[s, :-(-n // ps)]].transpose(1, 2, 0, 3, 4).reshape(2, Hkv, -1, hd)[:, :, :n]
        m = np.concatenate([np.ones((len(y), n), bool), sees[s]], 1)
        out, lse, bound = np.zeros((len(y), H, hd)), np.zeros((H, len(y))), np.zeros((len(y), H, hd))
        for h in range(H):
            j = h // (H // Hkv)
            k, v = np.concatenate([kv[0, j], y[:, H + j]]), np.concatenate([kv[1, j], y[:, H + Hkv + j]])
            if not len(y):
                continue
            sc = np.where(m, y[:, h] @ np.where(np.isfinite(k), k, 0).T / np.sqrt(hd), -np.inf)
            top = sc.max(1, keepdims=True)
            e = np.where(m, np.exp(sc - np.where(np.isfinite(top), top, 0)), 0)
            total = e.sum(1, keepdims=True)
            p = e / np.where(total > 0, total, 1)
            v = np.where(np.isfinite(v), v, 0)
            with np.errstate(divide="ignore"):
                lse[h] = (top + np.log(total))[:, 0]
            out[:, h] = p @ v
            bound[:, h] = R * (np.abs(out[:, h]) + p @ np.abs(v)) + 2.0 ** -15 * (p @ np.abs(v))
        res.append((out.reshape(len(y), H * hd), lse, bound.reshape(len(y), H * hd)))
    return res


def check(y, lse, starts, ref, rows=slice(None)):
    y, lse = f64(y), f64(lse)
    for s, (out, l, bound) in enumerate(ref):
        a = slice(starts[s], starts[s + 1])
        assert np.all(np.abs(y[a] - out) <= bound), s
        with np.errstate(invalid="ignore"):
            assert np.all((lse[:, a] == l) | (np.abs(lse[:, a] - l) <= 2.0 ** -18 * (1 + np.abs(l)))), s


@pytest.mark.parametrize("name", list(CASES))
def test_attention_against_the_definition(name):
    print(f"{name}: {CASES[name]}", flush=True)
    H, Hkv, hd, ps, lens, new, tree, max_new = CASES[name]
    c, x, starts, mask, sees = build(name, poison=True)
    for layer in (0, 1):
        y, lse = c.attention(x, ints(starts), max_new, mask=mask, layer=layer)
        torch.cuda.synchronize()
        ref = reference(c, x, starts, lens, sees, H, Hkv, hd, layer)
        check(y, lse, starts, ref)
    # the same bits again, into buffers of the caller's, whose other rows stay
    y2, lse2 = torch.full_like(y, 7), torch.full_like(lse, 7)
    c.attention(x, ints(starts), max_new, mask=mask, layer=1, out=y2, lse=lse2)
    used = slice(starts[0], starts[-1])
    assert torch.equal(y[used], y2[used]) and torch.equal(lse[:, used], lse2[:, used])
    for t in (y2[:starts[0]], y2[starts[-1]:], lse2[:, :starts[0]], lse2[:, starts[-1]:]):
        assert bool((t == 7).all())


def test_pages_that_the_table_does_not_name_are_not_seen():
    """Entries out of range, in the middle and at the end: the tokens there are
    left out, and the others' weights are those of a softmax without them."""
    H, Hkv, hd, ps, lens, new, tree, max_new = CASES["single_tokens"]
    c, x, starts, mask, sees = build("single_tokens")
    for s, i, page in ((0, 1, -1), (4, 0, c.pages.shape[1]), (4, 3, 2 ** 31 - 1), (5, 2, -2 ** 31), (1, 0, -5)):
        c.table[s, i] = page
    y, lse = c.attention(x, ints(starts), max_new, layer=1)
    torch.cuda.synchronize()
    table, pages = c.table.cpu().numpy(), c.pages
    for s, n in enumerate(lens):
        there = np.array([0 <= table[s, t // ps] < pages.shape[1] for t in range(n)], bool)
        good = np.where((table[s] >= 0) & (table[s] < pages.shape[1]), table[s], 0)
        k = torch.from_numpy(good[:-(-n // ps)]).long()
        kv = f64(pages[1][k.cuda()]).transpose(1, 2, 0, 3, 4).reshape(2, Hkv, -1, hd)[:, :, :n][:, :, there]
        row = f64(x[starts[s]]).reshape(H + 2 * Hkv, hd)
        for h in range(H):
            j = h // (H // Hkv)
            keys, values = np.vstack([kv[0, j], row[H + j]]), np.vstack([kv[1, j], row[H + Hkv + j]])
            e = keys @ row[h] / np.sqrt(hd)
            p = np.exp(e - e.max())
            want, size = (p @ values) / p.sum(), (p @ np.abs(values)) / p.sum()
            got = f64(y[starts[s]]).reshape(H, hd)[h]
            assert np.all(np.abs(got - want) <= R * (np.abs(want) + size) + 2.0 ** -15 * size), (s, h)
            assert abs(float(lse[h, starts[s]]) - (e.max() + np.log(p.sum()))) < 1e-4


@pytest.mark.parametrize("name", ["drafts", "drafts_wide", "drafts_hd64", "drafts_hd64_wide", "drafts_past_64", "chain"])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_what_a_token_does_not_see_does_not_reach_it(name, what):
    """One drafted token of each sequence holds NaN or infinity everywhere: the
    rows that do not see it stay what they were but for the rounding of their
    probabilities, those that do are not finite."""
    H, Hkv, hd, ps, lens, new, tree, max_new = CASES[name]
    c, x, starts, mask, sees = build(name)
    y, lse = c.attention(x, ints(starts), max_new, mask=mask)
    bad = x.clone()
    touched = torch.zeros(x.shape[0], dtype=torch.bool, device="cuda")
    for s, k in enumerate(new):
        at = (3 * s + 1) % k
        bad[starts[s] + at] = what
        touched[starts[s]:starts[s + 1]] = torch.from_numpy(sees[s][:, at]).cuda()
    z, zl = c.attention(bad, ints(starts), max_new, mask=mask)
    keep = ~touched
    keep[:starts[0]] = False
    keep[starts[-1]:] = False
    assert int(keep.sum()) > 0 and int(touched.sum()) > 0
    # a tile that holds it goes token by token, with probabilities that are not rounded: 2^-8 of them
    size = (y[keep].float().abs() + x[:, -Hkv * hd:].float().abs().max() * 2.0 ** -8) * 2.0 ** -7
    assert bool(((z[keep].float() - y[keep].float()).abs() <= size + 2.0 ** -6).all())
    assert bool((zl[:, keep] - lse[:, keep]).abs().max() < 1e-5)
    assert bool(torch.isnan(z[touched].float()).any(1).all())


def test_rows_past_max_new_are_left():
    c, x, starts, mask, sees = build("chain")
    y, lse = c.attention(x, ints(starts), 129)
    z, zl = torch.full_like(y, 7), torch.full_like(lse, 7)
    c.attention(x, ints(starts), 70, out=z, lse=zl)
    for s in range(3):
        a, n = starts[s], min(70, starts[s + 1] - starts[s])
        assert bool(((z[a:a + n].float() - y[a:a + n].float()).abs() < 2.0 ** -5).all())
        assert bool((z[a + n:starts[s + 1]] == 7).all()) and bool((zl[:, a + n:starts[s + 1]] == 7).all())


def test_rows_that_see_nothing():
    """No cached tokens and masks without a bit: 0, and -infinity."""
    c = db().PagedCache.empty(1, 4, 2, 16, 64, 3, 2)
    x = torch.randn(6, 8 * 64, device="cuda").bfloat16()
    mask = torch.zeros(6, 1, dtype=torch.int32, device="cuda")
    mask[1] = 2
    y, lse = c.attention(x, ints([0, 2, 2, 6]), 4, mask=mask)
    keep = torch.tensor([0, 2, 3, 4, 5], device="cuda")
    assert bool((y[keep] == 0).all()) and bool((lse[:, keep] == -float("inf")).all())
    assert torch.equal(y[1].view(2, 2, 64), x[1, 6 * 64:].view(2, 1, 64).expand(2, 2, 64))   # one key: its value


def test_two_calls_at_once_and_a_captured_one():
    """On two streams over one cache, and captured with lengths that change
    between the replays."""
    c, x, starts, mask, sees = build("long_drafts")
    st, n = ints(starts), CASES["long_drafts"][7]
    want = c.attention(x, st, n, mask=mask)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for k in range(6):
        with torch.cuda.stream(streams[k % 2]):
            got.append(c.attention(x, st, n, mask=mask))
    torch.cuda.synchronize()
    used = slice(starts[0], starts[-1])
    for y, lse in got:
        assert torch.equal(y[used], want[0][used]) and torch.equal(lse[:, used], want[1][:, used])
    out = tuple(torch.zeros_like(t) for t in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attention(x, st, n, mask=mask, out=out[0], lse=out[1])
    full = c.lens.clone()
    for cut in (0, 1, 700, 5000, 3):
        c.lens.copy_((full - cut).clamp(min=0))
        graph.replay()
        y, lse = c.attention(x, st, n, mask=mask)
        torch.cuda.synchronize()
        assert torch.equal(y[used], out[0][used]) and torch.equal(lse[:, used], out[1][:, used]), cut


def test_pages_past_4_gib():
    """A sequence's pages at both ends of 9 GiB of them: appended, read, copied on
    a fork, moved together; the same bits as in a small cache."""
    layers, Hkv, hd, ps, n_pages = 2, 4, 128, 64, 36864
    pages = torch.empty(layers, n_pages, 2, Hkv, ps, hd, dtype=torch.bfloat16, device="cuda")
    assert pages[0].numel() * 2 > 1 << 32
    refs = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    free = [0, 1, 20000, 36000, 36001, 36002, 36860, 36861, 36862, 36863]
    refs[free] = 0   # the others belong to a sequence that is not looked at
    one = lambda v: torch.full((1,), v, dtype=torch.int32, device="cuda")   # noqa: E731
    big = db().PagedCache(pages, torch.full((3, n_pages), -1, dtype=torch.int32, device="cuda"), ints([0, 0, 0]), refs, one(0))
    small = db().PagedCache.empty(layers, 12, Hkv, ps, hd, 3, 12)
    x = torch.randn(layers, 300, (8 + 2 * Hkv) * hd, device="cuda").bfloat16()
    q = torch.randn(3, (8 + 2 * Hkv) * hd, device="cuda").bfloat16()
    for c in (big, small):
        c.append(x, ints([0, 290, 290, 290]), 290)      # 5 pages
        c.fork(ints([0, 0, -1]))
        c.append(x, ints([290, 295, 300, 300]), 10)     # two copies of the last page
        assert c.short.item() == 0
    assert big.table[0, :5].tolist() == free[:4] + [free[5]] and big.table[1, 4].item() == free[6]
    for layer in range(layers):
        a, b = (c.attention(q, ints([0, 1, 2, 3]), 1, layer=layer) for c in (big, small))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # only the sequences that are looked at are left, and move to the front
    held = torch.zeros_like(refs)
    held.index_add_(0, big.table[:2, :5].flatten().long(), torch.ones(10, dtype=torch.int32, device="cuda"))
    big.refs.copy_(held)
    big.compact()
    assert big.table[:2, :5].max().item() == 5 and int((big.refs > 0).sum()) == 6
    for layer in range(layers):
        a, b = (c.attention(q, ints([0, 1, 2, 3]), 1, layer=layer) for c in (big, small))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_the_largest_number_of_sequences():
    """4,096 sequences forked from one, a token each stored and read."""
    n = 4096
    c = db().PagedCache.empty(1, n + 4, 1, 16, 64, n, 2)
    x = torch.randn(1, 21, 3 * 64, device="cuda").bfloat16()
    c.append(x, ints([0] + [21] * n), 21)
    c.fork(ints([0] * n))
    assert c.refs[:2].tolist() == [n, n]
    q = torch.randn(1, n, 3 * 64, device="cuda").bfloat16()
    st = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    y, lse = c.attention(q[0], st, 1)
    c.append(q, st, 1)
    assert c.short.item() == 0 and c.lens.tolist() == [22] * n and c.refs[:2].tolist() == [n, 0]
    assert sorted(c.table[:, 1].tolist()) == list(range(2, n + 2)) and c.table[5, 1].item() == 7
    # a sequence's new token is seen from the cache as it was from its row
    e = torch.zeros(n, 3 * 64, device="cuda").bfloat16()
    e[:, :64] = q[0, :, :64]
    mask = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    z, zl = c.attention(e, st, 1, mask=mask)
    # the same probabilities, rounded to bf16 in another tile, and the result rounded
    assert bool(((z.float() - y.float()).abs() <= 2.0 ** -6 * (1 + y.float().abs())).all())
    assert float((zl - lse).abs().max()) < 1e-5


def test_masks_without_words_are_refused():
    c = db().PagedCache.empty(1, 4, 1, 16, 64, 2, 4)
    x, starts = torch.zeros(4, 4 * 64, dtype=torch.bfloat16, device="cuda"), ints([0, 2, 4])
    for call in (lambda mask: c.attention(x, starts, 2, mask), lambda mask: c.positions(starts, 4, mask)):
        for mask in (torch.zeros(4, 0, dtype=torch.int32, device="cuda"), ints([0] * 4)):
            with pytest.raises(ValueError, match="word"):
                call(mask)


@pytest.mark.parametrize("H,Hkv,hd,new,lens", [
    (8, 8, 128, 1, [37 * s % 391 for s in range(40)]),      # 320 segments: every wave a worker, shares cut
    (8, 4, 64, 40, [61 * s % 1500 for s in range(70)]),     # planned, two blocks of rows to a workgroup
    (4, 4, 64, 5, [300, 0, 1, 17, 333, 64])])               # segments that are dealt and some that are whole
def test_divisions_of_ragged_lengths(H, Hkv, hd, new, lens):
    """Shares that end anywhere in a segment, segments of nothing, one part and several."""
    torch.manual_seed(9)
    n = len(lens)
    held = [-(-x // 16) for x in lens]
    pages = torch.randn(1, sum(held) + 1, 2, Hkv, 16, hd, device="cuda").bfloat16()
    table = torch.full((n, max(held)), -1, dtype=torch.int32)
    order, at = torch.randperm(sum(held)).int(), 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += h
    refs = torch.ones(sum(held) + 1, dtype=torch.int32)
    refs[-1] = 0
    c = db().PagedCache(pages, table.cuda(), ints(lens), refs.cuda(), ints([0]))
    news = [(7 * s) % (new + 1) for s in range(n)] if new > 1 else [1] * n
    starts = [sum(news[:s]) for s in range(n + 1)]
    x = torch.randn(starts[-1], (H + 2 * Hkv) * hd, device="cuda").bfloat16()
    y, lse = c.attention(x, ints(starts), max(news))
    again, _ = c.attention(x, ints(starts), max(news))
    assert torch.equal(y, again)
    sees = [np.tri(k, dtype=bool) for k in news]
    check(y, lse, starts, reference(c, x, starts, lens, sees, H, Hkv, hd, 0))


@pytest.mark.parametrize("n_rows", [2 ** 26 - 1, 2 ** 26 - 3])
def test_as_many_rows_as_a_call_takes(n_rows):
    """n_head * n_rows just below 2^26, where the workgroups that join parts have
    2^32 threads: one token of a sequence of many parts, in the last row."""
    torch.manual_seed(4)
    hd, n = 64, 600
    c = db().PagedCache.empty(1, 40, 1, 16, hd, 1, 40)
    x = torch.randn(1, n + 1, 3 * hd, device="cuda").bfloat16()
    c.append(x, ints([0, n]), n)
    qkv = torch.empty(n_rows, 3 * hd, dtype=torch.bfloat16, device="cuda")
    qkv[-1] = x[0, n]
    y, lse = c.attention(qkv, ints([n_rows - 1, n_rows]), 1)
    small = torch.empty(700, 3 * hd, dtype=torch.bfloat16, device="cuda")   # joined likewise, a wave a row
    small[-1] = x[0, n]
    z, zl = c.attention(small, ints([699, 700]), 1)
    assert torch.equal(y[-1], z[-1]) and torch.equal(lse[:, -1], zl[:, -1])
    check(y[-1:], lse[:, -1:], [0, 1], reference(c, x[0, n:], [0, 1], [n], [np.ones((1, 1), bool)], 1, 1, hd, 0))


@pytest.mark.parametrize("n_seq,piece,at", [(64, 2048, 63), (200, 3001, 137), (4096, 8192, 2500)])
def test_one_long_piece_appended_among_single_tokens(n_seq, piece, at):
    """Every third sequence gets nothing, one a piece, the others a token; rows
    before the first sequence's and behind the last one's are nobody's."""
    layers, H, Hkv, hd, ps = 2, 2, 1, 64, 16
    pages = -(-piece // ps) + 1
    c = db().PagedCache.empty(layers, pages + n_seq, Hkv, ps, hd, n_seq, pages)
    m = Model(pages + n_seq, n_seq, pages, ps)
    new = [0 if s % 3 == 2 else 1 for s in range(n_seq)]
    new[at] = piece
    lead = 5
    starts = (lead + np.concatenate([[0], np.cumsum(new)])).tolist()
    x = torch.randn(layers, starts[-1] + 3, (H + 2 * Hkv) * hd, generator=torch.Generator().manual_seed(8)).bfloat16()
    c.append(x.cuda(), ints(starts), piece)
    value = {(s, i): x[:, starts[s] + i].view(layers, H + 2 * Hkv, hd)[:, H:].reshape(layers, 2, Hkv, hd)
             for s, k in enumerate(new) for i in range(k)}
    assert m.append([[(s, i) for i in range(k)] for s, k in enumerate(new)]) == 0 == c.short.item()
    agree(c, m, value)


def pick(c, x, starts, lens, sees, some, heads):
    """reference() of some sequences: (their rows of an output, starts, the reference) of it."""
    from types import SimpleNamespace
    rows = torch.cat([torch.arange(starts[s], starts[s + 1]) for s in some]).cuda()
    at = np.concatenate([[0], np.cumsum([starts[s + 1] - starts[s] for s in some])]).tolist()
    part = SimpleNamespace(pages=c.pages, table=c.table[torch.tensor(some, device="cuda")])
    return rows, at, reference(part, x[rows], at, [lens[s] for s in some], [sees[s] for s in some], *heads, 0)


def test_one_long_piece_among_the_most_sequences():
    """4,096 sequences in a table for 131,072 tokens each, one with a piece of a
    prompt of 4,096, the others with a token or none: the same bits as in a table
    that is hardly wider than what they have, and what the definition says."""
    n, H, Hkv, hd, ps, at, piece = 4096, 16, 8, 128, 16, 1717, 4096
    torch.manual_seed(12)
    lens = [37 * s % 90 for s in range(n)]
    lens[at] = 777
    held = [-(-k // ps) for k in lens]
    pages = torch.randn(1, sum(held), 2, Hkv, ps, hd, device="cuda").bfloat16()
    new = [0 if s % 5 == 4 else 1 for s in range(n)]
    new[at] = piece
    starts = np.concatenate([[0], np.cumsum(new)]).tolist()
    order, x = torch.randperm(sum(held)).int(), torch.randn(starts[-1], (H + 2 * Hkv) * hd, device="cuda").bfloat16()
    got = []
    for width in (max(held) + 1, 8192):
        table, k = torch.full((n, width), -1, dtype=torch.int32), 0
        for s, h in enumerate(held):
            table[s, :h] = order[k:k + h]
            k += h
        refs = torch.ones(sum(held), dtype=torch.int32, device="cuda")
        c = db().PagedCache(pages, table.cuda(), ints(lens), refs, ints([0]))
        got.append(c.attention(x, ints(starts), piece))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    y, lse = got[1]
    some = list(range(0, n, 41)) + [at - 1, at, at + 1]
    sees = [None] * n
    for s in some:
        sees[s] = np.tri(new[s], dtype=bool)
    rows, k, ref = pick(c, x, starts, lens, sees, some, (H, Hkv, hd))
    check(y[rows], lse[:, rows], k, ref)


@pytest.mark.parametrize("n_seq", [4, 70])
def test_starts_that_fall_compute_nothing(n_seq):
    c = db().PagedCache.empty(1, 8, 1, 16, 64, n_seq, 64)
    c.lens[1] = 1000   # of no pages: tokens that nobody sees
    x = torch.randn(40, 3 * 64, device="cuda").bfloat16()
    out, lse = torch.full((40, 64), 7, dtype=torch.bfloat16, device="cuda"), torch.full((1, 40), 7.0, device="cuda")
    c.attention(x, ints([0, 20, 10] + [40] * (n_seq - 2)), 40, out=out, lse=lse)
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and bool((lse == 7).all())


def test_a_cache_let_go_while_another_stream_works_on_it():
    """Its memory is not another tensor's before that stream is done."""
    n, H, hd = 600, 2, 64
    x = torch.randn(1, n + 1, (H + 2) * hd, device="cuda").bfloat16()
    st, one = ints([0, n]), ints([0, 1])

    def use(sleep):
        c = db().PagedCache.empty(1, 40, 1, 16, hd, 1, 40)
        torch.cuda.current_stream().synchronize()
        with torch.cuda.stream(side):
            if sleep:
                torch.cuda._sleep(50_000_000)
            c.append(x, st, n)
            y = c.attention(x[0, n:], one, 1)
            p = c.positions(one, 1)
        shapes = [t.shape for t in (c.pages, c.table, c.lens, c.refs, c.short, c.scratch)]
        return y, p, shapes

    side = torch.cuda.Stream()
    (want, lse), place, _ = use(False)
    torch.cuda.synchronize()
    (y, l), p, shapes = use(True)
    # of the same sizes, on the stream that the cache was made on
    junk = [torch.full(s, 3, dtype=d, device="cuda") for s, d in
            zip(shapes, [torch.bfloat16] + [torch.int32] * 4 + [torch.uint8]) for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(l, lse) and torch.equal(p, place) and p.tolist() == [[n]]
    assert all(bool((t == 3).all()) for t in junk)


# ---- which kernel a call takes, and how it divides its work

def walk(H, Hkv, hd, lens, new, max_new):
    """(head size, blocks of 32 rows of a workgroup, division, planned): the rules of
    tree.hip's with_walk and cuts_of, so that the cases below reach what they are for."""
    G = H // Hkv
    rb = 1 if max_new * G <= 32 else 2 if max_new * G <= 64 else 4
    kt, groups, teams = 32 if hd == 128 and rb < 4 else 64, 4 // rb, 256 if rb == 1 else 512
    whole = max(2 * groups, 4)
    up = lambda a, b: -(-a // b)   # noqa: E731
    seqs = [(up(n, kt) + up(k, kt), up(k * G, 32 * rb) * Hkv) for n, k in zip(lens, new) if k]   # tiles, segments
    total, segments = sum(t * s for t, s in seqs), sum(s for _, s in seqs)
    even = max(whole // 2, up(total, teams))
    pieces = lambda share: sum((1 if t <= whole else up(t, share)) * s for t, s in seqs)   # noqa: E731
    dealt = segments <= teams and (max(t for t, _ in seqs) <= whole or pieces(even + (even * 14 + 31) // 32) <= teams)
    return hd, rb, "dealt" if dealt else "solo" if rb == 1 and segments > teams else "line", len(lens) > 64


def ragged(n, lo, hi, step):
    return [lo + (step * i) % (hi - lo + 1) for i in range(n)]


DIVIDED = {
    # as CASES, with the walk
    "dealt_128_2": ((4, 2, 128, 16, [3001, 0, 1700, 333, 64, 2222], [20, 32, 17, 31, 1, 29], True, 32), "dealt"),
    "dealt_128_2_chain": ((6, 2, 128, 64, [2500, 31, 900], [13, 21, 20], False, 21), "dealt"),
    "dealt_128_2_planned": ((2, 1, 128, 16, ragged(80, 0, 900, 311), ragged(80, 17, 32, 5), True, 32), "dealt"),
    "dealt_64_2": ((4, 2, 64, 32, [4000, 1, 1234, 777], [18, 32, 25, 3], True, 32), "dealt"),
    "dealt_64_2_planned": ((3, 1, 64, 16, ragged(70, 5, 1500, 407), ragged(70, 11, 21, 4), False, 21), "dealt"),
    "dealt_128_4": ((4, 2, 128, 32, [1800, 77, 640], [130, 40, 65], True, 130), "dealt"),
    "dealt_128_1_planned": ((4, 1, 128, 16, ragged(90, 0, 1200, 173), [1] * 90, False, 1), "dealt"),
    "line_128_1": ((6, 3, 128, 16, ragged(48, 950, 1150, 37), [1 + i % 4 for i in range(48)], False, 4), "line"),
    "line_64_1": ((6, 3, 64, 32, ragged(48, 1900, 2300, 71), [1 + i % 3 for i in range(48)], True, 3), "line"),
    "line_128_1_planned": ((4, 2, 128, 64, ragged(73, 950, 1150, 53), [1] * 73, False, 1), "line"),
    "line_64_1_planned": ((4, 2, 64, 16, ragged(73, 1900, 2300, 91), [2] * 73, True, 2), "line"),
    "line_128_2": ((18, 9, 128, 16, ragged(60, 0, 700, 263), ragged(60, 12, 32, 7), True, 32), "line"),
    "line_128_2_planned": ((8, 4, 128, 32, ragged(140, 0, 500, 119), ragged(140, 1, 24, 5), False, 24), "line"),
    "line_64_2": ((18, 9, 64, 64, ragged(60, 0, 1300, 571), ragged(60, 12, 32, 7), False, 32), "line"),
    "line_64_2_planned": ((8, 4, 64, 16, ragged(140, 0, 900, 313), ragged(140, 1, 24, 5), True, 24), "line"),
    "line_128_4": ((18, 9, 128, 128, ragged(60, 0, 900, 389), ragged(60, 20, 90, 17), True, 90), "line"),
    "line_128_4_planned": ((8, 4, 128, 16, ragged(140, 0, 600, 257), ragged(140, 1, 45, 8), False, 45), "line"),
    "line_64_4": ((18, 9, 64, 16, ragged(60, 0, 1100, 463), ragged(60, 20, 90, 17), False, 90), "line"),
    "line_64_4_planned": ((8, 4, 64, 32, ragged(140, 0, 800, 337), ragged(140, 1, 45, 8), True, 45), "line"),
    "solo_128_1_planned": ((8, 4, 128, 16, ragged(120, 0, 700, 97), [i % 3 for i in range(120)], False, 2), "solo"),
    "solo_64_1": ((20, 10, 64, 64, ragged(50, 0, 1500, 283), [1 + i % 5 for i in range(50)], True, 5), "solo"),
    # a piece of a prompt among single tokens
    "mixed": ((4, 2, 128, 16, ragged(64, 200, 2048, 709), [1] * 40 + [700] + [1] * 23, False, 700), "dealt"),
    "mixed_planned": ((4, 4, 64, 32, ragged(90, 200, 1500, 709), [1] * 70 + [333] + [1] * 19, False, 333), "line"),
}


def test_walks_and_divisions_are_all_reached():
    got = {k: walk(*c[:3], c[4], c[5], c[7]) for k, c in CASES.items()}
    for k, (c, division) in DIVIDED.items():
        got[k] = walk(*c[:3], c[4], c[5], c[7])
        assert got[k][2] == division, (k, got[k])
    ways = {(rb, d) for rb in (1, 2, 4) for d in ("dealt", "line")} | {(1, "solo")}
    assert {(hd, rb, d) for hd, rb, d, _ in got.values()} == {(hd, rb, d) for hd in (64, 128) for rb, d in ways}
    assert {(rb, d) for _, rb, d, planned in got.values() if planned} == ways


@pytest.mark.parametrize("name", list(DIVIDED))
def test_every_walk_and_division(name, monkeypatch):
    monkeypatch.setitem(CASES, name, DIVIDED[name][0])
    test_attention_against_the_definition(name)


def test_a_step_of_the_books_captured():
    """Forking, appending and compacting captured once: every replay, with other
    arguments and eager calls on another cache in between, as the lists say."""
    rng, gen = random.Random(5), torch.Generator().manual_seed(5)
    layers, H, Hkv, hd, ps, n_seq, n_pages, max_pages, rows, width = 2, 2, 1, 64, 16, 6, 60, 9, 64, 7
    c, m = db().PagedCache.empty(layers, n_pages, Hkv, ps, hd, n_seq, max_pages), Model(n_pages, n_seq, max_pages, ps)
    other = db().PagedCache.empty(layers, n_pages, Hkv, ps, hd, n_seq, max_pages)
    x = torch.zeros(layers, rows, (H + 2 * Hkv) * hd, dtype=torch.bfloat16, device="cuda")
    src, keep, counts = (torch.zeros(n_seq, dtype=torch.int32, device="cuda") for _ in range(3))
    starts, path = torch.zeros(n_seq + 1, dtype=torch.int32, device="cuda"), ints([[-1] * width] * n_seq)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.fork(src, keep)
        c.append(x, starts, width, counts=counts, path=path)
        c.append(x, starts, 40)
        c.compact()
    value = {}
    for step in range(12):
        s, k = [rng.choice((i, i, 0, -1)) for i in range(n_seq)], [rng.choice((10 ** 6, 3, ps, 21)) for _ in range(n_seq)]
        given = [rng.choice((0, 1, rng.randint(0, 10))) for _ in range(n_seq)]
        if step % 4 == 1:
            given[rng.randrange(n_seq)] = 40
            given = [g if g in (40, 1) else 0 for g in given]
        st = np.concatenate([[0], np.cumsum(given)]).tolist()
        assert st[-1] <= rows
        new = torch.randn(layers, rows, x.shape[2], generator=gen).bfloat16()
        taken = [sorted(rng.sample(range(g), rng.randint(0, min(g, width)))) for g in given]
        for t, v in ((src, s), (keep, k), (starts, st), (counts, [len(t) for t in taken]),
                     (path, [t + [-1] * (width - len(t)) for t in taken])):
            t.copy_(ints(v))
        x.copy_(new)
        graph.replay()
        other.append(x, starts, 40)   # eager work in between, until the pages are too few
        torch.cuda.synchronize()
        name = lambda q, i: (step, q, i)   # noqa: E731
        for q, g in enumerate(given):
            for i in range(g):
                row = new[:, st[q] + i].view(layers, H + 2 * Hkv, hd)[:, H:]
                value[name(q, i)] = row.reshape(layers, 2, Hkv, hd)
        m.fork(s, k)
        m.append([[name(q, i) for i in t] for q, t in enumerate(taken)])
        assert m.append([[name(q, i) for i in range(g)] for q, g in enumerate(given)]) == c.short.item()
        m.compact()
        agree(c, m, value)


@pytest.mark.parametrize("name", ["drafts", "drafts_wide", "drafts_hd64", "drafts_hd64_wide", "drafts_past_64", "chain",
                                  "chain_hd64"])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_rows_beside_one_that_is_not_finite_keep_their_bounds(name, what):
    """Against the definition, of which a token that a row does not see is no part."""
    H, Hkv, hd, ps, lens, new, tree, max_new = CASES[name]
    c, x, starts, mask, sees = build(name, seed=5)
    for s, k in enumerate(new):
        x[starts[s] + (2 * s + k // 3) % k] = what
    y, lse = c.attention(x, ints(starts), max_new, mask=mask)
    ref = reference(c, torch.where(x.isfinite(), x, 0), starts, lens, sees, H, Hkv, hd, 0)
    n = 0
    for s, k in enumerate(new):
        rows = np.flatnonzero(~sees[s][:, (2 * s + k // 3) % k])
        n += len(rows)
        out, l, bound = ref[s]
        at = torch.from_numpy(starts[s] + rows).cuda()
        assert np.all(np.abs(f64(y[at]) - out[rows]) <= bound[rows]), s
        assert np.all(np.abs(f64(lse[:, at]) - l[:, rows]) <= 2.0 ** -18 * (1 + np.abs(l[:, rows]))), s
    assert n > 0
