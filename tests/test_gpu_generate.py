"""Answers generated over a paged cache with the adapter model, on the GPU: every
logit that a token was chosen from against the oracle's forward over the whole
sequence, through prompts stored in pieces, forks, trees of drafted tokens,
penalties, freed sequences and compaction; and a step captured into a graph.

Logits within the bar of the other activations (2e-2 relative L2 a row)."""
import numpy as np
import pytest

from oracle import qwen3 as q3
from paper_2609_28568_amd import synth
from tests.util import REL_L2, rel_l2

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

W = dict(synth.QWEN3_WORKLOADS["qwen3_tiny"], B=1, T=64, max_seq_len=64, loss_from=0.0)
PS, N_SEQ = 16, 5


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Answers:
    """A model, a cache of its keys and values, and what every sequence holds."""

    def __init__(self, seed=51, pages=60):
        from paper_2609_28568_amd import decode_binding as db, qwen3_binding as qb
        self.db = db
        self.base, self.lora = synth.init_qwen3(W, seed=seed, b_std=0.02, norm_jitter=0.1)
        self.m = qb.Qwen3(qb.make_config(W, synth.QWEN3_OPTIM))
        self.m.set_base(self.base)
        self.m.set_lora(self.lora)
        self.cache = db.PagedCache.empty(W["n_layer"], pages, W["n_kv_head"], PS, W["head_dim"], N_SEQ, 12)
        self.tokens = [[] for _ in range(N_SEQ)]
        self.logits = [[] for _ in range(N_SEQ)]   # behind each token

    def forward(self, new, mask=None):
        """The logits behind new[s]: the new tokens of sequence s."""
        starts = np.concatenate([[0], np.cumsum([len(n) for n in new])]).tolist()
        self.starts = ints(starts)
        ids = np.zeros((1, 64), np.int64)
        ids[0, :starts[-1]] = [t for n in new for t in n]
        if mask is not None:
            full = torch.zeros(64, mask.shape[1], dtype=torch.int32, device="cuda")
            full[:mask.shape[0]] = mask
            mask = full
        self.m.set_cache(self.cache, self.starts, max(map(len, new)), mask)
        self.m.forward(torch.from_numpy(ids))
        y = self.m.logits()
        assert y.shape == (64, W["vocab"])
        return [y[a:b].clone() for a, b in zip(starts, starts[1:])]

    def extend(self, new):
        for s, y in enumerate(self.forward(new)):
            self.tokens[s] += new[s]
            self.logits[s] += list(y.float().cpu().numpy())
        self.m.keep_tokens(max(map(len, new)))
        assert self.cache.short.item() == 0

    def check(self):
        """Everything against the oracle over whole sequences."""
        assert self.cache.lens.tolist() == [len(t) for t in self.tokens]
        for s, t in enumerate(self.tokens):
            if not t:
                continue
            cfg = q3.Qwen3Config.from_dict(dict(W, T=len(t), max_seq_len=len(t)))
            ids = np.array([t])
            want = q3.forward(self.base, self.lora, ids, ids, cfg)["logits"][0]
            for i, (a, b) in enumerate(zip(self.logits[s], want)):
                assert rel_l2(a, b) < REL_L2, (s, i, rel_l2(a, b))


def prompt(n, seed):
    return synth.zipf_ids(np.random.default_rng(seed), n, W["vocab"]).tolist()


def test_prompts_in_pieces_forks_drafts_and_compaction():
    a = Answers()
    a.extend([prompt(20, 1), prompt(37, 2), [], prompt(1, 3), []])
    a.extend([[], prompt(33, 4), [], prompt(15, 5), prompt(2, 6)])   # pieces behind what is there; a page filled
    a.check()
    # two answers of sequence 1, one of them a shorter prompt; sequence 3 ends
    a.cache.fork(ints([0, 1, 1, -1, 1]), ints([100, 100, 100, 100, 61]))
    for to, n in ((2, 70), (4, 61)):
        a.tokens[to], a.logits[to] = a.tokens[1][:n], a.logits[1][:n]
    a.tokens[3], a.logits[3] = [], []
    assert a.cache.refs.max().item() == 3
    a.check()
    # tokens chosen greedily, with repetitions made less likely
    for _ in range(4):
        rows = [s for s in range(N_SEQ) if a.tokens[s]]
        x = torch.from_numpy(np.stack([a.logits[s][-1] for s in rows])).cuda()
        longest = max(len(a.tokens[s]) for s in rows)
        history = ints([a.tokens[s] + [-1] * (longest - len(a.tokens[s])) for s in rows])
        n = len(rows)
        y = a.db.adjust_logits(x, history, ints([len(a.tokens[s]) // 2 for s in rows]),
                               ints([len(a.tokens[s]) for s in rows]), torch.full((n,), 1.3, device="cuda"),
                               torch.full((n,), 0.2, device="cuda"), torch.full((n,), 0.4, device="cuda"))
        seen = torch.zeros_like(x, dtype=torch.bool)
        for r, s in enumerate(rows):
            seen[r, a.tokens[s]] = True
        assert torch.equal(x[~seen], y[~seen]) and bool((y[seen] < x[seen]).all())
        new = [[] for _ in range(N_SEQ)]
        for s, t in zip(rows, y.argmax(1).tolist()):
            new[s] = [t]
        a.extend(new)
    a.check()
    a.cache.compact()
    used = int((a.cache.refs > 0).sum())
    assert bool((a.cache.refs[:used] > 0).all()) and a.cache.table.max().item() == used - 1
    a.extend([[7], [], [8], [], [9]])
    a.check()


def test_drafted_trees():
    """Every branch of a tree against the oracle over its own path; one path is
    kept, and what follows goes on from it."""
    a = Answers(seed=53)
    a.extend([prompt(18, 7), prompt(16, 8), [], prompt(5, 9), []])
    parents = [[-1, 0, 0, 1, 1, 2, -1], [-1], [], [-1, -1, 0, 1, 3], []]
    drafts = [prompt(len(p), 20 + i) for i, p in enumerate(parents)]
    mask = a.db.tree_mask(parents)
    lens = a.cache.lens.tolist()
    ys = a.forward(drafts, mask)
    pos = a.cache.positions(a.starts, 64, torch.cat([mask, mask.new_zeros(64 - mask.shape[0], 1)])).tolist()[0]
    at = 0
    for s, (p, d, y) in enumerate(zip(parents, drafts, ys)):
        for i in range(len(p)):
            path, k = [], i
            while k >= 0:
                path.insert(0, k)
                k = p[k]
            assert pos[at + i] == lens[s] + len(path) - 1
            t = a.tokens[s] + [d[k] for k in path]
            cfg = q3.Qwen3Config.from_dict(dict(W, T=len(t), max_seq_len=len(t)))
            want = q3.forward(a.base, a.lora, np.array([t]), np.array([t]), cfg)["logits"][0, -1]
            assert rel_l2(y[i].float().cpu().numpy(), want) < REL_L2, (s, i)
        at += len(p)
    assert pos[at:] == [0] * (64 - at)
    kept = [[0, 1, 4], [0], [], [1, 3, 4], []]
    a.m.keep_tokens(3, ints([len(k) for k in kept]), ints([k + [-1] * (3 - len(k)) for k in kept]))
    for s, k in enumerate(kept):
        a.tokens[s] += [drafts[s][i] for i in k]
        a.logits[s] += [ys[s][i].float().cpu().numpy() for i in k]
    a.check()
    a.extend([[3], [4, 5], [], [6], []])
    a.check()


def test_a_captured_step_goes_on_as_the_eager_one():
    """Forward over the cache, adjusted logits, the choice, the token stored:
    replays with eager work of another cache in between give eager tokens."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a, b = Answers(seed=55), Answers(seed=55)
        runs = []
        for x in (a, b):
            x.extend([prompt(20, 1), prompt(31, 2), [], [], []])
            x.cache.fork(ints([0, 1, 1, 0, -1]))
            ids = torch.zeros(1, 64, dtype=torch.int32, device="cuda")
            ids[0, :4] = ints([5, 6, 7, 8])
            starts, history = ints([0, 1, 2, 3, 4, 4]), torch.full((4, 40), -1, dtype=torch.int32, device="cuda")
            lens, one = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.full((4,), 1.5, device="cuda")
            x.m.set_cache(x.cache, starts, 1)

            def step(x=x, ids=ids, history=history, lens=lens, one=one):
                x.m.forward(ids)
                x.m.keep_tokens(1)
                y = x.db.adjust_logits(x.m.logits()[:4], history, None, lens, one, one)
                new = y.float().argmax(1).int()
                history.scatter_(1, lens[:, None].long(), new[:, None])
                lens.add_(1)
                ids[0, :4] = new

            runs.append((step, history))
        runs[0][0]()
        runs[1][0]()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        runs[1][0]()
    for k in range(20):
        with torch.cuda.stream(side):
            runs[0][0]()
            if k == 7:
                runs[1][0]()
            else:
                graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(runs[0][1], runs[1][1]), k
        assert a.cache.lens.tolist() == b.cache.lens.tolist() and a.cache.table.tolist() == b.cache.table.tolist()
    assert len(set(runs[0][1][0, :20].tolist())) > 3 and a.cache.short.item() == 0


def test_the_forward_without_a_cache_is_as_before():
    from paper_2609_28568_amd import binding
    a = Answers(seed=57)
    ids = torch.from_numpy(np.array([prompt(64, 3)]))
    a.m.forward(ids, ids)
    loss = a.m.loss()
    a.m.backward()
    grads = a.m.adapters("lora_grads")
    with pytest.raises(binding.LibError, match="status 2"):   # the logits' gradient is there
        a.m.logits()
    a.extend([prompt(30, 4), [], [], [], []])
    for call in (a.m.backward, a.m.loss):
        with pytest.raises(binding.LibError, match="status 2"):
            call()
    with pytest.raises(binding.LibError, match="targets"):
        a.m.forward(ids, ids)
    with pytest.raises(binding.LibError, match="cache is set"):
        a.m.set_layout(60, [4])
    a.m.set_cache(None)
    a.m.forward(ids, ids)
    assert a.m.loss() == loss
    a.m.backward()
    again = a.m.adapters("lora_grads")
    assert all(np.array_equal(grads[k], again[k]) for k in grads)
    with pytest.raises(binding.LibError, match="status 2"):
        a.m.keep_tokens(1)


def test_the_model_refuses_caches_that_are_not_its_own():
    from paper_2609_28568_amd import binding
    a = Answers(seed=59)
    e, starts = a.db.PagedCache.empty, ints([0] * 4)
    for bad in (e(3, 4, 2, 16, 128, 3, 4), e(2, 4, 1, 16, 128, 3, 4), e(2, 4, 2, 16, 64, 3, 4)):
        with pytest.raises(binding.LibError, match="not the model's"):
            a.m.set_cache(bad, starts)
    good = e(2, 4, 2, 16, 128, 3, 4)
    with pytest.raises(binding.LibError, match="max_new"):
        a.m.set_cache(good, starts, 0)
    with pytest.raises(ValueError):
        a.m.set_cache(good, ints([0] * 3))
    with pytest.raises(ValueError):
        a.m.set_cache(good, starts, 1, ints([[1]] * 63))
    # no rows at all: every row is padding
    a.m.set_cache(good, starts)
    a.m.forward(torch.zeros(1, 64, dtype=torch.int32, device="cuda"))
    a.m.keep_tokens(1)
    assert good.lens.tolist() == [0, 0, 0] and good.short.item() == 0


def test_only_rows_that_the_forward_computed_are_kept():
    """A forward of two rows a sequence where one has four: more of them are
    refused, and a path that names the others leaves their places."""
    from paper_2609_28568_amd import binding
    a = Answers(seed=61)
    a.cache.pages.fill_(7)
    ids = torch.zeros(1, 64, dtype=torch.int32, device="cuda")
    ids[0, :5] = ints([3, 4, 5, 6, 7])
    a.m.set_cache(a.cache, ints([0, 4, 5, 5, 5, 5]), 2)
    a.m.forward(ids)
    for n in (3, 4, 64, 1000):
        with pytest.raises(binding.LibError, match="max_new"):
            a.m.keep_tokens(n)
    torch.cuda.synchronize()
    assert not a.cache.lens.any() and bool((a.cache.pages == 7).all())
    a.m.keep_tokens(4, ints([4, 2, 0, 0, 0]), ints([[1, 2, 0, 3], [0, 1, -1, -1]] + [[-1] * 4] * 3))
    torch.cuda.synchronize()
    assert a.cache.lens.tolist() == [4, 2, 0, 0, 0]
    left = (a.cache.pages == 7).all(-1)   # [layer, page, 2, head, token]
    assert not left[:, 0, :, :, [0, 2]].any() and bool(left[:, 0, :, :, [1, 3]].all())   # rows 1 and 0; 2 and 3
    assert not left[:, 1, :, :, 0].any() and bool(left[:, 1, :, :, 1].all())             # another sequence's row
    a.m.keep_tokens(2)
    assert a.cache.lens.tolist() == [6, 3, 0, 0, 0]
    # as many rows as there are, whatever the call says
    a.m.set_cache(a.cache, ints([0, 4, 5, 5, 5, 5]), 1000)
    a.m.forward(ids)
    a.m.keep_tokens(500)
    assert a.cache.lens.tolist() == [10, 4, 0, 0, 0] and a.cache.short.item() == 0


def test_logits_read_on_another_stream():
    """The stream that asks for them waits for the forward on the model's stream."""
    a = Answers(seed=63)
    a.extend([prompt(20, 1), prompt(3, 2), [], [], []])
    ids = torch.zeros(1, 64, dtype=torch.int32, device="cuda")
    starts, other = ints([0, 1, 2, 2, 2, 2]), torch.cuda.Stream()
    a.m.set_cache(a.cache, starts, 1)
    got = {}
    for token in (5, 9):
        ids[0, :2] = token
        torch.cuda._sleep(20_000_000)   # the forward is behind this, on the model's stream
        a.m.forward(ids)
        with torch.cuda.stream(other):
            got[token] = a.m.logits()[:2].clone()
        torch.cuda.current_stream().wait_stream(other)
        assert torch.equal(a.m.logits()[:2], got[token])
    assert not torch.equal(got[5], got[9])
    # captured on that stream, replayed behind forwards
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(got[5])
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=other):
        out.copy_(a.m.logits()[:2])
    for token in (5, 9, 5):
        ids[0, :2] = token
        a.m.forward(ids)
        graph.replay()
        assert torch.equal(out, got[token])
