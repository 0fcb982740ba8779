"""Attention over sequences that share a prefix on the GPU, forward and
backward, against its definition in 64 bits: groupings, head sizes, ragged and
empty sequences, single tokens, prefixes that end inside tiles, no prefix, no
sequence, walks long enough to be dealt to several workgroups; the adapter step
that uses it against the oracle.

Tolerances, element by element. Probabilities and score gradients are rounded
to bf16 (2^-8 of each at most) before the products that sum them, and results
once more; everything else is fp32 (2^-15 covers its sums and the exponents').
So with absolute values written |.|:
  out  2^-8 (|out| + P|V|) =: E_out             dV  2^-8 (|dV| + P^T|dO|)
  D = rowsum(dO out) moves by |dO| E_out, so dS = P (dP - D) by
  E_dS = 2^-8 |dS| + P rowsum(|dO| E_out); dQ and dK sum it against |K| and |Q|,
  and are rounded."""
import numpy as np
import pytest

from oracle import qwen3 as q3
from paper_2609_28568_amd import synth
from tests.util import LOSS_ATOL, REL_L2, rel_l2

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

R = 2.0 ** -8 * (1 + 2.0 ** -6)


def sees(P, lens, q0):
    """[rows, tokens]: which keys each token with a query sees."""
    N = P + sum(lens)
    own = np.concatenate([np.full(P, -1)] + [np.full(n, i) for i, n in enumerate(lens)]).astype(int)
    t = np.arange(N)
    return ((t[None] <= t[:, None]) & ((t[None] < P) | (own[None] == own[:, None])))[q0:]


def reference(qkv, dout, H, Hkv, hd, P, lens, q0):
    """(out, lse, dqkv) in float64 and the bounds of out and dqkv."""
    N = qkv.shape[0]
    x = qkv.astype(np.float64).reshape(N, H + 2 * Hkv, hd)
    do = dout.astype(np.float64).reshape(N - q0, H, hd)
    m = sees(P, lens, q0)
    scale = 1 / np.sqrt(hd)
    out, lse = np.zeros_like(do), np.zeros((H, N - q0))
    d, e_out, e_d = np.zeros_like(x), np.zeros_like(do), np.zeros_like(x)
    for h in range(H):
        kh, vh = H + h // (H // Hkv), H + Hkv + h // (H // Hkv)
        q, k, v = x[q0:, h], x[:, kh], x[:, vh]
        s = np.where(m, q @ k.T * scale, -np.inf)
        top = s.max(1, keepdims=True)
        e = np.exp(s - top)
        lse[h] = (top + np.log(e.sum(1, keepdims=True)))[:, 0]
        p = e / e.sum(1, keepdims=True)
        out[:, h] = p @ v
        e_out[:, h] = R * (np.abs(out[:, h]) + p @ np.abs(v)) + 2.0 ** -15 * (p @ np.abs(v))
        g = do[:, h]
        d[:, vh] += p.T @ g
        e_d[:, vh] += (R + 2.0 ** -15) * (p.T @ np.abs(g))
        dp = g @ v.T
        ds = p * (dp - (g * out[:, h]).sum(1, keepdims=True))
        e_ds = R * np.abs(ds) + p * ((np.abs(g) * e_out[:, h]).sum(1, keepdims=True) + 2.0 ** -15 * (np.abs(g) @ np.abs(v.T)))
        d[q0:, h] = ds @ k * scale
        e_d[q0:, h] = e_ds @ np.abs(k) * scale
        d[:, kh] += ds.T @ q * scale
        e_d[:, kh] += e_ds.T @ np.abs(q) * scale
    e_d += R * np.abs(d)
    return out.reshape(N - q0, -1), lse, d.reshape(N, -1), e_out.reshape(N - q0, -1), e_d.reshape(N, -1)


CASES = {
    # H, Hkv, hd, prefix, lengths, prefix_queries
    "answers": (4, 2, 128, 150, [40, 17, 64, 1], True),
    "answers_hd64": (4, 4, 64, 130, [33, 65, 2], True),
    "single_tokens": (4, 2, 128, 700, [1] * 9, False),
    "one_token_one_sequence": (2, 1, 128, 1, [1], False),
    "nothing_but_a_token": (2, 2, 64, 0, [1], True),
    "groups_of_three": (6, 2, 64, 77, [50, 0, 31], True),
    "groups_of_eight": (8, 1, 128, 65, [30, 100], True),
    "some_empty": (2, 1, 64, 64, [0, 0, 70, 0, 5, 0], True),
    "packed_without_prefix": (3, 3, 64, 0, [100, 3, 64, 129, 1, 40], True),
    "prefix_only": (4, 2, 128, 321, [], True),
    "known_prefix": (4, 2, 128, 200, [70, 9, 130], False),
    "known_prefix_hd64": (3, 1, 64, 64, [64, 1, 63], False),
    "many_short": (2, 1, 128, 10, [3, 1, 2, 5, 0, 7] * 25, True),
    "long_walks": (1, 1, 128, 2500, [30, 50], False),
    "long_walks_hd64": (2, 1, 64, 2100, [300, 11, 200], True),
    "prefix_of_one_tile": (2, 2, 128, 128, [128, 64], True),
    # more workgroups than CUs: one group of waves each, walks whole and shared
    "many_items": (16, 16, 64, 700, [250, 333], True),
    "many_items_wide": (12, 12, 128, 500, [700, 61], True),
    "few_rows_shared_widely": (2, 1, 128, 6000, [1, 2], False),
    "few_rows_shared_widely_hd64": (8, 2, 64, 5000, [3] * 7, False),
}


def inputs(name, seed=5):
    H, Hkv, hd, P, lens, queries = CASES[name]
    g = np.random.default_rng(seed)
    N, q0 = P + sum(lens), 0 if queries else P
    qkv = g.standard_normal((N, (H + 2 * Hkv) * hd)).astype(np.float32)
    qkv[:, :(H + Hkv) * hd] *= 1.4
    dout = g.standard_normal((N - q0, H * hd)).astype(np.float32) * np.float32(1e-2)
    return synth.round_to_bf16(qkv), synth.round_to_bf16(dout), (H, Hkv, hd, P, lens, q0)


def plan(name):
    from paper_2609_28568_amd import qwen3_binding as qb
    H, Hkv, hd, P, lens, queries = CASES[name]
    return qb.SharedPrefix(H, Hkv, hd, P, lens, prefix_queries=queries)


def dev(a):
    return torch.from_numpy(a).bfloat16().cuda()


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("name", list(CASES))
def test_against_the_definition(name):
    print(f"shared prefix {name}: {CASES[name]}", flush=True)
    qkv, dout, how = inputs(name)
    out, lse, d, e_out, e_d = reference(qkv, dout, *how)
    p = plan(name)
    x, g = dev(qkv), dev(dout)
    y, l = p.forward(x)
    torch.cuda.synchronize()
    assert np.all(np.abs(host(y) - out) <= e_out)
    assert np.all(np.abs(l.cpu().numpy() - lse) <= 2.0 ** -18 * (1 + np.abs(lse)))
    dx = p.backward(g, x, y, l)
    torch.cuda.synchronize()
    assert np.all(np.abs(host(dx) - d) <= e_d)
    # the same bits again, into buffers of the caller's
    y2, l2, d2 = torch.full_like(y, 7), torch.full_like(l, 7), torch.full_like(dx, 7)
    p.forward(x, out=y2, lse=l2)
    p.backward(g, x, y, l, dqkv=d2)
    assert torch.equal(y, y2) and torch.equal(l, l2) and torch.equal(dx, d2)
    p.close()


@pytest.mark.parametrize("name", ["answers_hd64", "nothing_but_a_token", "groups_of_eight", "packed_without_prefix", "many_short"])
def test_rows_of_one_key_have_no_score_gradient(name):
    """Such a row's probability is 1 and dP - D = 0. P comes from scores and a
    log-sum-exp below 32 in fp32, about eight roundings of them: |1 - P| <=
    2^-24 * 8 * 32 = 2^-16, so dS is at most 2^-16 |dP|, and its two roundings
    to bf16 do not double that. D from the bf16 output would leave 2^-9 |dP|."""
    qkv, dout, (H, Hkv, hd, P, lens, q0) = inputs(name)
    p = plan(name)
    x, g = torch.tensor(qkv).cuda().bfloat16(), torch.tensor(dout).cuda().bfloat16()
    out, lse = p.forward(x)
    dqkv = p.backward(g, x, out, lse).float().cpu().numpy().astype(np.float64).reshape(qkv.shape[0], -1, hd)
    xs, gs = np.abs(qkv.astype(np.float64)).reshape(-1, H + 2 * Hkv, hd), np.abs(dout.astype(np.float64)).reshape(-1, H, hd)
    rows = np.flatnonzero(sees(P, lens, q0).sum(1) == 1)
    assert len(rows) > 0
    for r in rows:
        for h in range(H):
            k, v = xs[q0 + r, H + h // (H // Hkv)], xs[q0 + r, H + Hkv + h // (H // Hkv)]
            assert (np.abs(dqkv[q0 + r, h]) <= 2.0 ** -15 * (gs[r, h] @ v) * k / np.sqrt(hd)).all(), (r, h)


def test_gradient_against_differences():
    name = "answers_hd64"
    qkv, dout, how = inputs(name)
    p = plan(name)
    x = dev(qkv)
    y, l = p.forward(x)
    d = host(p.backward(dev(dout), x, y, l))
    e_d = reference(qkv, dout, *how)[4]
    g = np.random.default_rng(2)
    for _ in range(3):
        v, h = g.standard_normal(qkv.shape), 1e-5
        f = [(reference(qkv + s * h * v, dout, *how)[0] * dout).sum() for s in (1, -1)]
        assert abs((f[0] - f[1]) / (2 * h) - (d * v).sum()) < 3 * np.linalg.norm(e_d * v) + 1e-6


def test_extreme_scores():
    """Scores far below zero, and one key that takes everything."""
    qkv, dout, how = inputs("answers")
    H, Hkv, hd, P, lens, q0 = how
    x = qkv.reshape(-1, H + 2 * Hkv, hd).copy()
    x[:, :H] = 0
    x[:, :H, 0] = 30000
    x[:, H:H + Hkv, 0] = -30000 - 1000 * np.arange(x.shape[0])[:, None]   # scores of -8e7 and below, falling
    x = synth.round_to_bf16(x.reshape(qkv.shape).astype(np.float32))
    out = reference(x, dout, *how)[0]
    p = plan("answers")
    d = dev(x)
    y, l = p.forward(d)
    assert torch.isfinite(y).all() and torch.isfinite(l).all()
    assert rel_l2(host(y), out) < 2.0 ** -7
    assert torch.isfinite(p.backward(dev(dout), d, y, l)).all()


def test_a_sequence_does_not_read_the_others():
    """Other sequences' queries and keys may hold anything finite, and lengths
    of the others do not show: the same bits as alone, up to the tiles' order."""
    qkv, _, how = inputs("answers")
    H, Hkv, hd, P, lens, _ = how
    y, _ = plan("answers").forward(dev(qkv))
    other = qkv.copy()
    other[P + 40:P + 57] = 3e38   # the second sequence
    z, _ = plan("answers").forward(dev(other))
    keep = np.r_[0:P + 40, P + 57:qkv.shape[0]]
    assert torch.equal(y[keep], z[keep])


def test_on_a_stream_of_its_own():
    """A layout made on one stream and used on another, and freed right after."""
    qkv, dout, how = inputs("long_walks")
    x, g = dev(qkv), dev(dout)
    y, l = plan("long_walks").forward(x)
    d = plan("long_walks").backward(g, x, y, l)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    p = plan("long_walks")
    size = p.plan.numel()
    with torch.cuda.stream(side):
        got = p.forward(x)
        grad = p.backward(g, x, *got)
    del p
    torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255)   # may not take the layout's place yet
    torch.cuda.synchronize()
    assert torch.equal(got[0], y) and torch.equal(got[1], l) and torch.equal(grad, d)


def test_a_captured_pass_replays():
    qkv, dout, how = inputs("long_walks_hd64")
    p = plan("long_walks_hd64")
    x, g = dev(qkv), dev(dout)
    y, l = p.forward(x)
    d = p.backward(g, x, y, l)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.forward(x, out=y, lse=l)
        p.backward(g, x, y, l, dqkv=d)
    for seed in (6, 7, 8):
        a, b, _ = inputs("long_walks_hd64", seed)
        x.copy_(dev(a))
        g.copy_(dev(b))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, l, d)]
        ey, el = p.forward(x)
        ed = p.backward(g, x, ey, el)
        assert all(torch.equal(s, t) for s, t in zip(got, (ey, el, ed)))


# ---- in the adapter step

def masked_attention(mask):
    def forward(q, k, v):
        grp = q.shape[1] // k.shape[1]
        ke, ve = np.repeat(k, grp, axis=1), np.repeat(v, grp, axis=1)
        s = np.where(mask, (q @ ke.transpose(0, 1, 3, 2)) * q.dtype.type(1.0 / np.sqrt(q.shape[3])), -np.inf)
        e = np.exp(s - s.max(axis=-1, keepdims=True))
        p = e / e.sum(axis=-1, keepdims=True)
        return p @ ve, p
    return forward


@pytest.mark.parametrize("P,lens", [(64, [40, 13, 60, 15]), (100, [92]), (0, [100, 28, 64]), (191, [1])])
def test_step_against_the_oracle(monkeypatch, P, lens):
    """The whole step with a layout, its positions the default ones and then
    given with several axes, and the orthogonalised update on its gradients."""
    from paper_2609_28568_amd import qwen3_binding as qb
    T = P + sum(lens)
    w = dict(synth.QWEN3_WORKLOADS["qwen3_tiny"], B=1, T=T, max_seq_len=T, loss_from=(P + 0.5) / T)
    base, lora = synth.init_qwen3(w, seed=51, b_std=0.02, norm_jitter=0.1)
    ids, tgt = synth.token_batch(w, seed=52)
    ocfg = q3.Qwen3Config.from_dict({**w, **synth.QWEN3_OPTIM})
    pos = np.concatenate([np.arange(P)] + [P + np.arange(n) for n in lens])
    axes = np.stack([pos, pos // 7, pos % 7]).astype(np.int32)
    inv = 1e6 ** (-np.arange(0, 128, 2, dtype=np.float64) / 128)
    monkeypatch.setattr(q3, "gqa_attention_forward", masked_attention(sees(P, lens, 0)))
    m = qb.Qwen3(qb.make_config(w, synth.QWEN3_OPTIM))
    m.set_base(base)
    m.set_lora(lora)
    m.set_layout(P, lens)
    for turn in ("default", "axes"):
        if turn == "default":
            ang = pos[:, None] * inv
        else:
            ang = axes[np.repeat([0, 1, 2], (24, 20, 20))].T * inv
            m.set_positions(torch.from_numpy(axes).cuda(), (24, 20, 20))
        monkeypatch.setattr(q3, "rope_tables", lambda T_, hd, th, dt: (np.cos(ang).astype(dt), np.sin(ang).astype(dt)))
        cache = q3.forward(base, lora, ids, tgt, ocfg)
        ref = q3.backward(base, lora, cache, ocfg)
        m.forward(torch.from_numpy(ids), torch.from_numpy(tgt))
        m.set_layout(P + 1 if P + 1 < T else P - 1, [T - P - 1 if P + 1 < T else T - P + 1])   # the next forward's
        m.backward()
        assert abs(m.loss() - float(cache["loss"])) < LOSS_ATOL, turn
        for k, v in m.adapters("lora_grads").items():
            assert rel_l2(v, ref[k]) < REL_L2, (turn, k)
        m.set_layout(P, lens)
    before = m.adapters()
    m.muon_step()
    after = m.adapters()
    for k in before:
        step = np.linalg.norm(after[k] - before[k])
        # an update of 0.2 sqrt(max side) times a matrix of singular values near 1, per layer
        sides = before[k].shape[1:]
        assert 0.3 < step / (synth.QWEN3_OPTIM["lr"] * 0.2 * np.sqrt(max(sides) * min(sides) * w["n_layer"])) < 1.5, k
    # and back to plain sequences
    m.set_layout()
    m.set_positions()
    m.forward(torch.from_numpy(ids), torch.from_numpy(tgt))
    m.backward()
    m.close()


def test_step_layout_of_one_causal_sequence_is_the_plain_step():
    from paper_2609_28568_amd import qwen3_binding as qb
    w = dict(synth.QWEN3_WORKLOADS["qwen3_tiny"], B=1, T=192, max_seq_len=192)
    base, lora = synth.init_qwen3(w, seed=51, b_std=0.02)
    ids, tgt = (torch.from_numpy(a) for a in synth.token_batch(w, seed=52))
    m = qb.Qwen3(qb.make_config(w, synth.QWEN3_OPTIM))
    m.set_base(base)
    m.set_lora(lora)
    got = []
    for layout in (None, (192, []), (0, [192]), (100, [92])):
        m.set_layout(*layout) if layout else m.set_layout()
        m.forward(ids, tgt)
        m.backward()
        got.append((m.loss(), m.adapters("lora_grads")))
    for loss, grads in got[1:]:
        assert abs(loss - got[0][0]) < 1e-3
        assert all(rel_l2(v, got[0][1][k]) < REL_L2 / 2 for k, v in grads.items())
    m.close()


def test_refusals_of_the_step():
    from paper_2609_28568_amd import binding, qwen3_binding as qb
    w = dict(synth.QWEN3_WORKLOADS["qwen3_tiny"], B=1, T=192, max_seq_len=192)
    m = qb.Qwen3(qb.make_config(w, synth.QWEN3_OPTIM))
    for P, lens, why in ((100, [91], "T tokens"), (-1, [193], "prefix_len"), (100, [-1, 93], "negative")):
        with pytest.raises(binding.LibError, match=why) as e:
            m.set_layout(P, lens)
        assert e.value.status == binding.GPT2_ERR_INVALID_ARG
    with pytest.raises(binding.LibError, match="backward"):
        m.muon_step()
    for kw, why in ((dict(momentum=1.0), "momentum"), (dict(iterations=0), "iterations"), (dict(scale=0.0), "scale")):
        with pytest.raises(binding.LibError, match=why):
            m.muon_step(**kw)
    with pytest.raises(ValueError):
        m.set_positions(torch.zeros(2, 191, dtype=torch.int32, device="cuda"), (32, 32))
    with pytest.raises(binding.LibError, match="sum"):
        m.set_positions(torch.zeros(2, 192, dtype=torch.int32, device="cuda"), (32, 31))
    m.close()
    two = qb.Qwen3(qb.make_config(dict(synth.QWEN3_WORKLOADS["qwen3_tiny"]), synth.QWEN3_OPTIM))
    with pytest.raises(binding.LibError, match="B = 1"):
        two.set_layout(96, [96])
    two.close()


@pytest.mark.parametrize("name,seq", [("answers", 1), ("answers_hd64", 0), ("long_walks_hd64", 1), ("known_prefix", 1),
                                      ("many_items_wide", 0)])
def test_gradients_of_a_sequence_do_not_read_the_others(name, seq):
    """As above for the backward: values whose products with a gradient of
    order 1 leave fp32's range reach no other sequence's gradients. The prefix'
    keys see every sequence, so theirs do depend on it."""
    qkv, dout, (H, Hkv, hd, P, lens, q0) = inputs(name)
    dout = synth.round_to_bf16(dout * np.float32(100))
    lo = P + sum(lens[:seq])
    hi = lo + lens[seq]
    other = qkv.copy()
    other[lo:hi] = 3e38
    p, g = plan(name), dev(dout)
    got = []
    for x in (dev(qkv), dev(other)):
        y, l = p.forward(x)
        got.append((y, l, p.backward(g, x, y, l)))
    (y, l, d), (y2, l2, d2) = got
    rows = np.r_[0:lo, hi:P + sum(lens)]
    seen = rows[rows >= q0] - q0
    assert torch.equal(y[seen], y2[seen]) and torch.equal(l[:, seen], l2[:, seen])
    own = rows[rows >= P]
    assert torch.isfinite(d2[own]).all() and torch.equal(d[own], d2[own])
    dq = slice(0, H * hd)
    assert torch.isfinite(d2[rows][:, dq]).all() and torch.equal(d[rows][:, dq], d2[rows][:, dq])


def test_step_set_up_with_another_stream_current():
    """Layout, positions and the update's workspace asked for while another
    stream is current and busy: the memory that stream's pool has free is still
    being written there, and the positions are not made yet."""
    from paper_2609_28568_amd import qwen3_binding as qb
    P, lens = 60, [50, 31, 51]
    w = dict(synth.QWEN3_WORKLOADS["qwen3_tiny"], B=1, T=192, max_seq_len=192)
    base, lora = synth.init_qwen3(w, seed=51, b_std=0.02)
    ids, tgt = (torch.from_numpy(a) for a in synth.token_batch(w, seed=52))
    axes = torch.randint(0, 300, (2, 192), dtype=torch.int32, device="cuda")
    side, got = torch.cuda.Stream(), []
    for busy in (False, True):
        m = qb.Qwen3(qb.make_config(w, synth.QWEN3_OPTIM))
        m.set_base(base)
        m.set_lora(lora)
        m.forward(ids, tgt)
        m.backward()
        torch.cuda.synchronize()
        with torch.cuda.stream(side if busy else torch.cuda.current_stream()):
            if busy:
                sizes = (got[0][3], got[0][4])
                blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
                torch.cuda._sleep(10 ** 7)
                for b in blocks:
                    b.fill_(255)
                del blocks, b
            pos = axes.clone()
            m.set_layout(P, lens)
            m.set_positions(pos, (30, 34))
            m.muon_step()
        m.forward(ids, tgt)
        m.backward()
        got.append((m.loss(), m.adapters("lora_grads"), m.adapters(), m._plan.numel(), m.muon_workspace.numel()))
        m.close()
    assert got[0][0] == got[1][0]
    for k in got[0][1]:
        assert np.array_equal(got[0][1][k], got[1][1][k]) and np.array_equal(got[0][2][k], got[1][2][k]), k


CASES.update({
    # short walks on more workgroups than CUs
    "many_short_walks": (16, 16, 64, 0, [64, 63, 1, 70] * 14, True),
    "many_short_walks_wide": (16, 16, 128, 3, [64, 63, 1, 70] * 14, True),
    # groups of heads that leave a block of rows inside a token, or make up two
    "groups_of_48": (48, 1, 128, 33, [2, 0, 1, 7], False),
    "groups_of_256": (256, 1, 64, 70, [5, 3], True),
    "groups_of_three_wide": (6, 2, 128, 129, [1, 64, 66], True),
})


@pytest.mark.parametrize("name", list(CASES)[-5:])
def test_short_walks_and_large_groups(name):
    test_against_the_definition(name)


def test_millions_of_single_tokens():
    """More rows than the division of walks is estimated for; the prefix' keys
    sum their gradients over all of them. Tolerances as above, and fp32 sums of
    up to 700 partial sums (540 products of 16 a workgroup, 130 workgroups):
    2^-24 700 < 2^-14 of the sum of absolute values."""
    from paper_2609_28568_amd import qwen3_binding as qb
    P, n, hd = 100, 2200000, 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(P + n, 3 * hd, generator=gen, device="cuda")
    x[:, :2 * hd] *= 1.4
    x, g = x.bfloat16(), (torch.randn(n, hd, generator=gen, device="cuda") * 1e-2).bfloat16()
    p = qb.SharedPrefix(1, 1, hd, P, [1] * n, prefix_queries=False)
    y, lse = p.forward(x)
    dx = p.backward(g, x, y, lse).double()
    del p
    q, do = x[P:, :hd].double(), g.double()
    kp, vp = x[:P, hd:2 * hd].double(), x[:P, 2 * hd:].double()
    k, v = x[P:, hd:2 * hd].double(), x[P:, 2 * hd:].double()
    s = torch.cat([q @ kp.T.contiguous(), (q * k).sum(1, keepdim=True)], 1) / hd ** 0.5
    ref = torch.logsumexp(s, 1)
    pr = torch.exp(s - ref[:, None])
    del s
    assert (lse[0].double() - ref).abs().max() <= 2.0 ** -18 * (1 + ref.abs().max())
    pp, ps = pr[:, :P].contiguous(), pr[:, P:]
    out, mass = pp @ vp + ps * v, pp @ vp.abs() + ps * v.abs()
    e_out = R * (out.abs() + mass) + 2.0 ** -15 * mass
    assert ((y.double() - out).abs() <= e_out).all()
    del mass
    noise = (do.abs() * e_out).sum(1, keepdim=True)
    D = (do * out).sum(1, keepdim=True)
    del out, e_out
    rest = R + 2.0 ** -14
    dv, e_dv = pp.T @ do, rest * (pp.T @ do.abs())
    assert ((dx[:P, 2 * hd:] - dv).abs() <= e_dv + R * dv.abs()).all()
    assert ((dx[P:, 2 * hd:] - ps * do).abs() <= 2 * R * (ps * do).abs() + 2.0 ** -15 * do.abs()).all()
    ds = pp * (do @ vp.T.contiguous() - D)
    e_ds = rest * ds.abs() + pp * (noise + 2.0 ** -15 * (do.abs() @ vp.abs().T.contiguous()))
    dk, e_dk = ds.T @ q / hd ** 0.5, e_ds.T @ q.abs() / hd ** 0.5
    assert ((dx[:P, hd:2 * hd] - dk).abs() <= e_dk + R * dk.abs()).all()
    dss = ps * ((do * v).sum(1, keepdim=True) - D)
    e_dss = rest * dss.abs() + ps * (noise + 2.0 ** -15 * (do.abs() * v.abs()).sum(1, keepdim=True))
    dq = (ds @ kp + dss * k) / hd ** 0.5
    e_dq = (e_ds @ kp.abs() + e_dss * k.abs()) / hd ** 0.5
    assert ((dx[P:, :hd] - dq).abs() <= e_dq + R * dq.abs()).all()
    assert (dx[:P, :hd] == 0).all()


def test_results_over_what_is_read_are_refused():
    from paper_2609_28568_amd import binding
    qkv, dout, (H, Hkv, hd, P, lens, q0) = inputs("groups_of_three")
    p = plan("groups_of_three")
    n, width = qkv.shape
    rows = n - q0
    x, g = dev(qkv), dev(dout)
    y, l = p.forward(x)
    with pytest.raises(binding.LibError, match="overlap"):
        p.forward(x, out=x.view(-1)[:rows * H * hd].view(rows, -1))
    with pytest.raises(binding.LibError, match="overlap"):
        p.forward(x, out=y, lse=y.view(torch.float32).view(-1)[:H * rows].view(H, rows))
    place = torch.empty(2 * n * width, dtype=torch.bfloat16, device="cuda")
    dx = place[64:64 + n * width].view(n, width)
    over = place[:rows * H * hd].view(rows, -1)
    lse = place.view(torch.float32)[40:40 + H * rows].view(H, rows)
    for a in ((over, x, y, l), (g, x, over, l), (g, x, y, lse), (g, place[:n * width].view(n, width), y, l)):
        with pytest.raises(binding.LibError, match="overlap"):
            p.backward(*a, dqkv=dx)
    p.close()


def test_a_layout_asked_for_in_a_capture_is_refused_and_the_capture_goes_on():
    from paper_2609_28568_amd import binding, qwen3_binding as qb
    qkv, dout, (H, Hkv, hd, P, lens, q0) = inputs("answers")
    p = plan("answers")
    x, g = dev(qkv), dev(dout)
    y, l = p.forward(x)
    w = dict(synth.QWEN3_WORKLOADS["qwen3_tiny"], B=1, T=192, max_seq_len=192)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    out, lse = torch.zeros_like(y), torch.zeros_like(l)
    with torch.cuda.stream(side):
        m = qb.Qwen3(qb.make_config(w, synth.QWEN3_OPTIM))
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        for make in (lambda: plan("answers"), lambda: m.set_layout(100, [92])):
            with pytest.raises(binding.LibError, match="captured") as e:
                make()
            assert e.value.status == binding.GPT2_ERR_STATE
        p.forward(x, out=out, lse=lse)
    for _ in range(3):
        out.zero_()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, y) and torch.equal(lse, l)
    m.set_layout(100, [92])
    m.close()
