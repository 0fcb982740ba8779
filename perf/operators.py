"""Performance cases of three operators of the training steps: the
orthogonalised update of a weight matrix (Newton-Schulz products), the head
norm and rotary embedding of queries and keys at positions with several axes,
and attention over packed sequences that share one prefix.

Every case is one pass as a program using this package makes it. `run` holds
each operator's plain form in elementary torch operations (32 bits, angles in
64) and, with `own`, the package's calls. `exact` computes the same outputs in
64 bits. Sizes are those of the package's own workloads
(paper_2609_28568_amd/synth.py), its tests' small models, and generic ones.
"""
import math
import random

import torch

own = False
DEV = "cuda"

# quintic Newton-Schulz coefficients of the orthogonalised update
NS = (3.4445, -4.7750, 2.0315)
ITERATIONS = 5
EPS = 1e-6


def _ortho(rows, cols, count):
    return dict(op="orthogonalise", rows=rows, cols=cols, count=count)


def _rotary(tokens, H, Hkv, hd, sections, interleaved, norm, max_pos, theta, backward):
    return dict(op="rotary", tokens=tokens, H=H, Hkv=Hkv, hd=hd, sections=sections, interleaved=interleaved, norm=norm,
                max_pos=max_pos, theta=theta, backward=backward)


def _prefix(H, Hkv, hd, prefix, n_seq, max_len, lens_seed, prefix_queries, backward):
    """lens_seed 0: n_seq sequences of max_len tokens; otherwise of 0..max_len tokens, drawn from it."""
    return dict(op="prefix", H=H, Hkv=Hkv, hd=hd, prefix=prefix, n_seq=n_seq, max_len=max_len, lens_seed=lens_seed,
                prefix_queries=prefix_queries, backward=backward)


def listed():
    return [
        # the smallest updates: the MLP matrices of a two-layer toy model
        dict(_ortho(64, 256, 2), name="ortho_tiny"),
        # the rank-16 A factors of 28 adapted layers (q, k, v and o)
        dict(_ortho(16, 1024, 112), name="ortho_adapters"),
        # a few matrices of odd shape, taller than wide
        dict(_ortho(333, 250, 3), name="ortho_odd"),
        # q, k, v and output projections of the 12 layers of the 124M model
        dict(_ortho(768, 768, 48), name="ortho_124m_attention"),
        # ... and its MLP up projections
        dict(_ortho(3072, 768, 12), name="ortho_124m_mlp"),
        # one new token of each of eight sequences, far into them
        dict(_rotary(8, 16, 8, 128, "24,20,20", True, True, 1 << 20, 1e6, False), name="rotary_tokens"),
        # a training micro-batch of text and images: time, height, width
        dict(_rotary(16384, 16, 8, 128, "16,24,24", False, True, 4096, 1e6, True), name="rotary_train"),
        # narrow heads without the norm, four axes, an odd number of tokens
        dict(_rotary(4097, 12, 4, 64, "8,8,8,8", True, False, 30000, 1e4, True), name="rotary_odd"),
        # one token for each of 64 candidates of one long prompt, whose keys and values are there
        dict(_prefix(16, 8, 128, 8192, 64, 1, 0, False, False), name="prefix_tokens"),
        # ragged candidate answers scored against one prompt, prompt included
        dict(_prefix(16, 8, 128, 1500, 12, 150, 7, True, False), name="prefix_score"),
        # training on 16 answers to one prompt
        dict(_prefix(16, 8, 128, 2048, 16, 256, 0, True, True), name="prefix_train"),
        # narrow heads without grouping, ragged answers, some empty
        dict(_prefix(12, 12, 64, 333, 9, 90, 5, True, True), name="prefix_odd"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _split(rng, total, parts):
    """`parts` numbers of at least 1 that sum to `total`."""
    cuts = sorted(rng.sample(range(1, total), parts - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def draw(rng):
    kind = rng.choice(("orthogonalise", "rotary", "prefix"))
    if kind == "orthogonalise":
        while True:
            rows, cols = _log_uniform(rng, 8, 2500), _log_uniform(rng, 8, 2500)
            count = _log_uniform(rng, 1, 64)
            c = _ortho(rows, cols, count)
            if work(c)["flops"] <= work(_ortho(768, 768, 48))["flops"]:
                return c
    if kind == "rotary":
        H, Hkv, hd = rng.choice(((16, 8, 128), (4, 2, 128), (12, 12, 64), (12, 4, 64), (9, 3, 32), (8, 1, 128)))
        axes = rng.randint(1, 4)
        interleaved = rng.random() < 0.5
        # interleaved axes take every axes-th pair: equal shares, and what is left goes to the first
        share = hd // 2 // axes
        sections = [hd // 2 - share * (axes - 1)] + [share] * (axes - 1) if interleaved else _split(rng, hd // 2, axes)
        return _rotary(_log_uniform(rng, 1, 16384), H, Hkv, hd, ",".join(map(str, sections)), interleaved,
                       rng.random() < 0.6, _log_uniform(rng, 64, 1 << 20), rng.choice((1e4, 1e6)), rng.random() < 0.5)
    H, Hkv, hd = rng.choice(((16, 8, 128), (4, 2, 128), (12, 12, 64), (12, 4, 64), (8, 1, 128), (6, 2, 64)))
    while True:
        queries = rng.random() < 0.6
        prefix = _log_uniform(rng, 1, 4096) if queries else _log_uniform(rng, 1, 16384)
        c = _prefix(H, Hkv, hd, prefix, _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 512), rng.randint(0, 9999),
                    queries, rng.random() < 0.5)
        n = _lens(c)
        if sum(n) and (sum(n) + prefix * queries) * (prefix + sum(n)) * H <= 16 * 6144 * 6144:
            return c


def _lens(case):
    if not case["lens_seed"]:
        return [case["max_len"]] * case["n_seq"]
    rng = random.Random(case["lens_seed"])
    return [rng.randint(0, case["max_len"]) for _ in range(case["n_seq"])]


def _sections(case):
    return [int(s) for s in case["sections"].split(",")]


def _pair_axis(case):
    """The axis whose position turns each of the hd/2 pairs."""
    s = _sections(case)
    if not case["interleaved"]:
        return [a for a, k in enumerate(s) for _ in range(k)]
    n = len(s)
    return [i % n if i // n < s[i % n] else 0 for i in range(case["hd"] // 2)]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 2 + 1)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    if case["op"] == "orthogonalise":
        # a gradient's spectrum: a few dozen strong directions over noise
        n, r, c = case["count"], case["rows"], case["cols"]
        k = min(r, c, 48)
        w = torch.arange(1, k + 1, device=DEV) ** -0.5
        x = torch.matmul(normal(n, r, k) * w, normal(n, k, c)) + 0.5 * normal(n, r, c)
        return dict(case=case, x=(x * 1e-3).contiguous())
    slots = case["H"] + 2 * case["Hkv"]
    if case["op"] == "rotary":
        t, hd = case["tokens"], case["hd"]
        s = dict(case=case, sections=_sections(case), qkv=normal(t, slots * hd).bfloat16(), q_norm=None, k_norm=None)
        s["positions"] = torch.randint(0, case["max_pos"], (len(s["sections"]), t), generator=g, device=DEV).int()
        s["axis"] = torch.tensor(_pair_axis(case), device=DEV)
        if case["norm"]:
            s["q_norm"], s["k_norm"] = ((1 + 0.2 * normal(hd)).bfloat16() for _ in range(2))
        if case["backward"]:
            s["dout"] = (normal(t, slots * hd) * 1e-3).bfloat16()
        return s
    lens = _lens(case)
    n, P, hd = case["prefix"] + sum(lens), case["prefix"], case["hd"]
    s = dict(case=case, qkv=normal(n, slots * hd))
    s["qkv"][:, :(case["H"] + case["Hkv"]) * hd] *= 1.4   # scores of twice the unit spread
    s["qkv"] = s["qkv"].bfloat16()
    rows = n if case["prefix_queries"] else n - P
    if case["backward"]:
        s["dout"] = (normal(rows, case["H"] * hd) * 1e-3).bfloat16()
    # the first row of each row's own sequence (0 in the prefix)
    first, at = [0] * P, P
    for k in lens:
        first += [at] * k
        at += k
    s["first"] = torch.tensor(first, device=DEV)
    s["plan"] = None
    if own:
        from paper_2609_28568_amd import qwen3_binding as qb
        s["plan"] = qb.SharedPrefix(case["H"], case["Hkv"], hd, P, lens, prefix_queries=case["prefix_queries"])
    return s


def _plain_orthogonalise(x):
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt().float()
    x = torch.where(norm > 0, x / norm, torch.zeros_like(x))
    a, b, c = NS
    for _ in range(ITERATIONS):
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return x.transpose(1, 2).contiguous() if tall else x


def _angles(s, dtype):
    case = s["case"]
    half = case["hd"] // 2
    freq = case["theta"] ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    ang = s["positions"].double()[s["axis"]].T * freq
    return ang.cos().to(dtype)[:, None], ang.sin().to(dtype)[:, None]


def _plain_rotary(s):
    case = s["case"]
    H, Hkv, hd, n = case["H"], case["Hkv"], case["hd"], case["tokens"]
    half = hd // 2
    cos, sin = _angles(s, torch.float32)
    raw = s["qkv"].view(n, H + 2 * Hkv, hd)
    x = raw[:, :H + Hkv].float()
    gain = rstd = None
    if case["norm"]:
        gain = torch.cat([s["q_norm"].expand(H, hd), s["k_norm"].expand(Hkv, hd)]).float()
        rstd = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
        x = x * rstd
    y = x * gain if case["norm"] else x
    y = torch.cat([y[..., :half] * cos - y[..., half:] * sin, y[..., half:] * cos + y[..., :half] * sin], -1)
    out = [torch.cat([y.bfloat16(), raw[:, H + Hkv:]], 1).view(n, -1)]
    if case["backward"]:
        dall = s["dout"].view(n, H + 2 * Hkv, hd)
        d = dall[:, :H + Hkv].float()
        d = torch.cat([d[..., :half] * cos + d[..., half:] * sin, d[..., half:] * cos - d[..., :half] * sin], -1)
        if case["norm"]:
            d = d * gain
            d = rstd * (d - x * (d * x).mean(-1, keepdim=True))
        out.append(torch.cat([d.bfloat16(), dall[:, H + Hkv:]], 1).view(n, -1))
    return out


def _plain_prefix(s):
    case = s["case"]
    H, Hkv, hd, P = case["H"], case["Hkv"], case["hd"], case["prefix"]
    G, n = H // Hkv, s["qkv"].shape[0]
    q0 = 0 if case["prefix_queries"] else P
    rows = n - q0
    x = s["qkv"].float().view(n, H + 2 * Hkv, hd)
    # [Hkv, G * rows, hd]: the rows of a key/value head's query heads, one after another
    q = x[q0:, :H].reshape(rows, Hkv, G, hd).permute(1, 2, 0, 3).reshape(Hkv, G * rows, hd).contiguous()
    k = x[:, H:H + Hkv].permute(1, 0, 2).contiguous()
    v = x[:, H + Hkv:].permute(1, 0, 2).contiguous()
    i, j = torch.arange(q0, n, device=DEV)[:, None], torch.arange(n, device=DEV)[None]
    seen = (j <= i) & ((j < P) | (j >= s["first"][q0:, None]))
    sc = torch.matmul(q, k.transpose(1, 2).contiguous()).view(Hkv, G, rows, n) * hd ** -0.5
    sc = sc.masked_fill(~seen, -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = (sc - top).exp()
    total = p.sum(-1, keepdim=True)
    p = (p / total).view(Hkv, G * rows, n)
    o = torch.matmul(p, v)
    lse = (top + total.log()).view(H, rows)
    out = [o.view(Hkv, G, rows, hd).permute(2, 0, 1, 3).reshape(rows, H * hd).bfloat16(), lse]
    if case["backward"]:
        do = s["dout"].float().view(rows, Hkv, G, hd).permute(1, 2, 0, 3).reshape(Hkv, G * rows, hd).contiguous()
        dv = torch.matmul(p.transpose(1, 2).contiguous(), do)
        ds = torch.matmul(do, v.transpose(1, 2).contiguous())
        ds = p * (ds - (do * o).sum(-1, keepdim=True)) * hd ** -0.5
        dq = torch.matmul(ds, k).view(Hkv, G, rows, hd).permute(2, 0, 1, 3).reshape(rows, H, hd)
        dk = torch.matmul(ds.transpose(1, 2).contiguous(), q)
        d = torch.zeros(n, H + 2 * Hkv, hd, device=DEV, dtype=torch.bfloat16)
        d[q0:, :H] = dq.bfloat16()
        d[:, H:H + Hkv] = dk.permute(1, 0, 2).bfloat16()
        d[:, H + Hkv:] = dv.permute(1, 0, 2).bfloat16()
        out.append(d.view(n, -1))
    return out


def run(state):
    case = state["case"]
    if own:
        from paper_2609_28568_amd import binding as gb, qwen3_binding as qb
        if case["op"] == "orthogonalise":
            return gb.orthogonalise(state["x"], iterations=ITERATIONS)
        if case["op"] == "rotary":
            how = dict(n_head=case["H"], n_kv_head=case["Hkv"], sections=state["sections"], theta=case["theta"],
                       interleaved=case["interleaved"], q_norm=state["q_norm"], k_norm=state["k_norm"], eps=EPS)
            out = [qb.rotary(state["qkv"], state["positions"], **how)]
            if case["backward"]:
                out.append(qb.rotary_backward(state["dout"], state["qkv"], state["positions"], **how))
            return out
        o, lse = state["plan"].forward(state["qkv"])
        if not case["backward"]:
            return [o, lse]
        return [o, lse, state["plan"].backward(state["dout"], state["qkv"], o, lse)]
    if case["op"] == "orthogonalise":
        return _plain_orthogonalise(state["x"])
    return _plain_rotary(state) if case["op"] == "rotary" else _plain_prefix(state)


def work(case):
    if case["op"] == "orthogonalise":
        a, b = sorted((case["rows"], case["cols"]))
        # the Gram matrix and its square are symmetric: half of each
        flops = ITERATIONS * (a * (a + 1) * b + a * a * (a + 1) + 2 * a * a * b)
        return {"bytes": 8.0 * a * b * case["count"], "flops": float(flops * case["count"])}
    slots = case["H"] + 2 * case["Hkv"]
    if case["op"] == "rotary":
        t, hd = case["tokens"], case["hd"]
        row, pos = 2.0 * slots * hd, 4.0 * (case["sections"].count(",") + 1)
        gains = 4.0 * hd if case["norm"] else 0.0
        nbytes = t * (2 * row + pos) + gains
        flops = 10.0 * t * (case["H"] + case["Hkv"]) * hd
        if case["backward"]:
            raw = 2.0 * (case["H"] + case["Hkv"]) * hd if case["norm"] else 0.0
            nbytes += t * (2 * row + pos + raw) + gains
            flops *= 2.4
        return {"bytes": nbytes, "flops": flops}
    lens, P, H, hd = _lens(case), case["prefix"], case["H"], case["hd"]
    n = P + sum(lens)
    rows = n if case["prefix_queries"] else n - P
    pairs = sum(k * P + k * (k + 1) // 2 for k in lens) + (P * (P + 1) // 2 if case["prefix_queries"] else 0)
    kv = 4.0 * n * case["Hkv"] * hd
    q = 2.0 * rows * H * hd
    nbytes, flops = kv + 2 * q + 4.0 * rows * H, 4.0 * hd * H * pairs
    if case["backward"]:
        nbytes += 2 * kv + 4 * q + 4.0 * rows * H
        flops += 10.0 * hd * H * pairs
    return {"bytes": nbytes, "flops": flops}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orthogonalise":
        # on the shorter side's Gram matrix from the right: Y <- Y (a + b G + c G^2), G = Y^T Y
        out = []
        for m in s["x"].double():
            y = m if m.shape[0] >= m.shape[1] else m.T.contiguous()
            norm = torch.linalg.norm(y)
            y = y / norm if norm > 0 else y
            for _ in range(ITERATIONS):
                gram = y.T.contiguous() @ y
                poly = torch.eye(gram.shape[0], device=DEV, dtype=torch.float64) * NS[0] + gram * NS[1]
                y = y @ (poly + gram @ gram * NS[2])
            out.append(y if m.shape[0] >= m.shape[1] else y.T.contiguous())
        return torch.stack(out)
    H, Hkv, hd = case["H"], case["Hkv"], case["hd"]
    x = s["qkv"].double().unflatten(1, (H + 2 * Hkv, hd))
    if case["op"] == "rotary":
        # pairs as complex numbers: a turn by e^{i angle}, gradients by its conjugate
        def pairs(z):
            return torch.complex(z[..., :hd // 2].contiguous(), z[..., hd // 2:].contiguous())

        def halves(z):
            return torch.cat([z.real, z.imag], -1)

        cos, sin = _angles(s, torch.float64)
        turn = torch.complex(cos, sin)
        qk, out = x[:, :H + Hkv], []
        if case["norm"]:
            gain = torch.cat([s["q_norm"].double().repeat(H, 1), s["k_norm"].double().repeat(Hkv, 1)])
            size = (qk.pow(2).sum(-1, keepdim=True) / hd + EPS).sqrt()
        y = qk / size * gain if case["norm"] else qk
        out.append(torch.cat([halves(pairs(y) * turn), x[:, H + Hkv:]], 1).flatten(1))
        if case["backward"]:
            d = s["dout"].double().unflatten(1, (H + 2 * Hkv, hd))
            e = halves(pairs(d[:, :H + Hkv]) * turn.conj())
            if case["norm"]:
                e = e * gain
                e = e / size - qk * (e * qk).sum(-1, keepdim=True) / (hd * size ** 3)
            out.append(torch.cat([e, d[:, H + Hkv:]], 1).flatten(1))
        return out
    # one query head after another, the sequences' rows by a mask of their own numbers
    P, n = case["prefix"], x.shape[0]
    q0 = 0 if case["prefix_queries"] else P
    lens = _lens(case)
    number = torch.tensor([-1] * P + [a for a, k in enumerate(lens) for _ in range(k)], device=DEV)
    at = torch.arange(n, device=DEV)
    hidden = (at[None] > at[q0:, None]) | ((number[None] >= 0) & (number[None] != number[q0:, None]))
    outs, lses = [], []
    grad = torch.zeros_like(x) if case["backward"] else None
    for h in range(H):
        q, k, v = x[q0:, h], x[:, H + h // (H // Hkv)], x[:, H + Hkv + h // (H // Hkv)]
        sc = (q @ k.T.contiguous() / math.sqrt(hd)).masked_fill(hidden, -math.inf)
        lse = torch.logsumexp(sc, 1)
        p = torch.exp(sc - lse[:, None])
        del sc
        outs.append(p @ v)
        lses.append(lse)
        if case["backward"]:
            d = s["dout"].double()[:, h * hd:(h + 1) * hd]
            grad[:, H + Hkv + h // (H // Hkv)] += p.T.contiguous() @ d
            e = p * (d @ v.T.contiguous() - (d * outs[-1]).sum(1, keepdim=True)) / math.sqrt(hd)
            del p
            grad[q0:, h] = e @ k
            grad[:, H + h // (H // Hkv)] += e.T.contiguous() @ q
    out = [torch.cat(outs, 1), torch.stack(lses)]
    return out + [grad.flatten(1)] if case["backward"] else out
