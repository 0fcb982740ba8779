"""Head norm and rotary embedding at positions with several axes on the GPU,
against the formulas in 64 bits: head widths, groupings, sections of both
kinds, far and negative positions, one token and many; the gradient against
the formula's and against differences; in place; and the adapter step that
uses it, against the oracle.

Tolerance: angles are exact to fp32's rounding of a value in [-1, 1], the
arithmetic between is fp32 over a head of at most 256 elements (2^-19 of the
largest term), and the result is rounded once to bf16, by at most 2^-8 of it."""
import numpy as np
import pytest

from oracle import qwen3 as q3
from paper_2609_28568_amd import synth
from tests.util import LOSS_ATOL, REL_L2, rel_l2

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EPS = 1e-6


def pair_axes(sections, interleaved):
    n = len(sections)
    if not interleaved:
        return np.repeat(np.arange(n), sections)
    half = sum(sections)
    axis = np.zeros(half, int)
    for a in range(1, n):
        axis[a:a + n * sections[a]:n] = a
    return axis


def tables(positions, hd, sections, interleaved, theta):
    """cos and sin [tokens, hd/2] in float64."""
    inv = theta ** (-np.arange(0, hd, 2, dtype=np.float64) / hd)
    ang = positions.astype(np.float64)[pair_axes(sections, interleaved)].T * inv
    return np.cos(ang), np.sin(ang)


def forward(x, cos, sin, H, Hkv, gq, gk):
    """x [tokens, H + 2 Hkv, hd] float64."""
    y = x.copy()
    for lo, hi, g in ((0, H, gq), (H, H + Hkv, gk)):
        n = q3.rmsnorm_forward(x[:, lo:hi], g, EPS)[0] if g is not None else x[:, lo:hi]
        y[:, lo:hi] = q3.rope_forward(n, cos[:, None], sin[:, None])
    return y


def backward(d, x, cos, sin, H, Hkv, gq, gk):
    y = d.copy()
    for lo, hi, g in ((0, H, gq), (H, H + Hkv, gk)):
        n = q3.rope_backward(d[:, lo:hi], cos[:, None], sin[:, None])
        if g is not None:
            n = q3.rmsnorm_backward(n, x[:, lo:hi], q3.rmsnorm_forward(x[:, lo:hi], g, EPS)[1], g)
        y[:, lo:hi] = n
    return y


def close(y, ref):
    """Within the rounding of the result, and fp32's of the head's largest element."""
    top = np.abs(ref).max(axis=-1, keepdims=True)
    return np.all(np.abs(y - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -17 * top + 1e-30)


CASES = {
    # tokens, H, Hkv, hd, sections, interleaved, norm, theta, position range
    "three_axes": (37, 16, 8, 128, (16, 24, 24), False, True, 1e6, (0, 5000)),
    "interleaved": (130, 16, 8, 128, (24, 20, 20), True, True, 1e6, (0, 5000)),
    "one_token_far": (1, 4, 2, 128, (22, 21, 21), True, True, 1e6, (1 << 30, 1 << 31)),
    "negative": (5, 2, 1, 128, (30, 34), False, True, 1e4, (-(1 << 31), 1 << 31)),
    "no_norm": (9, 4, 4, 128, (64,), False, False, 1e6, (0, 100)),
    "hd64_grouped_by_three": (67, 9, 3, 64, (8, 8, 8, 8), True, True, 1e4, (0, 30000)),
    "hd32_odd_heads": (3, 5, 5, 32, (5, 11), False, True, 1e4, (0, 400)),
    "hd256": (4, 3, 1, 256, (0, 100, 28), False, True, 1e6, (0, 400)),
    "empty_section": (6, 3, 1, 64, (30, 0, 2), True, False, 1e6, (0, 400)),
    "enough_for_one_wave_each": (1501, 1, 1, 64, (20, 12), False, True, 1e6, (0, 400)),
}


def setup(name):
    t, H, Hkv, hd, sections, inter, norm, theta, (lo, hi) = CASES[name]
    g = np.random.default_rng(17)
    x = synth.round_to_bf16(g.standard_normal((t, H + 2 * Hkv, hd)).astype(np.float32))
    d = synth.round_to_bf16(g.standard_normal(x.shape).astype(np.float32) * np.float32(1e-3))
    pos = g.integers(lo, hi, (len(sections), t)).astype(np.int32)
    gains = [synth.round_to_bf16((1 + 0.3 * g.standard_normal(hd)).astype(np.float32)) for _ in range(2)]
    how = dict(n_head=H, n_kv_head=Hkv, sections=sections, interleaved=inter, theta=theta, eps=EPS)
    if norm:
        how["q_norm"], how["k_norm"] = (torch.from_numpy(a).bfloat16().cuda() for a in gains)
    cos, sin = tables(pos, hd, sections, inter, theta)
    ref = (cos, sin, H, Hkv, *(gains if norm else (None, None)))
    dev = [torch.from_numpy(a.reshape(t, -1)).bfloat16().cuda() for a in (x, d)]
    return x.astype(np.float64), d.astype(np.float64), dev, torch.from_numpy(pos).cuda(), how, ref


def host(t, like):
    return t.float().cpu().numpy().astype(np.float64).reshape(like.shape)


@pytest.mark.parametrize("name", list(CASES))
def test_against_the_formulas(name):
    from paper_2609_28568_amd import qwen3_binding as qb
    print(f"rotary {name}", flush=True)
    x, d, (dx, dd), pos, how, ref = setup(name)
    y = qb.rotary(dx, pos, **how)
    assert close(host(y, x), forward(x, *ref))
    g = qb.rotary_backward(dd, dx, pos, **how)
    assert close(host(g, x), backward(d, x, *ref))
    # in place gives the same bits
    assert torch.equal(qb.rotary_backward(dd, dx, pos, out=dd, **how), g) and dd.data_ptr() != g.data_ptr()
    assert torch.equal(qb.rotary(dx, pos, out=dx, **how), y)


@pytest.mark.parametrize("name", ["three_axes", "hd64_grouped_by_three"])
def test_gradient_against_differences(name):
    from paper_2609_28568_amd import qwen3_binding as qb
    x, d, (dx, dd), pos, how, ref = setup(name)
    g = host(qb.rotary_backward(dd, dx, pos, **how), x)
    rng = np.random.default_rng(3)
    for _ in range(4):
        v, h = rng.standard_normal(x.shape), 1e-5
        num = (d * (forward(x + h * v, *ref) - forward(x - h * v, *ref))).sum() / (2 * h)
        # every element's rounding of 2^-8 at most, in a sum of independent terms
        assert abs(num - (g * v).sum()) < 4 * 2.0 ** -8 * np.linalg.norm(g * v) + 1e-6 * abs(num)


def test_no_tokens_and_a_replayed_graph():
    from paper_2609_28568_amd import qwen3_binding as qb
    x, d, (dx, dd), pos, how, ref = setup("interleaved")
    assert qb.rotary(dx[:0], pos[:, :0].contiguous(), **how).shape == (0, dx.shape[1])
    out, g = torch.empty_like(dx), torch.empty_like(dx)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qb.rotary(dx, pos, out=out, **how)
        qb.rotary_backward(dd, dx, pos, out=g, **how)
    for k in range(3):
        pos.add_(k * 11)
        graph.replay()
        a, b = qb.rotary(dx, pos, **how), qb.rotary_backward(dd, dx, pos, **how)
        torch.cuda.synchronize()
        assert torch.equal(out, a) and torch.equal(g, b)


# ---- in the adapter step

def step_case():
    w = dict(synth.QWEN3_WORKLOADS["qwen3_tiny"])
    base, lora = synth.init_qwen3(w, seed=51, b_std=0.02, norm_jitter=0.1)
    ids, tgt = synth.token_batch(w, seed=52)
    return w, base, lora, ids, tgt


def model(w, base, lora):
    from paper_2609_28568_amd import qwen3_binding as qb
    m = qb.Qwen3(qb.make_config(w, synth.QWEN3_OPTIM))
    m.set_base(base)
    m.set_lora(lora)
    return m


@pytest.mark.parametrize("sections,interleaved", [((16, 24, 24), False), ((24, 20, 20), True)])
def test_step_against_the_oracle(monkeypatch, sections, interleaved):
    w, base, lora, ids, tgt = step_case()
    B, T = w["B"], w["T"]
    g = np.random.default_rng(9)
    pos = np.stack([np.sort(g.integers(0, 400, (B, T)), axis=1) for _ in sections]).astype(np.int32)
    cos, sin = tables(pos.reshape(len(sections), -1), 128, sections, interleaved, synth.QWEN3_OPTIM["rope_theta"])
    tab = [a.reshape(B, 1, T, 64) for a in (cos, sin)]
    monkeypatch.setattr(q3, "rope_tables", lambda T_, hd, theta, dt: tuple(a.astype(dt) for a in tab))
    ocfg = q3.Qwen3Config.from_dict({**w, **synth.QWEN3_OPTIM})
    cache = q3.forward(base, lora, ids, tgt, ocfg)
    ref = q3.backward(base, lora, cache, ocfg)
    m = model(w, base, lora)
    m.set_positions(torch.from_numpy(pos.reshape(len(sections), -1)).cuda(), sections, interleaved)
    m.forward(torch.from_numpy(ids), torch.from_numpy(tgt))
    # a change between a forward and its backward is the next forward's
    m.set_positions(None)
    m.backward()
    assert abs(m.loss() - float(cache["loss"])) < LOSS_ATOL
    for k, v in m.adapters("lora_grads").items():
        assert rel_l2(v, ref[k]) < REL_L2, k
    m.close()


def test_step_with_the_default_positions_spelled_out():
    """The same angles from positions as from the default tables: equal to
    their rounding, and back to the same bits without them."""
    w, base, lora, ids, tgt = step_case()
    m = model(w, base, lora)
    batch = [torch.from_numpy(a) for a in (ids, tgt)]
    m.forward(*batch)
    loss = m.loss()
    m.backward()
    grads = m.adapters("lora_grads")
    pos = torch.arange(w["T"], dtype=torch.int32).repeat(1, w["B"]).cuda()
    m.set_positions(pos)
    m.forward(*batch)
    m.backward()
    assert abs(m.loss() - loss) < 1e-3
    for k, v in m.adapters("lora_grads").items():
        assert rel_l2(v, grads[k]) < REL_L2 / 2, k
    m.set_positions(None)
    m.forward(*batch)
    m.backward()
    assert m.loss() == loss
    assert all(np.array_equal(v, grads[k]) for k, v in m.adapters("lora_grads").items())
    m.close()


@pytest.mark.parametrize("name", ["three_axes", "hd256", "no_norm"])
def test_gradient_in_place_of_the_rows(name):
    from paper_2609_28568_amd import qwen3_binding as qb
    x, d, (dx, dd), pos, how, ref = setup(name)
    g = qb.rotary_backward(dd, dx, pos, **how)
    assert torch.equal(qb.rotary_backward(dd, dx, pos, out=dx, **how), g) and dx.data_ptr() != g.data_ptr()
