"""Orthogonalised updates on the GPU against their definition in 64 bits: the
operator over shapes that are odd, single rows, tall and wide, one and many;
special values; a captured call; and the optimizer steps that use it.

Tolerance. An operand is stored to 2^-22 of its value (two 11-bit halves), and
the product drops 2^-22 more. An iteration applies coefficients of at most
3.5 + 4.8 + 2.1 to three products of values of norm near 1, so it adds at most
about 2^5 2^-22 of the matrix's norm; the following iterations scale error and
signal of one direction alike. Five of them: 5 2^-17 = 4e-5 of the result's
norm, for matrices whose directions are not far below the strongest."""
import numpy as np
import pytest

from paper_2609_28568_amd import synth
from tests.util import rel_l2, workload

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TOL = 5 * 2.0 ** -17
NS = (3.4445, -4.7750, 2.0315)


def newton_schulz(x, iterations=5):
    """The definition, in float64 on the host."""
    x = np.asarray(x, np.float64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    n = np.sqrt((x * x).sum())
    x = x / n if n > 0 else x
    for _ in range(iterations):
        a = x @ x.T
        x = NS[0] * x + (NS[1] * a + NS[2] * (a @ a)) @ x
    return x.T if tall else x


def batch(count, rows, cols, seed, scale=1e-3):
    g = np.random.default_rng(seed)
    return (g.standard_normal((count, rows, cols)) * scale).astype(np.float32)


SHAPES = [(1, 1, 1), (2, 1, 77), (1, 300, 1), (3, 5, 7), (2, 64, 64), (1, 65, 63), (2, 63, 129), (2, 129, 130),
          (1, 200, 1000), (1, 1001, 190), (40, 16, 256), (5, 128, 384), (3, 384, 320), (9, 700, 513),
          # whole in LDS: one to four blocks of 32 rows, sides that do and do not fill them
          (2, 31, 992), (2, 1184, 32), (3, 64, 480), (2, 450, 50), (2, 96, 288), (2, 70, 301), (1, 128, 128), (2, 141, 97),
          # larger tiles of the products, odd sides in the last ones
          (24, 513, 700), (21, 570, 760), (30, 300, 2050), (26, 2050, 300)]


@pytest.mark.parametrize("count,rows,cols", SHAPES)
def test_against_the_definition(count, rows, cols):
    from paper_2609_28568_amd import binding
    print(f"orthogonalise {count} x {rows} x {cols}", flush=True)
    x = batch(count, rows, cols, 3)
    d = torch.from_numpy(x).cuda()
    y = binding.orthogonalise(d).cpu().numpy()
    assert np.array_equal(d.cpu().numpy(), x)   # the input stays
    for k in range(min(count, 3)):
        for i in {k, count - 1 - k}:
            assert rel_l2(y[i], newton_schulz(x[i])) < TOL, i


@pytest.mark.parametrize("iterations", [1, 2, 9])
def test_other_iteration_counts(iterations):
    from paper_2609_28568_amd import binding
    x = batch(2, 96, 150, 4)
    y = binding.orthogonalise(torch.from_numpy(x).cuda(), iterations=iterations).cpu().numpy()
    tol = TOL * max(1.0, iterations / 5)
    assert all(rel_l2(y[i], newton_schulz(x[i], iterations)) < tol for i in range(2))


@pytest.mark.parametrize("rows,cols", [(70, 90), (200, 190)])
@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e18])
def test_scale_does_not_matter(scale, rows, cols):
    from paper_2609_28568_amd import binding
    x = batch(1, rows, cols, 5, scale)
    y = binding.orthogonalise(torch.from_numpy(x).cuda()).cpu().numpy()
    assert rel_l2(y[0], newton_schulz(x[0])) < TOL


@pytest.mark.parametrize("rows,cols", [(40, 66), (140, 270)])
def test_zeros_and_invalid_numbers_stay_in_their_matrix(rows, cols):
    from paper_2609_28568_amd import binding
    x = batch(5, rows, cols, 6)
    x[1] = 0
    x[2, 3, 4] = np.nan
    x[3, rows - 1, cols - 1] = np.inf
    x[4, 7] = 0
    y = binding.orthogonalise(torch.from_numpy(x).cuda()).cpu().numpy()
    assert np.all(y[1] == 0)
    assert np.all(np.isnan(y[2])) and np.all(np.isnan(y[3]))
    assert np.all(y[4, 7] == 0)
    assert all(rel_l2(y[i], newton_schulz(x[i])) < TOL for i in (0, 4))


@pytest.mark.parametrize("rows,cols", [(33, 52), (260, 132)])
def test_in_place_unaligned_and_an_own_workspace(rows, cols):
    from paper_2609_28568_amd import binding
    x = batch(2, rows, cols, 7)
    flat = torch.zeros(x.size + 1, device="cuda")
    d = flat[1:].view(2, rows, cols)   # 4-byte alignment only
    d.copy_(torch.from_numpy(x))
    ws = torch.empty(binding.orthogonalise_size(rows, cols, 2), dtype=torch.uint8, device="cuda")
    whole = binding.orthogonalise(d.clone())
    assert binding.orthogonalise(d, out=d, workspace=ws) is d
    assert torch.equal(d, whole) and float(flat[0]) == 0.0


def test_runs_repeat_and_a_captured_call_replays():
    from paper_2609_28568_amd import binding
    x = torch.from_numpy(batch(3, 190, 260, 8)).cuda()
    ws = torch.empty(binding.orthogonalise_size(190, 260, 3), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.orthogonalise(x, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.orthogonalise(x, out=out, workspace=ws)
    for seed in (8, 9, 10):
        x.copy_(torch.from_numpy(batch(3, 190, 260, seed)))
        graph.replay()
        eager = binding.orthogonalise(x)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def muon(p, g, mom, coef, lr, wd, momentum, nesterov, scale, iterations=5):
    """One matrix's step in 64 bits: (p, momentum)."""
    g = g.astype(np.float64) * coef
    m = momentum * mom + g
    u = g + momentum * m if nesterov else m
    return p - lr * (wd * p + scale * np.sqrt(max(p.shape)) * newton_schulz(u, iterations)), m


@pytest.mark.parametrize("nesterov,wide", [(True, False), (False, False), (True, True)])
def test_gpt2_muon_step(nesterov, wide):
    """wide: matrices that go through the products, tall, wide and square; otherwise they stay in LDS."""
    from paper_2609_28568_amd import binding
    # one warmup step, so that the rate is the peak and the update is well above fp32's rounding of the weights
    w = workload("tiny", **(dict(d_model=256, d_ff=1024) if wide else {}))
    opt = dict(synth.OPTIM, lr_max=0.05, warmup_steps=1, grad_clip=0.5)
    m = binding.GPT2(binding.make_config(w, opt))
    other = binding.GPT2(binding.make_config(w, opt))
    p = synth.perturb_params(synth.init_params(w), 5)
    m.set_params(p)
    other.set_params(p)
    C, L = w["d_model"], w["n_layer"]
    mom = {}
    for step in range(2):
        ids, tgt = (torch.from_numpy(a) for a in synth.token_batch(w, micro=step))
        before = m.to_dict()
        m.forward(ids, tgt)
        m.backward()
        grads = m.to_dict("grads")
        norm = torch.zeros(1, device="cuda")
        lr = m.muon_step(step, norm_out=norm, momentum=0.9, nesterov=nesterov)
        torch.cuda.synchronize()
        assert abs(lr - m.lr_at(step)) < 1e-9
        total = np.sqrt(sum((g.astype(np.float64) ** 2).sum() for g in grads.values()))
        assert abs(float(norm) - total) < 1e-5 * total
        coef = min(1.0, 0.5 / total)
        after = m.to_dict()
        bf = m.flat_bf16().float().cpu().numpy()
        for kind, parts in (("qkvw", 3), ("attprojw", 1), ("fcw", 1), ("fcprojw", 1)):
            rows = before[kind].shape[1] // parts
            for l in range(L):
                for j in range(parts):
                    at = (l, slice(j * rows, (j + 1) * rows))
                    key = (kind, l, j)
                    ref, mom[key] = muon(before[kind][at].astype(np.float64), grads[kind][at],
                                         mom.get(key, 0.0), coef, lr, 0.1, 0.9, nesterov, 0.2)
                    step_ref = ref - before[kind][at]
                    # the step is read off fp32 weights: half a step of theirs besides the operator's own error
                    err = np.linalg.norm(after[kind][at] - before[kind][at] - step_ref)
                    assert err < 2 * TOL * np.linalg.norm(step_ref) + 2.0 ** -24 * np.linalg.norm(ref), key
            off, shape = m.kinds[kind]
            n = int(np.prod(shape))
            assert np.array_equal(bf[off:off + n], synth.round_to_bf16(after[kind]).ravel()), kind
        if step == 0:   # everything else takes the AdamW step, bit for bit
            other.forward(ids, tgt)
            other.backward()
            other.flat("grads").copy_(m.flat("grads"))
            other.adamw_step(0)
            ref = other.to_dict()
            for kind in ref:
                same = np.array_equal(ref[kind], after[kind])
                assert same != (kind in ("qkvw", "attprojw", "fcw", "fcprojw")), kind
    m.close()
    other.close()


@pytest.mark.parametrize("rank", [16, 1, 21, 32])
def test_qwen3_muon_step(rank):
    from paper_2609_28568_amd import qwen3_binding as qb
    # 1280 rows of gate and up: with the higher ranks more than a CU's LDS holds
    w = dict(synth.QWEN3_WORKLOADS["qwen3_tiny"], lora_rank=rank, d_ff=1280)
    opt = dict(synth.QWEN3_OPTIM, lr=0.05, grad_clip=0.1)
    m = qb.Qwen3(qb.make_config(w, opt))
    base, lora = synth.init_qwen3(w, b_std=0.02)
    m.set_base(base)
    m.set_lora(lora)
    mom = {}
    for step in range(2):
        ids, tgt = (torch.from_numpy(a) for a in synth.token_batch(w, micro=step))
        before = m.adapters()
        m.forward(ids, tgt)
        m.backward()
        grads = m.adapters("lora_grads")
        norm = torch.zeros(1, device="cuda")
        m.muon_step(norm_out=norm)
        after = m.adapters()
        total = np.sqrt(sum((g.astype(np.float64) ** 2).sum() for g in grads.values()))
        assert abs(float(norm) - total) < 1e-5 * total
        for k in grads:
            for l in range(w["n_layer"]):
                ref, mom[k, l] = muon(before[k][l].astype(np.float64), grads[k][l], mom.get((k, l), 0.0),
                                      min(1.0, 0.1 / total), 0.05, 0.1, 0.95, True, 0.2)
                step_ref = ref - before[k][l]
                err = np.linalg.norm(after[k][l] - before[k][l] - step_ref)
                assert err < 2 * TOL * np.linalg.norm(step_ref) + 2.0 ** -24 * np.linalg.norm(ref), (k, l)
        # the rank padding stays zero, and the bf16 copy follows
        packed, copy = m.packed(), m.packed("lora_bf16")
        for n, a in packed.items():
            assert np.array_equal(copy[n], synth.round_to_bf16(a)), n
            assert np.count_nonzero(a) <= sum(after[k].size for k in after if k.split("_")[-1] == n.split("_")[-1]), n
        r = w["lora_rank"]
        assert all(np.all(a[..., r:] == 0) for n, a in packed.items() if n.endswith("_B"))
        assert all(np.all(a.reshape(a.shape[0], -1, qb.RP, a.shape[2])[:, :, r:] == 0)
                   for n, a in packed.items() if n.endswith("_A"))
    m.close()


# 192-wide tiles for A and P (odd sides in the last ones), and for X of tall
# matrices; long contractions of few tiles for X, and for A and P
@pytest.mark.parametrize("count,rows,cols", [(12, 1100, 1100), (12, 1152, 1090), (21, 760, 570), (4, 1500, 1500),
                                             (1, 2030, 2040), (1, 2200, 2100)])
def test_large_tiles_against_the_definition(count, rows, cols):
    from paper_2609_28568_amd import binding
    print(f"orthogonalise {count} x {rows} x {cols}", flush=True)
    x = batch(count, rows, cols, 11)
    y = binding.orthogonalise(torch.from_numpy(x).cuda()).cpu().numpy()
    for i in {0, count - 1}:
        assert rel_l2(y[i], newton_schulz(x[i])) < TOL, i


@pytest.mark.parametrize("shape", [dict(n_layer=12, d_model=768, n_head=12, d_ff=3072),
                                   dict(n_layer=2, d_model=640, n_head=10, d_ff=2560)])
def test_gpt2_muon_step_of_real_widths(shape):
    """Square, tall and wide matrices together on the update's 192- and 128-wide
    tiles, one step from a momentum that is not zero; a few matrices against 64
    bits, every weight's bf16 copy, and the momenta."""
    from paper_2609_28568_amd import binding
    w = workload("tiny", **shape)
    opt = dict(synth.OPTIM, lr_max=0.05, warmup_steps=1, grad_clip=0.5)
    m = binding.GPT2(binding.make_config(w, opt), seed=3)
    m.forward(*(torch.from_numpy(a) for a in synth.token_batch(w)))
    m.backward()
    gen = torch.Generator(device="cuda").manual_seed(4)
    m.flat("grads").copy_(torch.randn(m.n_params, generator=gen, device="cuda") * 1e-3)
    m.flat("m").copy_(torch.randn(m.n_params, generator=gen, device="cuda") * 1e-3)
    before, grads, mom = m.to_dict(), m.to_dict("grads"), m.to_dict("m")
    lr = m.muon_step(0, momentum=0.9)
    torch.cuda.synchronize()
    after, mom2 = m.to_dict(), m.to_dict("m")
    total = np.sqrt(sum((g.astype(np.float64) ** 2).sum() for g in grads.values()))
    coef = min(1.0, 0.5 / total)
    bf = m.flat_bf16().float().cpu().numpy()
    last = shape["n_layer"] - 1
    for kind, parts, which in (("qkvw", 3, [(0, 1), (last, 2)]), ("attprojw", 1, [(last, 0)]),
                               ("fcw", 1, [(0, 0), (last, 0)]), ("fcprojw", 1, [(0, 0), (last, 0)])):
        rows = before[kind].shape[1] // parts
        for l, j in which:
            at = (l, slice(j * rows, (j + 1) * rows))
            ref, new = muon(before[kind][at].astype(np.float64), grads[kind][at], mom[kind][at].astype(np.float64),
                            coef, lr, 0.1, 0.9, True, 0.2)
            step = ref - before[kind][at]
            err = np.linalg.norm(after[kind][at] - before[kind][at] - step)
            assert err < 2 * TOL * np.linalg.norm(step) + 2.0 ** -24 * np.linalg.norm(ref), (kind, l, j)
        # two fp32 roundings of terms no larger than the sum of their sizes, and the clip coefficient's own
        size = 0.9 * np.abs(mom[kind]) + coef * np.abs(grads[kind])
        new = 0.9 * mom[kind].astype(np.float64) + coef * grads[kind].astype(np.float64)
        assert np.all(np.abs(mom2[kind] - new) <= 2.0 ** -20 * size), kind
        off, _ = m.kinds[kind]
        n = after[kind].size
        assert np.array_equal(bf[off:off + n], synth.round_to_bf16(after[kind]).ravel()), kind
    m.close()


@pytest.mark.parametrize("rows,cols", [(40, 66), (140, 270)])
@pytest.mark.parametrize("scale", [1e-42, 3e-40])
def test_subnormal_matrices(scale, rows, cols):
    """Whatever bits such numbers have are kept: the input is exact as it is."""
    from paper_2609_28568_amd import binding
    x = batch(1, rows, cols, 12, scale)
    assert np.count_nonzero(x) > 0.9 * x.size and np.abs(x).max() < 2.0 ** -126
    y = binding.orthogonalise(torch.from_numpy(x).cuda()).cpu().numpy()
    assert rel_l2(y[0], newton_schulz(x[0])) < TOL
