"""The three operators where offsets pass 32 bits, and the whole step that uses
them captured into a graph and replayed."""
import numpy as np
import pytest

from paper_2609_28568_amd import synth
from tests.test_gpu_orthogonalise import TOL, newton_schulz
from tests.test_gpu_prefix import R
from tests.util import rel_l2

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", [True, False])
def test_rotary_rows_past_4_gib(norm):
    """Every part of the rows gives the bits that it gives alone."""
    from paper_2609_28568_amd import qwen3_binding as qb
    H, Hkv, hd, n = 4, 2, 128, 2200001
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(n, (H + 2 * Hkv) * hd, generator=gen, device="cuda", dtype=torch.bfloat16)
    assert x.numel() * 2 > 1 << 32
    pos = torch.randint(-(1 << 31), 1 << 31, (3, n), generator=gen, device="cuda").int()
    how = dict(n_head=H, n_kv_head=Hkv, sections=(24, 20, 20), interleaved=True)
    if norm:
        how.update(q_norm=1 + 0.2 * torch.randn(hd, generator=gen, device="cuda"),
                   k_norm=1 + 0.2 * torch.randn(hd, generator=gen, device="cuda"))
        how = {k: v.bfloat16() if torch.is_tensor(v) else v for k, v in how.items()}
    y, g = qb.rotary(x, pos, **how), qb.rotary_backward(x, x.flip(0), pos, **how)
    for lo in (0, 2097152 - 700, n - 1500):
        part = slice(lo, lo + 1500)
        p = pos[:, part].contiguous()
        assert torch.equal(qb.rotary(x[part], p, **how), y[part])
        assert torch.equal(qb.rotary_backward(x[part], x.flip(0)[part].contiguous(), p, **how), g[part])


def test_orthogonalise_batch_past_4_gib():
    from paper_2609_28568_amd import binding
    n, r, c = 1100, 1024, 1000
    x = torch.randn(n, r, c, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda")
    assert x.numel() * 4 > 1 << 32
    y = binding.orthogonalise(x)
    for i in (0, 1047, n - 1):
        assert rel_l2(y[i].cpu().numpy(), newton_schulz(x[i].cpu().numpy())) < TOL, i


def test_shared_prefix_up_to_4_gib():
    """The longest prefix that rows of this width take; two of the eight
    key/value heads against the definition in 64 bits. Tolerances as in the
    smaller cases, and fp32 sums over 8,187 tiles, in workgroups and then over
    them, of at most 1,000 terms each: 2^-14."""
    from paper_2609_28568_amd import binding, qwen3_binding as qb
    H, Hkv, hd, P, n = 16, 8, 128, 523960, 64
    with pytest.raises(binding.LibError, match="32-bit"):
        qb.SharedPrefix(H, Hkv, hd, P + 80, [1] * n, prefix_queries=False)
    gen = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(P + n, (H + 2 * Hkv) * hd, generator=gen, device="cuda", dtype=torch.bfloat16)
    g = torch.randn(n, H * hd, generator=gen, device="cuda", dtype=torch.bfloat16)
    p = qb.SharedPrefix(H, Hkv, hd, P, [1] * n, prefix_queries=False)
    y, lse = p.forward(x)
    dx = p.backward(g, x, y, lse)
    xs, ds_, ys, gs = (t.view(t.shape[0], -1, hd) for t in (x, dx, y, g))
    rest, G = R + 2.0 ** -14, H // Hkv
    own = torch.arange(n, device="cuda")
    for j in (0, Hkv - 1):
        k, v = xs[:, H + j].double(), xs[:, H + Hkv + j].double()
        dk, dv = torch.zeros_like(k), torch.zeros_like(v)
        e_dk, e_dv = torch.zeros_like(k), torch.zeros_like(v)
        for h in range(j * G, (j + 1) * G):
            q, do = xs[P:, h].double(), gs[:, h].double()
            s = q @ k.T.contiguous() / hd ** 0.5
            s[:, P:] = torch.where(own[:, None] == own[None], s[:, P:], -torch.inf)
            ref = torch.logsumexp(s, 1)
            assert ((lse[h].double() - ref).abs() <= 2.0 ** -14).all()
            pr = torch.exp(s - ref[:, None])
            out, mass = pr @ v, pr @ v.abs()
            e_out = R * out.abs() + rest * mass
            assert ((ys[:, h].double() - out).abs() <= e_out).all()
            ds = pr * (do @ v.T.contiguous() - (do * out).sum(1, keepdim=True))
            e_ds = rest * ds.abs() + pr * ((do.abs() * e_out).sum(1, keepdim=True)
                                           + 2.0 ** -14 * (do.abs() @ v.abs().T.contiguous()))
            dq, e_dq = ds @ k / hd ** 0.5, e_ds @ k.abs() / hd ** 0.5
            assert ((ds_[P:, h].double() - dq).abs() <= e_dq + R * dq.abs()).all()
            dv += pr.T @ do
            e_dv += rest * (pr.T @ do.abs())
            dk += ds.T @ q / hd ** 0.5
            e_dk += e_ds.T @ q.abs() / hd ** 0.5
        assert ((ds_[:, H + j].double() - dk).abs() <= e_dk + R * dk.abs()).all()
        assert ((ds_[:, H + Hkv + j].double() - dv).abs() <= e_dv + R * dv.abs()).all()
    assert (ds_[:P, :H] == 0).all()


def test_the_step_of_all_three_captured_and_replayed():
    """Answers to one prompt at positions of three axes, the update orthogonalised:
    replays and eager steps in between give the bits of eager steps alone."""
    from paper_2609_28568_amd import qwen3_binding as qb
    P, lens = 60, [50, 31, 51]
    w = dict(synth.QWEN3_WORKLOADS["qwen3_tiny"], B=1, T=192, max_seq_len=192)
    base, lora = synth.init_qwen3(w, seed=51, b_std=0.02)
    ids, tgt = (torch.from_numpy(a).int().cuda() for a in synth.token_batch(w, seed=52))
    axes = torch.randint(0, 300, (3, 192), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()

    def model():
        with torch.cuda.stream(side):
            m = qb.Qwen3(qb.make_config(w, synth.QWEN3_OPTIM))
            m.set_base(base)
            m.set_lora(lora)
            m.set_layout(P, lens)
            m.set_positions(axes, (24, 20, 20), interleaved=True)
        return m

    def step(m):
        m.forward(ids, tgt)
        m.backward()
        m.muon_step()

    eager, captured = model(), model()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(eager)
        step(captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(captured)
    for k in range(5):
        with torch.cuda.stream(side):
            step(eager)
            if k == 2:
                step(captured)
            else:
                graph.replay()
        torch.cuda.synchronize()
        a, b = eager.adapters(), captured.adapters()
        assert all(np.array_equal(a[n], b[n]) for n in a), k
        assert eager.loss() == captured.loss()
    eager.close()
    captured.close()
