"""Host-side checks of the operator entry points: the library exports what the
headers declare, sizes are as documented, and malformed requests are refused
before anything is launched (no GPU here: a call that got through would fail
with a device error instead)."""
import ctypes
import os
import re

import pytest

from paper_2609_28568_amd import binding, qwen3_binding as qb, synth
from tests.util import workload

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, STATE = binding.GPT2_ERR_INVALID_ARG, binding.GPT2_ERR_STATE


def test_library_exports_the_prompt_header():
    text = open(os.path.join(ROOT, "include", "qwen3_prompt.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(qwen3_[a-z_0-9]+)\s*\(", text)))
    assert len(names) >= 2
    for n in names:
        assert hasattr(qb.lib(), n), n


# ---- orthogonalised updates

@pytest.mark.parametrize("shape", [(0, 4, 1), (4, 0, 1), (4, 4, 0), (-1, 4, 1), (1 << 16, 1 << 16, 1),
                                   (64, 64, 1 << 30), (8, 8, 1 << 18), (1 << 14, 1 << 14, 1 << 9)])
def test_orthogonalise_refuses_shapes(shape):
    with pytest.raises(binding.LibError) as e:
        binding.orthogonalise_size(*shape)
    assert e.value.status == INVALID and "rows, cols and count" in str(e.value)


def test_orthogonalise_size_grows_with_the_padded_shape():
    assert binding.orthogonalise_size(1, 1) == binding.orthogonalise_size(64, 64)
    assert binding.orthogonalise_size(64, 65) > binding.orthogonalise_size(64, 64)
    assert binding.orthogonalise_size(65, 200) == binding.orthogonalise_size(200, 65)


@pytest.mark.parametrize("x,y,it,ws,nbytes,why", [
    (0, 4096, 5, 8192, 1 << 30, "NULL"), (4096, 0, 5, 8192, 1 << 30, "NULL"), (4096, 4096, 5, 0, 1 << 30, "NULL"),
    (4098, 4096, 5, 8192, 1 << 30, "not aligned"), (4096, 4096, 5, 8200, 1 << 30, "256-byte"),
    (4096, 4096, 5, 8192, 100, "smaller"), (4096, 4096, 0, 8192, 1 << 30, "iterations"),
    (4096, 4096, 33, 8192, 1 << 30, "iterations")])
def test_orthogonalise_refuses_arguments(x, y, it, ws, nbytes, why):
    L = binding.lib()
    assert L.gpt2_orthogonalise(x, y, 8, 8, 1, it, ws, nbytes, None) == INVALID
    assert why in L.gpt2_last_error(None).decode()


def test_orthogonalise_binding_refuses_tensors():
    torch = pytest.importorskip("torch")
    for t in (torch.zeros(4, 4), torch.zeros(4), "x"):
        with pytest.raises(ValueError):
            binding.orthogonalise(t)


def test_muon_sizes():
    n = ctypes.c_size_t()
    cfg = binding.make_config(workload("gpt2_124m"), synth.OPTIM)
    assert binding.lib().gpt2_muon_size(ctypes.byref(cfg), ctypes.byref(n)) == 0
    # two planes of two bytes, twice, of every matrix, and its two Gram-sized ones
    C, F, L = 768, cfg.d_ff, 12
    want = 4 * L * (4 * (2 * C * C + 2 * C * C) + 2 * (2 * C * F + 2 * C * C))
    assert want <= n.value < want + (1 << 20)
    assert binding.lib().gpt2_muon_size(None, ctypes.byref(n)) == INVALID
    assert binding.lib().gpt2_muon_size(ctypes.byref(cfg), None) == INVALID
    assert binding.lib().gpt2_muon_step(None, 0, None, None, 0, None, None) == INVALID
    q = qb.make_config(synth.QWEN3_WORKLOADS["qwen3_tiny"], synth.QWEN3_OPTIM)
    assert qb.lib().qwen3_muon_size(ctypes.byref(q), ctypes.byref(n)) == 0 and n.value > 0
    assert qb.lib().qwen3_muon_size(ctypes.byref(q), None) == INVALID
    assert qb.lib().qwen3_muon_step(None, None, None, 0, None) == INVALID


# ---- rotary positions with several axes

def rotary_desc(**over):
    d = dict(n_tokens=8, n_head=4, n_kv_head=2, head_dim=128, n_axes=3, sections=(16, 24, 24), interleaved=0,
             theta=1e6, rms_eps=1e-6)
    d.update(over)
    d["sections"] = (ctypes.c_int32 * 4)(*d["sections"])
    return qb.Rotary(**d)


@pytest.mark.parametrize("over,why", [
    (dict(n_tokens=-1), "n_tokens"), (dict(n_tokens=(1 << 25) + 1), "n_tokens"), (dict(n_head=0), "n_head"), (dict(n_kv_head=0), "n_kv_head"),
    (dict(head_dim=96), "head_dim"), (dict(n_axes=0), "n_axes"), (dict(n_axes=5), "n_axes"),
    (dict(sections=(16, 24, 25)), "sum"), (dict(sections=(16, 24, 23)), "sum"), (dict(sections=(-1, 41, 24)), "range"),
    (dict(sections=(0, 40, 24), interleaved=1), "fit"), (dict(theta=0.0), "theta"), (dict(theta=float("inf")), "theta"),
    (dict(rms_eps=-1.0), "rms_eps"), (dict(rms_eps=float("nan")), "rms_eps")])
def test_rotary_refuses_descriptions(over, why):
    d = rotary_desc(**over)
    L = qb.lib()
    for call in (lambda: L.qwen3_rotary_forward(ctypes.byref(d), 4096, 4096, 4096, 4096, 8192, None),
                 lambda: L.qwen3_rotary_backward(ctypes.byref(d), 4096, 4096, 4096, 4096, 4096, 8192, None)):
        assert call() == INVALID
        assert why in L.qwen3_last_error(None).decode()


@pytest.mark.parametrize("args,why", [
    ((0, 4096, 4096, 4096, 8192), "null"), ((4096, 0, 4096, 4096, 8192), "null"), ((4096, 4096, 4096, 4096, 0), "null"),
    ((4096, 4096, 0, 4096, 8192), "together"), ((4096, 4096, 4096, 0, 8192), "together"),
    ((4104, 4096, 4096, 4096, 8192), "aligned"), ((4096, 4098, 4096, 4096, 8192), "aligned"),
    ((4096, 4096, 4098, 4096, 8192), "aligned"), ((4096, 4096, 4096, 4096, 8200), "aligned")])
def test_rotary_refuses_pointers(args, why):
    L, d = qb.lib(), rotary_desc()
    assert L.qwen3_rotary_forward(ctypes.byref(d), *args, None) == INVALID
    assert why in L.qwen3_last_error(None).decode()
    assert L.qwen3_rotary_forward(None, *args, None) == INVALID


def test_rotary_without_tokens_does_nothing():
    d = rotary_desc(n_tokens=0)
    assert qb.lib().qwen3_rotary_forward(ctypes.byref(d), None, None, None, None, None, None) == 0


def test_rotary_binding_refuses_tensors():
    torch = pytest.importorskip("torch")
    x, pos = torch.zeros(4, 8 * 128, dtype=torch.bfloat16), torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        qb.rotary(x, pos, n_head=4, n_kv_head=2, sections=(64,))   # not on a device
    assert qb.lib().qwen3_set_positions(None, None, 1, None, 0) == INVALID


# ---- attention over a shared prefix

def prefix_size(lens, **over):
    c = dict(n_head=4, n_kv_head=2, head_dim=128, prefix_len=100, n_seq=len(lens), prefix_queries=1)
    c.update(over)
    n = ctypes.c_size_t()
    arr = (ctypes.c_int32 * max(len(lens), 1))(*lens)
    st = qb.lib().qwen3_prefix_size(ctypes.byref(qb.PrefixConfig(**c)), arr, ctypes.byref(n))
    return st, n.value


@pytest.mark.parametrize("lens,over,why", [
    ([5], dict(n_head=0), "n_head"), ([5], dict(n_kv_head=3), "n_head"), ([5], dict(n_kv_head=0), "n_head"),
    ([5], dict(head_dim=96), "head_dim"), ([5], dict(prefix_len=-1), "prefix_len"), ([5], dict(n_seq=-1), "n_seq"),
    ([5, -1], {}, "negative"), ([0, 0], dict(prefix_queries=0), "query"), ([], dict(prefix_len=0), "query"),
    ([1 << 30], {}, "32-bit"), ([1 << 30] * 9, {}, "32-bit")])
def test_prefix_refuses_layouts(lens, over, why):
    st, _ = prefix_size(lens, **over)
    assert st == INVALID and why in qb.lib().qwen3_last_error(None).decode()


def test_prefix_sizes():
    st, n = prefix_size([10, 0, 3])
    assert st == 0 and n >= 113 * 12
    assert prefix_size([], prefix_len=7)[0] == 0
    assert prefix_size([1] * 64, prefix_len=8192, prefix_queries=0)[0] == 0
    assert qb.lib().qwen3_prefix_size(None, None, None) == INVALID


def test_prefix_refuses_arguments():
    L = qb.lib()
    c = qb.PrefixConfig(4, 2, 128, 100, 1, 1)
    lens, out = (ctypes.c_int32 * 1)(5), ctypes.c_void_p()
    for d_plan, nbytes, why in ((0, 1 << 30, "NULL"), (4100, 1 << 30, "aligned"), (4096, 64, "smaller")):
        assert L.qwen3_prefix_create(ctypes.byref(c), lens, d_plan, nbytes, None, ctypes.byref(out)) == INVALID
        assert why in L.qwen3_last_error(None).decode() and not out
    assert L.qwen3_prefix_create(ctypes.byref(c), lens, 4096, 1 << 30, None, None) == INVALID
    assert L.qwen3_prefix_forward(None, 4096, 4096, 4096, None) == INVALID
    assert L.qwen3_prefix_backward(None, 4096, 4096, 4096, 4096, 4096, None) == INVALID
    L.qwen3_prefix_destroy(None)
    n = ctypes.c_size_t()
    assert L.qwen3_layout_size(None, 1, 1, lens, ctypes.byref(n)) == INVALID
    assert L.qwen3_set_layout(None, 1, 1, lens, None, 0) == INVALID


@pytest.mark.parametrize("n_seq", [1500, 3000, 5000, 600000])
def test_prefix_refuses_lengths_whose_bytes_pass_64_bits(n_seq):
    """Sums of lengths whose bytes wrap around 64 bits, to either sign."""
    st, _ = prefix_size([2 ** 31 - 1] * n_seq, n_head=4096, n_kv_head=4096, prefix_len=0)
    assert st == INVALID and "32-bit" in qb.lib().qwen3_last_error(None).decode()


# ---- buffers of a model used with another stream current

class _Library:
    """Accepts every call."""
    def __getattr__(self, name):
        return lambda *args: 0


class _Stream:
    def __init__(self, name):
        self.name, self.waited = name, []

    def wait_stream(self, other):
        self.waited.append(other.name)


@pytest.fixture
def streams(monkeypatch):
    """(torch, model's stream, list of (stream current at the allocation)): a side stream is current."""
    import contextlib
    torch = pytest.importorskip("torch")
    current, made = [_Stream("side")], []

    @contextlib.contextmanager
    def on(s):
        current.append(s)
        yield
        current.pop()

    empty = torch.empty
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: made.append(current[-1].name) or empty(*a, **kw))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: None)
    monkeypatch.setattr(qb, "lib", _Library)
    return torch, _Stream("model"), made


def _bare_qwen3(torch, stream):
    m = qb.Qwen3.__new__(qb.Qwen3)
    m.torch, m.stream, m.h, m.bufs = torch, stream, None, {"workspace": torch.zeros(1, dtype=torch.uint8)}
    m.cfg = qb.make_config(synth.QWEN3_WORKLOADS["qwen3_tiny"], synth.QWEN3_OPTIM)
    m._positions = m._plan = m._in_use = None
    return m


def test_buffers_of_a_step_come_from_the_models_stream(streams):
    """The library writes them there at once: memory of another stream's pool
    may still be in that stream's use."""
    torch, stream, made = streams
    m = _bare_qwen3(torch, stream)
    m.set_layout(5, [3, 4])
    m.muon_step()
    g = binding.GPT2.__new__(binding.GPT2)
    g.torch, g.stream, g.handle, g.L, g.device = torch, stream, None, _Library(), torch.device("cpu")
    g.cfg = binding.make_config(workload("tiny"), synth.OPTIM)
    g.muon_step(0)
    assert made == ["model"] * 3


def test_positions_are_read_after_the_stream_that_made_them(streams):
    torch, stream, _ = streams
    m = _bare_qwen3(torch, stream)
    m.set_positions(torch.zeros(1, m.cfg.B * m.cfg.T, dtype=torch.int32))
    assert stream.waited == ["side"]
    m.set_positions(None)
    assert stream.waited == ["side"]


def test_a_forward_that_is_refused_keeps_the_last_ones_layout(streams, monkeypatch):
    """A backward may still follow the forward before it, and reads that one's
    positions and layout: they stay allocated."""
    torch, stream, _ = streams
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self: self)
    m = _bare_qwen3(torch, stream)
    ids = torch.zeros(1, 192, dtype=torch.int64)
    m.set_layout(100, [92])
    first = m._plan
    m.forward(ids, ids)
    m.set_layout(90, [102])
    with pytest.raises(AttributeError):
        m.forward("not a tensor")
    assert m._in_use[1] is first
    refuse = _Library()
    refuse.qwen3_forward = lambda *args: INVALID
    refuse.qwen3_last_error = lambda h: b"refused"
    monkeypatch.setattr(qb, "lib", lambda: refuse)
    with pytest.raises(binding.LibError):
        m.forward(ids, ids)
    assert m._in_use[1] is first
    monkeypatch.setattr(qb, "lib", _Library)
    m.forward(ids, ids)
    assert m._in_use[1] is m._plan is not first


# ---- workspace of matrices that a workgroup holds in LDS

@pytest.mark.parametrize("rows,cols", [(16, 16), (16, 1024), (128, 128), (64, 256), (1024, 32)])
def test_matrices_that_stay_in_lds_take_no_planes(rows, cols):
    """The size does not grow with their number, and is small against one of them."""
    one = binding.orthogonalise_size(rows, cols, 1)
    assert 0 < one == binding.orthogonalise_size(rows, cols, 100000) <= max(256, rows * cols)


def test_muon_size_leaves_out_the_small_adapters():
    """Ranks and widths of the small test model: everything stays in LDS but
    what its width forbids, whose planes are counted."""
    n = ctypes.c_size_t()
    w = dict(synth.QWEN3_WORKLOADS["qwen3_tiny"], lora_rank=8)
    q = qb.make_config(w, synth.QWEN3_OPTIM)
    assert qb.lib().qwen3_muon_size(ctypes.byref(q), ctypes.byref(n)) == 0
    assert n.value < 64 << 10
    # rank 32 and 1,280 rows of gate and up: past what LDS holds
    q = qb.make_config(dict(w, lora_rank=32, d_ff=1280), synth.QWEN3_OPTIM)
    assert qb.lib().qwen3_muon_size(ctypes.byref(q), ctypes.byref(n)) == 0
    L = w["n_layer"]
    # two matrices a layer of gate and up's B and one of down's A: four planes of X and of the Gram size, 64 rows padded
    assert 3 * L * 8 * 64 * (1280 + 64) <= n.value < 3 * L * 8 * 64 * (1280 + 64) + (64 << 10)


def test_a_long_walk_is_shared_out_among_many_short_ones():
    """2.2 million sequences of one token: the walk of the prefix' keys over all
    of them is 34,375 tiles beside 17,188 walks of two or three."""
    n = 2200000
    st, size = prefix_size([1] * n, n_head=1, n_kv_head=1, head_dim=64, prefix_queries=0)
    # tables and the backward's D, 16 bytes a token, and the partial results of 64 workgroups or more
    assert st == 0 and size >= 16 * n + 64 * 2 * 128 * 64 * 4


# ---- results that lie over what is still read

@pytest.mark.parametrize("x,y", [(4096, 4100), (4100, 4096), (4096, 4096 + 8 * 8 * 3 * 4 - 4)])
def test_orthogonalise_refuses_partial_overlap(x, y):
    L = binding.lib()
    assert L.gpt2_orthogonalise(x, y, 8, 8, 3, 5, 1 << 20, 1 << 30, None) == INVALID
    assert "overlap" in L.gpt2_last_error(None).decode()


@pytest.mark.parametrize("out", [(1 << 20) + 16, (1 << 20) - 16])
def test_rotary_refuses_partial_overlap(out):
    L, d = qb.lib(), rotary_desc()
    base, far, pos, gain = 1 << 20, 1 << 22, 4096, 8192
    calls = (lambda: L.qwen3_rotary_forward(ctypes.byref(d), base, pos, gain, gain, out, None),
             lambda: L.qwen3_rotary_backward(ctypes.byref(d), base, far, pos, gain, gain, out, None),
             lambda: L.qwen3_rotary_backward(ctypes.byref(d), far, base, pos, gain, gain, out, None))
    for call in calls:
        assert call() == INVALID
        assert "overlap" in L.qwen3_last_error(None).decode()


# ---- numbers as the bindings take them

@pytest.mark.parametrize("call", [
    lambda: binding.orthogonalise_size(2 ** 32 + 8, 8),
    lambda: binding.orthogonalise_size(8, 8, 2 ** 32 + 1),
    lambda: qb.SharedPrefix(4, 2, 128, 2 ** 32 + 100, [5]),
    lambda: qb.SharedPrefix(4, 2, 128, 100, [2 ** 32 + 5]),
    lambda: qb.SharedPrefix(2 ** 32 + 4, 2, 128, 100, [5]),
    lambda: qb._rotary_desc(8, 4, 2, 1024, (2 ** 32 + 64,), False, 1e6, 1e-6),
    lambda: binding.muon_settings(0.9, True, 2 ** 32 + 5, 0.2)])
def test_integers_past_32_bits_are_not_cut_off(call):
    with pytest.raises(ValueError, match="32 bits"):
        call()


def test_a_rotary_description_is_made_of_the_numbers_it_was_given(monkeypatch):
    """Descriptions are kept by their values: one of a tensor that has changed is another."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(qb, "_device_rows", lambda *a, **kw: a[0])
    x, pos = torch.zeros(4, 8 * 128, dtype=torch.bfloat16), torch.zeros(1, 4, dtype=torch.int32)
    theta, eps, section = torch.tensor(1e4), torch.tensor(1e-6), torch.tensor(64)
    made = []
    for _ in range(2):
        r = qb._rotary_args(x, pos, 4, 2, (section, 0), theta, None, None, eps, False)._obj
        made.append((r.theta, r.rms_eps, r.sections[0]))
        theta.mul_(4)
        eps.mul_(4)
        section.sub_(1)
    assert made[0] == (1e4, ctypes.c_float(1e-6).value, 64) and made[1] == (4e4, ctypes.c_float(4e-6).value, 63)
