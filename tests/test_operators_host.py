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
                                   (64, 64, 1 << 30)])
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
