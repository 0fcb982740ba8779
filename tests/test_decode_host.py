"""Host-side checks of the entry points of the paged cache, the attention over
it and the adjustment of logits: what the header declares is exported, sizes are
as documented, and malformed requests are refused before anything is launched
(no GPU here: a call that got through would fail with a device error instead)."""
import ctypes
import os
import re

import pytest

from paper_2609_28568_amd import binding, decode_binding as db, qwen3_binding as qb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID = binding.GPT2_ERR_INVALID_ARG
FAR = 1 << 50   # addresses that nothing else uses


def header():
    text = open(os.path.join(ROOT, "include", "qwen3_decode.h")).read()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_library_exports_the_header():
    names = sorted(set(re.findall(r"\b(qwen3_[a-z_0-9]+)\s*\(", header())))
    assert len(names) >= 7
    for n in names:
        assert hasattr(db.lib(), n), n


@pytest.mark.parametrize("name,struct", [("qwen3_cache", db.Cache), ("qwen3_tree", db.Tree),
                                         ("qwen3_logits", db.Logits)])
def test_structs_match_the_header(name, struct):
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), header(), re.S).group(1)
    fields = []
    for decl in body.split(";"):
        decl = decl.replace("const ", "").strip()
        if decl:
            fields += [f.replace("*", "").strip() for f in decl.split(None, 1)[1].split(",")]
    assert fields == [f for f, _ in struct._fields_]


def why():
    return qb.lib().qwen3_last_error(None).decode()


def cache(**over):
    d = dict(n_layer=2, n_kv_head=2, head_dim=128, page_size=16, n_pages=64, n_seq=4, max_pages=16, d_pages=FAR,
             d_table=FAR + (1 << 40), d_lens=FAR + (2 << 40), d_refs=FAR + (3 << 40), d_short=FAR + (4 << 40),
             d_scratch=FAR + (5 << 40))
    d.update(over)
    return db.Cache(**d)


BAD_SIZES = [(dict(head_dim=96), "head_dim"), (dict(head_dim=0), "head_dim"), (dict(page_size=8), "page_size"),
             (dict(page_size=24), "page_size"), (dict(page_size=512), "page_size"), (dict(page_size=-16), "page_size"),
             (dict(n_layer=0), "n_layer"), (dict(n_kv_head=0), "n_kv_head"), (dict(n_kv_head=4097), "n_kv_head"),
             (dict(n_pages=0), "n_pages"), (dict(n_pages=1 << 28), "n_pages"), (dict(n_seq=0), "n_seq"),
             (dict(n_seq=4097), "n_seq"), (dict(max_pages=0), "max_pages"), (dict(max_pages=1 << 27), "max_pages")]
BAD_BUFFERS = [(dict(d_pages=0), "null"), (dict(d_table=0), "null"), (dict(d_lens=0), "null"), (dict(d_refs=0), "null"),
               (dict(d_short=0), "null"), (dict(d_scratch=0), "null"), (dict(d_pages=FAR + 8), "aligned"),
               (dict(d_table=FAR + 2), "aligned"), (dict(d_scratch=FAR + 4), "aligned")]


@pytest.mark.parametrize("over,reason", BAD_SIZES + BAD_BUFFERS)
def test_a_cache_is_refused(over, reason):
    L, c, t = db.lib(), cache(**over), db.Tree(4, 8, 8, 0, 0)
    ref = ctypes.byref(c)
    n = ctypes.c_size_t()
    calls = [lambda: L.qwen3_cache_fork(ref, 4096, None, None),
             lambda: L.qwen3_cache_append(ref, 4096, 4, 8, 0, 4096, None, None, 8, None),
             lambda: L.qwen3_cache_compact(ref, None),
             lambda: L.qwen3_tree_attention(ref, ctypes.byref(t), 4096, 4096, None, 1 << 20, None, 1 << 21, 1 << 40, None)]
    if (over, reason) in BAD_SIZES:
        calls += [lambda: L.qwen3_cache_scratch(ref, ctypes.byref(n)),
                  lambda: L.qwen3_tree_size(ref, ctypes.byref(t), ctypes.byref(n))]
    for call in calls:
        assert call() == INVALID
        assert reason in why()


def test_null_descriptions():
    L, n, c = db.lib(), ctypes.c_size_t(), cache()
    assert L.qwen3_cache_scratch(None, ctypes.byref(n)) == INVALID
    assert L.qwen3_cache_scratch(ctypes.byref(c), None) == INVALID
    assert L.qwen3_cache_fork(None, 4096, None, None) == INVALID
    assert L.qwen3_cache_fork(ctypes.byref(c), None, None, None) == INVALID
    assert L.qwen3_cache_compact(None, None) == INVALID
    assert L.qwen3_tree_size(ctypes.byref(c), None, ctypes.byref(n)) == INVALID
    assert L.qwen3_tree_size(ctypes.byref(c), ctypes.byref(db.Tree(4, 8, 8, 0, 0)), None) == INVALID
    assert L.qwen3_adjust_logits(None, 4096, 4096, None) == INVALID


def test_sizes():
    L, n = db.lib(), ctypes.c_size_t()
    assert L.qwen3_cache_scratch(ctypes.byref(cache()), ctypes.byref(n)) == 0
    assert n.value >= 4 * (4 * 4 + 2 * 64)

    def tree(words=0, c=None, **over):
        d = dict(n_head=4, n_rows=64, max_new=1, layer=0, mask_words=words)
        d.update(over)
        assert L.qwen3_tree_size(ctypes.byref(c or cache(max_pages=512)), ctypes.byref(db.Tree(**d)), ctypes.byref(n)) == 0
        return n.value

    # partial results of as many rows as a sequence's tokens have, and none for short sequences
    assert tree() < tree(max_new=16) < tree(max_new=64)
    assert tree(c=cache(max_pages=4)) < 4096
    assert tree(n_rows=0) > 0


@pytest.mark.parametrize("over,reason", [
    (dict(n_head=0), "n_head"), (dict(n_head=3), "n_head"), (dict(n_head=8192), "n_head"), (dict(n_rows=-1), "n_rows"),
    (dict(n_rows=1 << 28), "n_rows"), (dict(n_rows=1 << 24), "2^26"), (dict(max_new=0), "max_new"), (dict(max_new=-1), "max_new"),
    (dict(layer=-1), "layer"), (dict(layer=2), "layer")])
def test_tree_descriptions_are_refused(over, reason):
    d = dict(n_head=4, n_rows=8, max_new=8, layer=0, mask_words=0)
    d.update(over)
    t, n, L = db.Tree(**d), ctypes.c_size_t(), db.lib()
    assert L.qwen3_tree_size(ctypes.byref(cache()), ctypes.byref(t), ctypes.byref(n)) == INVALID and reason in why()
    assert L.qwen3_tree_attention(ctypes.byref(cache()), ctypes.byref(t), 4096, 4096, None, 1 << 20, None, 1 << 21,
                                  1 << 40, None) == INVALID
    assert reason in why()


def test_tiles_past_32_bits_are_refused():
    t, n = db.Tree(64, 1 << 19, 1 << 19, 0, 0), ctypes.c_size_t()
    c = cache(n_seq=4096, max_pages=1 << 20, n_kv_head=2)
    assert db.lib().qwen3_tree_size(ctypes.byref(c), ctypes.byref(t), ctypes.byref(n)) == INVALID
    assert "too many or too long" in why()


# qkv, starts, mask, out, lse, workspace, workspace bytes
GOOD = (1 << 24, 1 << 25, 1 << 26, 1 << 27, 1 << 28, 1 << 29, 1 << 28)


@pytest.mark.parametrize("at,value,reason", [
    (0, 0, "null"), (1, 0, "null"), (3, 0, "null"), (0, (1 << 24) + 8, "aligned"), (1, (1 << 25) + 2, "aligned"),
    (2, (1 << 26) + 2, "aligned"), (3, (1 << 27) + 8, "aligned"), (4, (1 << 28) + 2, "aligned"), (5, 0, "workspace"),
    (5, (1 << 29) + 128, "workspace"), (6, 16, "workspace"),
    (3, (1 << 24) + 16, "overlap"), (3, 1 << 25, "overlap"), (3, 1 << 26, "overlap"), (3, 1 << 28, "overlap"),
    (3, 1 << 29, "overlap"), (3, FAR + 4096, "overlap"), (3, FAR + (1 << 40), "overlap"),
    (3, FAR + (2 << 40), "overlap"), (4, 1 << 24, "overlap"), (4, 1 << 25, "overlap"), (4, (1 << 27) + 64, "overlap"),
    (4, FAR, "overlap"), (4, FAR + (2 << 40) + 4, "overlap")])
def test_attention_refuses_arguments(at, value, reason):
    args = list(GOOD)
    args[at] = value
    t = db.Tree(4, 8, 8, 1, 1)
    assert db.lib().qwen3_tree_attention(ctypes.byref(cache()), ctypes.byref(t), *args, None) == INVALID
    assert reason in why()


def test_attention_refuses_a_mask_without_words():
    t = db.Tree(4, 8, 8, 1, 0)
    assert db.lib().qwen3_tree_attention(ctypes.byref(cache()), ctypes.byref(t), *GOOD, None) == INVALID
    assert "mask_words" in why()


def test_attention_of_no_rows_does_nothing():
    t = db.Tree(4, 0, 1, 0, 0)
    assert db.lib().qwen3_tree_attention(ctypes.byref(cache()), ctypes.byref(t), None, None, None, None, None, 1 << 29,
                                         1 << 30, None) == 0


@pytest.mark.parametrize("over,reason", [
    (dict(qkv=0), "null"), (dict(starts=0), "null"), (dict(n_head=3), "n_head"), (dict(n_rows=-1), "n_rows"),
    (dict(max_new=0), "max_new"), (dict(max_new=1 << 24), "max_new"), (dict(stride=12), "layer_stride"),
    (dict(stride=(1 << 40) + 8), "layer_stride"), (dict(path=1 << 20), "counts"), (dict(qkv=4104), "aligned"),
    (dict(starts=4098), "aligned"), (dict(counts=2), "aligned"), (dict(counts=1 << 20, path=(1 << 21) + 1), "aligned"),
    (dict(qkv=FAR + 64), "overlap"), (dict(starts=FAR + (1 << 40) + 8), "overlap"),
    (dict(counts=FAR + (2 << 40)), "overlap"), (dict(counts=1 << 20, path=FAR + (3 << 40)), "overlap")])
def test_append_refuses_arguments(over, reason):
    d = dict(qkv=4096, n_head=4, n_rows=8, stride=8 * 8 * 128, starts=1 << 22, counts=None, path=None, max_new=8)
    d.update(over)
    assert db.lib().qwen3_cache_append(ctypes.byref(cache()), *d.values(), None) == INVALID
    assert reason in why()


@pytest.mark.parametrize("src,keep,reason", [(4098, None, "aligned"), (4096, 2, "aligned"), (FAR + (2 << 40), None, "overlap"),
                                             (4096, FAR + (1 << 40) + 64, "overlap"), (FAR + (3 << 40), None, "overlap")])
def test_fork_refuses_arguments(src, keep, reason):
    assert db.lib().qwen3_cache_fork(ctypes.byref(cache()), src, keep, None) == INVALID
    assert reason in why()


@pytest.mark.parametrize("over,reason", [
    (dict(rows=-1), "rows"), (dict(rows=65536), "rows"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 26) + 1), "vocab"),
    (dict(dtype=2), "dtype"), (dict(logits_stride=99), "stride"), (dict(out_stride=99), "stride"),
    (dict(logits_stride=1 << 41), "stride"), (dict(n_bias=-1), "n_bias"), (dict(n_bias=1025), "n_bias"),
    (dict(n_bias=1), "null biases"), (dict(n_masks=-1), "n_masks"), (dict(n_masks=1), "null masks"),
    (dict(path_len=-1), "path_len"), (dict(path_len=1), "null path"), (dict(d_history=4096), "history"),
    (dict(d_history=4096, n_seq=1, history_stride=5), "history"), (dict(d_repetition=4097), "aligned"),
    (dict(d_history=4096, n_seq=1, history_stride=5, d_lens=4098), "aligned"), (dict(logits=0), "null"),
    (dict(out=0), "null"), (dict(logits=4097), "aligned"), (dict(out=(1 << 20) + 1), "aligned"),
    (dict(out=4096 + 2), "overlap"), (dict(out=4096, out_stride=101), "in place"), (dict(out=4096 + 3 * 200), "overlap"),
    (dict(d_presence=(1 << 20) + 4), "overlap"), (dict(n_masks=1, d_masks=1 << 20), "overlap"),
    (dict(d_history=(1 << 20) - 16, n_seq=1, history_stride=5, d_lens=4096), "overlap")])
def test_logits_refuse_arguments(over, reason):
    d = dict(rows=4, vocab=100, dtype=1, logits_stride=100, out_stride=100)
    args = dict(logits=4096, out=1 << 20)
    for k, v in over.items():
        (args if k in args else d)[k] = v
    assert db.lib().qwen3_adjust_logits(ctypes.byref(db.Logits(**d)), args["logits"], args["out"], None) == INVALID
    assert reason in why()


def test_bindings_refuse_tensors():
    torch = pytest.importorskip("torch")
    pages, i = torch.zeros(1, 4, 2, 1, 16, 64, dtype=torch.bfloat16), lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError):
        db.PagedCache(pages, i(2, 4), i(2), i(4), i(1))   # not on a device
    for x in (torch.zeros(2, 8), torch.zeros(8), "x"):
        with pytest.raises(ValueError):
            db.adjust_logits(x)
    with pytest.raises(ValueError, match="parent"):
        db.tree_mask([[-1, 1]], device="cpu")


def test_tree_masks():
    torch = pytest.importorskip("torch")
    m = db.tree_mask([[-1, 0, 0, 1], [], [-1] * 2 + list(range(1, 39))], device="cpu")
    assert m.shape == (44, 2) and m[:4, 0].tolist() == [1, 3, 5, 11] and not m[:4, 1].any()
    assert m[4:6, 0].tolist() == [1, 2]
    # a chain from token 1 on
    assert m[43].tolist() == [torch.tensor(-2, dtype=torch.int32).item(), 255]


# ---- positions, and the cache in the model

@pytest.mark.parametrize("starts,mask,words,out,reason", [
    (0, None, 0, 1 << 24, "null"), (4096, None, 0, 0, "null"), (4098, None, 0, 1 << 24, "aligned"),
    (4096, 2, 1, 1 << 24, "aligned"), (4096, None, 0, (1 << 24) + 1, "aligned"), (4096, 1 << 20, 0, 1 << 24, "mask_words"),
    (4096, None, 0, 4100, "overlap"), (4096, 1 << 20, 2, (1 << 20) + 60, "overlap"),
    (4096, None, 0, FAR + (2 << 40), "overlap")])
def test_positions_refuse_arguments(starts, mask, words, out, reason):
    t = db.Tree(4, 8, 8, 0, words)
    assert db.lib().qwen3_tree_positions(ctypes.byref(cache()), ctypes.byref(t), starts, mask, out, None) == INVALID
    assert reason in why()


def test_calls_without_a_model():
    L, n, r = db.lib(), ctypes.c_size_t(), ctypes.c_int32()
    assert L.qwen3_set_cache_size(None, ctypes.byref(cache()), 1, ctypes.byref(n)) == INVALID
    assert L.qwen3_set_cache(None, ctypes.byref(cache()), 4096, None, 0, 1, 4096, 1 << 30) == INVALID
    assert L.qwen3_keep_tokens(None, None, None, 1) == INVALID
    assert L.qwen3_logits_info(None, ctypes.byref(n), ctypes.byref(r)) == INVALID


def test_what_a_call_writes_may_not_be_its_input():
    """The scratch and the count of missing pages are written too."""
    L = db.lib()
    for at in (FAR + (4 << 40), FAR + (5 << 40) + 64):
        assert L.qwen3_cache_fork(ctypes.byref(cache()), at, None, None) == INVALID and "overlap" in why()
        assert L.qwen3_cache_append(ctypes.byref(cache()), 4096, 4, 8, 0, at, None, None, 8, None) == INVALID
        assert "overlap" in why()


@pytest.mark.parametrize("shape", [(3, 0), (0, 0), (3,), (3, 1, 1)])
def test_masks_without_words_are_refused(shape):
    """An empty tensor's address is null, which would mean no mask."""
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="word"):
        db.mask_words(torch.zeros(*shape, dtype=torch.int32))
    assert db.mask_words(torch.zeros(0, 2, dtype=torch.int32)) == 2


@pytest.mark.parametrize("n_seq,max_new,path,reason", [
    (4096, 8192, None, None), (4096, (1 << 22) - 1, None, None), (1, (1 << 25) - 1, None, None), (8, (1 << 22) - 1, None, None),
    (8, 1 << 22, None, "max_new"), (1, 1 << 25, None, "max_new"), (4096, 8191, 1 << 21, None), (4096, 8192, 1 << 21, "max_new")])
def test_appends_of_one_long_piece_among_many_sequences(n_seq, max_new, path, reason):
    """Without a path the rows bound the work, not n_seq * max_new: what is taken
    gets as far as the overlap of its counts with the cache's lengths."""
    c = cache(n_seq=n_seq)
    counts = FAR + (2 << 40)
    assert db.lib().qwen3_cache_append(ctypes.byref(c), 4096, 4, 8, 0, 1 << 22, counts, path, max_new, None) == INVALID
    assert (reason or "overlap") in why()


def test_tiles_are_bounded_by_the_rows():
    """4,096 sequences of up to 131,072 tokens, one of them with a piece of a prompt
    of 4,096: not as if all of them had one."""
    c, n, L = cache(n_kv_head=8, n_seq=4096, max_pages=8192), ctypes.c_size_t(), db.lib()
    assert L.qwen3_tree_size(ctypes.byref(c), ctypes.byref(db.Tree(16, 8191, 4096, 0, 0)), ctypes.byref(n)) == 0
    assert n.value > 0
    c.max_pages, t = 1 << 15, db.Tree(16, (1 << 22) - 1, 4096, 0, 0)   # 69,632 blocks of 8,256 tiles, 8 heads
    assert L.qwen3_tree_size(ctypes.byref(c), ctypes.byref(t), ctypes.byref(n)) == INVALID
    assert "too many or too long" in why()


def test_a_cache_on_another_device_than_the_model_is_refused():
    """Its addresses would be another card's."""
    torch = pytest.importorskip("torch")
    from types import SimpleNamespace
    m = qb.Qwen3.__new__(qb.Qwen3)
    m.bufs, m.cfg = {"workspace": torch.zeros(1)}, SimpleNamespace(B=1, T=64)
    c = SimpleNamespace(pages=torch.empty(1, 4, 2, 1, 16, 64, device="meta"), lens=torch.zeros(3, dtype=torch.int32, device="meta"))
    with pytest.raises(ValueError, match="device"):
        m.set_cache(c, torch.zeros(4, dtype=torch.int32))
