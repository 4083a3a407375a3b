"""What the operators refuse, and their sizes: host checks of the C ABI, which end before anything touches a device."""
import ctypes as C

import pytest

from paper_2509_24007_amd import sdlm

P = 0x10000      # a pointer that nothing follows: every call here is refused


def kv(**kw):
    base = dict(pool=P, layer_stride=8 * 2 * 2 * 16 * 64, n_layers=2, n_tiles=8, n_kv_heads=2, head_dim=64, dtype=1, n_pages=6, max_seqs=4, pages_per_seq=3, page_table=P, lengths=P,
                backed=P, page_refs=P, free_pages=P, free_count=P)
    return sdlm.KvDesc(**{**base, **kw})


def refused(rc, code, word):
    assert rc == code
    assert word in sdlm.load().sdlm_op_error().decode()


def sample_args(**kw):
    base = dict(logits=P, row_stride=100, dtype=0, rows=3, vocab=100, u=P, ids=P)
    return sdlm.SampleArgs(**{**base, **kw})


@pytest.mark.parametrize("kw,word", [(dict(rows=-1), "rows"), (dict(vocab=0), "vocab"), (dict(vocab=1 << 20, row_stride=1 << 20), "vocab"), (dict(dtype=2), "dtype"),
                                     (dict(row_stride=99), "row_stride"), (dict(logits=None), "required"), (dict(u=None), "required"), (dict(ids=None), "required"),
                                     (dict(logits=P + 2), "aligned")])
def test_sample_refuses(kw, word):
    refused(sdlm.load().sdlm_sample(C.byref(sample_args(**kw)), P, 1 << 30, None), sdlm.EINVAL, word)


def test_sample_workspace():
    L = sdlm.load()
    assert L.sdlm_sample_workspace_bytes(-1, 10) == 0 and L.sdlm_sample_workspace_bytes(1, 0) == 0 and L.sdlm_sample_workspace_bytes(1, (1 << 19) + 1) == 0
    need = L.sdlm_sample_workspace_bytes(3, 100)
    assert need > 0
    refused(L.sdlm_sample(C.byref(sample_args()), P, need - 1, None), sdlm.ECAPACITY, "workspace")
    refused(L.sdlm_sample(C.byref(sample_args()), P + 16, need, None), sdlm.EINVAL, "workspace")
    refused(L.sdlm_sample(C.byref(sample_args()), None, need, None), sdlm.EINVAL, "workspace")
    refused(L.sdlm_sample(None, P, need, None), sdlm.EINVAL, "null")
    assert L.sdlm_sample(C.byref(sample_args(rows=0)), None, 0, None) == 0      # nothing to draw


BAD_KV = [(dict(pool=None), "pool"), (dict(pool=P + 8), "pool"), (dict(dtype=3), "dtype"), (dict(head_dim=48), "head_dim"), (dict(n_layers=0), "sizes"), (dict(n_kv_heads=0), "sizes"),
          (dict(max_seqs=0), "sizes"), (dict(pages_per_seq=0), "sizes"), (dict(layer_stride=100), "layer_stride"), (dict(layer_stride=8 * 2 * 2 * 16 * 64 + 4), "layer_stride"),
          (dict(page_table=None), "page_table"), (dict(lengths=None), "lengths")]


@pytest.mark.parametrize("kw,word", BAD_KV + [(dict(n_pages=0), "n_pages"), (dict(n_pages=9), "n_pages"), (dict(backed=None), "backed"), (dict(page_refs=None), "page_refs"),
                                              (dict(free_pages=None), "free_pages"), (dict(free_count=None), "free_count")])
def test_fork_refuses_bad_caches(kw, word):
    L = sdlm.load()
    refused(L.sdlm_kv_fork(C.byref(kv(**kw)), P, 2, 1, P, P, 1 << 30, None), sdlm.EINVAL, word)
    assert L.sdlm_kv_fork_workspace_bytes(C.byref(kv(**kw))) == 0


def test_fork_refuses():
    L = sdlm.load()
    need = L.sdlm_kv_fork_workspace_bytes(C.byref(kv()))
    assert need > 0
    for n, parent, status, ws, size, code, word in [(5, P, P, P, need, sdlm.EINVAL, "room"), (-1, P, P, P, need, sdlm.EINVAL, "room"), (2, None, P, P, need, sdlm.EINVAL, "parent"),
                                                    (2, P, None, P, need, sdlm.EINVAL, "status"), (2, P, P, P, need - 1, sdlm.ECAPACITY, "workspace"), (2, P, P, P + 8, need, sdlm.EINVAL, "workspace")]:
        refused(L.sdlm_kv_fork(C.byref(kv()), parent, n, 1, status, ws, size, None), code, word)
    refused(L.sdlm_kv_fork(None, P, 1, 1, P, P, need, None), sdlm.EINVAL, "null")


@pytest.mark.parametrize("kw,word", BAD_KV)
def test_compact_and_tree_refuse_bad_caches(kw, word):
    L = sdlm.load()
    refused(L.sdlm_kv_compact(C.byref(kv(**kw)), 2, P, 4, P, 4, P, 1, None, None), sdlm.EINVAL, word)
    refused(L.sdlm_tree_attention(C.byref(kv(**kw)), 0, C.byref(tree()), P, 1 << 30, None), sdlm.EINVAL, word)
    assert L.sdlm_tree_attention_workspace_bytes(C.byref(kv(**kw)), 4, 2, 8, 0) == 0


def test_compact_refuses():
    L = sdlm.load()
    for args, word in [((5, P, 4, P, 4, P, 1), "sequences"), ((-1, P, 4, P, 4, P, 1), "sequences"), ((2, P, 3, P, 4, P, 1), "path_stride"), ((2, P, 4, P, -1, P, 1), "max_path"),
                       ((2, P, 4, P, 4, P, 0), "node_pages"), ((2, None, 4, P, 4, P, 1), "required"), ((2, P, 4, None, 4, P, 1), "required"), ((2, P, 4, P, 4, None, 1), "required")]:
        refused(L.sdlm_kv_compact(C.byref(kv()), *args, None, None), sdlm.EINVAL, word)
    assert L.sdlm_kv_compact(C.byref(kv()), 0, None, 0, None, 0, None, 1, None, None) == 0


def tree(**kw):
    base = dict(q=P, out=P, q_stride=256, out_stride=256, n_rows=10, n_seqs=2, n_q_heads=4, max_nodes=8, max_len=0, node_offsets=P, mask=P, mask_words=1, node_pages=1, node_table=P)
    return sdlm.TreeArgs(**{**base, **kw})


@pytest.mark.parametrize("kw,word", [(dict(n_q_heads=3), "n_q_heads"), (dict(n_q_heads=0), "n_q_heads"), (dict(max_nodes=0), "max_nodes"), (dict(max_nodes=1025, mask_words=17), "max_nodes"),
                                     (dict(n_seqs=5), "sequences"), (dict(n_seqs=-1), "n_seqs"), (dict(max_len=-1), "max_len"), (dict(n_rows=17), "rows"), (dict(n_rows=-1), "rows"),
                                     (dict(mask_words=0), "mask_words"), (dict(max_nodes=65, mask_words=1), "mask_words"), (dict(node_pages=0), "node_pages"), (dict(q_stride=248), "q_stride"),
                                     (dict(out_stride=257), "out_stride"), (dict(q=None), "required"), (dict(mask=None), "required"), (dict(node_table=None), "required"),
                                     (dict(node_offsets=None), "required"), (dict(out=P + 4), "aligned")])
def test_tree_attention_refuses(kw, word):
    refused(sdlm.load().sdlm_tree_attention(C.byref(kv()), 0, C.byref(tree(**kw)), P, 1 << 30, None), sdlm.EINVAL, word)


def test_tree_attention_layer_and_workspace():
    L = sdlm.load()
    for layer in (-1, 2):
        refused(L.sdlm_tree_attention(C.byref(kv()), layer, C.byref(tree()), P, 1 << 30, None), sdlm.EINVAL, "layer")
    need = L.sdlm_tree_attention_workspace_bytes(C.byref(kv()), 4, 2, 8, 0)
    assert need > 0
    refused(L.sdlm_tree_attention(C.byref(kv()), 0, C.byref(tree()), P, need - 1, None), sdlm.ECAPACITY, "workspace")
    assert L.sdlm_tree_attention(C.byref(kv()), 0, C.byref(tree(n_rows=0)), None, 0, None) == 0


@pytest.mark.parametrize("dtype,d,heads", [(0, 128, 600), (0, 32, 900), (1, 64, 400), (1, 128, 1200)])
def test_a_context_lends_the_trees_a_run_of_every_kv_head(dtype, d, heads):
    """Beyond a fixed room, a further kv head takes the places of a run's two parts as well: 64 queries (bf16: 128) with a sum of d and two numbers each."""
    def total(h):
        m = sdlm.ModelCfg(1, 64, h, h, d, 64, 300, 1e4, 1e-6, 1.0, dtype, 299, 0, 0)
        return sdlm.load().sdlm_workspace_bytes(C.byref(m), C.byref(sdlm.RunCfg(1, 64, 4, 0, 16, 0, 0.5, 0, 0, 32)))
    assert total(heads + 2) - total(heads) >= total(12) - total(10) + 2 * 2 * 64 * (1 + dtype) * (4 * d + 8)


BIG = 1 << 50      # a layer stride that holds anything


def test_sizes_beyond_a_launch_are_refused():
    """Grids and their threads have 16 and 32 bits: what does not fit is refused before the first launch."""
    L = sdlm.load()
    for rows, vocab in ((1 << 21, 10), ((1 << 20) + 1, 10), (1 << 20, 1 << 19)):
        assert L.sdlm_sample_workspace_bytes(rows, vocab) == 0
        refused(L.sdlm_sample(C.byref(sample_args(rows=rows, vocab=vocab, row_stride=vocab)), P, 1 << 62, None), sdlm.EINVAL, "rows")
    assert L.sdlm_sample_workspace_bytes(1 << 20, 10) > 0
    for kw, word in ((dict(n_kv_heads=65536, layer_stride=BIG), "heads"), (dict(n_layers=1 << 10, n_kv_heads=1 << 14, layer_stride=BIG), "layers"), (dict(max_seqs=(1 << 20) + 1), "max_seqs")):
        refused(L.sdlm_kv_fork(C.byref(kv(**kw)), P, 2, 1, P, P, 1 << 62, None), sdlm.EINVAL, word)
        refused(L.sdlm_kv_compact(C.byref(kv(**kw)), 2, P, 4, P, 4, P, 1, None, None), sdlm.EINVAL, word)
        refused(L.sdlm_tree_attention(C.byref(kv(**kw)), 0, C.byref(tree()), P, 1 << 62, None), sdlm.EINVAL, word)
    refused(L.sdlm_tree_attention(C.byref(kv()), 0, C.byref(tree(n_q_heads=65536, q_stride=BIG, out_stride=BIG)), P, 1 << 62, None), sdlm.EINVAL, "n_q_heads")
    assert L.sdlm_tree_attention_workspace_bytes(C.byref(kv(max_seqs=1 << 20, pages_per_seq=1)), 4, 1 << 20, 1024, 0) == 0


def test_largest_sample():
    """rows * ceil((vocab + 7) / 16384) below 2^24, as the header says."""
    need = sdlm.load().sdlm_sample_workspace_bytes
    assert need(1 << 20, 15 * 16384 - 7) > 0 and need(1 << 20, 15 * 16384 - 6) == 0
    assert need(508400, 1 << 19) > 0 and need(508401, 1 << 19) == 0      # 33 pieces a row


def test_struct_sizes_agree_with_the_header():
    """Sizes of the argument structs as a C compiler lays them out on this ABI."""
    assert C.sizeof(sdlm.SampleArgs) == 88 and C.sizeof(sdlm.KvDesc) == 96 and C.sizeof(sdlm.TreeArgs) == 96
