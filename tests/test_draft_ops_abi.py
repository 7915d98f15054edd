"""Refusals of the speculative decoding step's operators: found on the host before any device work, so they run without a
GPU (the pointers are stand-ins and never dereferenced), and the sizes of their workspaces."""

import ctypes
import os

import pytest

P = ctypes.c_void_p
BASE = 1 << 20  # a stand-in device address, 16-byte aligned

POINTERS = {"qkv_f32", "qkv_bf16", "q_gain", "k_gain", "rope", "pos", "slot", "q", "kv", "src", "dst", "offsets", "cu_q", "ctx",
            "mask", "block_tables", "out", "workspace", "logits", "temperature", "top_k", "top_p", "min_p", "u", "prob", "stream"}


@pytest.fixture(scope="module")
def metro(repo_root):
    if not os.path.exists(os.path.join(repo_root, "paper_2411_03519_amd", "libmetro.so")):
        pytest.skip("libmetro.so not built")
    from paper_2411_03519_amd import metro
    return metro


def call(metro, name, args):
    return getattr(metro.lib, name)(*[P(v) if k in POINTERS else v for k, v in args.items()])


def refused(metro, name, good, changes, word):
    """Every change of the good call is refused with E_INVAL and a message that names the operator."""
    for change in changes:
        assert call(metro, name, {**good, **change}) == -1, (name, change)
        msg = metro.lib.metro_last_error()
        assert word in msg, (name, change, msg)


def nulls(*names):
    return [{n: None} for n in names]


def off(by, *names):
    return [{n: BASE + by} for n in names]


APPEND = dict(qkv_f32=BASE, qkv_bf16=None, ld=1024, T=3, nq=8, nkv=4, hd=64, q_gain=BASE, k_gain=BASE, eps=1e-5, rope=BASE,
              n_pos=64, pos=BASE, slot=BASE, q=BASE, kv=BASE, n_pages=9, stream=None)
MOVE = dict(kv=BASE, layer_stride=9 * 2 * 4 * 16 * 64, n_layers=2, n_pages=9, nkv=4, hd=64, src=BASE, dst=BASE, offsets=BASE,
            n_groups=1, n_moves=3, stream=None)
TREE = dict(q=BASE, kv=BASE, n_pages=9, nq=8, nkv=4, hd=64, n_items=2, cu_q=BASE, rows=5, ctx=BASE, max_q=40, max_keys=64,
            mask=BASE, ldm=2, block_tables=BASE, ldb=4, out=BASE, workspace=BASE, workspace_bytes=1024, stream=None)
SAMPLE = dict(logits=BASE, ldl=101, rows=3, vocab=101, temperature=None, top_k=None, top_p=None, min_p=None, u=BASE, out=BASE,
              prob=None, workspace=BASE, workspace_bytes=1 << 40, stream=None)
CACHE = [{"hd": 32}, {"hd": 0}, {"hd": 256}, {"nkv": 0}, {"nkv": -1}, {"nkv": 257}, {"n_pages": 0}, {"n_pages": 1 << 27}] + off(8, "kv")


def test_rope_append_refusals(metro):
    refused(metro, "metro_op_rope_append", APPEND, CACHE + nulls("qkv_f32", "rope", "pos", "slot", "q", "kv") +
            off(8, "qkv_f32", "q_gain", "k_gain", "rope", "q") + off(2, "pos", "slot") +
            [{"qkv_bf16": BASE}, {"qkv_f32": None, "qkv_bf16": BASE + 8}, {"T": -1}, {"T": 1 << 22}, {"ld": 1016}, {"ld": 1028},
             {"nq": 0}, {"nq": 1025}, {"n_pos": 0}], b"rope_append")


def test_rope_append_takes_no_other_types(metro):
    """Rows of another type are not read as bf16 or as fp32."""
    torch = pytest.importorskip("torch")
    for dtype in (torch.float16, torch.float64, torch.int32, torch.int8, torch.float8_e4m3fn):
        with pytest.raises(ValueError, match="float32 or bfloat16"):
            metro.op_rope_append(torch.zeros(3, 1024, dtype=dtype), 3, 8, 4, 64, None, 64, None, None, None, None, 9, stream=0)
    # (none at all: the call of no rows)
    metro.op_rope_append(None, 0, 8, 4, 64, None, 64, None, None, None, None, 9, stream=0)


def test_kv_move_refusals(metro):
    refused(metro, "metro_op_kv_move", MOVE, CACHE + nulls("kv", "src", "dst", "offsets") + off(2, "src", "dst", "offsets") +
            [{"n_layers": -1}, {"n_layers": 65536}, {"n_groups": -1}, {"n_groups": 65536}, {"n_moves": -1},
             {"layer_stride": 9 * 2 * 4 * 16 * 64 - 8}, {"layer_stride": 9 * 2 * 4 * 16 * 64 + 4}], b"kv_move")


def test_attn_tree_refusals(metro):
    refused(metro, "metro_op_attn_tree", TREE, CACHE + nulls("q", "kv", "cu_q", "ctx", "block_tables", "out") +
            off(8, "q", "out", "workspace") + off(2, "cu_q", "ctx", "mask", "block_tables") +
            [{"nq": 6}, {"nq": 12}, {"nq": 64}, {"nq": 0}, {"n_items": -1}, {"rows": -1}, {"max_q": 0}, {"max_q": 4097, "ldm": 200},
             {"max_q": 65}, {"ldm": 1}, {"max_keys": 0}, {"max_keys": 65}, {"max_keys": (1 << 30) + 1, "ldb": 1 << 27}, {"ldb": 3}, {"workspace_bytes": -1},
             {"n_items": 1 << 21}], b"attn_tree")


def test_sample_refusals(metro):
    refused(metro, "metro_op_sample", SAMPLE, nulls("logits", "u", "out") +
            off(2, "logits", "temperature", "top_k", "top_p", "min_p", "u", "out", "prob") + off(8, "workspace") +
            [{"rows": -1}, {"rows": 65536}, {"vocab": 0}, {"vocab": (1 << 18) + 1, "ldl": 1 << 20}, {"ldl": 100}], b"sample")
    need = metro.op_sample_workspace(3, 101)
    if need:
        refused(metro, "metro_op_sample", SAMPLE, [{"workspace_bytes": need - 1}, {"workspace": None}], b"workspace")


def test_calls_of_nothing_take_null(metro):
    """Calls without rows, items or moves return before any device work."""
    assert call(metro, "metro_op_rope_append", {**APPEND, "T": 0, "qkv_f32": None, "rope": None, "pos": None, "slot": None,
                                                "q": None, "kv": None}) == 0
    for k in ("n_layers", "n_groups", "n_moves"):
        assert call(metro, "metro_op_kv_move", {**MOVE, k: 0, "kv": None, "src": None, "dst": None, "offsets": None}) == 0
    for k in ("n_items", "rows"):
        assert call(metro, "metro_op_attn_tree", {**TREE, k: 0, "q": None, "kv": None, "cu_q": None, "ctx": None,
                                                  "block_tables": None, "out": None}) == 0
    assert call(metro, "metro_op_sample", {**SAMPLE, "rows": 0, "logits": None, "u": None, "out": None, "workspace": None,
                                           "workspace_bytes": 0}) == 0


def test_workspace_queries(metro):
    n = ctypes.c_int64(-1)
    assert metro.lib.metro_op_sample_workspace(0, 128256, ctypes.byref(n)) == 0 and n.value == 0
    for rows, vocab in ((-1, 5), (1, 0), (1, (1 << 18) + 1)):
        assert metro.lib.metro_op_sample_workspace(rows, vocab, ctypes.byref(n)) == -1
    assert metro.lib.metro_op_sample_workspace(1, 5, None) == -1
    assert metro.op_attn_tree_workspace(32, 8, 128, 0, 0, 1, 1) == 0
    assert metro.op_attn_tree_workspace(32, 8, 128, 1, 1, 1, 16) == 0  # one page is one piece
    few, many = (metro.op_attn_tree_workspace(32, 8, 128, 1, 1, 1, k) for k in (256, 30000))
    assert 0 < few <= many and many % (32 * 130 * 4) == 0
    assert metro.op_attn_tree_workspace(32, 8, 128, 1000, 1000, 1, 30000) == 0  # workgroups enough without splits
    for bad in ((32, 8, 96, 1, 1, 1, 16), (32, 7, 128, 1, 1, 1, 16), (32, 8, 128, 1, 1, 0, 16), (32, 8, 128, 1, 1, 1, 0)):
        assert metro.lib.metro_op_attn_tree_workspace(*bad, ctypes.byref(n)) == -1
    assert metro.lib.metro_op_attn_tree_workspace(32, 8, 128, 1, 1, 1, 16, None) == -1
