"""The cache in 4 bits and the pages' operations on the host: the layout, the rounding, and what the entry points refuse; nothing here
reaches a GPU."""
import ctypes
import math
import os

import pytest
import torch

import kvq_helpers as K


@pytest.fixture(scope="module")
def R():
    from paper_2508_09072_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2508_09072_amd import build
        build.build()
    binding.load()
    return binding


ONE = ctypes.c_void_p(4096)
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, -1, -2, -3


@pytest.mark.parametrize("D", [64, 128])
def test_every_byte_of_a_block_belongs_to_one_row(D):
    at = torch.cat([K.row_bytes(D, s) for s in range(16)])
    assert sorted(at.tolist()) == list(range(17 * D))


def test_rounding_by_hand():
    x = torch.zeros(32, dtype=torch.bfloat16)
    x[:12] = torch.tensor([7.0, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, -0.74, -0.0]).bfloat16()
    codes, scale, kept = K.quantise(x)
    assert codes[:12].tolist() == [7, 0, 1, 2, 2, 4, 4, 6, 6, 7, 9, 8] and scale.tolist() == [127] and bool(kept.all())
    x[0] = 7.03125                                               # above 7: the next scale
    assert K.quantise(x)[1].tolist() == [128]
    x[0] = math.nan
    codes, scale, kept = K.quantise(x)
    assert codes.tolist() == [0] * 32 and scale.tolist() == [2] and not bool(kept.any())
    assert K.quantise(torch.zeros(64).bfloat16())[1].tolist() == [2, 2]


def test_no_value_moves_by_more_than_its_scale():
    gen = torch.Generator().manual_seed(1)
    x = (torch.randn((500, 64), generator=gen) * torch.randn((500, 1), generator=gen).mul(20).exp2()).bfloat16()
    codes, scale, _ = K.quantise(x)
    step = torch.exp2(scale.double() - 127).repeat_interleave(32, -1)
    assert bool(((K.CODES[codes] * step - x.double()).abs() <= step).all())


def dims(R, **kw):
    a = dict(B=2, T=4, Hq=8, Hkv=2, D=128, max_pages_per_seq=8, max_path=3, num_pages=20)
    a.update(kw)
    return R.make_dims(**a)


CALLS = {
    "reader_kvq_store": [("N", 10), ("k", ONE), ("v", ONE), ("cu_tokens", ONE), ("seq_lens", ONE), ("kvq_cache", ONE), ("page_table", ONE)],
    "reader_kvq_pack": [("num_layers", 2), ("k_cache", ONE), ("v_cache", ONE), ("from_pages", 30), ("from_table", ONE), ("starts", None),
                        ("seq_lens", ONE), ("max_seq_len", 100), ("kvq_cache", ONE), ("page_table", ONE)],
    "reader_kvq_compact_layers": [("num_layers", 2), ("path", ONE), ("accept_len", ONE), ("kvq_cache", ONE), ("page_table", ONE),
                                  ("seq_lens", ONE)],
    "reader_kvq_tree_attn": [("q", ONE), ("kvq_cache", ONE), ("page_table", ONE), ("seq_lens", ONE), ("parents", ONE), ("out", ONE),
                             ("lse", None), ("max_seq_len", 100), ("workspace", ONE), ("workspace_bytes", 1 << 40)],
    "reader_kvq_prompt_attn": [("N", 10), ("q", ONE), ("kvq_cache", ONE), ("page_table", ONE), ("cu_tokens", ONE), ("seq_lens", ONE),
                               ("out", ONE), ("lse", None), ("max_seq_len", 100), ("workspace", ONE), ("workspace_bytes", 1 << 40)],
    "reader_pages_reorder": [("sources", ONE), ("page_table", ONE), ("seq_lens", ONE), ("page_refs", ONE), ("workspace", ONE),
                             ("workspace_bytes", 1 << 40)],
    "reader_pages_reserve": [("num_layers", 2), ("page_bytes", 4096), ("seq_lens", ONE), ("new_lens", ONE), ("k_cache", ONE), ("v_cache", ONE),
                             ("page_table", ONE), ("page_refs", ONE), ("workspace", ONE), ("workspace_bytes", 1 << 40)],
}
OPTIONAL = {"starts", "lse", "cu_tokens", "v_cache"}
NAMES = list(CALLS)
KVQ = [n for n in NAMES if "kvq" in n]


def call(R, name, d, **change):
    """The entry point with arguments that are all right but for the named ones."""
    args = CALLS[name]
    unknown = set(change) - {k for k, _ in args}
    assert not unknown, unknown
    return getattr(R.load(), name)(ctypes.byref(d) if d is not None else None, *[change.get(k, v) for k, v in args], None, None)


def pointers(name):
    return [k for k, v in CALLS[name] if v is ONE]


@pytest.mark.parametrize("name", NAMES)
def test_dimensions(R, name):
    assert call(R, name, None) == EINVAL
    for bad in (dict(Hq=7), dict(B=-1), dict(T=0), dict(max_path=5)):
        assert call(R, name, dims(R, **bad)) == EINVAL, bad
    for bad in (dict(D=96), dict(page_size=32), dict(Hq=64), dict(B=5000), dict(T=200), dict(num_pages=1 << 31)):
        assert call(R, name, dims(R, **bad)) == EUNSUPPORTED, bad
    if name in KVQ:
        assert call(R, name, dims(R, variant=1)) == EINVAL
        assert call(R, name, dims(R, Hq=70000, Hkv=70000, num_pages=20)) == EUNSUPPORTED


@pytest.mark.parametrize("name", NAMES)
def test_null_pointers(R, name):
    for p in pointers(name):
        if p == "v_cache" and name == "reader_pages_reserve":
            continue
        want = EWORKSPACE if p == "workspace" else EINVAL
        if p == "cu_tokens" and name == "reader_kvq_store":
            want = EINVAL                                       # (packed rows without bounds: N is not B * T)
        assert call(R, name, dims(R), **{p: None}) == want, p


@pytest.mark.parametrize("name", NAMES)
def test_tensors_that_start_between_16_bytes(R, name):
    wide = {"k", "v", "k_cache", "v_cache", "kvq_cache", "q", "out"}
    for p in wide & set(pointers(name)):
        assert call(R, name, dims(R), **{p: ctypes.c_void_p(4096 + 8)}) == EINVAL, p


@pytest.mark.parametrize("name", NAMES)
def test_an_empty_batch_is_nothing_to_do(R, name):
    change = {p: None for p in pointers(name)}
    if name == "reader_kvq_store":
        change["N"] = 0
    assert call(R, name, dims(R, B=0), **change) == OK


@pytest.mark.parametrize("name", ["reader_kvq_store", "reader_kvq_prompt_attn"])
def test_packed_rows(R, name):
    assert call(R, name, dims(R), N=-1) == EINVAL
    assert call(R, name, dims(R), N=(1 << 25) + 1) == EUNSUPPORTED
    assert call(R, name, dims(R), N=0) == OK
    assert call(R, name, dims(R, Hq=1024, Hkv=64), N=1 << 22) == EUNSUPPORTED


@pytest.mark.parametrize("name", ["reader_kvq_tree_attn", "reader_kvq_prompt_attn"])
def test_lengths_and_workspaces_of_the_attention(R, name):
    assert call(R, name, dims(R), max_seq_len=-1) == EINVAL
    assert call(R, name, dims(R), max_seq_len=129) == EINVAL       # 8 pages of 16
    if "tree" in name:
        assert call(R, name, dims(R), max_seq_len=125) == EINVAL   # ... four of them for the tree
    # beyond what 31 bits count, a last block's tokens included
    assert call(R, name, dims(R, max_pages_per_seq=(1 << 27) + 10, B=1), max_seq_len=0x7fffffff) == EUNSUPPORTED
    assert call(R, name, dims(R, max_pages_per_seq=(1 << 26) + 10, B=1), max_seq_len=(1 << 30) + 1) == EUNSUPPORTED
    d = dims(R)
    N = 8 if "tree" in name else 10
    need = R.reader_kvq_workspace_bytes(d, N, 100)
    assert need > 0
    assert call(R, name, d, workspace_bytes=need - 1) == EWORKSPACE
    assert call(R, name, d, workspace=ctypes.c_void_p(4096 + 16)) == EWORKSPACE
    assert R.reader_kvq_workspace_bytes(dims(R, D=96), N, 100) == 0 and R.reader_kvq_workspace_bytes(d, -1, 100) == 0
    assert R.reader_kvq_workspace_bytes(d, N, -1) == 0


def test_layers_and_pages(R):
    assert call(R, "reader_kvq_pack", dims(R), num_layers=-1) == EINVAL
    assert call(R, "reader_kvq_pack", dims(R), num_layers=70000) == EUNSUPPORTED
    assert call(R, "reader_kvq_pack", dims(R), num_layers=0) == OK
    assert call(R, "reader_kvq_pack", dims(R), max_seq_len=-1) == EINVAL
    assert call(R, "reader_kvq_pack", dims(R), from_pages=-1) == EINVAL
    assert call(R, "reader_kvq_pack", dims(R), from_pages=0) == EINVAL
    assert call(R, "reader_kvq_pack", dims(R), from_pages=1 << 40) == EUNSUPPORTED
    assert call(R, "reader_kvq_pack", dims(R, Hq=8192, Hkv=8192), max_seq_len=1 << 20) == EUNSUPPORTED
    assert call(R, "reader_kvq_compact_layers", dims(R), num_layers=-1) == EINVAL
    assert call(R, "reader_kvq_compact_layers", dims(R), num_layers=70000) == EUNSUPPORTED
    for bad in (dict(num_layers=-1), dict(page_bytes=-16), dict(page_bytes=24), dict(page_bytes=0)):
        assert call(R, "reader_pages_reserve", dims(R), **bad) == EINVAL, bad
    for bad in (dict(num_layers=70000), dict(page_bytes=1 << 32)):
        assert call(R, "reader_pages_reserve", dims(R), **bad) == EUNSUPPORTED, bad


@pytest.mark.parametrize("name", ["reader_pages_reorder", "reader_pages_reserve"])
def test_workspaces_of_the_pages(R, name):
    d = dims(R)
    need = R.reader_pages_workspace_bytes(d)
    assert need >= 4 * max(20 + 2 * 2, 2 * 9)
    assert call(R, name, d, workspace_bytes=need - 1) == EWORKSPACE
    assert call(R, name, d, workspace=ctypes.c_void_p(4098)) == EWORKSPACE
    assert R.reader_pages_workspace_bytes(dims(R, D=96)) == 0


def test_the_binding_looks_at_shapes_and_places(R):
    i32, bf16, u8 = torch.zeros(1, dtype=torch.int32), torch.zeros((1, 1, 64), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.uint8)
    d = R.make_dims(1, 1, 1, 1, 64, 1, 1, 1)
    calls = [(R.reader_kvq_store, (bf16, bf16, i32, i32, u8, i32)), (R.reader_kvq_pack, (bf16, bf16, i32, None, i32, 1, u8, i32)),
             (R.reader_kvq_compact_layers, (i32, i32, u8, i32, i32)), (R.reader_kvq_tree_attn, (bf16, u8, i32, i32, i32, bf16, None, 1, None)),
             (R.reader_kvq_prompt_attn, (bf16, u8, i32, i32, i32, bf16, None, 1, None)), (R.reader_pages_reorder, (i32, i32, i32, i32, None)),
             (R.reader_pages_reserve, (i32, i32, None, None, i32, i32, None))]
    for f, rest in calls:
        with pytest.raises(TypeError):
            f(None, *rest)
        with pytest.raises(ValueError, match="GPU"):
            f(d, *rest)
