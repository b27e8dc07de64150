"""What the operators around the verification step refuse, on the host; nothing here reaches a GPU."""
import ctypes
import math
import os

import pytest
import torch


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


def dims(R, **kw):
    a = dict(B=2, T=4, Hq=8, Hkv=2, D=128, max_pages_per_seq=8, max_path=3, num_pages=20)
    a.update(kw)
    return R.make_dims(**a)


def call(R, name, d, **change):
    """The entry point with arguments that are all right but for the named ones."""
    calls = {
        "reader_tree_qkv": [("qkv", ONE), ("parents", ONE), ("seq_lens", ONE), ("positions", None), ("q_norm", ONE), ("k_norm", ONE), ("eps", 1e-6),
                            ("cos_sin", ONE), ("max_positions", 100), ("rot_dims", 64), ("interleaved", 0), ("q", ONE), ("k_tree", ONE),
                            ("v_tree", ONE), ("k_cache", ONE), ("v_cache", ONE), ("page_table", ONE)],
        "reader_prompt_qkv": [("N", 10), ("qkv", ONE), ("cu_tokens", ONE), ("seq_lens", ONE), ("positions", None), ("q_norm", ONE), ("k_norm", ONE),
                              ("eps", 1e-6), ("cos_sin", ONE), ("max_positions", 100), ("rot_dims", 64), ("interleaved", 0), ("q", ONE),
                              ("k_cache", ONE), ("v_cache", ONE), ("page_table", ONE)],
        "reader_prompt_attn": [("N", 10), ("q", ONE), ("k_cache", ONE), ("v_cache", ONE), ("page_table", ONE), ("cu_tokens", ONE), ("seq_lens", ONE),
                               ("out", ONE), ("lse", None), ("max_seq_len", 100), ("workspace", ONE), ("workspace_bytes", 1 << 40)],
        "reader_key_weights": [("q", ONE), ("lse", ONE), ("path", ONE), ("accept_len", ONE), ("k_cache", ONE), ("page_table", ONE), ("seq_lens", ONE),
                               ("decay", 1.0), ("weights", ONE), ("max_positions", 128), ("max_seq_len", 100)],
        "reader_prompt_key_weights": [("N", 10), ("q", ONE), ("lse", ONE), ("cu_tokens", ONE), ("window", 4), ("k_cache", ONE), ("page_table", ONE),
                                      ("seq_lens", ONE), ("decay", 1.0), ("weights", ONE), ("max_positions", 128), ("max_seq_len", 100)],
        "reader_kv_evict": [("num_layers", 2), ("keep", 50), ("recent", 5), ("k_cache", ONE), ("v_cache", ONE), ("page_table", ONE), ("seq_lens", ONE),
                            ("weights", ONE), ("max_positions", 128), ("workspace", ONE), ("workspace_bytes", 1 << 40)],
    }
    args = calls[name]
    unknown = set(change) - {k for k, _ in args}
    assert not unknown, unknown
    return getattr(R.load(), name)(ctypes.byref(d) if d is not None else None, *[change.get(k, v) for k, v in args], None, None)


NAMES = ["reader_tree_qkv", "reader_prompt_qkv", "reader_prompt_attn", "reader_key_weights", "reader_prompt_key_weights", "reader_kv_evict"]
POINTERS = {
    "reader_tree_qkv": ["qkv", "parents", "seq_lens", "cos_sin", "q", "q_norm", "k_norm", "k_tree", "v_tree"],
    "reader_prompt_qkv": ["qkv", "cu_tokens", "seq_lens", "cos_sin", "q", "q_norm", "k_norm", "k_cache", "v_cache", "page_table"],
    "reader_prompt_attn": ["q", "k_cache", "v_cache", "page_table", "cu_tokens", "seq_lens", "out"],
    "reader_key_weights": ["q", "lse", "path", "accept_len", "k_cache", "page_table", "seq_lens", "weights"],
    "reader_prompt_key_weights": ["q", "lse", "cu_tokens", "k_cache", "page_table", "seq_lens", "weights"],
    "reader_kv_evict": ["k_cache", "v_cache", "page_table", "seq_lens", "weights"],
}


@pytest.mark.parametrize("name", NAMES)
def test_dimensions(R, name):
    assert call(R, name, None) == EINVAL
    for bad in (dict(Hq=7), dict(B=-1), dict(T=0), dict(max_path=5)):
        assert call(R, name, dims(R, **bad)) == EINVAL, bad
    for bad in (dict(D=96), dict(page_size=32), dict(Hq=64), dict(B=5000), dict(T=200), dict(num_pages=1 << 31)):
        assert call(R, name, dims(R, **bad)) == EUNSUPPORTED, bad


@pytest.mark.parametrize("name", NAMES)
def test_null_pointers(R, name):
    for p in POINTERS[name]:
        assert call(R, name, dims(R), **{p: None}) == EINVAL, p


@pytest.mark.parametrize("name", NAMES)
def test_tensors_that_start_between_16_bytes(R, name):
    wide = {"qkv", "cos_sin", "q", "q_norm", "k_norm", "k_tree", "v_tree", "k_cache", "v_cache", "out"}
    for p in wide & set(POINTERS[name]):
        assert call(R, name, dims(R), **{p: ctypes.c_void_p(4096 + 8)}) == EINVAL, p


@pytest.mark.parametrize("name", NAMES)
def test_an_empty_batch_is_nothing_to_do(R, name):
    assert call(R, name, dims(R, B=0), **{p: None for p in POINTERS[name]}) == OK


@pytest.mark.parametrize("name", ["reader_prompt_qkv", "reader_prompt_attn"])
def test_no_rows_are_nothing_to_do(R, name):
    assert call(R, name, dims(R), N=0, **{p: None for p in POINTERS[name]}) == OK


@pytest.mark.parametrize("name", ["reader_prompt_qkv", "reader_prompt_attn", "reader_prompt_key_weights"])
def test_number_of_rows(R, name):
    assert call(R, name, dims(R), N=-1) == EINVAL
    assert call(R, name, dims(R), N=(1 << 25) + 1) == EUNSUPPORTED
    assert call(R, name, dims(R, Hq=1024, Hkv=512), N=1 << 25) == EUNSUPPORTED


@pytest.mark.parametrize("name", ["reader_prompt_qkv", "reader_prompt_attn", "reader_key_weights", "reader_kv_evict"])
def test_no_cache(R, name):
    assert call(R, name, dims(R, num_pages=0)) == EINVAL
    assert call(R, name, dims(R, max_pages_per_seq=0)) == EINVAL


@pytest.mark.parametrize("name", ["reader_tree_qkv", "reader_prompt_qkv"])
def test_rotation_and_norm(R, name):
    for bad in (dict(rot_dims=-16), dict(rot_dims=144), dict(max_positions=-1), dict(interleaved=2), dict(eps=-1e-6), dict(eps=2.0),
                dict(eps=math.nan), dict(eps=math.inf)):
        assert call(R, name, dims(R), **bad) == EINVAL, bad
    for bad in (8, 20, 100):
        assert call(R, name, dims(R), rot_dims=bad) == EUNSUPPORTED
    assert call(R, name, dims(R, D=64), rot_dims=128) == EINVAL


def test_tree_rows_in_the_cache_need_one(R):
    for gone in ("k_cache", "v_cache", "page_table"):
        assert call(R, "reader_tree_qkv", dims(R), k_tree=None, v_tree=None, **{gone: None}) == EINVAL


def test_prompt_attention(R):
    assert call(R, "reader_prompt_attn", dims(R), max_seq_len=-1) == EINVAL
    assert call(R, "reader_prompt_attn", dims(R), max_seq_len=129) == EINVAL          # eight pages
    assert call(R, "reader_prompt_attn", dims(R, variant=2)) == EINVAL
    assert call(R, "reader_prompt_attn", dims(R), workspace=None) == EWORKSPACE
    assert call(R, "reader_prompt_attn", dims(R), workspace=ctypes.c_void_p(4096 + 64)) == EWORKSPACE
    d = dims(R)
    need = R.reader_prompt_workspace_bytes(d, 10, 100)
    assert need >= 256 and call(R, "reader_prompt_attn", d, workspace_bytes=need - 1) == EWORKSPACE
    assert call(R, "reader_prompt_attn", dims(R, variant=1), N=1 << 23) == EUNSUPPORTED
    assert R.reader_prompt_workspace_bytes(dims(R, D=96), 10, 100) == 0
    assert R.reader_prompt_workspace_bytes(d, -1, 100) == 0 and R.reader_prompt_workspace_bytes(d, 10, -1) == 0


@pytest.mark.parametrize("name", ["reader_key_weights", "reader_prompt_key_weights"])
def test_key_weights(R, name):
    for bad in (dict(decay=-0.1), dict(decay=1.5), dict(decay=math.nan), dict(max_positions=-1), dict(max_seq_len=-1)):
        assert call(R, name, dims(R), **bad) == EINVAL, bad
    assert call(R, name, dims(R, Hq=70000, Hkv=70000, num_pages=20)) == EUNSUPPORTED


def test_window(R):
    assert call(R, "reader_prompt_key_weights", dims(R), window=-1) == EINVAL
    assert call(R, "reader_prompt_key_weights", dims(R), window=65537) == EUNSUPPORTED


def test_evict(R):
    for bad in (dict(num_layers=0), dict(num_layers=-1), dict(keep=-1), dict(recent=-1), dict(recent=51), dict(max_positions=-1)):
        assert call(R, "reader_kv_evict", dims(R), **bad) == EINVAL, bad
    assert call(R, "reader_kv_evict", dims(R), num_layers=1 << 19) == EUNSUPPORTED
    d = dims(R)
    need = R.reader_kv_evict_workspace_bytes(d, 2, 50)
    assert need >= 2 * 2 * 2 * 51 * 4
    assert call(R, "reader_kv_evict", d, workspace_bytes=need - 1) == EWORKSPACE
    assert call(R, "reader_kv_evict", d, workspace=None) == EWORKSPACE
    assert call(R, "reader_kv_evict", d, workspace=ctypes.c_void_p(4098)) == EWORKSPACE


def test_binding_asks_for_tensors_on_the_gpu(R):
    bf, i, f = torch.zeros(1, 1, 1, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32), torch.zeros(1)
    d = dims(R)
    for c, rest in ((R.reader_tree_qkv, (bf, i, i, None, None, None, 1e-6, None, 0, bf, bf, bf, None, None, None)),
                    (R.reader_prompt_qkv, (bf, i, i, None, None, None, 1e-6, None, 0, bf, bf, bf, i)),
                    (R.reader_prompt_attn, (bf, bf, bf, i, i, i, bf, None, 1, None)),
                    (R.reader_key_weights, (bf, f, i, i, bf, i, i, 1.0, f, 1)),
                    (R.reader_prompt_key_weights, (bf, f, i, 1, bf, i, i, 1.0, f, 1)),
                    (R.reader_kv_evict, (1, 0, bf, bf, i, i, f, None))):
        with pytest.raises(ValueError, match="GPU"):
            c(d, *rest)
        with pytest.raises(TypeError):
            c(None, *rest)


def test_rows_of_a_prompt(R):
    def rows(B, N, bound, **kw):
        return R.reader_prompt_rows(dims(R, B=B, Hq=32, Hkv=8, max_pages_per_seq=4096, **kw), N, bound)
    assert rows(16, 16, 16384) == 16                     # single tokens
    assert rows(8, 64, 9000) == 32                       # chunks of eight
    assert rows(1, 100, 100) == R.PROMPT_ROWS_32_UNCUT and rows(1, 400, 400) == R.PROMPT_ROWS_32_UNCUT and rows(16, 16, 300) == R.PROMPT_ROWS_32_UNCUT
    assert rows(1, 1500, 1500) == 64
    assert rows(16, 16 * 300, 300) == 128
    assert rows(1, 16384, 16384) == 256 and rows(1, 256, 8000) == 256
    assert rows(1, 0, 0) == 16 and rows(0, 0, 0) == 16
    assert rows(1, 16384, 16384, variant=1) == 0
    for forced in (16, 32, 33, 64, 128, 256):
        R.reader_tuning_override(R.TUNE_PROMPT_ROWS, forced)
        try:
            assert rows(1, 100, 100) == forced
        finally:
            R.reader_tuning_override(R.TUNE_PROMPT_ROWS, -1)
    with pytest.raises(R.ReaderError):
        rows(1, -1, 10)
    with pytest.raises(R.ReaderError):
        rows(1, 10, 10, variant=3)


@pytest.mark.parametrize("big", [1 << 32, (1 << 32) + 5, 1 << 31, -(1 << 31) - 1, 1 << 62])
def test_numbers_that_32_bits_do_not_hold_are_refused(R, big):
    """... and not taken for their last 32 bits: 2^32 + 5 kept rows are not five."""
    bf, i, f = torch.zeros(1, 1, 1, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32), torch.zeros(1)
    d = dims(R)
    for args in ((big, 0), (50, big)):
        with pytest.raises(ValueError, match="32 bits"):
            R.reader_kv_evict(d, *args, bf, bf, i, i, f, None)
