"""Host-side checks of the calls around the model's own attention that need no GPU."""
import ctypes as C

import pytest
import torch

import paper_2411_03786_b200 as ngs


def test_every_new_call_is_declared_and_exported():
    lib = ngs.load_library()
    names = {"spec_rope_rows", "spec_cache_write", "spec_cache_read", "spec_tree_mask", "spec_tree_attention_bytes", "spec_tree_attention",
             "spec_score_bytes", "score_tokens"}
    assert names <= set(ngs.declared_symbols()) and all(hasattr(lib, n) for n in names)


def test_a_context_is_asked_for():
    lib = ngs.load_library()
    z = None
    assert lib.spec_rope_rows(z, z, z, 1, 64, 64, z, z, 0, 0, 0, z, 64, z, 1, z) == -1 and b"spec_rope_rows" in lib.spec_last_error(None)
    assert lib.spec_cache_write(z, z, z, 64, 64, z, 64, 64, 1, 1, 1, z, z, z, z, z) == -1 and b"spec_cache_write" in lib.spec_last_error(None)
    assert lib.spec_cache_read(z, z, 1, 1, z, z, z, z, z) == -1 and b"spec_cache_read" in lib.spec_last_error(None)
    assert lib.spec_tree_mask(z, z, 1, 1, z, z, z, z) == -1 and b"spec_tree_mask" in lib.spec_last_error(None)
    assert lib.spec_tree_attention_bytes(z, z, 1, 1, 1) == 0 and lib.spec_score_bytes(z, 1, 0) == 0
    assert lib.spec_tree_attention(z, z, z, 64, 64, z, 64, 64, z, 64, 64, 1, 1, 1, z, z, z, C.c_float(1.0), z, z, z, 0, z) == -1
    assert b"spec_tree_attention" in lib.spec_last_error(None)
    assert lib.score_tokens(z, z, 1, z, 0, z, z, z, z, z, 0, z) == -1 and b"score_tokens" in lib.spec_last_error(None)


def test_tensors_have_to_be_on_a_gpu():
    kv = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16)
    table = torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ngs.SpecError):
        ngs.KVCache(kv, kv, table)
    with pytest.raises(ngs.SpecError):
        ngs.Rope(torch.zeros(32))


def test_strides_of_rows():
    """Token and head strides that the calls are given, and the layouts that have none."""
    from paper_2411_03786_b200.binding import _strides
    t = torch.zeros(4, 3, 12, 64)
    assert _strides(t, "t") == (768, 64) and _strides(t[:, :, :8], "t") == (768, 64) and _strides(t[0], "t") == (768, 64)
    fused = torch.zeros(4, 12, 64)
    assert _strides(fused[:, :8].unsqueeze(1), "t") == (768, 64)  # one node to a sequence
    assert _strides(t[:, 2:], "t") == (3 * 768, 64) and _strides(t[:1, 1:], "t") == (768, 64)
    for bad in (t[:, :2], t[..., ::2], t.transpose(0, 1)):
        with pytest.raises(ngs.SpecError):
            _strides(bad, "t")


def test_strides_of_more_dimensions():
    from paper_2411_03786_b200.binding import _strides
    t = torch.zeros(2, 5, 3, 12, 64)
    assert _strides(t, "t") == (768, 64) and _strides(t[:, :, :, 4:], "t") == (768, 64)
    assert _strides(t[:, :1, :1], "t") == (5 * 3 * 768, 64) and _strides(t[:1, :, 1:2], "t") == (3 * 768, 64) and _strides(t[1:, 2:3], "t") == (768, 64)
    assert _strides(t[:, :0], "t")[1] == 64 and _strides(torch.zeros(1, 1, 1, 2, 16), "t")[1] == 16
    for bad in (t[:, :, :2], t[:, :4], t.transpose(0, 1), t.transpose(1, 2)):
        with pytest.raises(ngs.SpecError):
            _strides(bad, "t")
