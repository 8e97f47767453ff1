"""What the paged cache's entry points refuse before they touch a GPU."""
import pytest

GOOD = dict(B=2, K=3, n_q=8, n_kv=2, head_dim=128, page_size=16, n_pages=10, table_width=4)


@pytest.mark.parametrize("bad", [
    dict(B=-1), dict(K=-1), dict(K=1024), dict(B=1 << 14, K=1023), dict(n_q=7), dict(n_q=0), dict(n_kv=0), dict(n_q=65536, n_kv=1), dict(head_dim=0),
    dict(head_dim=24), dict(head_dim=272), dict(dtype=2), dict(kv_dtype=2), dict(dtype=0, kv_dtype=1), dict(page_size=0), dict(page_size=24),
    dict(page_size=1 << 17), dict(n_pages=0), dict(table_width=0), dict(table_width=1 << 27), dict(window=-1), dict(sinks=4), dict(window=8, sinks=-1),
    dict(rot_dim=8), dict(rot_dim=144), dict(rot_dim=-16), dict(rope=2), dict(page_stride=4096), dict(page_stride=4096, slot_stride=256, head_stride=64),
    dict(page_stride=4096, slot_stride=260, head_stride=128), dict(page_stride=-4096, slot_stride=256, head_stride=128), dict(qkv_stride=1000),
    dict(qkv_stride=1540), dict(qkv_stride=-1), dict(q_stride=1016), dict(q_stride=1028), dict(flags=1)], ids=str)
def test_bad_configurations(bad):
    import paper_2504_20039_amd as aj
    with pytest.raises(aj.AjError) as e:
        aj.aj_cache_create(**{**GOOD, **bad})
    assert e.value.status == -1


def test_null_handles_and_pointers():
    import paper_2504_20039_amd as aj
    lib = aj.load_library()
    assert lib.aj_cache_create(None, None) == -1
    assert lib.aj_cache_destroy(None) == -1
    assert lib.aj_cache_append(None, 0, 0, 0, 0, 0, 0.0, 0, 0, 0, 0, 0, 1.0, 1.0, 0, 0, 0, None) == -1
    assert lib.aj_cache_attend(None, 0, 0, 0, 0, 0, 0, 0, 0, 1.0, 1.0, 1.0, 0, 0, None) == -1
    assert lib.aj_cache_commit(None, 0, 0, 0, 0, 1, 0, 0, 0, 0, None) == -1
    for bad in ((-1, 4, 16, 16, 16), (1, 0, 16, 16, 16), (1, 1024, 16, 16, 16), (1 << 14, 1023, 16, 16, 16), (1, 4, 0, 16, 16), (1, 4, 16, 0, 16),
                (1, 4, 16, 16, 0), (1, 4, 18, 16, 16), (1, 4, 16, 17, 16), (1, 4, 16, 16, 19)):
        assert lib.aj_tree_mask(*bad, None) == -1, bad
    assert lib.aj_tree_mask(0, 4, None, None, None, None) == 0


def test_the_binding_takes_device_tensors():
    import torch
    import paper_2504_20039_amd as aj
    x = torch.zeros(64, dtype=torch.int32)
    with pytest.raises(ValueError):
        aj.aj_tree_mask(1, 4, x, x, x, stream=0)
    with pytest.raises(ValueError):
        aj.aj_cache_attend(None, x, x, x, x, x, 1.0, x, stream=0)
