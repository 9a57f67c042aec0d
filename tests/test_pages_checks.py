"""Checks of the paged cache's arguments that need no GPU."""
import pytest
import torch


def config(**kw):
    from paper_2602_14236_amd import binding
    return binding.make_pages_config(**dict(dict(n_kv_heads=8, n_heads=32, n_pages=100), **kw))


def test_sizes():
    from paper_2602_14236_amd import binding
    for store, per_block in (("16", 64), ("int8", 36), ("int4", 22)):
        for dim in (64, 128):
            pool, scratch = binding.pages_bytes(config(n_layers=3, head_dim=dim, page_tokens=32, store=store))
            assert pool == 3 * 100 * 8 * 2 * per_block * dim
            assert scratch > 0


@pytest.mark.parametrize("bad", [dict(n_layers=0), dict(n_kv_heads=0), dict(n_heads=0), dict(n_heads=33), dict(head_dim=96), dict(head_dim=0),
                                 dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512), dict(page_tokens=0), dict(n_pages=0),
                                 dict(n_pages=(1 << 24) + 1), dict(n_heads=70000, n_kv_heads=1)])
def test_configurations_that_are_none(bad):
    from paper_2602_14236_amd import binding
    with pytest.raises(binding.SaliError) as e:
        binding.pages_bytes(config(**bad))
    assert e.value.code == -4


def test_types_that_are_none():
    with pytest.raises(ValueError):
        config(dtype=torch.float32)
    with pytest.raises(ValueError):
        config(store="int2")


def test_codes_that_are_none():
    from paper_2602_14236_amd import binding
    for field in ("dtype", "store"):
        cfg = config()
        setattr(cfg, field, 3)
        with pytest.raises(binding.SaliError):
            binding.pages_bytes(cfg)


def test_null_arguments():
    import ctypes as C
    from paper_2602_14236_amd import binding
    lib = binding.load_library()
    b, r = binding.sali_page_batch(), binding.sali_rows()
    assert lib.sali_pages_bytes(None, None, None) == -1
    assert lib.sali_pages_create(config(), None, None, None) == -1
    h = C.c_void_p()
    assert lib.sali_pages_create(config(), None, None, C.byref(h)) == -1 and h.value is None
    assert lib.sali_pages_create(config(), 256, 264, C.byref(h)) == -3
    assert lib.sali_pages_append(None, 0, b, r, r, None) == -1
    assert lib.sali_pages_read(None, 0, b, r, r, None) == -1
    assert lib.sali_pages_attend(None, 0, b, r, 1.0, 0, 0, None, None, r, None, None) == -1
    assert lib.sali_pages_get_status(None, None, None) == -1
    lib.sali_pages_destroy(None)


def test_batches_that_are_none():
    from paper_2602_14236_amd.binding import PageBatch
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    PageBatch(i(4), i(3), i(3, 5), 7, max_kv=80)
    for args in ((i(3), i(3), i(3, 5)), (i(4), i(3), i(2, 5)), (i(4).long(), i(3), i(3, 5)), (i(4), i(6)[::2], i(3, 5)), (i(4), i(3), i(15)),
                 (i(4), i(3), i(5, 3).t())):
        with pytest.raises(ValueError):
            PageBatch(*args, 7, max_kv=80)


def test_pages_are_on_the_gpu():
    from paper_2602_14236_amd import binding
    with pytest.raises(ValueError):
        binding.SaliPages(config(), "cpu")


def test_reports_of_spilled_registers_are_read():
    from paper_2602_14236_amd import build
    line = "a.hip:1:1: remark: {} [-Rpass-analysis=kernel-resource-usage]"
    report = "\n".join(line.format(x) for x in ("Function Name: good", "    SGPRs Spill: 3", "    VGPRs Spill: 0", "Function Name: bad",
                                                "    SGPRs Spill: 0", "    VGPRs Spill: 12"))
    assert build.spilled(report) == ["bad"]
