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


@pytest.fixture
def pages_elsewhere(monkeypatch):
    """A SaliPages whose GPU (number -1, as CPU tensors have it) is not the current one, over a library that notes the device and stream of its calls."""
    from types import SimpleNamespace
    from paper_2602_14236_amd import binding
    state = SimpleNamespace(device=0, calls=[])

    class On:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.before, state.device = state.device, self.device

        def __exit__(self, *_):
            state.device = self.before

    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state.device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index, raising=False)
    pages = object.__new__(binding.SaliPages)

    def entry(name):
        def call(*args):
            state.calls.append((name, state.device, args[-1]))
            return 0
        return call

    names = ("sali_pages_append", "sali_pages_read", "sali_pages_attend", "sali_pages_get_status")
    pages.lib = SimpleNamespace(**{name: entry(name) for name in names})
    pages.handle, pages.index, pages.device, pages.dtype = None, -1, torch.device("cpu"), torch.float16
    pages.n_heads, pages.n_kv_heads, pages.head_dim = 4, 2, 64
    return pages, state


def test_calls_run_on_the_pages_gpu(pages_elsewhere):
    from types import SimpleNamespace
    from paper_2602_14236_amd.binding import PageBatch
    pages, state = pages_elsewhere
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    batch = PageBatch(i(2), i(1), i(1, 5), 3, max_kv=80)
    kv, q = torch.zeros((3, 2, 64), dtype=torch.float16), torch.zeros((3, 4, 64), dtype=torch.float16)
    for stream, handle in ((None, 999), (SimpleNamespace(cuda_stream=77, device_index=-1), 77)):
        pages.append(0, batch, kv, kv, stream=stream)
        pages.read(0, batch, kv, kv, stream=stream)
        pages.attend(0, batch, q, 1.0, q, stream=stream)
        assert state.calls == [(f"sali_pages_{name}", -1, handle) for name in ("append", "read", "attend")]
        state.calls.clear()
    pages.get_status()
    assert state.calls == [("sali_pages_get_status", -1, 999)] and state.device == 0
    with pytest.raises(ValueError):
        pages.append(0, batch, kv, kv, stream=SimpleNamespace(cuda_stream=77, device_index=0, device="cuda:0"))


def test_a_pool_lies_on_the_pages_gpu(monkeypatch):
    from types import SimpleNamespace
    from paper_2602_14236_amd import binding
    cfg = config()
    need = binding.pages_bytes(cfg)[0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)

    def pool(device, size=need):
        return SimpleNamespace(is_contiguous=lambda: True, numel=lambda: size, element_size=lambda: 1, device=torch.device(device))

    for device, bad in (("cuda:0", pool("cuda:1")), ("cuda:1", pool("cuda:0")), ("cuda", pool("cuda:0")), ("cuda:0", pool("cpu")),
                        ("cuda:0", pool("cuda:0", need - 1))):
        with pytest.raises(ValueError):
            binding.SaliPages(cfg, device, pool=bad)
