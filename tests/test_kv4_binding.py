"""The 4-bit cache's binding on the CPU: what its calls hand to the library, with the library's functions replaced."""
import pytest
import torch

from paper_2504_12329_amd import binding as B

needs_cuda_build = pytest.mark.skipif(not hasattr(torch._C, "_cuda_getDevice"), reason="torch without GPU support")


class Device:
    """Stands for torch's current device: what is current now, and the guard that changes it."""

    def __init__(self, monkeypatch, current):
        self.current = current
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: self.current)
        outer = self

        class Guard:
            def __init__(self, index):
                self.index = index

            def __enter__(self):
                self.was, outer.current = outer.current, self.index

            def __exit__(self, *a):
                outer.current = self.was

        monkeypatch.setattr(torch.cuda, "device", Guard)


def cache_on(index, seen, rc=B.ST_OK):
    """A cache whose library functions note the device that is current when they are called."""
    kv = B.Kv4Cache.__new__(B.Kv4Cache)
    kv._h, kv._index, kv._dev, kv._own_stream = None, index, torch.device("cuda", index), True
    kv._nq, kv._nkv, kv._d, kv._slots = 4, 2, 64, (1, 1, 2, 8)
    kv._alloc = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16)
    kv._matrix = lambda name, x, rows, heads: (x.data_ptr(), heads * 64)
    for name in ("append", "attend", "evict", "read"):
        def call(*a, name=name):
            seen.append((name, torch._C._cuda_getDevice()))
            return rc
        setattr(kv, "_" + name, call)
    return kv


def every_call(kv):
    one, x = B.Kv4Spans([(0, 0, 0, 1)]), torch.zeros(1, 8 * 64, dtype=torch.bfloat16)
    return {"append": lambda: kv.append(0, one, x), "attend": lambda: kv.attend(0, one, x[:, :256]), "evict": lambda: kv.evict(0, 1, one, 1, 0, None),
            "read": lambda: kv.read(0, 1, one)}


@needs_cuda_build
@pytest.mark.parametrize("current", [0, 1, 3])
def test_calls_go_to_the_device_of_the_cache(monkeypatch, current):
    """Whichever GPU is current (the default streams of all have one handle, so the stream's check does not tell)."""
    seen, device = [], Device(monkeypatch, current)
    for call in every_call(cache_on(1, seen)).values():
        call()
    assert seen == [(name, 1) for name in ("append", "attend", "evict", "read")]
    assert device.current == current


@needs_cuda_build
def test_errors_of_the_library_are_raised_on_any_device(monkeypatch):
    B.lib()
    for current in (0, 1):
        device = Device(monkeypatch, current)
        for call in every_call(cache_on(1, [], rc=B.ST_EINVAL)).values():
            with pytest.raises(B.StError) as e:
                call()
            assert e.value.code == B.ST_EINVAL and device.current == current


class Test32Bits:
    """Numbers past 32 bits are refused: ctypes would cut them down, and position 2^32 + 5 would be position 5."""

    @pytest.mark.parametrize("field", range(4))
    @pytest.mark.parametrize("value", [2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 63, -2 ** 31 - 1, -2 ** 32])
    def test_spans(self, field, value):
        span = [0, 1, 2, 1]
        span[field] = value
        for spans in ([span], [(0, 0, 0, 1), span], [span, (3, 0, 0, 1)]):
            with pytest.raises(B.StError) as e:
                B.Kv4Spans(spans)
            assert e.value.code == B.ST_ERANGE

    def test_spans_that_fit(self):
        s = B.Kv4Spans([(0, 2 ** 31 - 1, 2 ** 31 - 1, 1), (-2 ** 31, -1, 0, 0)])
        assert [(x.seq, x.len, x.pos, x.rows) for x in s.c] == s.spans == [(0, 2 ** 31 - 1, 2 ** 31 - 1, 1), (-2 ** 31, -1, 0, 0)]
        assert B.Kv4Spans([]).rows == 0 and B.Kv4Spans(iter([[1, 2, 3, 4]])).spans == [(1, 2, 3, 4)]

    @pytest.mark.parametrize("past", [2 ** 32, -2 ** 32])
    def test_arguments(self, past, monkeypatch):
        seen, one, x = [], B.Kv4Spans([(0, 0, 0, 1)]), torch.zeros(1, 8 * 64, dtype=torch.bfloat16)
        kv = cache_on(1, seen)
        monkeypatch.setattr(kv, "_elsewhere", lambda: False, raising=False)
        for call in (lambda: kv.append(past, one, x), lambda: kv.attend(past, one, x[:, :256]), lambda: kv.evict(past, past + 1, one, 1, 0, None),
                     lambda: kv.evict(0, past + 1, one, 1, 0, None), lambda: kv.evict(0, 1, one, past + 1, 0, None), lambda: kv.evict(0, 1, one, 1, past, None),
                     lambda: kv.read(past, past + 1, one), lambda: kv.read(0, past + 1, one)):
            with pytest.raises(B.StError) as e:
                call()
            assert e.value.code == B.ST_ERANGE
        assert not seen

    def test_configurations(self):
        cfg = dict(n_layers=1, n_seq=1, n_q_heads=2, n_kv_heads=1, head_dim=64, max_seq=8, max_rows=8, max_pos=8, rms_eps=1e-6)
        for name in set(cfg) - {"rms_eps"}:
            with pytest.raises(B.StError) as e:
                B.Kv4Cache(dict(cfg, **{name: cfg[name] + 2 ** 32}), torch.zeros(8, 32, 2))
            assert e.value.code == B.ST_ERANGE
