"""CPU-only checks of where the serving calls of the binding allocate and launch: the library's functions and torch.cuda are replaced by
recorders, the tensors are the CPU's."""
import contextlib

import pytest
import torch

from paper_1804_01526_amd import hbfp


class _Stream:
    device = torch.device("cpu")


def _calls(hb):
    cache, spare = (hb.cache_alloc(2, 2, 9000, 64, device="cpu") for _ in range(2))
    lengths = torch.zeros(2, dtype=torch.int32)
    new, q, lse = torch.zeros(2, 1, 2, 64), torch.zeros(2, 1, 8, 64), torch.zeros(2, 1, 8)
    weights, x = torch.zeros(2, 2, 9000), torch.zeros(100, 256)
    codes = hb.RowCodes(torch.zeros(128, 256, dtype=torch.int8), torch.zeros(128), 256)
    rows = hb.RowCodes(torch.zeros(100, 256, dtype=torch.int8), torch.zeros(100), 256)
    return {
        "hbfp_cache_append": lambda s: hb.cache_append(cache, new, new, lengths, values=True, stream=s),
        "hbfp_cache_read": lambda s: hb.cache_read(cache, lengths, stream=s),
        "hbfp_cache_attend": lambda s: hb.cache_attend(cache, q, lengths, stream=s),
        "hbfp_cache_weigh_longest": lambda s: hb.cache_weigh(cache, q, lse, lengths, weights, stream=s),
        "hbfp_cache_evict": lambda s: hb.cache_evict(cache, weights, lengths, spare, 10, 5, stream=s),
        "hbfp_quant_rows": lambda s: hb.quant_rows(x, stream=s),
        "hbfp_gemm_rows": lambda s: hb.gemm_rows(rows, codes, stream=s),
        "hbfp_linear_i8": lambda s: hb.linear_i8(x, codes, stream=s),
    }


NAMES = ["hbfp_cache_append", "hbfp_cache_read", "hbfp_cache_attend", "hbfp_cache_weigh_longest", "hbfp_cache_evict", "hbfp_quant_rows", "hbfp_gemm_rows",
         "hbfp_linear_i8"]


@pytest.fixture
def recorded(monkeypatch):
    """(the name of every call's library function -> the call, the log): where the call was when it allocated and launched, which
    stream its results were recorded for."""
    calls, where, log = _calls(hbfp), ["caller's"], []

    @contextlib.contextmanager
    def there(what):
        where.append(what)
        yield
        where.pop()
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: (log.append(("alloc", where[-1])), empty(*a, **k))[1])
    monkeypatch.setattr(torch.cuda, "stream", there)
    monkeypatch.setattr(torch.cuda, "device", lambda d: there("device"))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: "the caller's stream")
    current = {"caller's": None}                                # None: the index of the tensors' device
    monkeypatch.setattr(hbfp, "_current_device", lambda: current.get(where[-1]))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: log.append(("record", s)))
    monkeypatch.setattr(hbfp, "_matrix", lambda t: t.stride(0))
    monkeypatch.setattr(hbfp, "_raw_stream", lambda d: where[-1])
    for name in NAMES:
        def launch(*args):
            log.append(("launch", where[-1], args[-1]))                     # (the stream is the last argument)
            return hbfp.OK
        monkeypatch.setattr(hbfp._lib, name, launch)
    return calls, log, current


@pytest.mark.parametrize("name", NAMES)
def test_a_call_on_a_stream_allocates_there(recorded, name):
    """Memory that the caller's stream has freed may still be in use there; outputs may be in use there when they are freed."""
    calls, log, _ = recorded
    side = _Stream()
    calls[name](side)
    assert [e for e in log if e[0] == "launch"] == [("launch", side, side)]
    assert all(e[1] is side for e in log if e[0] == "alloc")
    outputs = {"hbfp_cache_weigh_longest": 1, "hbfp_cache_evict": 3, "hbfp_gemm_rows": 1, "hbfp_linear_i8": 1}.get(name, 2)
    assert [e for e in log if e[0] == "record"] == [("record", "the caller's stream")] * outputs


@pytest.mark.parametrize("name", NAMES)
def test_a_call_without_one_goes_to_its_tensors_device(recorded, name):
    calls, log, current = recorded
    calls[name](None)
    assert log[-1] == ("launch", "caller's", "caller's") and all(e[0] == "launch" or e == ("alloc", "caller's") for e in log)
    log.clear()
    current["caller's"] = 5
    calls[name](None)
    assert log[-1] == ("launch", "device", "device") and all(e[0] == "launch" or e == ("alloc", "device") for e in log)


def test_a_stream_of_another_device_is_refused(recorded):
    side = _Stream()
    side.device = torch.device("meta")
    with pytest.raises(AssertionError):
        recorded[0]["hbfp_quant_rows"](side)


def test_weigh_longest_refusals():
    import ctypes
    at = 0x100000                                              # nothing reads it: every call below is refused on the host
    c = hbfp.cache_plan(2, 2, 100, 64)
    c.k, c.v, c.k_exps, c.v_exps = at, at + (1 << 24), at + (2 << 24), at + (3 << 24)
    q = hbfp.Heads(at, 1, 0, 1024, 256, 64)
    weigh = lambda longest=0, ld=100, w=at, heads=8: hbfp._lib.hbfp_cache_weigh_longest(
        ctypes.byref(c), ctypes.byref(q), 1, heads, at, longest, 0.1, 1, at, 1.0, w, at, ld, None)
    assert weigh(longest=-1) == hbfp.ERR_ARG and weigh(ld=99) == hbfp.ERR_ARG and weigh(w=None) == hbfp.ERR_ARG and weigh(heads=7) == hbfp.ERR_ARG


def test_linear_refuses_to_write_the_tokens_it_still_reads():
    at = 0x100000
    lin = lambda x, y, m, k, n, ldx, ldy, dtype=1: hbfp._lib.hbfp_linear_i8(x, dtype, m, k, ldx, at + (1 << 28), at + (2 << 28), None, n, y, ldy, None, 0, None)
    for m, k, n, ldx, ldy, shift in ((1, 256, 256, 256, 256, 0), (1, 256, 64, 256, 64, 510), (1, 64, 256, 64, 256, -510),
                                     (2, 512, 100, 512, 512, 1024), (2, 512, 100, 700, 300, 1400), (2, 300, 300, 300, 600, 2 * 599)):
        assert hbfp.linear_i8_workspace(m, n, k) == 0
        assert lin(at, at + shift, m, k, n, ldx, ldy) == hbfp.ERR_ARG, (m, k, n, shift)
