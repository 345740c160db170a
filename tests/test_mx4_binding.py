"""CPU-only checks of where the calls of the microscaled 4-bit operators and of the norm allocate and launch: the library's functions and
torch.cuda are replaced by recorders, the tensors are the CPU's.  And what the binding itself refuses."""
import contextlib

import pytest
import torch

from paper_1804_01526_amd import hbfp


class _Stream:
    device = torch.device("cpu")


def _calls(hb):
    x, w, r = torch.zeros(40, 300), torch.zeros(300), torch.zeros(40)
    a, b = hb.mx4_alloc(40, 300, device="cpu"), hb.mx4_alloc(24, 300, device="cpu")
    return {
        "hbfp_quant_mx4": lambda s: hb.quant_mx4(x, stream=s),
        "hbfp_quant_mx4 both": lambda s: hb.quant_mx4_both(x, stream=s),
        "hbfp_read_mx4": lambda s: hb.read_mx4(a, stream=s),
        "hbfp_gemm_mx4": lambda s: hb.gemm_mx4(a, b, stream=s),
        "hbfp_linear_mx4": lambda s: hb.linear_mx4(x, b, stream=s),
        "hbfp_norm_i8": lambda s: hb.norm_i8(x, w, residual=x, values=True, stream=s),
        "hbfp_norm_mx4": lambda s: hb.norm_mx4(x, w, residual=x, stream=s),
        "hbfp_norm_grad": lambda s: hb.norm_grad(x, x, r, w, stream=s),
    }


OUTPUTS = {"hbfp_quant_mx4": 1, "hbfp_quant_mx4 both": 2, "hbfp_read_mx4": 1, "hbfp_gemm_mx4": 1, "hbfp_linear_mx4": 1, "hbfp_norm_i8": 5,
           "hbfp_norm_mx4": 3, "hbfp_norm_grad": 2}


@pytest.fixture
def recorded(monkeypatch):
    """(every call, the log, the current devices): where the call was when it allocated and launched, which stream its results were
    recorded for."""
    calls, where, log = _calls(hbfp), ["caller's"], []

    @contextlib.contextmanager
    def there(what):
        where.append(what)
        yield
        where.pop()
    for name in ("empty", "empty_like"):
        real = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, real=real, **k: (log.append(("alloc", where[-1])), real(*a, **k))[1])
    monkeypatch.setattr(torch.cuda, "stream", there)
    monkeypatch.setattr(torch.cuda, "device", lambda d: there("device"))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: "the caller's stream")
    current = {"caller's": None}                                # None: the index of the tensors' device
    monkeypatch.setattr(hbfp, "_current_device", lambda: current.get(where[-1]))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: log.append(("record", s)))
    monkeypatch.setattr(hbfp, "_matrix", lambda t: t.stride(0))
    monkeypatch.setattr(hbfp, "_raw_stream", lambda d: where[-1])
    for name in {n.split()[0] for n in OUTPUTS}:
        def launch(*args):
            log.append(("launch", where[-1], args[-1]))                     # (the stream is the last argument)
            return hbfp.OK
        monkeypatch.setattr(hbfp._lib, name, launch)
    return calls, log, current


@pytest.mark.parametrize("name", list(OUTPUTS))
def test_a_call_on_a_stream_allocates_there(recorded, name):
    calls, log, _ = recorded
    side = _Stream()
    calls[name](side)
    assert [e for e in log if e[0] == "launch"] == [("launch", side, side)]
    assert all(e[1] is side for e in log if e[0] == "alloc")
    assert [e for e in log if e[0] == "record"] == [("record", "the caller's stream")] * OUTPUTS[name]


@pytest.mark.parametrize("name", list(OUTPUTS))
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
    for name in OUTPUTS:
        with pytest.raises(AssertionError):
            recorded[0][name](side)


def test_what_the_binding_refuses(recorded):
    hb, log = hbfp, recorded[1]
    x, w, r = torch.zeros(40, 300), torch.zeros(300), torch.zeros(40)
    a, b = hb.mx4_alloc(40, 300, device="cpu"), hb.mx4_alloc(24, 301, device="cpu")
    log.clear()
    for call in (lambda: hb.linear_mx4(x, b),                                                       # contractions that differ
                 lambda: hb.gemm_mx4(a, a, bias=torch.zeros(39)), lambda: hb.gemm_mx4(a, a, bias=torch.zeros(40, dtype=torch.float64)),
                 lambda: hb.gemm_mx4(a, a, out=torch.zeros(40, 41)), lambda: hb.linear_mx4(x, a, out=torch.zeros(40, 40, dtype=torch.bfloat16)),
                 lambda: hb.quant_mx4(x, axis=2),
                 lambda: hb.norm_i8(x, torch.zeros(299)), lambda: hb.norm_mx4(x, w.double()), lambda: hb.norm_i8(x, w, residual=x.bfloat16()),
                 lambda: hb.norm_i8(x, w, residual=x[:39]), lambda: hb.norm_mx4(x, w, residual=x, out_sum=x[:, :299]),
                 lambda: hb.norm_grad(x, x[:39], r, w), lambda: hb.norm_grad(x, x, torch.zeros(39), w), lambda: hb.norm_grad(x, x, r, torch.zeros(301)),
                 lambda: hb.norm_grad(x, x, r, w, g_sum=x.half()), lambda: hb.norm_grad(x, x, r, w, out=x.double())):
        with pytest.raises(AssertionError):
            call()
    assert not [e for e in log if e[0] == "launch"]


def test_results_of_a_norm_without_a_residual():
    """The sum is x itself where nothing was added and nothing asked for."""
    assert hbfp._buffers((hbfp.mx4_alloc(3, 5, device="cpu"), None, (torch.zeros(1),)))[1].numel() == 1
    t = hbfp.mx4_alloc(3, 600, device="cpu")
    assert tuple(t.codes.shape) == (3, 3, 128) and tuple(t.scales.shape) == (3, 16, 8) and t.buffer.numel() == t.desc.code_bytes + t.desc.scale_bytes
    assert t.scales.data_ptr() == t.desc.scales and t.codes.data_ptr() == t.desc.codes
