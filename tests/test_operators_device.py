"""An operator's handle belongs to one device: the binding makes it current for every call, the C calls refuse another one.  Without
a second GPU (or a first): the library and torch's device functions are replaced by recorders."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class _Recorder:
    """Stands in for the library: notes which device was current at each call."""
    def __init__(self, state):
        self.state, self.seen = state, []

    def __getattr__(self, name):
        def function(*args):
            self.seen.append((name, self.state["current"]))
            return 0
        return function


@pytest.fixture
def fake(monkeypatch):
    import torch
    from paper_2507_20055_b200 import build
    build.build()
    from paper_2507_20055_b200 import binding
    state = {"current": 0, "entered": 0}

    class device:
        def __init__(self, d):
            self.index = d.index

        def __enter__(self):
            self.before, state["current"] = state["current"], self.index
            state["entered"] += 1

        def __exit__(self, *_):
            state["current"] = self.before

    lib = _Recorder(state)
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_current_device", lambda: state["current"])
    monkeypatch.setattr(binding, "_current_raw_stream", lambda index: 0)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(binding, "_check_rows", lambda *a: None)
    monkeypatch.setattr(binding, "_empty", lambda shape, *a, **k: torch.empty(shape))
    return binding, state, lib


@pytest.mark.parametrize("index", [0, 1])
def test_every_call_runs_with_its_operators_device_current(fake, index):
    import torch
    binding, state, lib = fake
    on, x = torch.device("cuda", index), torch.zeros(4, 8)
    xent, clip, layer = (c.__new__(c) for c in (binding.LinearCrossEntropy, binding.GradClipper, binding.Int4Weight))
    for op in (xent, clip, layer):
        op._h, op.device, op.dtype = 1, on, torch.float32
    xent.features, xent.classes, xent._number, clip._number = 8, 20, None, None
    xent._weight_shape, xent._bias_shape = torch.Size((20, 8)), torch.Size((20,))
    layer.in_features, layer.out_features = 8, 20
    w, y = torch.zeros(20, 8), torch.zeros(4, dtype=torch.int64)
    xent.loss(x, w, y)
    xent.loss_and_grad(x, w, y)
    clip.clip(1.0)
    layer.matvec(x)
    layer.dequantize()
    for op in (xent, clip, layer):
        op.last_status()
        op.check_guards()
        op.destroy()
    assert [n for n, _ in lib.seen] == ["cert_xent_run", "cert_xent_run", "cert_clip_run", "cert_int4_matvec", "cert_int4_dequantize"] + \
        [f"cert_{k}_{f}" for k in ("xent", "clip", "int4") for f in ("last_status", "check_guards", "destroy")]
    assert {d for _, d in lib.seen} == {index}
    assert state["current"] == 0
    assert state["entered"] == (len(lib.seen) if index else 0)       # the usual path does not switch


def test_a_stream_of_another_device_is_refused(fake):
    import torch
    binding = fake[0]

    class Stream:
        device, cuda_stream = torch.device("cuda", 0), 0             # its default stream's handle is every device's
    assert binding._stream_ptr(Stream(), torch.device("cuda", 0)) == 0
    with pytest.raises(ValueError):
        binding._stream_ptr(Stream(), torch.device("cuda", 1))


def test_c_calls_on_a_handle_ask_for_its_device():
    for name in ("linear_xent.cu", "clip.cu", "int4.cu"):
        with open(os.path.join(ROOT, "paper_2507_20055_b200", "csrc", name)) as f:
            text = f.read()
        text = text[text.index('extern "C" {'):]
        calls = re.findall(r"^(?:cert_status_t|int) (cert_\w+)\((cert_(?:xent|clip|int4)_t \*op\b.*?)\n\}", text, re.M | re.S)
        assert len(calls) >= 4
        for call, body in calls:
            first_use = min(body.index(w) for w in ("op->mem", "op->status", "cudaDeviceSynchronize", "run(op", "static_cast<cudaStream_t>") if w in body)
            assert "on_device(op->device)" in body[:first_use], call


def test_calls_that_use_a_handles_workspace_are_taken_one_at_a_time():
    """Two host threads on one stream: what the handle remembers and the order of the launches are one call's at a time."""
    for name, call, work in (("linear_xent.cu", "cert_xent_run", "return run("), ("clip.cu", "cert_clip_run", "launch_chained(")):
        with open(os.path.join(ROOT, "paper_2507_20055_b200", "csrc", name)) as f:
            body = f.read().split(f"cert_status_t {call}(")[1].split("\n}\n")[0]
        assert "const OpLock lock(op->calls);" in body[:body.index(work)]


def test_sizes_that_an_int_does_not_hold_are_refused(fake):
    """They would arrive cut to 32 bits: a layer of 2^32 + 3 outputs as one of 3, whose others nobody writes."""
    import torch
    binding, _, lib = fake
    meta, many = torch.device("meta"), 2 ** 32 + 3
    xent, layer = binding.LinearCrossEntropy.__new__(binding.LinearCrossEntropy), binding.Int4Weight.__new__(binding.Int4Weight)
    for op in (xent, layer):
        op._h, op.device, op.dtype = 1, torch.device("cuda", 0), torch.float32
    xent.features, xent.classes, xent._weight_shape = 1, 20, torch.Size((20, 1))
    layer.in_features, layer.out_features = 1, 20
    x, w, y = torch.empty(many, 1, device=meta), torch.empty(20, 1, device=meta), torch.empty(many, dtype=torch.int64, device=meta)
    codes, scales = torch.empty(many, 1, dtype=torch.uint8, device=meta), torch.empty(many, 1, device=meta)
    for call in (lambda: xent.loss(x, w, y), lambda: xent.loss_and_grad(x, w, y), lambda: layer.matvec(x, out=x),
                 lambda: binding.int4_quantize(x, 32), lambda: binding.Int4Weight(codes, scales, 1, 32),
                 lambda: binding.Int4Weight(codes[:20], scales[:20], 1, many), lambda: binding.int4_quantize(w, many),
                 lambda: binding.LinearCrossEntropy(many, 1, 20, device=torch.device("cuda", 0)),
                 lambda: binding.LinearCrossEntropy(1, 1, many, device=torch.device("cuda", 0))):
        with pytest.raises(ValueError, match="does not fit"):
            call()
    assert lib.seen == []
