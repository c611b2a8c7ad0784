"""Calls of the region block on a stream that is not the current one, and on a device that is not
(the GPU tests; the others need none)."""
import pytest
import torch

from paper_2605_09204_amd import block

gpu = pytest.mark.gpu
DEV = "cuda:0"


def calls():
    """Every operator: (name, call with keyword arguments, workspace bytes)."""
    g = torch.Generator()
    g.manual_seed(21)
    n = [900, 0, 5, 300]
    T, S, D, N = sum(n), len(n), 200, 16

    def r(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g).to(dtype).to(DEV)
    f32 = torch.float32
    off = torch.tensor([0, *n]).cumsum(0).to(DEV)
    x, dy, w, cw, cb = r(T, D), r(T, D), r(D, dtype=f32), r(D, 4, dtype=f32), r(D, dtype=f32)
    args = (x, r(T, D), -torch.rand(D, N, generator=g).to(DEV), r(T, 2, N), r(T, 2, N))
    rest = {"skip": w, "z": r(T, D), "delta_bias": cb, "offsets": off, "state_in": r(S, D, N, dtype=f32)}
    one = tuple(t if t.shape[0] == D else t[:S] for t in args)
    cs, c_new, s_new = r(S, 3, D), r(S, 3, D), r(S, D, N, dtype=f32)
    return [
        ("norm", lambda **k: block.lbi_rms_norm(x, w, dy, **k), 0),
        ("norm q8", lambda **k: block.lbi_rms_norm_q8(x, w, dy, group=64, **k), 0),
        ("norm backward", lambda **k: block.lbi_rms_norm_backward(dy, x, w, **k),
         block.lbi_rms_norm_backward_workspace_bytes(T, D)),
        ("conv", lambda **k: block.lbi_ssm_conv(x, cw, cb, offsets=off, state_in=cs, **k), 0),
        ("conv backward", lambda **k: block.lbi_ssm_conv_backward(x, cw, dy, cb, offsets=off,
                                                                  state_in=cs, **k),
         block.lbi_ssm_conv_backward_workspace_bytes(T, D, 4)),
        ("conv step", lambda **k: block.lbi_ssm_conv_step(x[:S], cw, cs, c_new, cb, **k), 0),
        ("scan", lambda **k: block.lbi_ssm_scan(*args, **rest, **k),
         block.lbi_ssm_scan_workspace_bytes(T, S, D, N, 2, True)),
        ("scan backward", lambda **k: block.lbi_ssm_scan_backward(*args, dy, **rest, **k),
         block.lbi_ssm_scan_backward_workspace_bytes(T, S, D, N, 2, True)),
        ("scan step", lambda **k: block.lbi_ssm_scan_step(*one, rest["state_in"], s_new, **k), 0),
    ]


def tensors(results):
    results = results.values() if isinstance(results, dict) else \
        results if isinstance(results, tuple) else (results,)
    return [t for t in results if t is not None]


def bits(t):
    return t.contiguous().view(torch.uint8).clone()


@gpu
@pytest.mark.parametrize("handle", [False, True])
def test_memory_of_a_call_on_another_stream(handle):
    """The other stream is busy when the call comes, so its kernels run after the call has returned:
    what the current stream allocates and fills meanwhile must not be the call's memory, and what
    the call allocates must not be memory that the current stream is still filling."""
    every = calls()
    want = [[bits(t) for t in tensors(f())] for _, f, _ in every]
    side = torch.cuda.Stream()
    busy = torch.zeros(1 << 26, device=DEV)
    assert sum(need > 0 for _, _, need in every) == 4
    for (name, f, need), w in zip(every, want):
        print(f"[streams] {name}, workspace of {need} bytes", flush=True)
        sizes = sorted({need, *(t.numel() for t in w)} - {0})
        torch.cuda.synchronize()
        # blocks of these sizes lie free, and the current stream still writes to them
        for _ in range(40):
            busy.add_(1.0)
        for size in sizes:
            for _ in range(2):
                torch.empty(size, dtype=torch.uint8, device=DEV).fill_(170)
        with torch.cuda.stream(side):
            for _ in range(20):
                busy.add_(1.0)
        results = f(stream=side.cuda_stream if handle else side)
        junk = [torch.empty(size, dtype=torch.uint8, device=DEV).fill_(85)
                for size in sizes for _ in range(3)]
        torch.cuda.synchronize()
        got = tensors(results)
        assert len(got) == len(w)
        for a, b in zip(got, w):
            assert torch.equal(bits(a), b), name
        assert all((j == 85).all() for j in junk), f"{name} wrote to memory of the current stream"


@gpu
def test_the_callers_stream_stays_current():
    side = torch.cuda.Stream()
    x, w = torch.ones(4, 8, device=DEV), torch.ones(8, device=DEV)
    before = torch.cuda.current_stream()
    block.lbi_rms_norm(x, w, stream=side)
    with pytest.raises(ValueError):
        block.lbi_rms_norm(x, w[:4], stream=side)
    assert torch.cuda.current_stream() == before
    torch.cuda.synchronize()


def test_tensors_off_the_gpu_are_refused_with_a_stream_too():
    x = torch.ones(4, 8)
    with pytest.raises(ValueError):
        block.lbi_rms_norm(x, torch.ones(8), stream=7)


def test_a_workspace_off_the_gpu_is_refused():
    for need in (0, 16):
        with pytest.raises(ValueError):
            block._scratch(need, torch.empty(256, dtype=torch.uint8), 0)


@gpu
def test_a_workspace_with_gaps_is_refused():
    """What lies between its values is not its own."""
    x, w = torch.ones(6, 8, device=DEV), torch.ones(8, device=DEV)
    need = block.lbi_rms_norm_backward_workspace_bytes(6, 8)
    with pytest.raises(ValueError):
        block.lbi_rms_norm_backward(x, x, w, workspace=torch.empty(2 * need, dtype=torch.uint8,
                                                                  device=DEV)[::2])
    block.lbi_rms_norm_backward(x, x, w, workspace=torch.empty(need, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()


def test_a_call_makes_its_device_current(monkeypatch):
    """The default stream of every device has the same handle: the kernels go to the current device."""
    entered = []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            entered.append(self.index)

        def __exit__(self, *exc):
            entered.append("left")

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(block, "_current_device", lambda: 0)
    block._run(0, lambda *a: entered.append(a) or 0, 3)
    assert entered == [(3,)]
    entered.clear()
    block._run(1, lambda *a: entered.append(a) or 0, 4, 5)
    assert entered == [1, (4, 5), "left"]
    entered.clear()
    with pytest.raises(block.binding.LbiError):
        block._run(1, lambda: 2)
    assert entered == [1, "left"]
    # no entry point is called past it
    calls_of = open(block.__file__).read()
    assert calls_of.count("_check(") == 2 and calls_of.count("    _run(dev, ") == 9


@gpu
@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
def test_tensors_on_another_device():
    x = torch.randn(6, 8)
    want = block.lbi_rms_norm(x.to(DEV), torch.ones(8, device=DEV))[0].cpu()
    with torch.cuda.device(0):
        got = block.lbi_rms_norm(x.to("cuda:1"), torch.ones(8, device="cuda:1"))[0]
        assert torch.cuda.current_device() == 0
    assert got.device.index == 1 and torch.equal(got.cpu(), want)


@gpu
def test_outputs_by_a_name_that_no_input_has_are_refused():
    x, A, B = torch.zeros(6, 8, device=DEV), -torch.ones(8, 2, device=DEV), torch.zeros(6, 2, device=DEV)
    for name in ("du", "dout", "state_out"):
        with pytest.raises(ValueError):
            block.lbi_ssm_scan_backward(x, x, A, B, B, x, outputs={name: torch.empty_like(x)})
    torch.cuda.synchronize()
