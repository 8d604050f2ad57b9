"""The native argument marshalling (_otbind.so) of the MX4 entry points: it takes
exactly the arguments that the Python checks take, and leaves every other one to
them."""
import pytest
import torch

from paper_2406_18832_amd import ot

M, K, N = 5, 96, 33
E, F, TOP_K = 4, 64, 2


def _calls(device):
    """(native name, public function, arguments) of each marshalled call."""
    g = torch.Generator().manual_seed(3)
    u8 = lambda *s: torch.randint(0, 256, s, generator=g, dtype=torch.uint8).to(device)
    exps = lambda *s: torch.randint(120, 130, s, generator=g, dtype=torch.uint8).to(device)
    f32 = lambda *s: (torch.rand(*s, generator=g) + 0.1).to(device)
    f16 = lambda *s: torch.randn(*s, generator=g).half().to(device)
    packed = lambda n, k: exps(ot.ot_packed_weights_mx4_size(n, k))
    empty = lambda *s: torch.empty(s, dtype=torch.uint8, device=device)
    Xc, Xe = u8(M, K // 2), exps(1, M, 8)
    ws = empty(max(64, ot.ot_moe_mx4_workspace_size(M, K, F, E, TOP_K)))
    y = lambda n: torch.empty(M, n, dtype=torch.float16, device=device)
    return {
        "quantize_act_mx4": (ot.ot_quantize_act_mx4,
                             [f16(M, K), f32(K), f32(K), empty(M, K // 2), empty(1, M, 8)]),
        "ln_quantize_act_mx4": (ot.ot_ln_quantize_act_mx4,
                                [f16(M, K), f16(K), f16(K), 1e-5, f32(K), f32(K),
                                 empty(M, K // 2), empty(1, M, 8)]),
        "dequantize_mx4": (ot.ot_dequantize_mx4, [Xc, Xe, torch.empty(M, K, device=device)]),
        "qlinear_mx4": (ot.ot_qlinear_mx4, [Xc, Xe, packed(N, K), N, f32(N), y(N), ws]),
        "moe_mx4": (ot.ot_moe_mx4,
                    [Xc, Xe, f16(M, E), TOP_K, packed(E * 2 * F, K), f32(E, 2 * F),
                     packed(E * K, F), f32(E, K), F, "swiglu", y(K), ws]),
    }


NAMES = list(ot._BOUND_MX4)


def _native(name, args, stream=None):
    """The native call, as the public function makes it."""
    if name == "moe_mx4":
        args = args[:9] + [ot.MOE_ACTIVATIONS.get(args[9], 7)] + args[10:]
    return getattr(ot, "_n_" + name)(*args, stream)


def _wrong_arguments(args):
    """Each argument in turn replaced by ones the call does not take as it is."""
    for i, a in enumerate(args):
        if isinstance(a, str):
            yield args[:i] + ["gelu"] + args[i + 1:]
            continue
        wrong = [3.0 if isinstance(a, int) else 3]
        if isinstance(a, torch.Tensor):
            wrong += [a.to(torch.int16), a.reshape(-1)[:-1], a.unsqueeze(0)]
            if a.dim() == 2:
                wrong += [a.t(), torch.cat([a, a], 1)[:, ::2],
                          a.new_empty(a.shape[0], a.shape[1] + 16)]
            if a.dim() == 3:
                wrong += [a.transpose(1, 2), a.new_empty(2, *a.shape[1:])]
            if a.is_cuda:
                wrong.append(a.cpu())
        for w in wrong:
            yield args[:i] + [w] + args[i + 1:]


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_are_left_to_the_python_checks(name):
    ot.lib()
    call, args = _calls("cpu")[name]
    assert _native(name, args) is None
    with pytest.raises(ValueError, match="must be on the GPU"):
        call(*args)
    for wrong in _wrong_arguments(args):
        assert _native(name, wrong) is None
    assert getattr(ot, "_n_" + name)() is None


@pytest.mark.parametrize("name", NAMES)
def test_every_wrong_argument_is_named_by_an_error(name):
    """None of them reaches the library: on host tensors every call ends in an
    error of the binding."""
    call, args = _calls("cpu")[name]
    for wrong in _wrong_arguments(args):
        with pytest.raises((TypeError, ValueError, AttributeError)):
            call(*wrong)


def _outcome(call, args):
    try:
        call(*args)
    except Exception as e:
        return type(e).__name__, str(e)
    torch.cuda.synchronize()
    return [a.cpu().clone() if isinstance(a, torch.Tensor) else a for a in args]


def _same(a, b):
    if isinstance(a, tuple) or isinstance(b, tuple):
        return a == b
    return all(torch.equal(x.nan_to_num(), y.nan_to_num()) if isinstance(x, torch.Tensor)
               and x.is_floating_point() else torch.equal(x, y) if isinstance(x, torch.Tensor)
               else x == y for x, y in zip(a, b))


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_native_and_python_marshalling_agree(name, monkeypatch):
    print(f"[case] binding {name}", flush=True)
    ot.lib()
    call, args = _calls("cuda")[name]
    assert _native(name, args, ot._stream(None)) == ot.OT_OK
    torch.cuda.synchronize()
    refused = list(_wrong_arguments(args))
    first = [_outcome(call, c) for c in [args, *refused]]
    monkeypatch.setattr(ot, "_n_" + name, ot._unbound)
    second = [_outcome(call, c) for c in [args, *refused]]
    for i, (a, b) in enumerate(zip(first, second)):
        assert _same(a, b), (i, a, b)
    assert not isinstance(first[0], tuple)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device_are_refused(name, monkeypatch):
    """The launch goes to the current device; here that is said to be another one
    (the native side asks the runtime itself, and leaves such calls to this check)."""
    ot.lib()
    call, args = _calls("cuda")[name]
    monkeypatch.setattr(ot, "_n_" + name, ot._unbound)
    monkeypatch.setattr(ot, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device 1, not cuda:0"):
        call(*args)
