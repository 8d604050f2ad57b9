"""The native argument marshalling (_otbind.so) of the 8-bit cache's entry points: it
takes exactly the arguments that the Python checks take, and leaves every other one to
them."""
import pytest
import torch

from paper_2406_18832_amd import ot

T, B, H, G, D, PAGES = 5, 2, 3, 2, 80, 7


def _calls(device):
    """(native name, public function, arguments) of each marshalled call."""
    g = torch.Generator().manual_seed(3)
    f16 = lambda *s: torch.randn(*s, generator=g).half().to(device)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=device)
    cu, kv_len, table = i32(0, 2, 5), i32(70, 3), i32([0, 1, -1], [2, -1, -1])

    def cache():
        c = ot.kv8_cache(PAGES, H, D, device)
        for t in c[:2]:
            t.random_(generator=torch.Generator(device=device).manual_seed(4))
        for t in c[2:]:
            t.fill_(0.01)
        return c
    x = f16(T, (G + 2) * H * D)
    q, k, v = x.split((G * H * D, H * D, H * D), 1)
    q, k, v = q.view(T, G * H, D), k.view(T, H, D), v.view(T, H, D)
    need = ot.ot_attn_kv8_workspace_size(T, B, G * H, H, D, 3)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    zeros = lambda *s: torch.zeros(s, dtype=torch.float16, device=device)
    return {
        "kv8_append": (ot.ot_kv8_append, [k, v, cu, kv_len, table, *cache()]),
        "kv8_read": (ot.ot_kv8_read, [*cache(), cu, i32(66, 0), table, zeros(T, H, D), zeros(T, H, D)]),
        "attn_kv8": (ot.ot_attn_kv8, [q, cu, kv_len, table, *cache(), 0.1, True, 0, 3,
                                      zeros(T, G * H, D), torch.zeros(T, G * H, device=device), ws]),
    }


NAMES = list(ot._BOUND_KV8)


def _native(name, args, stream=None):
    return getattr(ot, "_n_" + name)(*args, stream)


def _wrong_tensors(args):
    """Each tensor in turn replaced by ones the call does not take."""
    for i, a in enumerate(args):
        if isinstance(a, torch.Tensor):
            wrong = [3, None if i not in (len(args) - 1, len(args) - 2) else 3, a.to(torch.int16),
                     a.reshape(-1)[:-1], a.unsqueeze(0)]
            if a.dim() >= 2:
                wrong += [a.transpose(-1, -2).contiguous().transpose(-1, -2),
                          torch.cat([a, a], 0)[::2][:, : a.shape[1] - 1],
                          torch.cat([a, a], -1)[..., ::2]]
            if a.is_cuda:
                wrong.append(a.cpu())
            for w in wrong:
                yield args[:i] + [w] + args[i + 1:]


def _wrong_numbers(name, args):
    if name == "attn_kv8":
        yield args[:8] + ["0.1"] + args[9:]
        yield args[:10] + ["0"] + args[11:]
        yield args[:11] + [None] + args[12:]


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_are_left_to_the_python_checks(name):
    ot.lib()
    call, args = _calls("cpu")[name]
    assert _native(name, args) is None
    with pytest.raises(ValueError, match="must be on the GPU"):
        call(*args)
    for wrong in _wrong_tensors(args):
        assert _native(name, wrong) is None
    assert getattr(ot, "_n_" + name)() is None


@pytest.mark.parametrize("name", NAMES)
def test_every_wrong_argument_is_named_by_an_error(name):
    """None of them reaches the library: on host tensors every call ends in an error of
    the binding."""
    call, args = _calls("cpu")[name]
    for wrong in [*_wrong_tensors(args), *_wrong_numbers(name, args)]:
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
    refused = [*_wrong_tensors(args), *_wrong_numbers(name, args)]
    if name == "attn_kv8":  # taken by Python alone, or refused by the library
        refused += [args[:8] + [1] + args[9:], args[:9] + [1] + args[10:], args[:11] + [0] + args[12:],
                    args[:10] + [-1] + args[11:], args[:-1] + [None], args[:-2] + [None, None]]
    first = [_outcome(call, c) for c in [args, *refused]]
    monkeypatch.setattr(ot, "_n_" + name, ot._unbound)
    second = [_outcome(call, c) for c in [args, *refused]]
    for i, (a, b) in enumerate(zip(first, second)):
        assert _same(a, b), (i, a, b)
    assert not isinstance(first[0], tuple)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device_are_refused(name, monkeypatch):
    ot.lib()
    call, args = _calls("cuda")[name]
    monkeypatch.setattr(ot, "_n_" + name, ot._unbound)
    monkeypatch.setattr(ot, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device 1, not cuda:0"):
        call(*args)
