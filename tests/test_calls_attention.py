"""The binding's native calls of the cache and of attention: what reaches the C function, and what is left to the Python function."""
import ctypes
import inspect

import pytest

from test_calls import F, INT, L, P, Stream, Tensor, Z, forget_streams

ROWS = [P, L, L]
KINDS = {                                                # the C functions' arguments as include/ngemm.h declares them
    "move": ("ngemm_kv_write", [P, P, INT, L, L] + ROWS + ROWS + [P, P, P, L, P]),
    "decode": ("ngemm_attention_decode", [P, P, INT, L, L] + ROWS + [P, L, P, L, F] + ROWS + [P, Z, P]),
    "prompt": ("ngemm_attention_prompt", [P, INT, L, L, L, L, L] + ROWS + [L] + ROWS + ROWS + [P, P, INT, F] + ROWS + [P, Z, P]),
}


@pytest.fixture
def both():
    from paper_1910_00178_amd import binding
    forget_streams()
    keep = []

    def make(kind, status=0):
        seen, given = [], []
        fn = ctypes.CFUNCTYPE(INT, *KINDS[kind][1])(lambda *a: (seen.append(a), status)[1])
        keep.append(fn)

        def slow(*a, **kw):
            given.append(a)
            return "slow"
        slow.__name__ = KINDS[kind][0]
        return binding._calls.Call(slow, kind, ctypes.cast(fn, P).value), seen, given
    yield make
    forget_streams()


def usual(kind):
    from paper_1910_00178_amd import binding
    args, want = [], []
    for n, name in enumerate(inspect.signature(getattr(binding, KINDS[kind][0])).parameters):
        at = 0x1000 * (n + 1)
        if name in ("ctx", "cache"): a, w = P(at), at
        elif name == "hip_stream": a, w = Stream(), 0x5eed
        elif name == "scale": a, w = 0.1, F(0.1).value
        elif name == "causal": a, w = True, 1
        elif name == "type": a, w = 2, 2
        elif name.endswith("_dev"): a, w = Tensor(at), at
        else: a, w = (1 << 40) + n, (1 << 40) + n
        args.append(a)
        want.append(w)
    return args, want


@pytest.mark.parametrize("kind", KINDS)
def test_native_call(both, kind):
    call, seen, given = both(kind)
    args, want = usual(kind)
    assert call(*args) is None and not given and list(seen[0]) == want
    call(*[a.value if type(a) is P else None if isinstance(a, Tensor) else a for a in args])
    assert not given and list(seen[1]) == [None if isinstance(a, Tensor) else w for a, w in zip(args, want)]
    # every other way of saying it goes to the Python function untouched, nothing having been called
    others = {P: ("0", 1.5, -1), Tensor: ("0", 1.5, -1, object()), Stream: ("0", 1.5, -1), float: (1, "x"), bool: ("x", None), int: (1.0, "1", 1 << 70, True)}
    for n, a in enumerate(args):
        for other in others[type(a)]:
            bad = args[:n] + [other] + args[n + 1:]
            assert call(*bad) == "slow" and given.pop() == tuple(bad)
    assert call() == "slow" and call(*args, 1) == "slow" and len(seen) == 2


@pytest.mark.parametrize("kind", KINDS)
def test_binding_holds_them(both, kind):
    from paper_1910_00178_amd import binding
    for name in [KINDS[kind][0]] + (["ngemm_kv_read"] if kind == "move" else []):
        fn = getattr(binding, name)
        assert type(fn) is binding._calls.Call and inspect.signature(fn) == inspect.signature(fn.__wrapped__)
        assert list(getattr(binding._lib, name).argtypes) == KINDS[kind][1]
    call, _, _ = both(kind, status=-2)
    with pytest.raises(binding.NgemmError, match=KINDS[kind][0] + ": bad shape"):
        call(*usual(kind)[0])
