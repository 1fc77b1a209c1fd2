"""The marshalling module by itself, on stand-ins: tensors that are ordinary objects, and entry points of a small C library.  A copy of the module
is loaded, so that the package's own keeps its entry points."""
import ctypes as C
import importlib.util
import os
import shutil
import subprocess
import threading
import time

import pytest

CODE = r"""
#include <unistd.h>
#include <stdint.h>
volatile int entered, released;
/* any entry point: waits until it is released, 2 s at most, and says whether it was */
int hold(void) {
  entered = 1;
  for (int i = 0; i < 2000 && !released; ++i) usleep(1000);
  return released ? 0 : -100;
}
int64_t nothing(void) { return 0; }
"""


class Tensor:
    def __init__(self, dtype, *shape, device=0, pointer=4096):
        self.dtype, self.shape, self.device, self.pointer = dtype, shape, device, pointer

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return True

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def dim(self):
        return len(self.shape)

    def size(self, i):
        return self.shape[i]

    def stride(self, i):
        n = 1
        for s in self.shape[i + 1:]:
            n *= s
        return n

    def data_ptr(self):
        return self.pointer


I32, I64, F32, F64, BF16, F16 = KINDS = tuple(object() for _ in range(6))


@pytest.fixture(scope="module")
def loaded(tmp_path_factory):
    from paper_2608_16305_b200 import build
    build.build_library()
    d = tmp_path_factory.mktemp("marshal")
    copy = os.path.join(d, "_marshal.so")
    shutil.copy(os.path.join(build.HERE, "_marshal.so"), copy)
    spec = importlib.util.spec_from_file_location("_marshal", copy)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    src, lib = os.path.join(d, "fake.c"), os.path.join(d, "fake.so")
    with open(src, "w") as f:
        f.write(CODE)
    subprocess.check_call([os.environ.get("CC", "gcc"), "-shared", "-fPIC", "-O1", "-o", lib, src])
    fake = C.CDLL(lib)
    addr = lambda f: C.cast(f, C.c_void_p).value
    m.init(KINDS, lambda: 0, lambda d: 0, tuple(addr(fake.nothing if i == 5 else fake.hold) for i in range(7)))
    return m, fake


def _calls():
    n, H, KV, D, S, P = 3, 4, 2, 8, 5, 50
    t = lambda k, *s: Tensor(k, *s)
    st = t(I32, 1)
    bias = [t(F32, H, 6), t(F64, 5), t(F64, n)]
    slot = [t(F32, n, H, D), t(F32, n, S, KV, D), t(F32, n, S, KV, D), t(I32, n), None, *bias, t(F64, n, S)]
    move = [4096, 0, 10, KV, D, t(F32, 7, KV, D), st, t(I64, 4), t(I64, 4), t(F64, 7)]
    return {
        "sample_window": [t(I64, 4), t(I32, P), t(I32, P), t(F64, P), t(I32, n), t(F64, n), 4, 1, t(I32, n, 5), t(I32, n, 5), t(F64, n, 5), t(I32, n),
                          t(I64, n), t(I32, n), st],
        "cache_write": [True, *move],
        "cache_read": [False, *move],
        "cached_attend": [4096, 4096, 0, P, D, t(F32, n, H, D), t(I64, n), t(I32, n), 4, 1, 0, None, t(F32, n, H, D), st, *bias, t(F64, P)],
        "slot_attend": [*slot, t(F32, n, H, D)],
        "slot_attend_backward": [*slot, t(F32, n, H, D), t(F32, n, H, D), t(F32, n, S, KV, D), t(F32, n, S, KV, D), t(F32, H, 6), t(F32, 1)],
    }


def _function(m, name):
    return getattr(m, "cache_move" if name.startswith("cache_") else name)


@pytest.mark.parametrize("name", list(_calls()))
def test_other_threads_run_while_the_library_is_called(loaded, name):
    """A launch may wait (for a full queue, for a module's first loading): the interpreter is free meanwhile, as it is under ctypes."""
    m, fake = loaded
    entered, released = (C.c_int.in_dll(fake, x) for x in ("entered", "released"))
    entered.value = released.value = 0
    got = []
    th = threading.Thread(target=lambda: got.append(_function(m, name)(*_calls()[name])))
    th.start()
    end = time.monotonic() + 30
    while not entered.value and th.is_alive() and time.monotonic() < end:
        time.sleep(0.001)
    released.value = 1
    th.join()
    assert got == [None]


class _Broken(Tensor):
    def __init__(self, method, error, *a):
        super().__init__(*a)

        def fail(*args):
            raise error
        setattr(self, method, fail)


def _tensors(name):
    return [i for i, a in enumerate(_calls()[name]) if isinstance(a, Tensor)]


@pytest.mark.parametrize("method", ["data_ptr", "numel", "get_device", "is_contiguous", "dim", "size", "stride"])
@pytest.mark.parametrize("name", list(_calls()))
def test_what_a_tensors_method_raises_is_what_the_call_raises(loaded, name, method):
    """A tensor without storage (a fake one) raises when it is asked for its address: the caller sees that, not an address that is refused."""
    m, fake = loaded
    C.c_int.in_dll(fake, "released").value = 1
    for error in (RuntimeError("it has no storage"), KeyboardInterrupt()):
        seen = 0
        for i in _tensors(name):
            args = _calls()[name]
            args[i] = _Broken(method, error, args[i].dtype, *args[i].shape)
            try:
                assert _function(m, name)(*args) is None           # (not every tensor is asked everything)
            except type(error) as e:
                assert e is error
                seen += 1
        # dimensions are asked for where a shape is looked at, strides of rows that are apart (below) only
        asks = name != "sample_window" if method in ("dim", "size") else method != "stride"
        assert seen >= (len(_tensors(name)) if method == "data_ptr" else int(asks))


@pytest.mark.parametrize("name", ["cache_write", "cache_read"])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_what_the_strides_of_rows_raise(loaded, name, which):
    m, fake = loaded
    C.c_int.in_dll(fake, "released").value = 1
    args, error = _calls()[name], ValueError("no strides")

    class Apart(Tensor):
        def is_contiguous(self):
            return False

        def stride(self, i):
            if i == which:
                raise error
            return super().stride(i)
    args[6] = Apart(F32, 7, 2, 8)
    with pytest.raises(ValueError) as e:
        _function(m, name)(*args)
    assert e.value is error


@pytest.mark.parametrize("name", list(_calls()))
def test_what_is_no_tensor_raises_type_error(loaded, name):
    m, fake = loaded
    C.c_int.in_dll(fake, "released").value = 1

    class Bare:
        pass
    for i in _tensors(name):
        for gone in ("data_ptr", "numel", "get_device"):
            args = _calls()[name]
            t, bare = args[i], Bare()
            for method in ("get_device", "is_contiguous", "numel", "dim", "size", "stride", "data_ptr"):
                if method != gone:
                    setattr(bare, method, getattr(t, method))
            bare.dtype = t.dtype
            args[i] = bare
            try:
                assert _function(m, name)(*args) is None and gone != "data_ptr"
            except TypeError as e:
                assert str(e)
    assert _function(m, name)(*_calls()[name]) is None             # and nothing of it is left behind
