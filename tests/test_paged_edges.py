"""Refusals of the paged cache's calls over buffers that overlap: no GPU."""
import ctypes

from tests.test_paged import abi, cache  # noqa: F401


def test_arguments_inside_the_state_are_refused(abi, cache):  # noqa: F811
    """The calls write what follows the tables in the state, so their arguments
    must not lie there; assign writes the tables too, and takes them in place
    only."""
    f, c, sz = abi.lib(), ctypes.byref(cache), cache.sz
    at = lambda word: ctypes.c_void_p(cache.state + 4 * word)  # noqa: E731
    far, end = ctypes.c_void_p(0x100000), sz.state_bytes // 4
    for w in (0, 60, sz.lens_word + 1, sz.lens_word - 1, sz.table_word, sz.table_word - 1, sz.refs_word, sz.scratch_word, end - 1):
        assert f.semkv_paged_assign(c, at(w), far, None) == -1, w
    for w in (-1, 0, sz.lens_word, sz.table_word - 1, sz.table_word + 50, sz.refs_word, end - 1):
        assert f.semkv_paged_assign(c, far, at(w), None) == -1, w
    for w in (sz.refs_word - 1, sz.refs_word, sz.free_word, sz.scratch_word, end - 1):
        assert f.semkv_paged_reserve(c, at(w), None) == -1, w
        assert f.semkv_paged_fork(c, at(w), None) == -1, w
        assert f.semkv_paged_compact(c, far, 8, at(w), None) == -1, w
        assert f.semkv_paged_compact(c, at(w), 8, far, None) == -1, w
    assert f.semkv_paged_compact(c, at(sz.refs_word - 31), 8, far, None) == -1     # its last entry lies there


def test_set_up_publishes_its_lookups_at_once(monkeypatch):
    """A second thread's first call may look while the first one's is setting up:
    it must find everything or nothing."""
    import sys
    import types
    from paper_2608_28911_amd import paged
    seen = []

    class C:
        def __getattr__(self, name):                     # every lookup that the set-up makes
            seen.append(paged._torch)
            return lambda *a: 0

    for name in ("_torch", "_device", "_stream_of"):
        monkeypatch.setattr(paged, name, None, raising=False)
    fake = types.SimpleNamespace(_C=C(), cuda=C())
    monkeypatch.setitem(sys.modules, "torch", fake)
    paged._setup()
    assert len(seen) >= 2 and all(t is None for t in seen)
    assert paged._torch is fake and paged._device is not None and paged._stream_of is not None


def test_library_is_published_with_its_signatures(monkeypatch):
    """Without them ctypes passes addresses as 32-bit integers: a second thread's
    first call must not find the library before it has them all."""
    from paper_2608_28911_amd import _abi
    seen = []

    class Function:
        def __setattr__(self, name, value):
            seen.append(_abi._lib)
            object.__setattr__(self, name, value)

    class Library:
        def __init__(self, path):
            self.f = {}

        def __getattr__(self, name):
            return self.f.setdefault(name, Function())

    monkeypatch.setattr(_abi, "_lib", None)
    monkeypatch.setattr(_abi.ctypes, "CDLL", Library)
    got = _abi.lib()
    assert len(seen) == 2 * len(_abi.EXPORTS) and all(x is None for x in seen)
    assert _abi._lib is got and all(f.argtypes == _abi.EXPORTS[n][1] for n, f in got.f.items())
