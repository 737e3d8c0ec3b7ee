"""Streams and devices of the helpers' calls.

What the helpers make for a call on another stream is allocated (and filled)
with that stream current, so that the fill and whatever used the memory before come
ahead of the kernels, and outputs are kept from reuse until the caller's own stream is
done with them.  Calls on another device than the current one are refused.  Tensors,
streams and the library are stand-ins: nothing is launched."""
import contextlib
import math

import pytest
import torch

from paper_2609_06663_gb300 import ecokv as E

D = 128


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class World:
    """Torch's current stream, and a library that notes the calls it gets."""

    def __init__(self):
        self.here = self.current = Stream(0)
        self.made, self.calls, self.device = [], [], 0

    @contextlib.contextmanager
    def stream(self, s):
        before, self.current = self.current, s
        yield
        self.current = before

    def __getattr__(self, name):  # the library's functions; sizes are asked for, the rest is launched
        def call(*args):
            if "workspace_size" in name:
                return 4096
            if "params" not in name:
                self.calls.append((name, args))
            return 0
        return call


class Tensor:
    def __init__(self, world, *shape, dtype=torch.bfloat16, device="cuda:0"):
        self.world, self.shape, self.dtype, self.device = world, shape, dtype, torch.device(device)
        self.made_on, self.kept_for, self.is_cuda = world.current, [], True
        world.made.append(self)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def stride(self):
        return tuple(math.prod(self.shape[i + 1:]) for i in range(len(self.shape)))

    def data_ptr(self):
        return 1 << 20

    def get_device(self):
        return -1 if self.device.type == "cpu" else self.device.index

    def is_contiguous(self):
        return True

    def new_empty(self, shape):
        return Tensor(self.world, *shape, dtype=self.dtype)

    def record_stream(self, s):
        self.kept_for.append(s)

    def item(self):
        assert self.world.current.cuda_stream == self.world.calls[-1][1][-1]  # else it would not wait for the call
        return 0


class Host:
    """A tensor in host memory: not of any stream."""
    dtype = torch.bfloat16

    def pin_memory(self):
        return self

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def world(monkeypatch):
    w = World()

    def make(*shape, dtype=None, device=None):
        if device is None:
            return Host()
        return Tensor(w, *(shape[0] if isinstance(shape[0], tuple) else shape), dtype=dtype)

    monkeypatch.setattr(E, "_lib", w)
    monkeypatch.setattr(E, "_raw_stream", lambda dev: w.current.cuda_stream)
    monkeypatch.setattr(E, "_get_device", lambda: w.device, raising=False)
    monkeypatch.setattr(torch, "zeros", make)
    monkeypatch.setattr(torch, "empty", make)
    monkeypatch.setattr(torch, "full", lambda shape, value, dtype, device: make(shape, dtype=dtype, device=device))
    for like in ("empty_like", "zeros_like"):
        monkeypatch.setattr(torch, like, lambda x: x.new_empty(x.shape))
    monkeypatch.setattr(torch.cuda, "stream", w.stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: w.current)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda dev=None: w.here)

    def external(handle, device=None):
        assert handle != 0  # (to torch that means any stream of its pool)
        return Stream(handle)

    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    return w


def decode_calls(w, stream):
    t = lambda *n, **kw: Tensor(w, *n, **kw)  # noqa: E731
    i32 = dict(dtype=torch.int32)
    q, k, v = t(3, 8, D), t(3, 4, D), t(3, 4, D)
    cache = E.PagedCache(t(10, 4, 16, D), t(10, 4, 16, D), t(3, 5, **i32), t(3, **i32))
    rot = E.ecokv_rotary(rot_dim=D, axes=1)
    pos = t(1, 3, **i32)
    del w.made[:]
    yield "ecokv_rotate", lambda: E.rotate(rot, pos, q, k, stream=stream), 2
    yield "ecokv_append", lambda: (E.append(cache, k, v, None, rot, pos, q, stream=stream),), 1
    yield "ecokv_attend", lambda: (E.attend(q, None, cache, stream=stream),), 1


@pytest.mark.parametrize("raw", [False, True])
def test_decode_helpers_make_tensors_on_the_stream_of_the_call(world, raw):
    side = Stream(4096)
    for name, call, outs in decode_calls(world, 4096 if raw else side):
        got = call()
        assert world.calls[-1][0] == name and world.calls[-1][1][-1] == 4096
        assert len(world.made) >= outs and world.current is world.here
        for x in world.made:
            assert x.made_on.cuda_stream == 4096, name
        for x in got:
            assert x in world.made and world.here in x.kept_for, name
        del world.made[:]


def test_decode_helpers_without_a_stream_run_on_torchs_current_one(world):
    side = Stream(8192)
    for name, call, outs in decode_calls(world, None):
        with world.stream(side):
            call()
        assert world.calls[-1][0] == name and world.calls[-1][1][-1] == 8192
        assert len(world.made) >= outs and all(x.made_on is side for x in world.made)
        del world.made[:]


def test_a_raw_handle_of_the_default_stream(world):
    side = Stream(8192)
    for name, call, _ in decode_calls(world, 0):
        with world.stream(side):
            call()
        assert world.calls[-1][1][-1] == 0 and all(x.made_on is world.here for x in world.made), name
        del world.made[:]


def evict_calls(w, stream):
    p = E.ecokv_params(n_layers=1, h_kv=4, h_q=8, n=500, d=D, window=4, budget=50)
    K, Q, S, idx = Tensor(w, 1, 4, 500, D), Tensor(w, 1, 8, 4, D), Tensor(w, 1, 4, 496), Tensor(w, 1, 4, 50)
    kw = dict(stream=stream)
    del w.made[:]
    yield "ecokv_score", lambda: E.score(p, K, Q, dbg=True, **kw)
    yield "ecokv_select", lambda: (E.select(p, S, **kw),)
    yield "ecokv_compact", lambda: E.compact(p, K, K, idx, **kw)
    yield "ecokv_evict", lambda: E.evict(p, K, K, Q, want_scores=True, **kw)
    yield "ecokv_evict_adaptive", lambda: E.evict_adaptive(p, K, K, Q, **kw)
    yield "ecokv_evict_layered", lambda: E.evict_layered(p, K, K, Q, [50], want_scores=True, **kw)
    yield "ecokv_evict_host", lambda: E.evict_host(p, Host(), Host(), Host(), **kw)
    yield "ecokv_evict_noalloc", lambda: E.evict_noalloc(p, K, K, Q, want_scores=True, **kw)


@pytest.mark.parametrize("raw", [False, True])
def test_eviction_helpers_make_tensors_on_the_stream_of_the_call(world, raw):
    for name, call in evict_calls(world, 4096 if raw else Stream(4096)):
        got = call()
        assert world.calls[-1][0] == name and world.calls[-1][1][-1] == 4096 and world.current is world.here
        assert world.made and all(x.made_on.cuda_stream == 4096 for x in world.made), name
        outs = [x for x in got if isinstance(x, Tensor)]
        assert (outs or name == "ecokv_evict_host") and all(world.here in x.kept_for for x in outs), name
        del world.made[:]


def test_eviction_helpers_without_a_stream_run_on_torchs_current_one(world):
    side = Stream(8192)
    for name, call in evict_calls(world, None):
        with world.stream(side):
            call()
        assert world.calls[-1][0] == name and world.calls[-1][1][-1] == 8192, name
        assert world.made and all(x.made_on is side for x in world.made), name
        del world.made[:]


@pytest.mark.parametrize("own_stream", [False, True])
def test_calls_on_another_device_than_the_current_one_are_refused(world, own_stream):
    """The library launches on the current device: a stream of another one's tensors would not be that device's."""
    stream = Stream(4096) if own_stream else None
    calls = [c[:2] for c in decode_calls(world, stream)]
    calls += [c for c in evict_calls(world, stream) if c[0] != "ecokv_evict_host"]  # (host tensors)
    world.device = 1
    for name, call in calls:
        with pytest.raises(ValueError):
            call()
        assert not world.calls, name


@pytest.mark.parametrize("where", ["cuda:1", "cpu"])
def test_every_tensor_of_a_call_is_on_its_device(world, where):
    t = lambda *n, **kw: Tensor(world, *n, **kw)  # noqa: E731
    i32, there = dict(dtype=torch.int32), dict(device=where)
    u8, f32 = dict(dtype=torch.uint8), dict(dtype=torch.float32)
    q, k = t(3, 8, D), t(3, 4, D)
    pages, table, lengths = t(10, 4, 16, D), t(3, 5, **i32), t(3, **i32)
    cache = E.PagedCache(pages, pages, table, lengths)
    rot, pos = E.ecokv_rotary(rot_dim=D, axes=1), t(1, 3, **i32)
    refused = [
        lambda: E.rotate(rot, t(1, 3, **i32, **there), q),
        lambda: E.append(cache, k, k, None, rot, t(1, 3, **i32, **there)),
        lambda: E.append(cache, k, k, t(4, **i32, **there)),
        lambda: E.append(cache, k, k, ws=t(4096, **u8, **there)),
        lambda: E.attend(q, None, cache, t(4, **i32, **there)),
        lambda: E.attend(q, None, cache, lse=t(3, 8, **f32, **there)),
        lambda: E.attend(q, None, cache, ws=t(4096, **u8, **there)),
        lambda: E.PagedCache(pages, pages, t(3, 5, **i32, **there), lengths),
        lambda: E.PagedCache(pages, pages, table, t(3, **i32, **there)),
        lambda: E.Prefix(t(30, D), t(30, D), t(5, **i32, **there)),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(i))
        assert not world.calls, i
    E.rotate(rot, pos, q)
    E.append(cache, k, k, t(4, **i32), rot, pos, ws=t(4096, **u8))
    E.attend(q, None, cache, t(4, **i32), lse=t(3, 8, **f32), ws=t(4096, **u8))
    assert len(world.calls) == 3


def test_handles_keep_the_tensors_whose_addresses_they_hold(world):
    t = lambda *n, **kw: Tensor(world, *n, **kw)  # noqa: E731
    i32 = dict(dtype=torch.int32)
    cache = E.PagedCache(t(10, 4, 16, D), t(10, 4, 16, D), t(3, 5, **i32), t(3, **i32))
    prefix = E.Prefix(t(30, D), t(30, D), t(5, **i32))
    for handle, names in ((cache, ("k_pages", "v_pages", "table", "lengths")), (prefix, ("k", "v", "head_off"))):
        for name in names:
            x = getattr(handle, name)
            with pytest.raises(AttributeError):
                setattr(handle, name, t(*x.shape, dtype=x.dtype))
            assert getattr(handle, name) is x
            setattr(handle, name, x)  # (what an operation in place does: cache.lengths += 1)
