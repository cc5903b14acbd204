"""What objects with a call's parameters keep between calls, threads and copies (CPU)."""
import copy
import dataclasses
import pickle
import threading

import pytest
import torch

import paper_2604_16429_amd as M
from paper_2604_16429_amd import binding

FAKE = 0x1000


class OnGpu:
    """What the binding looks at of a tensor, without its memory."""

    is_cuda = True

    def __init__(self, strides, *shape):
        self.shape, self.dtype, self.strides = torch.Size(shape), torch.bfloat16, strides

    def stride(self):
        return self.strides

    def data_ptr(self):
        return FAKE


def heads_first(b, h, n, d=64):
    return OnGpu((h * n * d, n * d, d, 1), b, h, n, d)


def tokens_first(b, h, n, d=64):
    return OnGpu((n * h * d, d, h * d, 1), b, h, n, d)


def strides_of(x):
    return x.batch, x.head, x.token


class Stub:
    """In place of the C library: the first call waits for another thread's whole call, then reads
    the parameters that it was given, as C code that runs without the interpreter's lock does."""

    def __init__(self, between, look):
        self.between, self.look, self.seen = between, look, []

    def __getattr__(self, name):
        def call(*args):
            if self.between is not None:
                between, self.between = self.between, None
                t = threading.Thread(target=between)
                t.start()
                t.join()
            self.seen.append(self.look(name, args))
            return 0
        return call


OBJECTS = pytest.mark.parametrize("other", [lambda p: p, copy.copy], ids=["shared", "copied"])


@OBJECTS
def test_windows_of_two_threads(other, monkeypatch):
    p = M.WindowParams(2, 4, 8, 64, 64, kv_heads=2, window_left=15, n_sink=4)
    tensors = [[make(2, h, n) for h, n in ((4, 8), (2, 64), (2, 64), (4, 8))] for make in (heads_first,
                                                                                           tokens_first)]
    M.mosaic_bsa_window_workspace_bytes(p, binding.OP_FWD)
    p2 = other(p)
    stub = Stub(lambda: M.mosaic_bsa_window_fwd(p2, *tensors[1], stream=0),
                lambda name, args: [strides_of(getattr(args[0]._obj, f)) for f in ("q", "k", "v", "out")])
    monkeypatch.setattr(binding, "_lib", stub)
    M.mosaic_bsa_window_fwd(p, *tensors[0], stream=0)
    assert len(stub.seen) == 2
    for seen, given in zip(stub.seen, (tensors[1], tensors[0])):
        assert seen == [t.strides[:3] for t in given]


@OBJECTS
def test_norm_gradients_of_two_threads(other, monkeypatch):
    p, rot = M.HeadsParams(2, 8, 4, 64, kv_heads=2, cache_tokens=16), M.Rotation(64)

    def grads(make):
        q, k = make(2, 4, 8), make(2, 2, 8)
        M.mosaic_bsa_qk_norm_rope_bwd(p2 if make is tokens_first else p, rot, FAKE, q, k, FAKE, FAKE, q, k, q, k,
                                      FAKE, FAKE, FAKE, stream=0, workspace_bytes=1 << 30)

    def forward():
        q, k, cache = tokens_first(2, 4, 8), tokens_first(2, 2, 8), tokens_first(2, 2, 16)
        M.mosaic_bsa_qk_norm_rope_fwd(p2, rot, FAKE, q, k, FAKE, FAKE, q, cache, v=k, v_out=cache, rows=FAKE,
                                      stream=0)

    def look(name, args):
        c = args[0]._obj
        if name.endswith("bwd"):
            return [strides_of(x) for x in (c.q, c.k, c.q_out, c.k_out, args[9]._obj, args[10]._obj)]
        return [strides_of(x) for x in (c.q, c.k, c.v, c.q_out, c.k_out, c.v_out)]

    M.mosaic_bsa_qk_norm_rope_workspace_bytes(p)
    p2 = other(p)
    for between in (lambda: grads(tokens_first), forward):
        stub = Stub(between, look)
        monkeypatch.setattr(binding, "_lib", stub)
        grads(heads_first)
        q, k = heads_first(2, 4, 8).strides[:3], heads_first(2, 2, 8).strides[:3]
        assert stub.seen[1] == [q, k, q, k, q, k]
        q, k, c = (tokens_first(2, h, n).strides[:3] for h, n in ((4, 8), (2, 8), (2, 16)))
        assert stub.seen[0] == ([q, k, q, k, q, k] if between is not forward else [q, k, k, q, c, c])


def test_positions_of_two_threads(monkeypatch):
    """Positions of each batch entry in one thread, shared ones in the other."""
    p, rot = M.HeadsParams(2, 8, 4, 64), M.Rotation(64)
    q = heads_first(2, 4, 8)

    class Positions(OnGpu):
        def __init__(self, *shape):
            super().__init__(None, *shape)
            self.dtype = torch.int32

        def is_contiguous(self):
            return True

    def call(pos):
        M.mosaic_bsa_rope_fwd(p, rot, pos, q, None, q, None, stream=0)

    stub = Stub(lambda: call(Positions(2, 8)), lambda name, args: args[0]._obj.position_batch)
    monkeypatch.setattr(binding, "_lib", stub)
    call(Positions(8))
    assert stub.seen == [8, 0]


def test_fields_set_between_calls(monkeypatch):
    """A field that was set counts from the next call on, also where the tensors are as before."""
    p = M.WindowParams(2, 4, 8, 64, 64, kv_heads=2, window_left=15)
    tensors = [heads_first(2, h, n) for h, n in ((4, 8), (2, 64), (2, 64), (4, 8))]
    stub = Stub(None, lambda name, args: args[0]._obj.window_left)
    monkeypatch.setattr(binding, "_lib", stub)
    for left in (15, 20, 15, 3):
        p.window_left = left
        M.mosaic_bsa_window_fwd(p, *tensors, stream=0)
    assert stub.seen == [15, 20, 15, 3]


def test_many_layouts_of_one_object(monkeypatch):
    """What an object keeps of its calls does not grow with them."""
    p = M.WindowParams(1, 1, 8, 8, 64)
    stub = Stub(None, lambda name, args: args[0]._obj.q.token)
    monkeypatch.setattr(binding, "_lib", stub)
    tokens = [64 + 8 * i for i in range(1000)]
    for t in tokens:
        q = OnGpu((8 * t, 8 * t, t, 1), 1, 1, 8, 64)
        M.mosaic_bsa_window_fwd(p, q, q, q, q, stream=0)
    assert stub.seen == tokens
    assert all(len(x) <= 64 for x in p.__dict__.values() if isinstance(x, dict))


COPIES = pytest.mark.parametrize("copied", [copy.copy, copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x))],
                                 ids=["copy", "deepcopy", "pickle"])


@COPIES
@pytest.mark.parametrize("used", [False, True])
def test_copies_of_parameters(copied, used):
    """Also after a call, which leaves a struct in the object."""
    for p in (M.HeadsParams(2, 8, 4, 64, kv_heads=2, norm_eps=1e-5), M.WindowParams(2, 4, 8, 64, 64, n_sink=3)):
        size = (M.mosaic_bsa_qk_norm_rope_workspace_bytes if isinstance(p, M.HeadsParams) else
                lambda x: M.mosaic_bsa_window_workspace_bytes(x, binding.OP_BWD))
        want = size(p) if used else size(dataclasses.replace(p))
        c = copied(p)
        assert c == p and type(c) is type(p) and size(c) == want
        c.batch = 1
        assert p.batch == 2 and size(p) == want


@COPIES
def test_copies_of_rotations(copied):
    a = M.Rotation(64, axes=2, layout=binding.ROTATE_PAIRS, theta=500.0)
    b = copied(a)
    assert bytes(a.c) == bytes(b.c) and b.axes == 2
    b.c.turns[0] = 5
    b.c.rotary_dim = 32
    assert a.c.turns[0] != 5 and a.c.rotary_dim == 64          # memory of its own
    assert b.ref._obj is b.c
