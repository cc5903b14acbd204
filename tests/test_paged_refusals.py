"""What the entry points of the cache in pages refuse, on the host, before anything is launched."""
import copy
import ctypes
import pickle

import pytest
import torch

import paper_2604_16429_amd as M
from paper_2604_16429_amd import binding

FAKE = 0x1000            # never read: the checks fail first


def params(**kw):
    base = dict(batch=2, heads=4, q_tokens=8, head_dim=64, pages=16, page_tokens=16, table_pages=4,
                dtype=binding.BF16, kv_heads=2, prefix_tokens=20)
    base.update(kw)
    return M.PagedParams(**base)


def code_of(call):
    with pytest.raises(M.BsaError) as e:
        call()
    return e.value.code


def append(p, rot=None, pos=None, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, q_weight=FAKE, k_weight=FAKE, q_lens=FAKE, k_lens=FAKE,
             page_table=FAKE, prefix_len=FAKE, q_out=FAKE, k_pages=FAKE, v_pages=FAKE)
    a.update(kw)
    M.mosaic_bsa_paged_append(p, rot or M.Rotation(64), pos, *a.values(), stream=0)


def attend(p, nbytes=1 << 40, **kw):
    a = dict(q=FAKE, k_pages=FAKE, v_pages=FAKE, q_lens=FAKE, k_lens=FAKE, page_table=FAKE,
             prefix_table=FAKE, prefix_len=FAKE, out=FAKE, lse=FAKE, workspace=FAKE)
    a.update(kw)
    M.mosaic_bsa_paged_fwd(p, *a.values(), stream=0, workspace_bytes=nbytes)


def test_struct_layout_matches_the_header():
    assert ctypes.sizeof(binding._CPagedParams) == 64 + 6 * 24


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -2), (dict(heads=0), -2), (dict(q_tokens=0), -2), (dict(kv_heads=-1), -2),
    (dict(kv_heads=3), -2), (dict(kv_heads=8), -2), (dict(head_dim=48), -4), (dict(head_dim=256), -4),
    (dict(dtype=2), -5), (dict(pages=0), -13), (dict(page_tokens=0), -13), (dict(page_tokens=24), -13),
    (dict(page_tokens=-16), -13), (dict(page_tokens=1 << 17), -13), (dict(table_pages=0), -13),
    (dict(table_pages=1 << 25), -13), (dict(prefix_tokens=-1), -13), (dict(prefix_tokens=1 << 29), -13),
    (dict(q_tokens=1 << 28), -2), (dict(batch=1 << 21), -2),
])
def test_parameters(kw, code):
    p = params(**kw)
    assert code_of(lambda: append(p)) == code
    assert code_of(lambda: attend(p)) == code
    assert M.mosaic_bsa_paged_workspace_bytes(p) == 0


def test_parameters_of_one_entry_point():
    assert code_of(lambda: attend(params(n_sink=-1))) == -12
    assert code_of(lambda: attend(params(batch=1 << 20, kv_heads=1, q_tokens=128))) == -2
    assert code_of(lambda: append(params(norm_eps=-1.0))) == -2
    assert code_of(lambda: append(params(norm_eps=float("nan")))) == -2
    assert code_of(lambda: append(params(batch=1 << 20, q_tokens=1 << 11))) == -2
    assert code_of(lambda: append(params(head_dim=32))) == -10                  # rotation wider than the head
    assert code_of(lambda: append(params(), M.Rotation(64, axes=2))) == -1      # no positions


@pytest.mark.parametrize("name", ["q", "k", "v", "k_lens", "page_table", "q_out", "k_pages", "v_pages"])
def test_append_needs(name):
    assert code_of(lambda: append(params(), **{name: None})) == -1


@pytest.mark.parametrize("name", ["q_weight", "k_weight"])
def test_append_takes_both_weights_or_none(name):
    assert code_of(lambda: append(params(), **{name: None})) == -1


@pytest.mark.parametrize("name", ["q", "k_pages", "v_pages", "k_lens", "page_table", "prefix_table", "out"])
def test_attention_needs(name):
    assert code_of(lambda: attend(params(), **{name: None})) == -1


@pytest.mark.parametrize("name", ["q", "k_pages", "v_pages", "out", "workspace"])
def test_attention_wants_16_bytes(name):
    assert code_of(lambda: attend(params(), **{name: FAKE + 8})) == -7


@pytest.mark.parametrize("name", ["q_lens", "k_lens", "page_table", "prefix_table", "prefix_len", "lse"])
def test_attention_wants_whole_words(name):
    assert code_of(lambda: attend(params(), **{name: FAKE + 2})) == -7


@pytest.mark.parametrize("name,by", [("q", 1), ("k", 1), ("v", 1), ("q_out", 1), ("k_pages", 1), ("v_pages", 1),
                                     ("q_weight", 2), ("k_weight", 2), ("q_lens", 2), ("k_lens", 2),
                                     ("page_table", 2), ("prefix_len", 2)])
def test_append_wants_whole_elements(name, by):
    assert code_of(lambda: append(params(), **{name: FAKE + by})) == -7


def test_workspace():
    p = params(batch=24, heads=16, q_tokens=1, head_dim=128, table_pages=100, prefix_tokens=28800)
    n = M.mosaic_bsa_paged_workspace_bytes(p)
    if n:
        assert code_of(lambda: attend(p, nbytes=n - 1)) == -6
        assert code_of(lambda: attend(p, workspace=None)) == -6


@pytest.mark.parametrize("field,strides,code", [
    ("q", (8 * 512, -64, 64), -11), ("out", (8 * 4 * 64, 8 * 64, 32), -11), ("out", (64, 64, 64), -11),
    ("out", (2048, 512, 60), -11), ("k_pages", (1 << 41, 1024, 64), -11), ("q", (2048, 512, 68), -7),
    ("v_pages", (2048, 1020, 64), -7)])
def test_strides(field, strides, code):
    p = params()
    c = p._new_struct()
    setattr(c, field, binding._CStrides(*strides))
    got = M.load_library().mosaic_bsa_paged_fwd(ctypes.byref(c), *([FAKE] * 11), 1 << 40, None)
    assert got == code


@pytest.mark.parametrize("field,strides", [("k_pages", (1024, 1024, 64)), ("v_pages", (2048, 1024, 32)),
                                           ("out", (2048, 512, 0x7fffffffffff)), ("k", (0, 0, -1))])
def test_strides_of_append(field, strides):
    p, rot = params(), M.Rotation(64)
    c = p._new_struct()
    setattr(c, field, binding._CStrides(*strides))
    assert M.load_library().mosaic_bsa_paged_append(ctypes.byref(c), rot.ref, *([FAKE] * 13), None) == -11


def test_tensors_of_another_shape_or_place():
    p = params()
    q = torch.zeros(2, 4, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        attend(p, q=q)                                   # on the CPU
    with pytest.raises(ValueError):
        attend(p, k_pages=torch.zeros(2, 2, 16, 64))
    with pytest.raises(ValueError):
        attend(p, k_lens=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        attend(p, page_table=torch.zeros(2, 5, dtype=torch.int32))
    with pytest.raises(ValueError):
        append(p, prefix_len=torch.zeros(1, dtype=torch.int64))


class OnGpu:
    """A tensor of some GPU: shape, strides and an address, nothing behind it."""

    def __init__(self, device, *shape, dtype=torch.bfloat16):
        self.t, self.index = torch.empty(shape, dtype=dtype, device="meta"), device
        self.shape, self.dtype, self.is_cuda, self.device = self.t.shape, dtype, True, f"cuda:{device}"

    def stride(self):
        return self.t.stride()

    def numel(self):
        return self.t.numel()

    def is_contiguous(self):
        return True

    def element_size(self):
        return self.t.element_size()

    def get_device(self):
        return self.index

    def data_ptr(self):
        return FAKE


class Library:
    """Takes every call."""

    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return 0
        return call


def tensors(device):
    i32 = torch.int32
    return dict(q=OnGpu(device, 2, 4, 8, 64), k_pages=OnGpu(device, 16, 2, 16, 64),
                v_pages=OnGpu(device, 16, 2, 16, 64), q_lens=OnGpu(device, 2, dtype=i32),
                k_lens=OnGpu(device, 2, dtype=i32), page_table=OnGpu(device, 2, 4, dtype=i32),
                prefix_table=OnGpu(device, 2, dtype=i32), prefix_len=OnGpu(device, 1, dtype=i32),
                out=OnGpu(device, 2, 4, 8, 64), lse=OnGpu(device, 2, 4, 8, dtype=torch.float32),
                workspace=OnGpu(device, 1 << 20, dtype=torch.uint8))


def append_tensors(device):
    t = tensors(device)
    new = {n: OnGpu(device, 2, c, 8, 64) for n, c in (("q", 4), ("k", 2), ("v", 2), ("q_out", 4))}
    w = {n: OnGpu(device, 64, dtype=torch.float32) for n in ("q_weight", "k_weight")}
    return {**new, **w, **{n: t[n] for n in ("q_lens", "k_lens", "page_table", "prefix_len", "k_pages", "v_pages")}}


@pytest.mark.parametrize("call,make", [(attend, tensors), (append, append_tensors)], ids=["attend", "append"])
def test_tensors_of_two_gpus(monkeypatch, call, make):
    lib, p = Library(), params()
    rot = M.Rotation(64)
    monkeypatch.setattr(binding, "_lib", lib)
    extra = {"rot": rot} if call is append else {}
    for device in (1, 0):
        monkeypatch.setattr(binding, "_raw_stream", (lambda device: 0, lambda: device))
        call(p, **extra, **make(device))
        with pytest.raises(ValueError):
            call(p, **extra, **make(1 - device))           # (stream 0 is the current GPU's)
    assert lib.calls == 2
    for name in make(0):
        with pytest.raises(ValueError):
            call(p, **extra, **{**make(0), name: make(1)[name]})
    assert lib.calls == 2
    monkeypatch.setattr(binding, "_raw_stream", (lambda device: 0, lambda: 1))     # GPU 1 is the current one
    t = make(0)
    if call is attend:
        with pytest.raises(ValueError):
            M.mosaic_bsa_paged_fwd(p, *t.values())
        M.mosaic_bsa_paged_fwd(p, *make(1).values())
    else:
        order = ("q", "k", "v", "q_weight", "k_weight", "q_lens", "k_lens", "page_table", "prefix_len", "q_out",
                 "k_pages", "v_pages")
        with pytest.raises(ValueError):
            M.mosaic_bsa_paged_append(p, rot, None, *(t[n] for n in order))
        M.mosaic_bsa_paged_append(p, rot, None, *(make(1)[n] for n in order))
    assert lib.calls == 3


@pytest.mark.parametrize("copied", [copy.copy, copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x))])
def test_copies_of_parameters(copied):
    p = params()
    n = M.mosaic_bsa_paged_workspace_bytes(p)
    c = copied(p)
    assert c == p and M.mosaic_bsa_paged_workspace_bytes(c) == n
    c.batch = 1
    assert p.batch == 2


@pytest.mark.parametrize("call,make", [(attend, tensors), (append, append_tensors)], ids=["attend", "append"])
@pytest.mark.parametrize("stream", [0, 12345], ids=["default", "handle"])
def test_tensors_on_the_cpu_after_a_call_on_a_gpu(monkeypatch, call, make, stream):
    """A device of -1 is no GPU, whatever the call before with the same shapes had."""
    lib, p, rot = Library(), params(), M.Rotation(64)
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_raw_stream", (lambda device: 0, lambda: 0))

    def go(t):
        if call is attend:
            M.mosaic_bsa_paged_fwd(p, *t.values(), stream=stream)
        else:
            order = ("q", "k", "v", "q_weight", "k_weight", "q_lens", "k_lens", "page_table", "prefix_len", "q_out",
                     "k_pages", "v_pages")
            M.mosaic_bsa_paged_append(p, rot, None, *(t[n] for n in order), stream=stream)

    go(make(0))
    assert lib.calls == 1
    with pytest.raises(ValueError):
        go(make(-1))
    for name in make(0):
        with pytest.raises(ValueError):
            go({**make(0), name: make(-1)[name]})
    assert lib.calls == 1


def test_a_workspace_on_the_cpu_beside_addresses(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "_lib", lib)
    with pytest.raises(ValueError):
        attend(params(), workspace=torch.zeros(1 << 10, dtype=torch.uint8))
    assert lib.calls == 0


@pytest.mark.parametrize("call,make", [(attend, tensors), (append, append_tensors)], ids=["attend", "append"])
def test_page_tables_the_other_way_round(monkeypatch, call, make):
    """As many entries in another order: [table_pages, batch]."""
    lib, p = Library(), params()
    extra = {"rot": M.Rotation(64)} if call is append else {}
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_raw_stream", (lambda device: 0, lambda: 0))
    for shape in ((4, 2), (1, 8), (2, 2, 2), (2, 4, 1)):
        with pytest.raises(ValueError, match="page_table"):
            call(p, **extra, **{**make(0), "page_table": OnGpu(0, *shape, dtype=torch.int32)})
    assert lib.calls == 0
    for shape in ((2, 4), (8,)):                           # (a flat one has one order only)
        call(p, **extra, **{**make(0), "page_table": OnGpu(0, *shape, dtype=torch.int32)})
    assert lib.calls == 2


@pytest.mark.parametrize("kw", [dict(batch=24, heads=16, q_tokens=1, head_dim=128, table_pages=100, prefix_tokens=28800),
                                dict(batch=2, heads=4, q_tokens=50, table_pages=60, prefix_tokens=0)], ids=["shares", "chunks"])
def test_workspaces_that_are_needed(kw):
    p = params(**kw)
    n = M.mosaic_bsa_paged_workspace_bytes(p)
    assert n > 0
    for short in (dict(nbytes=n - 1), dict(nbytes=0), dict(workspace=None), dict(workspace=None, nbytes=0)):
        assert code_of(lambda: attend(p, **short)) == -6
