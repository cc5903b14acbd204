"""What the entry points of the rotation, the head norms and the windowed attention refuse,
on the host, before anything is launched."""
import ctypes

import pytest
import torch

import paper_2604_16429_amd as M
from paper_2604_16429_amd import binding

FAKE = 0x1000            # never read: the checks fail first


def heads(**kw):
    base = dict(batch=2, tokens=8, heads=4, head_dim=64, dtype=binding.BF16, kv_heads=2)
    base.update(kw)
    return M.HeadsParams(**base)


def window(**kw):
    base = dict(batch=2, heads=4, q_tokens=8, k_tokens=64, head_dim=64, dtype=binding.BF16,
                kv_heads=2, window_left=15, n_sink=4)
    base.update(kw)
    return M.WindowParams(**base)


def code_of(call):
    with pytest.raises(M.BsaError) as e:
        call()
    return e.value.code


def rope(p, rot, q=FAKE, k=FAKE, qo=FAKE, ko=FAKE, pos=FAKE, **kw):
    M.mosaic_bsa_rope_fwd(p, rot, pos, q, k, qo, ko, stream=0, **kw)


def win_fwd(p, q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=FAKE, q_lens=None, k_lens=None, ws=FAKE,
            nbytes=1 << 40):
    M.mosaic_bsa_window_fwd(p, q, k, v, out, lse, q_lens, k_lens, ws, stream=0, workspace_bytes=nbytes)


def win_bwd(p, ptrs=None, ws=FAKE, nbytes=1 << 40):
    M.mosaic_bsa_window_bwd(p, *(ptrs or [FAKE] * 9), ws, stream=0, workspace_bytes=nbytes)


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(binding._CStrides) == 24
    assert ctypes.sizeof(binding._CRotation) == 16 + 8 * 64
    assert ctypes.sizeof(binding._CHeadsParams) == 40 + 6 * 24
    assert ctypes.sizeof(binding._CWindowParams) == 48 + 8 * 24


@pytest.mark.parametrize("kw", [
    dict(rotary_dim=63), dict(rotary_dim=-2), dict(rotary_dim=130), dict(rotary_dim=62, axes=2),
    dict(rotary_dim=64, axes=3), dict(rotary_dim=64, axes=0), dict(rotary_dim=64, layout=2),
    dict(rotary_dim=64, theta=0.0), dict(rotary_dim=64, theta=float("nan")),
    dict(rotary_dim=64, scaling=4), dict(rotary_dim=64, scaling=-1),
    dict(rotary_dim=64, scaling=binding.SCALE_LINEAR, factor=0.5),
    dict(rotary_dim=64, scaling=binding.SCALE_BASE, factor=float("inf")),
    dict(rotary_dim=64, scaling=binding.SCALE_RAMP, factor=2.0),
    dict(rotary_dim=64, scaling=binding.SCALE_RAMP, factor=2.0, original_tokens=10, beta_fast=1,
         beta_slow=2),
    dict(rotary_dim=4, inv_freq=[1.0, float("nan")]),
])
def test_rotations_that_are_none(kw):
    assert code_of(lambda: M.Rotation(**kw)) == -10


def test_number_of_given_frequencies():
    with pytest.raises(ValueError):
        M.Rotation(8, inv_freq=[1.0, 0.5])


def test_frequencies_are_turns_in_units_of_2_to_the_minus_64():
    import math
    rot = M.Rotation(8, inv_freq=[2.0 * math.pi * 0.25, -2.0 * math.pi * 0.25, 0.0, math.pi])
    turns = list(rot.c.turns)[:4]
    assert turns[2] == 0
    for have, want in zip(turns, (1 << 62, 3 << 62, 0, 1 << 63)):
        assert abs(have - want) <= 1 << 12
    rot = M.Rotation(64, scaling=binding.SCALE_RAMP, factor=8.0, original_tokens=4096)
    assert abs(rot.c.magnitude - (0.1 * math.log(8.0) + 1.0)) < 1e-6
    # the fastest pair is kept, the slowest divided by the factor
    plain = M.Rotation(64)
    assert abs(rot.c.turns[0] - plain.c.turns[0]) <= 1 << 12
    assert abs(rot.c.turns[31] * 8 - plain.c.turns[31]) <= 1 << 12


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -2), (dict(tokens=0), -2), (dict(heads=0), -2), (dict(kv_heads=-1), -2),
    (dict(cache_tokens=-1), -2), (dict(batch=1 << 20, tokens=1 << 20), -2), (dict(head_dim=48), -4),
    (dict(dtype=2), -5), (dict(norm_eps=-1.0), -2), (dict(norm_eps=float("nan")), -2),
])
def test_heads_parameters(kw, code):
    rot = M.Rotation(32)
    p = heads(**kw)
    assert code_of(lambda: rope(p, rot)) == code
    assert code_of(lambda: M.mosaic_bsa_rope_bwd(p, rot, FAKE, FAKE, FAKE, FAKE, FAKE, stream=0)) == code
    assert code_of(lambda: M.mosaic_bsa_qk_norm_rope_fwd(
        p, rot, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, stream=0)) == code
    assert code_of(lambda: M.mosaic_bsa_qk_norm_rope_bwd(
        p, rot, *([FAKE] * 11), FAKE, stream=0, workspace_bytes=1 << 40)) == code
    assert M.mosaic_bsa_qk_norm_rope_workspace_bytes(p) == 0


def test_heads_pointers_rotation_and_strides():
    rot = M.Rotation(64)
    assert code_of(lambda: rope(heads(head_dim=32), rot)) == -10        # wider than the head
    assert code_of(lambda: rope(heads(), rot, q=None)) == -1
    assert code_of(lambda: rope(heads(), rot, ko=None)) == -1
    assert code_of(lambda: rope(heads(), rot, qo=None)) == -1
    assert code_of(lambda: rope(heads(), rot, v=FAKE)) == -1            # v without v_out
    assert code_of(lambda: rope(heads(), rot, q=FAKE + 1)) == -7
    assert code_of(lambda: rope(heads(), rot, pos=FAKE + 2)) == -7
    assert code_of(lambda: rope(heads(), rot, rows=FAKE)) == -2         # cache without rows
    assert code_of(lambda: rope(heads(), M.Rotation(64, axes=2), pos=None)) == -1
    p = heads()
    p._c().q_out.token = -64
    assert code_of(lambda: M.load_library() and binding._check(
        M.load_library().mosaic_bsa_rope_fwd(p._ref, rot.ref, *([FAKE] * 2), None, None, None, FAKE,
                                             None, None, None))) == -11
    p._struct.q_out = binding._CStrides(0, 512, 64)                     # batch entries on each other
    assert code_of(lambda: binding._check(
        M.load_library().mosaic_bsa_rope_fwd(p._ref, rot.ref, *([FAKE] * 2), None, None, None, FAKE,
                                             None, None, None))) == -11
    p = heads()
    n = M.mosaic_bsa_qk_norm_rope_workspace_bytes(p)
    args = [p, rot] + [FAKE] * 11
    assert n > 0
    assert code_of(lambda: M.mosaic_bsa_qk_norm_rope_bwd(*args, FAKE, stream=0, workspace_bytes=n - 1)) == -6
    assert code_of(lambda: M.mosaic_bsa_qk_norm_rope_bwd(*args, None, stream=0, workspace_bytes=n)) == -6
    args[5] = None                                                       # q_weight
    assert code_of(lambda: M.mosaic_bsa_qk_norm_rope_bwd(*args, FAKE, stream=0, workspace_bytes=n)) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -2), (dict(heads=0), -2), (dict(q_tokens=0), -2), (dict(k_tokens=0), -2),
    (dict(kv_heads=3), -2), (dict(kv_heads=8), -2), (dict(kv_heads=-2), -2),
    (dict(batch=1 << 22, q_tokens=1 << 20), -2), (dict(k_tokens=1 << 30), -2), (dict(head_dim=96), -4),
    (dict(dtype=5), -5), (dict(n_sink=-1), -12), (dict(ring=-1), -12), (dict(ring=64), -12),
    (dict(ring=60, window_left=-1), -12), (dict(ring=60, window_left=53), -12),
])
def test_window_parameters(kw, code):
    p = window(**kw)
    assert code_of(lambda: win_fwd(p, k_lens=FAKE)) == code
    assert code_of(lambda: win_bwd(p)) == code
    assert M.mosaic_bsa_window_workspace_bytes(p, binding.OP_FWD) == 0
    assert M.mosaic_bsa_window_workspace_bytes(p, binding.OP_BWD) == 0


def test_window_pointers_and_strides():
    p = window()
    for name in ("q", "k", "v", "out"):
        assert code_of(lambda: win_fwd(p, **{name: None})) == -1
        assert code_of(lambda: win_fwd(p, **{name: FAKE + 8})) == -7
    assert code_of(lambda: win_fwd(p, lse=FAKE + 2)) == -7
    assert code_of(lambda: win_fwd(p, k_lens=FAKE + 1)) == -7
    ring = window(ring=60, window_left=52)
    assert code_of(lambda: win_fwd(ring)) == -1                          # k_lens
    assert code_of(lambda: win_bwd(ring)) == -12
    for i in range(9):
        ptrs = [FAKE] * 9
        ptrs[i] = None
        assert code_of(lambda: win_bwd(p, ptrs)) == -1
    n = M.mosaic_bsa_window_workspace_bytes(p, binding.OP_BWD)
    assert n > 0
    assert code_of(lambda: win_bwd(p, nbytes=n - 1)) == -6
    assert code_of(lambda: win_bwd(p, ws=None)) == -6
    lib = M.load_library()
    for strides, code in (((512, 64, -64), -11), ((512, 64, 4), -11), ((2048, 68, 256), -7),
                          ((1 << 41, 64, 256), -11)):
        p._struct.out = binding._CStrides(*strides)
        assert code_of(lambda: binding._check(lib.mosaic_bsa_window_fwd(
            p._ref, FAKE, FAKE, FAKE, None, None, FAKE, None, FAKE, 1 << 40, None))) == code


def test_tensors_that_do_not_fit_the_parameters():
    """The binding refuses host tensors, other shapes and other types."""
    x = torch.zeros(2, 4, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        win_fwd(window(), q=x)                                            # on the host
    with pytest.raises(ValueError):
        win_fwd(window(), q=x[:, :3])
    with pytest.raises(ValueError):
        rope(heads(), M.Rotation(64), q=x.float())
    with pytest.raises(ValueError):
        rope(heads(), M.Rotation(64), pos=torch.zeros(8, dtype=torch.int64))


class OnGpu:
    """What the binding looks at of a tensor, without its memory."""

    def __init__(self, *shape, strides=None):
        x = torch.empty(shape, dtype=torch.bfloat16, device="meta")
        self.shape, self.dtype, self.is_cuda = x.shape, x.dtype, True
        self.strides = x.stride() if strides is None else strides

    def stride(self):
        return self.strides

    def data_ptr(self):
        return FAKE


def test_a_field_that_two_calls_use_is_looked_at_for_each():
    """v of the forward and dq of the norm's gradient share a field, with other numbers of heads."""
    p, rot = heads(), M.Rotation(64)
    q, k = OnGpu(2, 4, 8, 64), OnGpu(2, 2, 8, 64)
    n = M.mosaic_bsa_qk_norm_rope_workspace_bytes(p)
    # (a missing weight ends both calls on the host)
    assert code_of(lambda: M.mosaic_bsa_qk_norm_rope_fwd(p, rot, FAKE, q, k, None, FAKE, q, k, v=k, v_out=k,
                                                         stream=0)) == -1
    with pytest.raises(ValueError):
        M.mosaic_bsa_qk_norm_rope_bwd(p, rot, FAKE, q, k, None, FAKE, q, k, k, k, FAKE, FAKE, FAKE,
                                      stream=0, workspace_bytes=n)
    assert code_of(lambda: M.mosaic_bsa_qk_norm_rope_bwd(p, rot, FAKE, q, k, None, FAKE, q, k, q, k, FAKE,
                                                         FAKE, FAKE, stream=0, workspace_bytes=n)) == -1
    with pytest.raises(ValueError):
        M.mosaic_bsa_qk_norm_rope_fwd(p, rot, FAKE, q, k, None, FAKE, q, k, v=q, v_out=k, stream=0)


@pytest.mark.parametrize("strides,bad", [
    ((64, 64, 64), True),            # heads and tokens on each other
    ((4096, 64, 128), True),         # four heads of 64 channels in tokens 128 apart
    ((4096, 64, 255), True),
    ((1024, 512, 64), True),         # batch entries inside each other
    ((2048, 64, 256), False), ((2048, 512, 64), False), ((64, 1024, 128), False),
    ((1 << 40, 64, 256), False),
])
def test_rows_of_an_output_that_share_memory(strides, bad):
    rot, p = M.Rotation(64), heads()
    p._c().q_out = binding._CStrides(*strides)
    lib = M.load_library()
    # (k without k_out ends the call on the host where the strides pass)
    assert code_of(lambda: binding._check(lib.mosaic_bsa_rope_fwd(
        p._ref, rot.ref, FAKE, FAKE, FAKE, None, None, FAKE, None, None, None))) == (-11 if bad else -1)
    if strides[2] % 8 == 0:
        p = window()
        p._c().dq = binding._CStrides(*strides)
        # (no workspace)
        assert code_of(lambda: win_bwd_as_it_is(p)) == (-11 if bad else -6)


def win_bwd_as_it_is(p):
    """The C entry point with the strides that the struct has."""
    binding._check(M.load_library().mosaic_bsa_window_bwd(
        p._ref, *([FAKE] * 6), None, None, *([FAKE] * 3), None, 0, None))


@pytest.mark.parametrize("code", [-10, -11, -12])
def test_error_texts(code):
    assert M.mosaic_bsa_strerror(code) not in ("", "unknown error code")
