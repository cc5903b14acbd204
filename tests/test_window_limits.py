"""Which sizes the windowed attention takes: as many as its launches hold (CPU)."""
import pytest

import paper_2604_16429_amd as M
from paper_2604_16429_amd import binding

FAKE = 0x1000


def forward(p):
    """Error code of a call that has no out: -1 where the sizes pass."""
    with pytest.raises(M.BsaError) as e:
        M.mosaic_bsa_window_fwd(p, FAKE, FAKE, FAKE, None, stream=0, workspace_bytes=0)
    return e.value.code


def backward(p):
    """... that has no dv."""
    with pytest.raises(M.BsaError) as e:
        M.mosaic_bsa_window_bwd(p, *([FAKE] * 8), None, FAKE, stream=0, workspace_bytes=1 << 60)
    return e.value.code


@pytest.mark.parametrize("kw", [
    dict(batch=256, heads=32, kv_heads=8, q_tokens=1, k_tokens=131072),        # 256 sequences, long caches
    dict(batch=1, heads=64, kv_heads=64, q_tokens=100, k_tokens=1 << 22),
    dict(batch=(1 << 22) - 1, heads=1, kv_heads=1, q_tokens=1, k_tokens=1 << 20),
    dict(batch=24, heads=16, kv_heads=16, q_tokens=1038240, k_tokens=1038240),  # 0.25 degrees, 24 members
    dict(batch=24, heads=16, kv_heads=4, q_tokens=1038240, k_tokens=1038240),
])
def test_large_forwards(kw):
    assert forward(M.WindowParams(head_dim=64, window_left=1023, n_sink=4, **kw)) == -1


@pytest.mark.parametrize("kw", [
    dict(batch=24, heads=16, kv_heads=16, q_tokens=1038240, k_tokens=1038240),
    dict(batch=24, heads=16, kv_heads=4, q_tokens=1038240, k_tokens=1038240),
])
def test_large_trainings(kw):
    p = M.WindowParams(head_dim=32, window_left=1023, n_sink=4, **kw)
    assert forward(p) == -1 and backward(p) == -1
    assert M.mosaic_bsa_window_workspace_bytes(p, binding.OP_BWD) > 0


@pytest.mark.parametrize("kw,fwd,bwd", [
    (dict(batch=1 << 22, q_tokens=1, k_tokens=1), -2, -2),             # slices
    (dict(batch=1 << 16, q_tokens=(1 << 15) + 1, k_tokens=1), -2, -2),  # tiles of 128 rows
    (dict(batch=1 << 16, q_tokens=1, k_tokens=(1 << 15) + 1), -1, -2),  # tiles of 128 keys
    (dict(batch=1 << 16, q_tokens=1, k_tokens=1 << 13, n_sink=(1 << 12) + 1), -1, -2),  # groups of sinks
    (dict(batch=1, q_tokens=1 << 29, k_tokens=1), -2, -2),
    (dict(batch=1, q_tokens=1, k_tokens=1 << 29), -2, -2),
])
def test_what_launches_do_not_hold(kw, fwd, bwd):
    p = M.WindowParams(heads=1, head_dim=32, window_left=15, **kw)
    assert forward(p) == fwd and backward(p) == bwd
    if fwd == -2:
        assert M.mosaic_bsa_window_workspace_bytes(p, binding.OP_FWD) == 0
    assert M.mosaic_bsa_window_workspace_bytes(p, binding.OP_BWD) == 0


def test_chunks_on_rings():
    """Chunk lengths that leave the sum of a position and the chunk below 2^31."""
    p = dict(batch=1, heads=1, head_dim=32, window_left=15)
    assert forward(M.WindowParams(q_tokens=1 << 28, k_tokens=1 << 28 | 16, ring=1 << 28 | 16, **p)) == -2
    assert forward(M.WindowParams(q_tokens=(1 << 28) - 1, k_tokens=1 << 28 | 16, ring=1 << 28 | 16, **p)) == -1


@pytest.mark.parametrize("kw,split", [
    (dict(heads=1, q_tokens=3000, k_tokens=3000, window_left=63, window_right=-1), True),
    (dict(heads=1, q_tokens=3000, k_tokens=3000, window_left=63, window_right=2000), True),
    (dict(heads=1, q_tokens=3000, k_tokens=3000, window_left=63, window_right=0), False),
])
def test_keys_to_the_right_count(kw, split):
    """Few workgroups with many keys share them out (which takes a workspace), on whichever side they are."""
    p = M.WindowParams(batch=1, k_tokens=kw["k_tokens"], head_dim=64, dtype=binding.BF16,
                       **{k: v for k, v in kw.items() if k != "k_tokens"})
    assert (M.mosaic_bsa_window_workspace_bytes(p, binding.OP_FWD) > 0) == split
