"""Calls that the binding refuses before anything is launched (host tensors and a stand-in library that succeeds)."""
import ctypes

import pytest
import torch

from paper_2606_04302_amd import ops


@pytest.fixture
def calls(monkeypatch):
    """The names of the library's functions that were called; type and device checks are off."""
    names = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                names.append(name)
                return 64 if name.endswith("_size") else 0
            return call

    library = Library()
    monkeypatch.setattr(ops, "lib", lambda: library)
    monkeypatch.setattr(ops, "_dev", lambda *a: None)
    monkeypatch.setattr(ops, "_chunks", lambda *a: None)
    return names


def bf16(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


@pytest.mark.parametrize("which", ["dk_pool", "dv_pool"])
@pytest.mark.parametrize("of", ["k_pool", "v_pool"])
@pytest.mark.parametrize("shift", [-1, 0, 1, 999, 1000])
def test_gradient_pools_may_not_overlap_the_pools(calls, which, of, shift):
    """Not in part either: a view of the pool's memory, shifted.  Memory that only touches is fine."""
    store = bf16(4000)
    pools = dict(k_pool=store[1000:2000], v_pool=bf16(1000))
    if of == "v_pool":
        pools = dict(k_pool=pools["v_pool"], v_pool=pools["k_pool"])
    grads = dict(dk_pool=bf16(1000), dv_pool=bf16(1000))
    grads[which] = store[1000 + shift:2000 + shift]
    q, lse = bf16(3, 2, 64), torch.zeros(3, 2)
    plan = ops.BackwardPlan(torch.zeros(0, dtype=torch.uint8), ops.BackwardInfo())

    def call():
        ops.prefill_backward(ops.Config(2, 1, 64, 1e4), q, i32(0, 3), i32(0), pools["k_pool"], pools["v_pool"],
                             torch.zeros(32, dtype=torch.uint8), i32(0, 1), q, lse, q, plan, dq=q, **grads, stream=0,
                             workspace=torch.zeros(64, dtype=torch.uint8))

    if shift == 1000:
        call()
        assert calls[-1] == "lazy_attn_prefill_backward"
    else:
        with pytest.raises(ValueError, match=which):
            call()
        assert "lazy_attn_prefill_backward" not in calls


@pytest.mark.parametrize("shift", [-3, 0, 4, 7, 8])
def test_compacted_weights_may_not_overlap_the_weights(calls, shift):
    """Kept keys move to lower places: one workgroup would overwrite weights that another has yet to read."""
    w = torch.zeros(24)
    weights, out = w[8:16], w[8 + shift:8 + shift + 8]
    if shift == -3:
        out = w[1:9]  # its last entry is the first weight

    def call():
        ops.cache_compact(ops.Config(2, 1, 64, 1e4), bf16(512), bf16(512), torch.zeros(32, dtype=torch.uint8), i32(0, 1),
                          i32(0, 3), i32(0, 2), 2, torch.zeros(32, dtype=torch.uint8), bf16(512), bf16(512),
                          key_start=i32(0, 8), weights=weights, weights_out=out, stream=0)

    if shift == 8:
        call()
        assert calls == ["lazy_cache_compact"]
    else:
        with pytest.raises(ValueError, match="weights_out"):
            call()
        assert not calls


def test_compaction_in_place_is_refused_by_the_library():
    p, one = ops.Config(4, 2, 64, 1e4).c(), 4096  # addresses that are never read
    args = [one] * 4 + [1, one, one, 10, one, 0, one, one]
    assert ops.lib().lazy_cache_compact(ctypes.byref(p), *args, one, one, one, None) == ops.LAZY_EINVAL


@pytest.mark.parametrize("shift", [0, 3, 8])
def test_running_weights_are_the_weights_or_apart(calls, shift):
    w = torch.zeros(24)
    q, lse = bf16(1, 2, 64), torch.zeros(1, 2)

    def call():
        ops.decode_key_weights(ops.Config(2, 1, 64, 1e4), q, i32(7), bf16(512), torch.zeros(32, dtype=torch.uint8),
                               i32(0, 1), i32(0, 8), 8, lse, w[8:16], weights_in=w[8 + shift:16 + shift], stream=0,
                               workspace=torch.zeros(64, dtype=torch.uint8))

    if shift == 3:
        with pytest.raises(ValueError, match="weights_in"):
            call()
    else:
        call()
        assert calls[-1] == "lazy_attn_decode_key_weights"


def test_workspaces_that_the_kernels_cannot_write_are_refused(calls):
    """A tensor elsewhere, or one whose bytes do not lie together."""
    here, other = torch.device("cpu"), torch.zeros(64, dtype=torch.uint8, device="meta")
    fine = torch.zeros(64, dtype=torch.uint8)
    assert ops._workspace(64, here, fine) is fine
    assert ops._workspace(0, here, other) is None
    assert ops._workspace(65, here, fine).numel() == 65
    for bad in (other, torch.zeros(128, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="workspace"):
            ops._workspace(64, here, bad)
    with pytest.raises(ValueError, match="workspace"):
        ops.decode(ops.Config(2, 1, 64, 1e4), bf16(1, 2, 64), i32(7), bf16(512), bf16(512),
                   torch.zeros(32, dtype=torch.uint8), i32(0, 1), 8, out=bf16(1, 2, 64), workspace=other, stream=0)
    assert "lazy_attn_decode" not in calls


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_weights_reserve_angles_where_they_are_read(d):
    """A table of 32 positions' (cos, sin), and only for keys that are stored without positions."""
    def size(**kw):
        return ops.prefill_key_weights_workspace_size(ops.Config(4, 2, d, 1e4, **kw), 2, 6, 3, 100, 200)

    for style in (ops.ROPE_HALF, ops.ROPE_INTERLEAVED):
        assert size(rope_style=style) - size(rope_style=style, key_positions=ops.KEYS_LOCAL) == 32 * (d // 2) * 8
    # ALiBi keeps one part of the queries, too: 6 tokens of 4 heads
    assert size(key_positions=ops.KEYS_LOCAL) - size(rope_style=ops.ALIBI) == 6 * 4 * d * 2
