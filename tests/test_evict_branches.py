"""Eviction at the borders between its kernels: selections at the sizes where the form changes and over several slices
(ties, special values and protected keys across them), single tokens' weights in each of their forms (heads shared by the
waves, plain, storage order) for ALiBi and several KV heads, several passes over head groups with running sums, and
rotated copies against lazy_materialize_k's."""
import numpy as np
import pytest
import torch

from oracle import eviction_oracle as E
from paper_2606_04302_amd import ops
from paper_2606_04302_amd import workloads as W
from tests.test_backward import oracle_kw, shared
from tests.test_backward_precision import long_context
from tests.test_evict import check_weights, decode_of, i32, run_select

SLICE, RESIDENT = 16384, 35840  # keys of a slice; most keys that one workgroup holds


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ops.lib()
    torch.cuda.init()


def values(kind, n):
    rng = np.random.default_rng([n, len(kind)])
    if kind == "distinct":
        return np.exp(2 * rng.standard_normal(n)).astype(np.float32)
    if kind == "four values":
        return rng.integers(0, 4, n).astype(np.float32)
    if kind == "one value":
        return np.full(n, 2.5, np.float32)
    if kind == "zeros of both signs":
        return np.where(rng.random(n) < 0.5, np.float32(0.0), np.float32(-0.0)).astype(np.float32)
    if kind == "denormals":
        return (rng.integers(0, 5, n) * np.float32(1e-45)).astype(np.float32)
    w = rng.standard_normal(n).astype(np.float32)  # "special": not a number, both infinities, among others
    w[::7], w[5::11], w[3::13] = np.nan, np.inf, -np.inf
    return w


def check(w, budgets, sink, recent):
    """One request, all budgets as a batch of its copies, against a sort."""
    got = run_select([w] * len(budgets), budgets, sink=sink, recent=recent, room=1)
    for b, kept in zip(budgets, got):
        want = E.select(w, b, sink, recent)
        assert kept == want + [-1] * (b - len(want)), f"{len(w)} keys, budget {b}, sink {sink}, recent {recent}"


def test_borders_of_the_forms_without_a_gpu():
    """The sizes above are the library's: no workspace up to what a workgroup holds, one slice more behind each 16384."""
    size = ops.cache_select_workspace_size
    assert size(1, RESIDENT) == 0 and size(1, RESIDENT + 1) > 0
    one = size(1, RESIDENT + 1) // 3
    assert size(1, 3 * SLICE) == 3 * one and size(1, 3 * SLICE + 1) == 4 * one


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["distinct", "four values", "special"])
@pytest.mark.parametrize("n", [SLICE - 1, SLICE, SLICE + 1, RESIDENT - 1, RESIDENT, RESIDENT + 1, 3 * SLICE, 3 * SLICE + 1])
def test_selection_where_its_form_changes(gpu, n, kind):
    w = values(kind, n)
    check(w, [1, n // 3, n - 1, n, n + 2], 0, 0)
    check(w, [1, n // 3, n - 1], 5, 700)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["four values", "one value", "zeros of both signs", "denormals", "special"])
def test_selection_ties_across_slices(gpu, kind):
    """Budgets that end within a run of equal scores, at the slices' borders and elsewhere."""
    n = 4 * SLICE + 777
    w = values(kind, n)
    check(w, [1, SLICE - 1, SLICE, SLICE + 1, 2 * SLICE + 5, n - 1], 0, 0)
    check(w, [9, 17, SLICE + 13, 3 * SLICE], 7, 9)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["distinct", "four values", "special"])
def test_protected_keys_across_slices(gpu, kind):
    n, sink, recent = 5 * SLICE + 1, SLICE + 900, 2 * SLICE + 3
    w = values(kind, n)
    check(w, [100, sink, sink + 1, sink + recent - 1, sink + recent, sink + recent + 1, n - 2], sink, recent)
    check(w, [3, SLICE, n - 1], n, 0)
    check(w, [3, SLICE, n - 1], 0, n + 5)
    check(w, [3, SLICE, n - 1], 2 ** 31 - 1, 2 ** 31 - 1)


# Single tokens.  Up to 256 tiles in all and several KV heads: the waves of a workgroup share the heads.  More tiles, or one
# KV head: plain.  Half a megabyte or more of keys a workgroup: records in storage order.
ALIBI, IL = dict(rope_style=ops.ALIBI), dict(rope_style=ops.ROPE_INTERLEAVED)
TOKENS = {
    "alibi, one KV head": (lambda: shared(100, 4, 1, 128, [300, 70], [5]), ALIBI),
    "alibi d64, one KV head, group 20": (lambda: shared(101, 20, 1, 64, [300, 70], [5]), ALIBI),
    "alibi, plain": (lambda: shared(102, 8, 2, 128, [2500, 500], [3], reqs=6), ALIBI),
    "alibi d64, plain, group 12": (lambda: shared(103, 24, 2, 64, [2500, 500], [3], reqs=6), ALIBI),
    "alibi, storage order": (lambda: shared(104, 8, 4, 128, [230, 264, 70], [1], reqs=770), ALIBI),
    "alibi, group 12, storage order": (lambda: shared(105, 24, 2, 128, [500, 40, 517], [1], reqs=769), ALIBI),
    "plain": (lambda: shared(106, 8, 2, 128, [2500, 500], [3], reqs=6), {}),
    "plain, 12 KV heads, interleaved": (lambda: shared(107, 12, 12, 64, [2500, 500], [3], reqs=6), IL),
    "plain, group 12": (lambda: shared(108, 24, 2, 128, [2500, 500], [3], reqs=6), {}),
    "plain, local, group 10": (lambda: shared(109, 20, 2, 64, [2500, 500], [3], reqs=6),
                               dict(key_positions=ops.KEYS_LOCAL)),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", TOKENS)
def test_token_weights_in_every_form(gpu, name):
    make, ckw = TOKENS[name]
    check_weights(decode_of(make()), ckw, name)


# More query heads than are held in LDS at once: later passes go on with the sums of the earlier ones.
PASSES = {
    "group 20, shared heads": (lambda: shared(110, 40, 2, 128, [200, 7], [9, 40]), {}),
    "group 20, plain": (lambda: shared(111, 40, 2, 128, [2500, 500], [3], reqs=6), {}),
    "group 20, alibi, plain": (lambda: shared(112, 40, 2, 64, [2500, 500], [3], reqs=6), ALIBI),
    "48 heads of their own": (lambda: shared(113, 48, 48, 64, [200, 7], [9, 40]), {}),
    "group 8, 8 KV heads, local": (lambda: shared(114, 64, 8, 64, [2500, 500], [3], reqs=6),
                                   dict(key_positions=ops.KEYS_LOCAL)),
    "group 20, storage order": (lambda: shared(115, 80, 4, 128, [230, 264, 70], [1], reqs=768), IL),
}


def passes_of(w):
    """Passes over the query heads: 32 rows at a time, in groups of up to 16 of one KV head, up to 16 groups."""
    group = w.num_q_heads // w.num_kv_heads
    groups = w.num_kv_heads * -(-group // 16)
    return -(-groups // min(16, 32 // min(group, 16)))


@pytest.mark.gpu
@pytest.mark.parametrize("name", PASSES)
@pytest.mark.parametrize("decay", [0.9, 0.0])
def test_running_sums_over_several_passes(gpu, name, decay):
    """Beside the bound of what a call adds: every pass rounds the sum once (2^-24), and the decay is an fp32 number
    (0.9 is off by 0.44 2^-24, relative): passes + 1/2 halves of an fp32 step in all, as sums of what is not negative
    never exceed the last one."""
    make, ckw = PASSES[name]
    w = decode_of(make())
    passes = passes_of(w)
    assert passes > 1
    cfg, dw = ops.config_of(w, **ckw), ops.upload(w)
    _, lse = ops.run_lazy(dw, cfg)
    n, room = w.kv_lens, 3
    ks = np.concatenate([[0], np.cumsum(n + room)])
    old = torch.empty(int(ks[-1]), device="cuda").uniform_(0, 3, generator=torch.Generator("cuda").manual_seed(5))
    out = torch.full_like(old, -7.0)

    def call(win, to):
        ops.decode_key_weights(cfg, dw.q, dw.q_pos0, dw.pool, dw.chunks, dw.chunk_start, i32(ks), w.max_kv_len, lse, to,
                               weights_in=win, decay=decay)

    call(old, out)
    got, before = (t.cpu().numpy().astype(np.float64) for t in (out, old))
    ref = E.key_weights(w.q, w.q_start, w.q_pos0, w.pool, w.chunks, w.chunk_start, w.num_q_heads, w.num_kv_heads,
                        w.head_dim, w.rope_base, w.causal, lse.cpu().numpy(), **oracle_kw(ckw))
    worst = 0.0
    for r, (x, bound) in enumerate(ref):
        mine = slice(ks[r], ks[r] + n[r])
        x = x + decay * before[mine]
        worst = max(worst, (np.abs(got[mine] - x) / (bound + (passes + 0.5) * 2.0 ** -24 * np.abs(x))).max())
        assert (got[ks[r] + n[r]:ks[r + 1]] == -7.0).all()
    print(f"{name}, decay {decay}: {passes} passes, largest error over its bound {worst:.3f}", flush=True)
    assert worst <= 1.0
    call(old, old)  # in place
    for r in range(w.batch):
        assert torch.equal(old[ks[r]:ks[r] + n[r]], out[ks[r]:ks[r] + n[r]])


@pytest.mark.gpu
@pytest.mark.parametrize("d,ckw", [(128, {}), (64, IL), (128, dict(key_positions=ops.KEYS_LOCAL)),
                                   (64, dict(IL, key_positions=ops.KEYS_LOCAL))])
def test_rotated_copies_against_lazy_materialize_k(gpu, d, ckw):
    """All keys kept and rotated: within one bf16 step of lazy_materialize_k's copy.  Both round once, what they round
    differs by their angles' sums (4e-6 for elements of at most 8, as for the oracle): another neighbour at most."""
    w = shared(116, 8, 2, d, [130, 64, 33], [9], reqs=1)
    cfg, dw = ops.config_of(w, **ckw), ops.upload(w)
    n, hkv = int(w.kv_lens[0]), w.num_kv_heads
    out = torch.zeros(2 * n * hkv * d, dtype=torch.bfloat16, device="cuda")
    dst = np.array([(0, n * hkv * d, n, 0, n, n)], dtype=W.CHUNK_DTYPE)
    ops.cache_compact(cfg, dw.pool, dw.pool, dw.chunks, dw.chunk_start, i32(np.arange(n)), i32([0, n]), n,
                      torch.from_numpy(dst.view(np.uint8).copy()).cuda(), out, out, rotate=True)
    copy, table = ops.materialize_k(cfg, dw.pool, dw.chunks, int(w.chunks["len"].max()), n)
    torch.cuda.synchronize()
    got = out[:n * hkv * d].view(hkv, n, d).float().cpu().numpy()
    copy = copy.float().cpu().numpy()
    want = np.concatenate([copy[int(c["k_offset"]):int(c["k_offset"]) + hkv * int(c["len"]) * d].reshape(hkv, -1, d)
                           for c in ops.chunks_from_tensor(table)], axis=1)
    assert want.shape == got.shape and np.abs(want).max() > 1
    step = np.maximum(np.abs(want), np.abs(got)) * 2.0 ** -7
    assert (np.abs(got - want) <= step + 4e-6).all()
    assert (got == want).mean() > 0.99


FAR = {
    "d128": lambda: long_context(117, 8, 2, 128, 500, 4, gap=20000),
    "d64, one KV head": lambda: long_context(118, 8, 1, 64, 500, 40, gap=20000),
    "d128, plain": lambda: long_context(119, 8, 2, 128, 17000, 4, gap=300000),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", FAR)
@pytest.mark.parametrize("kind", ["prompt", "token"])
def test_alibi_weights_far_from_the_keys(gpu, name, kind):
    """Bias and log-sum-exp are far larger than their difference, the score: what the call is given decides (the slopes
    of eight heads are powers of two, exact in fp32), so the bound is that of keys nearby."""
    w = FAR[name]()
    check_weights(w if kind == "prompt" else decode_of(w), ALIBI, f"{name}, {kind}")
