"""Eviction by accumulated attention weight: key weights, selection and compaction against the fp64 oracle, and the three
together with decoding over the compacted cache.

Key-weight tolerances (``oracle/eviction_oracle.py``): element by element the worst case; over a request a relative
2-norm of 2e-5 (root mean squares of the same roundings: u / sqrt(3) in place of u for each factor, over 64 to 128
products of random sign, leave less than 2^-17 of a score's spread).  Selected indices
and copied values are exact; rotated copies are rounded to bf16 once, half a step plus the hardware sine's error.
"""
import ctypes
import dataclasses
import math

import numpy as np
import pytest
import torch

from oracle import eviction_oracle as E
from oracle import lazy_oracle as O
from paper_2606_04302_amd import ops
from paper_2606_04302_amd import workloads as W
from tests.test_backward import oracle_kw, shared

REL = 2.0e-5


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ops.lib()
    torch.cuda.init()


def i32(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def starts(n, room=0):
    """Prefix sums with `room` unused entries behind each request's keys."""
    return np.concatenate([[0], np.cumsum(np.asarray(n, np.int64) + room)])


# ---------------------------------------------------------------------------------------------------------------
# CPU: refusals, and the oracle's selection against a sort
# ---------------------------------------------------------------------------------------------------------------
def test_refusals_without_a_gpu():
    """Every check comes before any launch, so addresses that are never read may be given."""
    lib, one = ops.lib(), 4096
    p = ops.Config(4, 2, 64, 1e4).c()
    ok = dict(p=p, q=one, qs=one, qp=one, k=one, c=one, cs=one, ks=one, batch=2, tq=6, mq=3, mk=100, nk=200, lse=one,
              win=None, decay=1.0, w=one, ws=one, nb=1 << 40)

    def prompt(**kw):
        a = dict(ok, **kw)
        return lib.lazy_attn_prefill_key_weights(
            None if a["p"] is None else ctypes.byref(a["p"]), a["q"], a["qs"], a["qp"], a["k"], a["c"], a["cs"],
            a["ks"], a["batch"], a["tq"], a["mq"], a["mk"], a["nk"], a["lse"], a["win"], a["decay"], a["w"], a["ws"],
            a["nb"], None)

    def token(**kw):
        a = dict(ok, **kw)
        return lib.lazy_attn_decode_key_weights(
            None if a["p"] is None else ctypes.byref(a["p"]), a["q"], a["qp"], a["k"], a["c"], a["cs"], a["ks"],
            a["batch"], a["mk"], a["lse"], a["win"], a["decay"], a["w"], None, 0, None)

    for f in (prompt, token):
        assert f(p=None) == ops.LAZY_EINVAL
        assert f(p=ops.Config(4, 3, 64, 1e4).c()) == ops.LAZY_EINVAL
        assert f(p=ops.Config(4, 2, 80, 1e4).c()) == ops.LAZY_EUNSUPPORTED
        for name in ("q", "qp", "k", "c", "cs", "ks", "lse", "w"):
            assert f(**{name: None}) == ops.LAZY_EINVAL, name
        assert f(batch=-1) == ops.LAZY_EINVAL and f(mk=-1) == ops.LAZY_EINVAL
        assert f(decay=math.inf) == ops.LAZY_EINVAL and f(decay=math.nan) == ops.LAZY_EINVAL
        assert f(batch=0) == ops.LAZY_OK and f(mk=0) == ops.LAZY_OK
        assert f(batch=70000) == ops.LAZY_EUNSUPPORTED
    assert prompt(qs=None) == ops.LAZY_EINVAL and prompt(mq=0) == ops.LAZY_EINVAL and prompt(nk=-1) == ops.LAZY_EINVAL
    assert prompt(ws=None) == ops.LAZY_EWORKSPACE and prompt(ws=one + 4) == ops.LAZY_EWORKSPACE
    need = lib.lazy_attn_prefill_key_weights_workspace_size(ctypes.byref(p), 2, 6, 3, 100, 200)
    assert need > 0 and prompt(nb=need - 1) == ops.LAZY_EWORKSPACE
    wide = ops.Config(1 << 15, 1, 64, 1e4).c()
    assert prompt(p=wide, tq=1 << 10) == ops.LAZY_EUNSUPPORTED

    def select(w=one, ks=one, os=one, batch=2, mk=10, sink=0, recent=0, kept=one, ws=one, nb=1 << 40):
        return lib.lazy_cache_select(w, ks, None, os, batch, mk, sink, recent, kept, ws, nb, None)

    for kw in (dict(w=None), dict(ks=None), dict(os=None), dict(kept=None), dict(batch=-1), dict(mk=-1), dict(sink=-1),
               dict(recent=-1)):
        assert select(**kw) == ops.LAZY_EINVAL, kw
    assert select(batch=0) == ops.LAZY_OK

    def compact(p=p, ptr={}, batch=2, mk=10, rotate=0, three=(None, None, None)):
        a = [ptr.get(n, one) for n in ("k", "v", "c", "cs")]
        b = [ptr.get(n, one) for n in ("kept", "os")]
        return lib.lazy_cache_compact(ctypes.byref(p), *a, batch, *b, mk, ptr.get("dst", one), rotate,
                                      ptr.get("ko", one), ptr.get("vo", one), *three, None)

    for name in ("k", "v", "c", "cs", "kept", "os", "dst", "ko", "vo"):
        assert compact(ptr={name: None}) == ops.LAZY_EINVAL, name
    assert compact(rotate=2) == ops.LAZY_EINVAL and compact(batch=-1) == ops.LAZY_EINVAL and compact(mk=-1) == ops.LAZY_EINVAL
    assert compact(three=(one, None, one)) == ops.LAZY_EINVAL
    assert compact(p=ops.Config(4, 2, 64, 1e4, rope_style=ops.ALIBI).c(), rotate=1) == ops.LAZY_EUNSUPPORTED
    assert compact(batch=0) == ops.LAZY_OK and compact(mk=0) == ops.LAZY_OK and compact(batch=70000) == ops.LAZY_EUNSUPPORTED


def test_python_refusals():
    t = torch.zeros(4)
    with pytest.raises(ValueError):
        ops.cache_select(t, t.int(), t.int(), 4, t.int())
    with pytest.raises(ValueError):
        ops.decode_key_weights(ops.Config(2, 1, 64, 1e4), t, t, t, t, t, t, 4, t, t)


def test_oracle_selection():
    w = np.array([3.0, 1.0, np.nan, 3.0, 0.0, 5.0, -1.0])
    assert E.select(w, 3, 0, 0) == [0, 3, 5]
    assert E.select(w, 2, 0, 0) == [0, 5]  # the tie goes to the lowest index
    assert E.select(w, 3, 1, 1) == [0, 5, 6]
    assert E.select(w, 6, 0, 0) == [0, 1, 3, 4, 5, 6]  # NaN last
    assert E.select(w, 9, 0, 0) == list(range(7))
    assert E.select(w, 2, 3, 3) == [0, 1]


# ---------------------------------------------------------------------------------------------------------------
# GPU: key weights
# ---------------------------------------------------------------------------------------------------------------
def check_weights(w, ckw, tag, room=0, decay=None):
    cfg = ops.config_of(w, **ckw)
    dw = ops.upload(w)
    _, lse = ops.run_lazy(dw, cfg)
    n = w.kv_lens
    ks = starts(n, room)
    gen = torch.Generator("cuda").manual_seed(5)
    win = None if decay is None else torch.empty(int(ks[-1]), device="cuda").uniform_(0, 3, generator=gen)
    out = torch.full((int(ks[-1]),), -7.0, device="cuda")
    kw = dict(weights_in=win, decay=1.0 if decay is None else decay)
    if w.kind == "decode":
        args = (cfg, dw.q, dw.q_pos0, dw.pool, dw.chunks, dw.chunk_start, i32(ks), max(1, w.max_kv_len), lse)
        fn = ops.decode_key_weights
    else:
        args = (cfg, dw.q, dw.q_start, dw.q_pos0, dw.pool, dw.chunks, dw.chunk_start, i32(ks), max(1, w.max_q_len),
                max(1, w.max_kv_len), lse)
        fn = ops.prefill_key_weights
    fn(*args, out, **kw)
    torch.cuda.synchronize()
    ref = E.key_weights(w.q, w.q_start, w.q_pos0, w.pool, w.chunks, w.chunk_start, w.num_q_heads, w.num_kv_heads,
                        w.head_dim, w.rope_base, w.causal, lse.cpu().numpy(), **oracle_kw(ckw))
    got = out.cpu().numpy().astype(np.float64)
    old = None if win is None else win.cpu().numpy().astype(np.float64)
    for r, (x, bound) in enumerate(ref):
        mine = got[ks[r]:ks[r] + n[r]]
        if old is not None:
            add = decay * old[ks[r]:ks[r] + n[r]]
            x, bound = x + add, bound + 2.0 ** -23 * np.abs(x + add)
        assert np.isfinite(mine).all(), tag
        worst = (np.abs(mine - x) / bound).max(initial=0.0)
        norm = np.linalg.norm(x)
        rel = np.linalg.norm(mine - x) / norm if norm else np.abs(mine).max(initial=0.0)
        print(f"{tag} request {r}: largest error over its bound {worst:.3f}, relative 2-norm {rel:.5f}", flush=True)
        assert worst <= 1.0 and rel <= REL, tag
        assert (got[ks[r] + n[r]:ks[r + 1]] == -7.0).all(), f"{tag}: written behind request {r}'s keys"
    if w.causal and old is None:  # every row that sees a key gives a weight of one in all, as near as the forward pass has its lse
        rows = (~torch.isneginf(lse)).sum().item()
        assert abs(sum(got[ks[r]:ks[r] + n[r]].sum() for r in range(w.batch)) - rows) <= 0.01 * rows + 1e-6
    again = torch.empty_like(out)
    fn(*args, again, **kw)
    for r in range(w.batch):
        assert torch.equal(again[ks[r]:ks[r] + n[r]], out[ks[r]:ks[r] + n[r]])
    if win is not None:  # in place
        fn(*args, win, **kw)
        for r in range(w.batch):
            assert torch.equal(win[ks[r]:ks[r] + n[r]], out[ks[r]:ks[r] + n[r]])


def decode_of(w):
    """One new token per request: the last query row of each of a prefill workload's requests."""
    last = w.q_start[1:] - 1
    return dataclasses.replace(w, kind="decode", q=np.ascontiguousarray(w.q[last]),
                               q_start=np.arange(w.batch + 1, dtype=np.int32),
                               q_pos0=(w.q_pos0 + w.q_lens - 1).astype(np.int32))


WEIGHTS = {
    "tiny": (lambda: W.tiny_rag_prefill(0, slack_fill=float("nan")), {}),
    "one query, one key": (lambda: W.custom(1, 2, 1, 64, 1e4, [dict(chunks=[(1, 0)], q_len=1, q_pos0=0)]), {}),
    "d128": (lambda: shared(50, 8, 2, 128, [130, 64, 33], [17, 40, 3]), {}),
    "d64 group 7": (lambda: shared(51, 14, 2, 64, [129, 63], [11, 50]), {}),
    "group 1, 12 heads": (lambda: shared(52, 12, 12, 64, [100, 20], [33, 64]), {}),
    "group 20": (lambda: shared(53, 40, 2, 128, [200, 7], [9, 40]), {}),
    "group 16, many rows": (lambda: shared(54, 16, 1, 128, [70], [300]), {}),
    "interleaved": (lambda: shared(55, 4, 2, 128, [70, 90], [20, 31]), dict(rope_style=ops.ROPE_INTERLEAVED)),
    "interleaved local d64": (lambda: shared(56, 4, 1, 64, [70, 90], [20, 31], twice=True),
                              dict(rope_style=ops.ROPE_INTERLEAVED, key_positions=ops.KEYS_LOCAL)),
    "local": (lambda: shared(57, 8, 2, 128, [70, 90, 128], [20, 31]), dict(key_positions=ops.KEYS_LOCAL)),
    "alibi": (lambda: shared(58, 8, 2, 128, [70, 90], [20, 31]), dict(rope_style=ops.ALIBI)),
    "alibi d64 not causal": (lambda: shared(59, 6, 2, 64, [70, 90], [20, 31], causal=False), dict(rope_style=ops.ALIBI)),
    "not causal": (lambda: shared(60, 8, 2, 128, [70, 90], [20, 31], causal=False), {}),
    "prerotated": (lambda: shared(61, 8, 2, 128, [70, 90], [20, 31]), dict(q_prerotated=True)),
    "scale": (lambda: shared(62, 8, 2, 64, [70, 90], [20, 31]), dict(softmax_scale=0.05)),
    "paged": (lambda: W.paginate(shared(63, 8, 2, 128, [170, 45], [38, 3]), 32), {}),
    "paged 16": (lambda: W.paginate(shared(64, 8, 2, 64, [700, 45], [38, 3], reqs=2), 16), {}),
    "own tokens": (lambda: W.custom(65, 8, 2, 128, 1e4, [dict(chunks=[(517, 0)], q_len=517, q_pos0=0)]), {}),
    "rows that see nothing": (lambda: W.custom(66, 4, 2, 128, 1e4, [
        dict(chunks=[("a", 100, 37)], q_len=90, q_pos0=3), dict(chunks=[("a", 100, 0), ("b", 65, 100)], q_len=40, q_pos0=20),
        dict(chunks=[("b", 65, 30)], q_len=5, q_pos0=1)], slack_fill=float("nan")), {}),
    "long": (lambda: shared(67, 4, 1, 64, [5000], [3], reqs=1), {}),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", WEIGHTS)
def test_prompt_weights(gpu, name):
    make, ckw = WEIGHTS[name]
    check_weights(make(), ckw, name)


@pytest.mark.gpu
@pytest.mark.parametrize("name", WEIGHTS)
def test_token_weights(gpu, name):
    make, ckw = WEIGHTS[name]
    check_weights(decode_of(make()), ckw, name)


@pytest.mark.gpu
@pytest.mark.parametrize("decay", [1.0, 0.9, 0.0])
def test_running_sums_and_room_behind_the_keys(gpu, decay):
    w = shared(70, 8, 2, 128, [130, 64], [17, 40, 3])
    check_weights(w, {}, f"prompt decay {decay}", room=37, decay=decay)
    check_weights(decode_of(w), {}, f"token decay {decay}", room=5, decay=decay)


# Batches whose requests are walked in storage order: a workgroup reads half a megabyte or more.
BATCHES = {
    "group 4": (lambda: shared(75, 16, 4, 128, [230, 264, 70], [1], reqs=770), {}),
    "group 12, interleaved": (lambda: shared(76, 24, 2, 128, [500, 40, 517], [1], reqs=769),
                              dict(rope_style=ops.ROPE_INTERLEAVED)),
    "local, d64": (lambda: shared(77, 8, 4, 64, [600, 500], [1], reqs=768), dict(key_positions=ops.KEYS_LOCAL)),
    "more records than are sorted": (lambda: W.paginate(shared(78, 4, 4, 128, [270, 260], [1], reqs=768), 1), {}),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", BATCHES)
def test_token_weights_of_many_requests(gpu, name):
    make, ckw = BATCHES[name]
    check_weights(decode_of(make()), ckw, name)


@pytest.mark.gpu
def test_requests_without_queries_or_keys(gpu):
    w = W.custom(71, 4, 2, 64, 1e4, [dict(chunks=[(70, 0)], q_len=0, q_pos0=0), dict(chunks=[], q_len=3, q_pos0=0),
                                     dict(chunks=[(9, 0)], q_len=2, q_pos0=9)])
    check_weights(w, {}, "empty requests", room=3)
    check_weights(w, {}, "empty requests", room=3, decay=0.5)


@pytest.mark.gpu
def test_keys_without_room_are_passed_over(gpu):
    w = decode_of(shared(72, 4, 2, 64, [100], [4], reqs=2))
    dw = ops.upload(w)
    cfg = ops.config_of(w)
    _, lse = ops.run_lazy(dw, cfg)
    full = torch.full((int(w.kv_lens.sum()),), -7.0, device="cuda")
    ops.decode_key_weights(cfg, dw.q, dw.q_pos0, dw.pool, dw.chunks, dw.chunk_start, i32(starts(w.kv_lens)),
                           w.max_kv_len, lse, full)
    ks = starts(w.kv_lens, -9)
    part = torch.full((int(ks[-1]) + 50,), -7.0, device="cuda")
    ops.decode_key_weights(cfg, dw.q, dw.q_pos0, dw.pool, dw.chunks, dw.chunk_start, i32(ks), w.max_kv_len, lse, part)
    n = int(w.kv_lens[0])
    for r in range(2):
        assert torch.equal(part[ks[r]:ks[r + 1]], full[r * n:r * n + n - 9])
    assert (part[ks[-1]:] == -7.0).all()


# ---------------------------------------------------------------------------------------------------------------
# GPU: selection
# ---------------------------------------------------------------------------------------------------------------
def run_select(ws, budgets, sink=0, recent=0, room=0, counts=True):
    n = [len(w) for w in ws]
    ks, os = starts(n, room), starts(budgets)
    flat = np.full(int(ks[-1]), np.inf, np.float32)  # what lies behind a request's keys would win if it were read
    for r, w in enumerate(ws):
        flat[ks[r]:ks[r] + n[r]] = w
    kept = torch.full((int(os[-1]) + 3,), -9, dtype=torch.int32, device="cuda")
    ops.cache_select(torch.from_numpy(flat).cuda(), i32(ks), i32(os), max(n + [0]), kept, sink=sink, recent=recent,
                     key_count=i32(n) if counts else None)
    kept = kept.cpu().numpy()
    assert (kept[int(os[-1]):] == -9).all()
    return [kept[os[r]:os[r + 1]].tolist() for r in range(len(ws))]


def check_select(ws, budgets, **kw):
    got = run_select(ws, budgets, **kw)
    for r, (w, b) in enumerate(zip(ws, budgets)):
        want = E.select(w, b, kw.get("sink", 0), kw.get("recent", 0))
        assert got[r] == want + [-1] * (b - len(want)), f"request {r}: {len(w)} keys, budget {b}"


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 1000, 1024, 1025, 5000, 33068, 131073])
def test_selection_sizes(gpu, n):
    rng = np.random.default_rng(n)
    w = np.exp(2 * rng.standard_normal(n)).astype(np.float32)
    for b in sorted({1, max(1, n // 8), max(1, n - 1), n, n + 2}):
        check_select([w], [b], counts=False)
        check_select([w], [b], sink=min(4, b), recent=min(100, max(0, b - 4)))


@pytest.mark.gpu
def test_selection_ties_and_special_values(gpu):
    rng = np.random.default_rng(3)
    ties = rng.integers(0, 4, 3000).astype(np.float32)
    same = np.full(700, 2.5, np.float32)
    zeros = np.where(rng.random(500) < 0.5, np.float32(0.0), np.float32(-0.0)).astype(np.float32)
    odd = rng.standard_normal(900).astype(np.float32)
    odd[::7], odd[5::11], odd[3::13] = np.nan, np.inf, -np.inf
    tiny = (rng.integers(0, 5, 400) * np.float32(1e-45)).astype(np.float32)
    for b in (1, 7, 350, 399):
        check_select([ties, same, zeros, odd, tiny], [b] * 5, room=3)
        check_select([ties, same, zeros, odd, tiny], [b] * 5, sink=5, recent=9, room=1)


@pytest.mark.gpu
def test_selection_of_ragged_batches(gpu):
    rng = np.random.default_rng(4)
    ws = [rng.random(n).astype(np.float32) for n in (0, 5, 2000, 1, 700, 64)]
    check_select(ws, [3, 0, 777, 1, 900, 63], room=2)
    check_select(ws, [3, 0, 777, 1, 900, 63], sink=1000, recent=2)


# ---------------------------------------------------------------------------------------------------------------
# GPU: compaction
# ---------------------------------------------------------------------------------------------------------------
def check_compact(w, ckw, rotate, tag, one_pool=True):
    cfg = ops.config_of(w, **ckw)
    dw = ops.upload(w)
    rng = np.random.default_rng(9)
    hkv, d = w.num_kv_heads, w.head_dim
    n = w.kv_lens
    kept = [np.sort(rng.choice(int(k), int(b), replace=False)) if k else np.zeros(0, int)
            for k, b in zip(n, [max(1, int(0.4 * k)) if k else 0 for k in n])]
    kept = [np.concatenate([k, [-1, int(n[r]) + 5]]) if r == 1 else k for r, k in enumerate(kept)]  # entries passed over
    os, ks = starts([len(k) for k in kept]), starts(n, 3)
    dst, at = [], 0
    for r, k in enumerate(kept):
        cap = len(k) + 4 if r != 2 else max(1, len(k) - 3)  # the third record is too small for its keys
        dst.append((at, at + cap * hkv * d if one_pool else at, len(k), 0, cap, cap))
        at += (2 if one_pool else 1) * cap * hkv * d
    dst = np.array(dst, dtype=W.CHUNK_DTYPE)
    ko = torch.full((at,), 5.0, dtype=torch.bfloat16, device="cuda")
    vo = ko if one_pool else torch.full_like(ko, 5.0)
    wt = torch.rand(int(ks[-1]), device="cuda")
    wo = torch.full((int(os[-1]),), -7.0, device="cuda")
    ops.cache_compact(cfg, dw.pool, dw.pool, dw.chunks, dw.chunk_start, i32(np.concatenate(kept)), i32(os),
                      max(len(k) for k in kept), torch.from_numpy(dst.view(np.uint8).copy()).cuda(), ko, vo,
                      rotate=rotate, key_start=i32(ks), weights=wt, weights_out=wo)
    torch.cuda.synchronize()
    ko, vo, wt, wo = ko.float().cpu().numpy(), vo.float().cpu().numpy(), wt.cpu().numpy(), wo.cpu().numpy()
    want_k, want_v = np.full(at, 5.0), np.full(at, 5.0)
    if one_pool:
        want_v = want_k
    exact = not rotate and not ckw.get("key_positions")
    pairing = "interleaved" if ckw.get("rope_style") == ops.ROPE_INTERLEAVED else "half"
    theta = O.rope_frequencies(d, w.rope_base)
    for r, idx in enumerate(kept):
        K, V, kpos, offs = O.request_kv(w.pool, w.pool, w.chunks, int(w.chunk_start[r]), int(w.chunk_start[r + 1]), hkv, d,
                                        with_offsets=True)
        for i, j in enumerate(idx):
            ok = 0 <= j < n[r]
            assert wo[os[r] + i] == (wt[ks[r] + j] if ok else 0.0), tag
            if not ok or i >= dst[r]["k_stride"]:
                continue
            k = K[:, j:j + 1]
            if rotate:
                k = O.rotate(k, [kpos[j] if not ckw.get("key_positions") else offs[j]], theta, pairing)
            elif ckw.get("key_positions"):
                k = O.rotate(k, [i - (kpos[j] - offs[j])], theta, pairing)
            for g in range(hkv):
                a = int(dst[r]["k_offset"]) + (g * int(dst[r]["k_stride"]) + i) * d
                want_k[a:a + d] = k[g, 0]
                a = int(dst[r]["v_offset"]) + (g * int(dst[r]["v_stride"]) + i) * d
                want_v[a:a + d] = V[g, j]
    # one rounding, and the hardware sine and cosine (1.3e-7 each) times two elements of at most 8
    tol = 0.0 if exact else 2.0 ** -8 * np.abs(want_k) + 4e-6
    assert (np.abs(ko - want_k) <= tol).all(), tag
    if not one_pool:
        assert (vo == want_v).all(), tag


COMPACT = {
    "nope d128": ((lambda: shared(80, 8, 2, 128, [130, 64, 33], [17, 40, 3])), {}),
    "nope d64 paged": ((lambda: W.paginate(shared(81, 4, 2, 64, [530, 64], [17, 40, 3]), 16)), {}),
    "local": ((lambda: shared(82, 4, 2, 128, [130, 64], [17, 40, 3])), dict(key_positions=ops.KEYS_LOCAL)),
    "local interleaved d64": ((lambda: shared(83, 3, 3, 64, [130, 64], [17, 40, 3])),
                              dict(key_positions=ops.KEYS_LOCAL, rope_style=ops.ROPE_INTERLEAVED)),
    "interleaved": ((lambda: shared(84, 4, 1, 128, [130, 64], [17, 40, 3])), dict(rope_style=ops.ROPE_INTERLEAVED)),
    "many blocks": ((lambda: W.paginate(shared(85, 2, 1, 64, [9000], [3, 1], reqs=3), 16)), {}),
    "a request without keys": ((lambda: W.custom(86, 2, 1, 64, 1e4, [
        dict(chunks=[(40, 0)], q_len=1, q_pos0=40), dict(chunks=[(20, 0)], q_len=1, q_pos0=20),
        dict(chunks=[(30, 0)], q_len=1, q_pos0=30), dict(chunks=[], q_len=1, q_pos0=0)])), {}),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", COMPACT)
@pytest.mark.parametrize("rotate", [False, True])
def test_compaction(gpu, name, rotate):
    make, ckw = COMPACT[name]
    check_compact(make(), ckw, rotate, name, one_pool=not rotate)


@pytest.mark.gpu
def test_rotated_copies_are_the_materialised_keys(gpu):
    """All keys kept and rotated: the bits of lazy_materialize_k's copy up to one step (its angles are added up from
    two parts), and the same attention."""
    w = shared(87, 8, 2, 128, [130, 64], [9], reqs=1)
    cfg, dw = ops.config_of(w), ops.upload(w)
    n = int(w.kv_lens[0])
    per = w.num_kv_heads * w.head_dim
    out = torch.zeros(2 * n * per, dtype=torch.bfloat16, device="cuda")
    dst = np.array([(0, n * per, n, 0, n, n)], dtype=W.CHUNK_DTYPE)
    table = torch.from_numpy(dst.view(np.uint8).copy()).cuda()
    ops.cache_compact(cfg, dw.pool, dw.pool, dw.chunks, dw.chunk_start, i32(np.arange(n)), i32([0, n]), n, table, out,
                      out, rotate=True)
    a, _ = ops.prefill(cfg, dw.q, dw.q_start, dw.q_pos0, out, out, table, i32([0, 1]), w.max_q_len, n, plain=True)
    b, _ = ops.run_lazy(dw, cfg)
    torch.cuda.synchronize()
    assert (a.float() - b.float()).abs().max().item() <= 2e-2


# ---------------------------------------------------------------------------------------------------------------
# GPU: the whole path, and the same path in a graph
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("rotate", [False, True])
def test_prompt_then_eviction_then_decoding(gpu, rotate):
    """Weights of a prompt, selection, compaction, and a decode step over the compacted cache, whose outputs and whose
    own key weights are those of the oracle over the kept keys (positions closed up, or as they were)."""
    w = shared(90, 8, 2, 128, [300, 211, 64], [40], reqs=3)
    cfg, dw = ops.config_of(w), ops.upload(w)
    hkv, d = w.num_kv_heads, w.head_dim
    n, budget, cap = w.kv_lens, 100, 116
    ks, os = starts(n), starts([budget] * 3)
    _, lse = ops.run_lazy(dw, cfg)
    weights = torch.empty(int(ks[-1]), device="cuda")
    ops.prefill_key_weights(cfg, dw.q, dw.q_start, dw.q_pos0, dw.pool, dw.chunks, dw.chunk_start, i32(ks), w.max_q_len,
                            w.max_kv_len, lse, weights)
    kept = torch.empty(3 * budget, dtype=torch.int32, device="cuda")
    ops.cache_select(weights, i32(ks), i32(os), w.max_kv_len, kept, sink=4, recent=16)
    store = torch.zeros(3 * 2 * cap * hkv * d, dtype=torch.bfloat16, device="cuda")
    dst = np.array([(2 * r * cap * hkv * d, (2 * r + 1) * cap * hkv * d, budget, 0, cap, cap) for r in range(3)],
                   dtype=W.CHUNK_DTYPE)
    table = torch.from_numpy(dst.view(np.uint8).copy()).cuda()
    room = starts([budget] * 3, 16)
    running = torch.zeros(int(room[-1]), device="cuda")
    wo = torch.empty(3 * budget, device="cuda")
    ops.cache_compact(cfg, dw.pool, dw.pool, dw.chunks, dw.chunk_start, kept, i32(os), budget, table, store, store,
                      rotate=rotate, key_start=i32(ks), weights=weights, weights_out=wo)
    running.view(3, -1)[:, :budget] = wo.view(3, -1)
    host_w, host_kept = weights.cpu().numpy(), kept.cpu().numpy()
    rng = np.random.default_rng(1)
    q = W.bf16_round(rng.standard_normal((3, w.num_q_heads, d), dtype=np.float32))
    # closed up: the next position is the budget; rotated: positions go on where the prompt ended
    q_pos = np.full(3, budget, np.int32) if not rotate else (w.q_pos0 + w.q_lens).astype(np.int32)
    qd = torch.from_numpy(W.bf16_bits(q).view(np.int16)).cuda().view(torch.bfloat16)
    args = (cfg, qd, i32(q_pos), store, store, table, i32(np.arange(4)), budget)
    lse2 = torch.empty(3, w.num_q_heads, device="cuda")
    out, lse2 = ops.decode(*args, lse=lse2, plain=rotate)
    torch.cuda.synchronize()
    for r in range(3):
        mine = host_kept[os[r]:os[r + 1]]
        assert mine.tolist() == E.select(host_w[ks[r]:ks[r + 1]], budget, 4, 16)
        K, V, kpos = O.request_kv(w.pool, w.pool, w.chunks, int(w.chunk_start[r]), int(w.chunk_start[r + 1]), hkv, d)
        theta = O.rope_frequencies(d, w.rope_base)
        pos = kpos[mine] if rotate else np.arange(budget)
        Kr = O.rotate(K[:, mine], pos, theta)
        qr = O.rotate(q[r][:, None], [q_pos[r]], theta)[:, 0]
        for h in range(w.num_q_heads):
            s = Kr[h // 4] @ qr[h] / math.sqrt(d)
            p = np.exp(s - s.max())
            want = (p / p.sum()) @ V[h // 4][mine]
            assert np.abs(out[r, h].float().cpu().numpy() - want).max() <= 2e-2
            assert abs(lse2[r, h].item() - (s.max() + math.log(p.sum()))) <= 2e-2
    if not rotate:  # the decode step's own weights are added to what the kept keys had
        before = running.clone()
        ops.decode_key_weights(cfg, qd, i32(q_pos), store, table, i32(np.arange(4)), i32(room), budget, lse2, running,
                               weights_in=running)
        more = (running - before).view(3, -1)
        assert torch.allclose(more[:, :budget].sum(1), torch.full((3,), 8.0, device="cuda"), atol=0.08)
        assert not more[:, budget:].any()


@pytest.mark.gpu
def test_eviction_in_a_graph(gpu):
    w = shared(91, 8, 2, 64, [300, 211, 64], [40], reqs=3)
    cfg, dw = ops.config_of(w), ops.upload(w)
    hkv, d, n, budget = w.num_kv_heads, w.head_dim, w.kv_lens, 100
    ks, os, cs = i32(starts(n)), i32(starts([budget] * 3)), i32(np.arange(4))
    _, lse = ops.run_lazy(dw, cfg)
    weights = torch.zeros(int(n.sum()), device="cuda")
    kept = torch.empty(3 * budget, dtype=torch.int32, device="cuda")
    store = torch.zeros(3 * 2 * budget * hkv * d, dtype=torch.bfloat16, device="cuda")
    dst = np.array([(2 * r * budget * hkv * d, (2 * r + 1) * budget * hkv * d, budget, 0, budget, budget)
                    for r in range(3)], dtype=W.CHUNK_DTYPE)
    table = torch.from_numpy(dst.view(np.uint8).copy()).cuda()
    token = torch.zeros(3 * budget, device="cuda")
    q1, p1 = dw.q[::40].contiguous(), i32(np.full(3, budget))
    l1 = torch.zeros(3, w.num_q_heads, device="cuda")
    ws = torch.empty(ops.prefill_key_weights_workspace_size(cfg, 3, w.total_q, w.max_q_len, w.max_kv_len,
                                                            weights.numel()), dtype=torch.uint8, device="cuda")
    sws = torch.empty(max(1, ops.cache_select_workspace_size(3, w.max_kv_len)), dtype=torch.uint8, device="cuda")
    dws = torch.empty(max(1, ops.decode_workspace_size(cfg, 3, budget)), dtype=torch.uint8, device="cuda")
    tws = torch.empty(max(1, ops.decode_key_weights_workspace_size(cfg, 3, budget)), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q1)

    def path():
        ops.prefill_key_weights(cfg, dw.q, dw.q_start, dw.q_pos0, dw.pool, dw.chunks, dw.chunk_start, ks, w.max_q_len,
                                w.max_kv_len, lse, weights, workspace=ws)
        ops.cache_select(weights, ks, os, w.max_kv_len, kept, sink=2, recent=8, workspace=sws)
        ops.cache_compact(cfg, dw.pool, dw.pool, dw.chunks, dw.chunk_start, kept, os, budget, table, store, store)
        ops.decode(cfg, q1, p1, store, store, table, cs, budget, out=out, lse=l1, workspace=dws)
        ops.decode_key_weights(cfg, q1, p1, store, table, cs, os, budget, l1, token, workspace=tws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        path()
    side.synchronize()
    bufs = (weights, kept, store, out, token)
    want = [b.clone() for b in bufs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        path()
    for _ in range(4):
        for b in bufs + (ws,):
            b.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bufs, want))
        torch.mm(torch.ones(64, 64, device="cuda"), torch.ones(64, 64, device="cuda"))


# ---------------------------------------------------------------------------------------------------------------
# Calls at the edges
# ---------------------------------------------------------------------------------------------------------------
def test_largest_bounds_without_a_gpu():
    """Bounds near 2^31: sizes do not wrap, and what no launch holds is refused."""
    most, one = (1 << 31) - 1, 4096
    slices = -(-most // 16384)
    assert ops.cache_select_workspace_size(1, most) >= slices * 3 * 2048 * 4
    assert ops.cache_select_workspace_size(3, most) == 3 * ops.cache_select_workspace_size(1, most)
    p = ops.Config(1, 1, 64, 1e4).c()
    assert ops.lib().lazy_cache_compact(ctypes.byref(p), one, one, one, one, 1, one, one, most, one, 0, one, one, None,
                                        None, None, None) == ops.LAZY_EUNSUPPORTED
    assert ops.lib().lazy_attn_prefill_key_weights(
        ctypes.byref(p), one, one, one, one, one, one, one, 1, most - 1, 4, 4, 4, one, None, 1.0, one, one, 1 << 50,
        None) == ops.LAZY_EUNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,style", [(4, 2, 64, ops.ROPE_HALF), (12, 1, 128, ops.ROPE_INTERLEAVED),
                                            (8, 2, 128, ops.ALIBI)])
def test_rows_that_are_left_out_may_hold_anything(gpu, hq, hkv, d, style):
    """Rows whose log-sum-exp is -inf give nothing, whatever their queries hold."""
    w = W.custom(92, hq, hkv, d, 1e4, [dict(chunks=[("a", 100, 0), (30, 100)], q_len=30, q_pos0=100),
                                       dict(chunks=[("a", 100, 7)], q_len=9, q_pos0=110)])
    cfg, dw = ops.config_of(w, rope_style=style), ops.upload(w)
    _, lse = ops.run_lazy(dw, cfg)
    lse[5:11] = -math.inf
    lse[:, hq // 2] = -math.inf
    dead, ks = torch.isneginf(lse), i32(starts(w.kv_lens))
    out = []
    for fill in (0.0, math.nan, math.inf):
        q = dw.q.clone()
        q[dead] = fill
        a = torch.empty(int(w.kv_lens.sum()), device="cuda")
        ops.prefill_key_weights(cfg, q, dw.q_start, dw.q_pos0, dw.pool, dw.chunks, dw.chunk_start, ks, w.max_q_len,
                                w.max_kv_len, lse, a)
        b = torch.empty_like(a)
        rows = [7, 38]
        ops.decode_key_weights(cfg, q[rows].contiguous(), i32([107, 118]), dw.pool, dw.chunks, dw.chunk_start, ks,
                               w.max_kv_len, lse[rows].contiguous(), b)
        out.append((a, b))
    assert torch.isfinite(out[0][0]).all() and out[0][0].any()
    assert not out[0][1][:130].any() and out[0][1][130:].any()
    for a, b in out[1:]:
        assert torch.equal(a, out[0][0]) and torch.equal(b, out[0][1])


@pytest.mark.gpu
def test_kept_keys_without_room_have_no_weight(gpu):
    w = shared(93, 4, 2, 64, [100], [4], reqs=2)
    cfg, dw = ops.config_of(w), ops.upload(w)
    n, room, cap = int(w.kv_lens[0]), 50, 8
    kept = np.array([0, 20, 49, 50, 60, n - 1] * 2)
    ks, os = starts([room, room]), starts([6, 6])
    weights = torch.arange(1, 2 * room + 1, device="cuda", dtype=torch.float32)
    per = cap * w.num_kv_heads * w.head_dim
    dst = np.array([(2 * r * per, (2 * r + 1) * per, 6, 0, cap, cap) for r in range(2)], dtype=W.CHUNK_DTYPE)
    store = torch.zeros(4 * per, dtype=torch.bfloat16, device="cuda")
    wo = torch.full((12,), -7.0, device="cuda")
    ops.cache_compact(cfg, dw.pool, dw.pool, dw.chunks, dw.chunk_start, i32(kept), i32(os), 6,
                      torch.from_numpy(dst.view(np.uint8).copy()).cuda(), store, store, key_start=i32(ks),
                      weights=weights, weights_out=wo)
    assert wo.tolist() == [1, 21, 50, 0, 0, 0, 51, 71, 100, 0, 0, 0]


@pytest.mark.gpu
def test_nothing_is_kept(gpu):
    w = shared(94, 4, 2, 64, [100], [4], reqs=2)
    cfg, dw = ops.config_of(w), ops.upload(w)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    weights = torch.rand(int(w.kv_lens.sum()), device="cuda")
    assert ops.cache_select(weights, i32(starts(w.kv_lens)), i32([0, 0, 0]), w.max_kv_len, none) is none
    store = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    ops.cache_compact(cfg, dw.pool, dw.pool, dw.chunks, dw.chunk_start, none, i32([0, 0, 0]), 5,
                      torch.zeros(64, dtype=torch.uint8, device="cuda"), store, store)
    assert (store == 1).all()


@pytest.mark.gpu
def test_selection_of_a_long_request_in_a_graph(gpu):
    n, budget = [40000, 17, 70001], [5000, 4, 70000]
    gen = torch.Generator("cuda").manual_seed(3)
    weights = torch.empty(sum(n), device="cuda")
    ks, os = i32(starts(n)), i32(starts(budget))
    kept = torch.empty(sum(budget), dtype=torch.int32, device="cuda")
    ws = torch.empty(ops.cache_select_workspace_size(3, max(n)), dtype=torch.uint8, device="cuda")
    weights.uniform_(generator=gen)

    def call():
        ops.cache_select(weights, ks, os, max(n), kept, sink=3, recent=7, workspace=ws)

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        weights.uniform_(generator=gen)
        ws.fill_(171 + step)
        graph.replay()
        torch.cuda.synchronize()
        host, at, to = weights.cpu().numpy(), 0, 0
        for k, b in zip(n, budget):
            assert kept[to:to + b].tolist() == E.select(host[at:at + k], b, 3, 7)
            at, to = at + k, to + b
