"""The backward pass: its planner on the CPU (every visible pair of query row and stored key covered once, refusals),
its oracle against differences of the forward oracle, and the kernels against the oracle on the GPU.

GPU tolerances, both derived in ``oracle/gradient_oracle.py`` from the roundings to bf16 that the method makes.
Element by element: the first-order bound of the worst case.  Over a whole tensor: roundings are independent, each with
a root mean square of at most u / sqrt(3) = 0.00226 relative; a score error has sqrt(2) of that for inputs of unit
variance, P and dS, the other operand and the result one more each, together sqrt(2 + 4) 0.00226 = 0.0056 of the
gradient's 2-norm; three times that is allowed.
"""
import ctypes
import dataclasses

import numpy as np
import pytest
import torch

from oracle import gradient_oracle as GO
from oracle import lazy_oracle as O
from paper_2606_04302_amd import ops
from paper_2606_04302_amd import workloads as W

REL = 0.017

HALF = np.dtype([("k_off", "<i8"), ("v_off", "<i8"), ("kst", "<i4"), ("vst", "<i4"), ("keys", "<i4"),
                 ("reserved", "<i4")])
TILE = np.dtype([("half", HALF, 2), ("seg_begin", "<i4"), ("seg_end", "<i4"), ("part", "<i4"), ("reserved", "<i4")])
SEG_HALF = np.dtype([(n, "<i4") for n in ("pos", "record_pos", "key_begin", "key_end")])
SEG = np.dtype([(n, "<i4") for n in ("row_begin", "row_end", "pos_shift", "full_from")] + [("half", SEG_HALF, 2)])
MERGE = np.dtype([("half", HALF, 2), ("part", "<i4"), ("parts", "<i4"), ("reserved", "<i4", 2)])
ROW = np.dtype([(n, "<i4") for n in ("request", "row0", "split", "splits")])
BLOCK = np.dtype([(n, "<i4") for n in ("t0", "tokens", "pos_shift", "splits")])


def arrays(plan):
    """The plan's arrays: blocks, row items, segments, tiles, merges."""
    i, at, out = plan.info, 0, []
    for dt, n in ((BLOCK, i.num_blocks), (ROW, i.num_row_items), (SEG, i.num_segments), (TILE, i.num_tiles),
                  (MERGE, i.num_merges)):
        out.append(plan.data[at:at + n * dt.itemsize].view(dt))
        at += n * dt.itemsize
    assert at == plan.data.size
    return out


def make_plan(w, **kw):
    cfg = ops.config_of(w, **kw)
    return cfg, ops.backward_plan(cfg, w.q_start, w.q_pos0, w.chunks, w.chunk_start)


def sub_records(w, length, cuts):
    """Copy of a workload whose records of `length` keys keep only a part of them, in turn: (first key, keys)."""
    chunks = w.chunks.copy()
    for i, (b, n) in zip(np.flatnonzero(chunks["len"] == length), cuts):
        chunks[i]["k_offset"] += b * w.head_dim
        chunks[i]["v_offset"] += b * w.head_dim
        chunks[i]["len"] = n
        chunks[i]["pos_offset"] += b
    return dataclasses.replace(w, chunks=chunks)


def shared(seed, hq, hkv, d, lens, q_lens, reqs=3, causal=True, gap=0, twice=False, slack=float("nan")):
    """Requests that read common chunks of the given lengths in orders of their own, then their own tokens."""
    rng = np.random.default_rng(seed)
    requests = []
    for r in range(reqs):
        u, pos = [], gap
        for c in rng.permutation(len(lens)):
            u.append((f"c{c}", lens[c], pos))
            pos += lens[c]
        if twice:
            u.append(("c0", lens[0], pos))
            pos += lens[0]
        n = q_lens[r % len(q_lens)]
        if n:
            u.append((n, pos))
        requests.append(dict(chunks=u, q_len=n, q_pos0=pos))
    return W.custom(seed, hq, hkv, d, 1.0e4, requests, causal=causal, slack_fill=slack)


# ---------------------------------------------------------------------------------------------------------------
# CPU: planner
# ---------------------------------------------------------------------------------------------------------------
def covered(w, plan, G):
    """{(token, k element offset of head 0, position): rows} over the plan's tiles and segments."""
    _, _, segs, tiles, _ = arrays(plan)
    pos_of = w.q_positions()
    seen = {}
    for t in tiles:
        for s in segs[t["seg_begin"]:t["seg_end"]]:
            assert 0 <= s["row_begin"] < s["row_end"] <= w.total_q * G
            for h, sh in zip(t["half"], s["half"]):
                assert 0 <= sh["key_begin"] <= sh["key_end"] <= h["keys"]
                for tok in range(int(s["row_begin"]) // G, -(-int(s["row_end"]) // G)):
                    # rows of a token may be divided between parts: count rows
                    rows = min(int(s["row_end"]), (tok + 1) * G) - max(int(s["row_begin"]), tok * G)
                    assert pos_of[tok] == tok + int(s["pos_shift"])
                    full = tok * G >= s["full_from"]
                    assert not full or (sh["key_begin"] == 0 and sh["key_end"] == h["keys"])
                    for key in range(int(sh["key_begin"]), int(sh["key_end"])):
                        if not w.causal or int(sh["pos"]) + key <= pos_of[tok]:
                            at = (tok, int(h["k_off"]) + key * w.head_dim, int(sh["pos"]) + key)
                            seen[at] = seen.get(at, 0) + rows
                        else:
                            assert not full
    return seen


def expected(w, G):
    pos_of = w.q_positions()
    want = {}
    for r in range(w.batch):
        for c in w.chunks[w.chunk_start[r]:w.chunk_start[r + 1]]:
            for j in range(int(c["len"])):
                for tok in range(int(w.q_start[r]), int(w.q_start[r + 1])):
                    if not w.causal or int(c["pos_offset"]) + j <= pos_of[tok]:
                        at = (tok, int(c["k_offset"]) + j * w.head_dim, int(c["pos_offset"]) + j)
                        want[at] = want.get(at, 0) + G
    return want


PLAN_CASES = {
    "tiny": lambda: W.tiny_rag_prefill(0),
    "shared": lambda: shared(1, 4, 2, 64, [70, 33, 128], [5, 1, 9]),
    "twice": lambda: shared(2, 3, 1, 64, [65, 7], [4], twice=True),
    "not causal": lambda: shared(3, 2, 2, 64, [40, 64], [3, 2], causal=False),
    "gap": lambda: W.custom(4, 2, 1, 64, 1e4, [dict(chunks=[("a", 20, 6)], q_len=12, q_pos0=3),
                                               dict(chunks=[("a", 20, 0)], q_len=0, q_pos0=0)]),
    "sub-records": lambda: sub_records(shared(5, 2, 1, 64, [150, 30], [6], reqs=3), 150, [(10, 77), (64, 20)]),
    "paged": lambda: W.paginate(shared(6, 7, 1, 64, [70, 45], [8, 3]), 32),
    "parts": lambda: shared(7, 1, 1, 64, [64], [300, 301], reqs=5),
}


@pytest.mark.parametrize("name", PLAN_CASES)
def test_plan_covers_every_visible_pair_once(name):
    w = PLAN_CASES[name]()
    G = w.num_q_heads // w.num_kv_heads
    _, plan = make_plan(w)
    assert covered(w, plan, G) == expected(w, G)
    blocks, rows, segs, tiles, merges = arrays(plan)
    # Every stored key belongs to one tile (or to the parts of one), and parts are numbered without a gap.
    keys = {}
    for t in tiles:
        for h in t["half"]:
            for k in range(int(h["keys"])):
                keys.setdefault(int(h["k_off"]) + k * w.head_dim, []).append(int(t["part"]))
    for c in w.chunks:
        for j in range(int(c["len"])):
            parts = keys[int(c["k_offset"]) + j * w.head_dim]
            assert parts == [-1] or -1 not in parts
    assert sorted(int(t["part"]) for t in tiles if t["part"] >= 0) == list(range(plan.info.num_parts))
    assert sum(int(m["parts"]) for m in merges) == plan.info.num_parts
    # Tokens belong to one block each; every row of a request is in one row item for each of its splits.
    toks = np.concatenate([np.arange(b["t0"], b["t0"] + b["tokens"]) for b in blocks]) if len(blocks) else []
    assert sorted(toks) == list(range(w.total_q))
    bm = 128 * plan.info.row_blocks
    for r in range(w.batch):
        mine = rows[rows["request"] == r]
        n = int(w.q_lens[r]) * G
        got = sorted((int(m["row0"]), int(m["split"])) for m in mine)
        splits = int(mine["splits"][0]) if len(mine) else 0
        assert got == [(x, s) for x in range(0, n, bm) for s in range(splits)]


def test_plan_cuts_heavy_tiles_into_parts():
    w = shared(8, 1, 1, 64, [64], [300, 301], reqs=5)
    _, plan = make_plan(w)
    assert plan.info.num_merges >= 1 and plan.info.num_parts >= 2 * plan.info.num_merges


def test_plan_refusals():
    w = shared(9, 2, 1, 64, [70, 33], [5])
    cfg = ops.config_of(w)

    def code(chunks=None, q_start=w.q_start, q_pos0=w.q_pos0, chunk_start=w.chunk_start, cfg=cfg):
        with pytest.raises(ops.LazyAttnError) as e:
            ops.backward_plan(cfg, q_start, q_pos0, w.chunks if chunks is None else chunks, chunk_start)
        return e.value.code

    for field, value in (("len", -1), ("k_stride", 1), ("v_stride", 1), ("k_offset", 4), ("v_offset", -8),
                         ("pos_offset", -1), ("pos_offset", (1 << 24) - 3)):
        c = w.chunks.copy()
        c[0][field] = value
        assert code(c) == ops.LAZY_EDATA, (field, value)
    same = next(i for i in range(1, w.chunks.size) if w.chunks[i]["k_offset"] == w.chunks[0]["k_offset"])
    for field, delta in (("k_offset", 8), ("v_offset", 64), ("k_stride", 1)):  # overlaps that no single gradient fits
        c = w.chunks.copy()
        c[same][field] += delta
        assert code(c) == ops.LAZY_EDATA, (field, delta)
    assert code(q_pos0=w.q_pos0 - 1000) == ops.LAZY_EDATA
    assert code(q_start=w.q_start + 1) == ops.LAZY_EDATA
    assert code(q_start=w.q_start[::-1].copy() - w.q_start[-1]) == ops.LAZY_EDATA
    assert code(chunk_start=w.chunk_start[::-1].copy()) in (ops.LAZY_EDATA,)
    assert code(cfg=dataclasses.replace(cfg, head_dim=96)) == ops.LAZY_EUNSUPPORTED
    assert code(cfg=dataclasses.replace(cfg, num_q_heads=0)) == ops.LAZY_EINVAL
    wide = dataclasses.replace(cfg, num_q_heads=1 << 16, num_kv_heads=1)
    assert code(cfg=wide) == ops.LAZY_EUNSUPPORTED
    # zero-length records are passed over
    c = w.chunks.copy()
    c[0]["len"] = 0
    ops.backward_plan(cfg, w.q_start, w.q_pos0, c, w.chunk_start)
    # a capacity that is too small still tells the size
    p, info = cfg.c(), ops.BackwardInfo()
    buf = np.zeros(8, np.uint8)
    args = [w.q_start.ctypes.data, w.q_pos0.ctypes.data, w.chunks.ctypes.data, w.chunk_start.ctypes.data]
    assert ops.lib().lazy_attn_backward_plan(ctypes.byref(p), *args, w.batch, buf.ctypes.data, 8,
                                             ctypes.byref(info)) == ops.LAZY_EINVAL
    assert info.plan_bytes > 8 and not buf.any()
    for hole in range(2):
        bad = list(args)
        bad[2 * hole if hole else 0] = None
        assert ops.lib().lazy_attn_backward_plan(ctypes.byref(p), *bad, w.batch, None, 0,
                                                 ctypes.byref(info)) == ops.LAZY_EINVAL


def test_backward_call_refusals_without_a_gpu():
    """Checks that come before any launch: a null or foreign plan record, null tensors, a missing workspace."""
    w = W.tiny_rag_prefill(0)
    cfg, plan = make_plan(w)
    fn, p = ops.lib().lazy_attn_prefill_backward, cfg.c()
    one = 4096  # a non-null, aligned address that is never read: every call below is refused

    def call(info=plan.info, q=one, table=one, plan_ptr=one, dq=one, ws=one, nbytes=1 << 40, total_q=w.total_q, p=p):
        return fn(ctypes.byref(p), q, table, table, one, one, table, table, w.batch, total_q, one, one, one, None,
                  plan_ptr, ctypes.byref(info) if info is not None else None, dq, one, one, ws, nbytes, None)

    need = ops.backward_workspace_size(cfg, plan)
    assert need > 0
    assert call(info=None) == ops.LAZY_EINVAL
    assert call(total_q=w.total_q + 1) == ops.LAZY_EINVAL
    for field in ("batch", "num_q_heads", "num_kv_heads", "head_dim", "causal", "key_positions", "plan_bytes",
                  "num_tiles"):
        other = ops.BackwardInfo.from_buffer_copy(plan.info)
        setattr(other, field, getattr(other, field) + 1)
        assert call(info=other) == ops.LAZY_EINVAL, field
    assert call(q=None) == ops.LAZY_EINVAL and call(table=None) == ops.LAZY_EINVAL and call(dq=None) == ops.LAZY_EINVAL
    assert call(plan_ptr=None) == ops.LAZY_EINVAL and call(plan_ptr=one + 8) == ops.LAZY_EINVAL
    assert call(ws=None) == ops.LAZY_EWORKSPACE and call(nbytes=need - 1) == ops.LAZY_EWORKSPACE
    assert call(ws=one + 4) == ops.LAZY_EWORKSPACE
    assert call(p=dataclasses.replace(cfg, head_dim=32).c()) == ops.LAZY_EUNSUPPORTED
    with pytest.raises(ValueError):  # host tensors
        t = torch.zeros(1, dtype=torch.bfloat16)
        ops.prefill_backward(cfg, t, t, t, t, t, t, t, t, t, t, plan)


# ---------------------------------------------------------------------------------------------------------------
# CPU: the oracle against differences of the forward oracle
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("pairing,keys,causal", [("half", "nope", True), ("interleaved", "local", True),
                                                 ("alibi", "nope", False)])
def test_oracle_against_differences(pairing, keys, causal):
    w = shared(11, 4, 2, 64, [9, 5], [4, 2], reqs=2, causal=causal, twice=True, slack=None)
    rng = np.random.default_rng(0)
    dout, dlse = rng.standard_normal(w.q.shape), rng.standard_normal(w.q.shape[:2])
    q, pool = w.q.astype(np.float64) * 0.5, w.pool.astype(np.float64) * 0.5
    args = (w.chunks, w.chunk_start, 4, 2, 64, w.rope_base)
    kw = dict(pairing=pairing, key_positions=keys)

    def loss(q, pool):
        o, l = O.lazy_attention(q, w.q_start, w.q_pos0, pool, pool, *args, causal, **kw)
        return (o * dout).sum() + (l * dlse).sum()

    out, lse = O.lazy_attention(q, w.q_start, w.q_pos0, pool, pool, *args, causal, **kw)
    (dq, dk, dv), _ = GO.lazy_backward(q, w.q_start, w.q_pos0, pool, pool, *args, causal, out, lse, dout, dlse, **kw)
    dpool = dk + dv  # K and V ranges of the one pool are disjoint
    h = 1e-5
    for flat, grad, which in ((q.reshape(-1), dq.reshape(-1), 0), (pool, dpool, 1)):
        for i in rng.choice(flat.size, 25, replace=False):
            old = flat[i]
            flat[i] = old + h
            up = loss(q, pool)
            flat[i] = old - h
            down = loss(q, pool)
            flat[i] = old
            # central differences: error of order h^2 times a third derivative of order 10, and rounding 1e-15 / h
            assert abs((up - down) / (2 * h) - grad[i]) < 1e-7, (which, i)


# ---------------------------------------------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ops.lib()
    torch.cuda.init()


def oracle_kw(ckw):
    style = {ops.ROPE_HALF: "half", ops.ROPE_INTERLEAVED: "interleaved", ops.ALIBI: "alibi"}[ckw.get("rope_style", 0)]
    kw = dict(pairing=style, key_positions="local" if ckw.get("key_positions") else "nope")
    if "softmax_scale" in ckw:
        kw["softmax_scale"] = ckw["softmax_scale"]
    if "q_prerotated" in ckw:
        kw["q_prerotated"] = ckw["q_prerotated"]
    if ckw.get("inv_freq") is not None:
        kw["inv_freq"] = ckw["inv_freq"].cpu().numpy()
    return kw


def close(got, ref, bound, tag):
    got = got.float().cpu().numpy().astype(np.float64).reshape(ref.shape)
    assert np.isfinite(got).all(), tag
    err = np.abs(got - ref)
    worst = (err / bound).max() if err.size else 0.0
    norm = np.linalg.norm(ref)
    rel = np.linalg.norm(got - ref) / norm if norm > 0 else np.abs(got).max(initial=0.0)
    print(f"{tag}: largest error over its bound {worst:.3f}, relative 2-norm {rel:.5f}", flush=True)
    assert worst <= 1.0, f"{tag}: an element is {worst} times its bound off"
    assert rel <= REL, f"{tag}: relative 2-norm {rel}"


def run(w, ckw, dlse=False, seed=0, fill=3.0):
    """Forward and backward on the GPU; (dq, dk, dv) tensors and the oracle's gradients and bounds."""
    cfg = ops.config_of(w, **ckw)
    dw = ops.upload(w)
    out, lse = ops.run_lazy(dw, cfg)
    gen = torch.Generator("cuda").manual_seed(seed)
    dout = torch.empty_like(dw.q).normal_(generator=gen)
    dl = torch.empty_like(lse).normal_(generator=gen) if dlse else None
    plan = ops.upload_backward_plan(ops.backward_plan(cfg, w.q_start, w.q_pos0, w.chunks, w.chunk_start))
    dk, dv = (torch.full_like(dw.pool, fill) for _ in range(2))
    dq = torch.full_like(dw.q, float("nan"))
    args = (cfg, dw.q, dw.q_start, dw.q_pos0, dw.pool, dw.pool, dw.chunks, dw.chunk_start, out, lse, dout, plan)
    ops.prefill_backward(*args, dlse=dl, dq=dq, dk_pool=dk, dv_pool=dv)
    torch.cuda.synchronize()
    f64 = lambda t: t.float().cpu().numpy().astype(np.float64)  # noqa: E731
    ref, bound = GO.lazy_backward(w.q, w.q_start, w.q_pos0, w.pool, w.pool, w.chunks, w.chunk_start, w.num_q_heads,
                                  w.num_kv_heads, w.head_dim, w.rope_base, w.causal, f64(out), f64(lse), f64(dout),
                                  f64(dl) if dlse else None, **oracle_kw(ckw))
    return args, dl, (dq, dk, dv), ref, bound


def cover_masks(w):
    ck, cv = np.zeros(w.pool.size, bool), np.zeros(w.pool.size, bool)
    for c in w.chunks:
        for g in range(w.num_kv_heads):
            for m, off, st in ((ck, "k_offset", "k_stride"), (cv, "v_offset", "v_stride")):
                at = int(c[off]) + g * int(c[st]) * w.head_dim
                m[at:at + int(c["len"]) * w.head_dim] = True
    return ck, cv


def check(w, ckw, tag, dlse=False, fill=3.0):
    args, dl, got, ref, bound = run(w, ckw, dlse=dlse, fill=fill)
    close(got[0], ref[0], bound[0], f"{tag} dq")
    for t, r, b, m, name in zip(got[1:], ref[1:], bound[1:], cover_masks(w), ("dk", "dv")):
        flat = t.float().cpu().numpy().reshape(-1)
        assert (flat[~m] == fill).all(), f"{tag}: {name} written outside the records"
        close(t.reshape(-1)[torch.from_numpy(m).to(t.device)], r[m], b[m], f"{tag} {name}")
    return args, dl, got


CASES = {
    "tiny": (lambda: W.tiny_rag_prefill(0, slack_fill=float("nan")), {}),
    "one query, one key": (lambda: W.custom(1, 2, 1, 64, 1e4, [dict(chunks=[(1, 0)], q_len=1, q_pos0=0)]), {}),
    "d128 shared": (lambda: shared(20, 8, 2, 128, [130, 64, 33], [17, 40, 3]), {}),
    "d64 shared, group 7": (lambda: shared(21, 14, 2, 64, [129, 63], [11, 50]), {}),
    "d128 group 1": (lambda: shared(22, 3, 3, 128, [100, 20], [33, 64]), {}),
    "d128 group 16": (lambda: shared(23, 16, 1, 128, [200], [9, 40]), {}),
    "interleaved": (lambda: shared(24, 4, 2, 128, [70, 90], [20, 31]), dict(rope_style=ops.ROPE_INTERLEAVED)),
    "interleaved local d64": (lambda: shared(25, 4, 1, 64, [70, 90], [20, 31], twice=True),
                              dict(rope_style=ops.ROPE_INTERLEAVED, key_positions=ops.KEYS_LOCAL)),
    "local": (lambda: shared(26, 8, 2, 128, [70, 90, 128], [20, 31]), dict(key_positions=ops.KEYS_LOCAL)),
    "alibi": (lambda: shared(27, 8, 2, 128, [70, 90], [20, 31]), dict(rope_style=ops.ALIBI)),
    "alibi d64 not causal": (lambda: shared(28, 6, 2, 64, [70, 90], [20, 31], causal=False), dict(rope_style=ops.ALIBI)),
    "not causal": (lambda: shared(29, 8, 2, 128, [70, 90], [20, 31], causal=False), {}),
    "prerotated": (lambda: shared(30, 8, 2, 128, [70, 90], [20, 31]), dict(q_prerotated=True)),
    "scale": (lambda: shared(31, 8, 2, 64, [70, 90], [20, 31]), dict(softmax_scale=0.05)),
    "same chunk twice": (lambda: shared(32, 8, 2, 128, [70, 90], [20, 31], twice=True), {}),
    "rows that see nothing": (lambda: W.custom(33, 4, 2, 128, 1e4, [
        dict(chunks=[("a", 100, 37)], q_len=90, q_pos0=3), dict(chunks=[("a", 100, 0), ("b", 65, 100)], q_len=40, q_pos0=20),
        dict(chunks=[], q_len=5, q_pos0=0), dict(chunks=[("b", 65, 3)], q_len=0, q_pos0=9)], slack_fill=float("nan")), {}),
    "parts of a tile": (lambda: shared(34, 4, 1, 128, [64], [300, 301], reqs=5), {}),
    "parts of a tile, interleaved d64": (lambda: shared(35, 4, 1, 64, [64], [300, 301], reqs=5),
                                         dict(rope_style=ops.ROPE_INTERLEAVED)),
    "own tokens": (lambda: W.custom(36, 8, 2, 128, 1e4, [dict(chunks=[(517, 0)], q_len=517, q_pos0=0)]), {}),
    "sub-records": (lambda: sub_records(shared(37, 4, 2, 128, [150, 30], [26], reqs=3), 150, [(10, 77), (64, 20)]), {}),
    "paged": (lambda: W.paginate(shared(38, 8, 2, 128, [170, 45], [38, 3]), 32), {}),
    "far positions": (lambda: W.custom(39, 4, 2, 128, 5e5, [
        dict(chunks=[("a", 90, (1 << 24) - 200)], q_len=30, q_pos0=(1 << 24) - 110),
        dict(chunks=[("a", 90, 5)], q_len=30, q_pos0=95)]), {}),
    "many keys, splits": (lambda: shared(40, 4, 1, 128, [4000], [20], reqs=1), {}),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_gradients(gpu, name):
    make, ckw = CASES[name]
    check(make(), ckw, name)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["d128 shared", "d64 shared, group 7", "alibi", "rows that see nothing"])
def test_gradients_of_the_log_sum_exps(gpu, name):
    make, ckw = CASES[name]
    check(make(), ckw, name + " dlse", dlse=True)


@pytest.mark.gpu
def test_frequency_and_slope_tables(gpu):
    w = shared(41, 8, 2, 128, [70, 90], [20, 31])
    table = torch.from_numpy((0.5 * 1e4 ** (-2.0 * np.arange(64) / 128)).astype(np.float32)).cuda()
    check(w, dict(inv_freq=table), "frequency table")
    slopes = torch.linspace(0.01, 0.4, 8).cuda()
    check(w, dict(rope_style=ops.ALIBI, inv_freq=slopes), "slope table")


@pytest.mark.gpu
def test_equal_calls_give_equal_bits_and_pools_may_be_one(gpu):
    w = shared(42, 8, 2, 128, [130, 64, 33], [17, 40, 3])
    args, _, first = check(w, {}, "first")
    dq, dk, dv = ops.prefill_backward(*args)  # gradients allocated here; one pool for both
    assert dk.data_ptr() == dv.data_ptr()
    ck, cv = (torch.from_numpy(m).cuda() for m in cover_masks(w))
    assert torch.equal(dq, first[0])
    assert torch.equal(dk.reshape(-1)[ck], first[1].reshape(-1)[ck])
    assert torch.equal(dv.reshape(-1)[cv], first[2].reshape(-1)[cv])
    assert not dk.reshape(-1)[~(ck | cv)].any()


@pytest.mark.gpu
def test_backward_in_a_graph_and_on_another_stream(gpu):
    w = shared(43, 8, 2, 128, [130, 64, 33], [17, 40, 3], slack=None)
    args, _, want = run(w, {})[:3]
    nbytes = ops.backward_workspace_size(args[0], args[-1])
    bufs = [torch.empty_like(want[0]), torch.zeros_like(want[1]), torch.zeros_like(want[2]),
            torch.empty(nbytes, dtype=torch.uint8, device="cuda")]
    side = torch.cuda.Stream()

    def call():
        ops.prefill_backward(*args, dq=bufs[0], dk_pool=bufs[1], dv_pool=bufs[2], workspace=bufs[3])

    ck, cv = (torch.from_numpy(m).cuda() for m in cover_masks(w))

    def same():
        return torch.equal(bufs[0], want[0]) and all(
            torch.equal(b.reshape(-1)[m], t.reshape(-1)[m]) for b, t, m in zip(bufs[1:3], want[1:], (ck, cv)))

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        for b in bufs:
            b.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same()
        torch.mm(torch.ones(64, 64, device="cuda"), torch.ones(64, 64, device="cuda"))


# ---------------------------------------------------------------------------------------------------------------
# Calls at the edges
# ---------------------------------------------------------------------------------------------------------------
def test_refusals_of_plans_and_pools_without_a_gpu():
    """More work items than a launch holds, offsets whose sums would overflow, gradients over what they are made from."""
    heads = 60000
    cfg = ops.Config(heads, heads, 64, 1e4)
    with pytest.raises(ops.LazyAttnError) as e:
        ops.backward_plan(cfg, np.arange(151, dtype=np.int32), np.zeros(150, np.int32), np.zeros(0, W.CHUNK_DTYPE),
                          np.zeros(151, np.int32))
    assert e.value.code == ops.LAZY_EUNSUPPORTED
    w = W.tiny_rag_prefill(0)
    cfg, plan = make_plan(w)
    for field in ("k_offset", "v_offset"):
        c = w.chunks.copy()
        c[0][field] = (1 << 63) - 8
        with pytest.raises(ops.LazyAttnError) as e:
            ops.backward_plan(cfg, w.q_start, w.q_pos0, c, w.chunk_start)
        assert e.value.code == ops.LAZY_EDATA
    p, one = cfg.c(), 4096  # addresses that are never read
    for k, v, dk, dv in ((1, 2, 1, 3), (1, 2, 2, 3), (1, 2, 3, 1), (1, 2, 3, 2), (1, 1, 1, 1)):
        assert ops.lib().lazy_attn_prefill_backward(
            ctypes.byref(p), one, one, one, k * one, v * one, one, one, w.batch, w.total_q, one, one, one, None, one,
            ctypes.byref(plan.info), one, dk * one, dv * one, one, 1 << 40, None) == ops.LAZY_EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("d,style", [(64, ops.ROPE_HALF), (128, ops.ROPE_INTERLEAVED), (128, ops.ALIBI)])
def test_rows_that_see_nothing_may_hold_anything(gpu, d, style):
    """Queries, outputs and their gradients of rows with a log-sum-exp of -inf are not finite: no other gradient changes,
    and theirs is zero."""
    w = W.custom(44, 4, 2, d, 1e4, [dict(chunks=[("a", 100, 37)], q_len=90, q_pos0=3),
                                    dict(chunks=[("a", 100, 0), ("b", 65, 100)], q_len=40, q_pos0=20)])
    args, dl, want = run(w, dict(rope_style=style), dlse=True)[:3]
    cfg, q, q_start, q_pos0, kp, vp, chunks, chunk_start, out, lse, dout, plan = args
    dead = torch.isneginf(lse)
    assert dead.any() and not dead.all()
    q, out, dout, dl = q.clone(), out.clone(), dout.clone(), dl.clone()
    q[dead], out[dead], dout[dead], dl[dead] = float("nan"), float("inf"), float("nan"), float("inf")
    got = [torch.full_like(t, 3.0) for t in want]
    ops.prefill_backward(cfg, q, q_start, q_pos0, kp, vp, chunks, chunk_start, out, lse, dout, plan, dlse=dl, dq=got[0],
                         dk_pool=got[1], dv_pool=got[2])
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert not got[0][dead].any()


@pytest.mark.gpu
def test_memory_allocated_for_another_stream(gpu):
    """Gradients and workspace that the call allocates belong to the stream it runs on."""
    w = shared(45, 8, 2, 128, [130, 64, 33], [17, 40, 3], slack=None)
    args, _, want = run(w, {})[:3]
    ck, cv = (torch.from_numpy(m).cuda() for m in cover_masks(w))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        dq, dk, dv = ops.prefill_backward(*args, stream=stream)
        side.synchronize()
        assert torch.equal(dq, want[0])
        assert torch.equal(dk.reshape(-1)[ck], want[1].reshape(-1)[ck])
        assert torch.equal(dv.reshape(-1)[cv], want[2].reshape(-1)[cv])
        assert not dk.reshape(-1)[~(ck | cv)].any()


# Work beyond what one launch takes for all three gradients: 128-row and 256-row items of head_dim 128, and head_dim 64.
LARGE = {
    "d128, 128 rows": (lambda: shared(46, 32, 32, 128, [1030, 700, 517], [20, 33], reqs=2), {}),
    "d128, 128 rows, interleaved local": (lambda: shared(47, 32, 32, 128, [1030, 700, 517], [20, 33], reqs=2),
                                          dict(rope_style=ops.ROPE_INTERLEAVED, key_positions=ops.KEYS_LOCAL)),
    "d128, 128 rows, alibi": (lambda: shared(48, 32, 32, 128, [1030, 700, 517], [20, 33], reqs=2),
                              dict(rope_style=ops.ALIBI)),
    "d128, 256 rows": (lambda: shared(49, 64, 16, 128, [1030, 700, 517, 2000], [128, 60], reqs=2), {}),
    "d128, 256 rows, interleaved": (lambda: shared(50, 64, 16, 128, [1030, 700, 517, 2000], [128, 60], reqs=2),
                                    dict(rope_style=ops.ROPE_INTERLEAVED)),
    "d64": (lambda: shared(51, 64, 64, 64, [1030, 700, 517, 500], [20, 33], reqs=2), {}),
    "d64, interleaved local": (lambda: shared(52, 64, 64, 64, [1030, 700, 517, 500], [20, 33], reqs=2),
                               dict(rope_style=ops.ROPE_INTERLEAVED, key_positions=ops.KEYS_LOCAL)),
    "d64, alibi": (lambda: shared(53, 64, 64, 64, [1030, 700, 517, 500], [20, 33], reqs=2), dict(rope_style=ops.ALIBI)),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", LARGE)
def test_gradients_in_separate_launches(gpu, name):
    make, ckw = LARGE[name]
    w = make()
    info = make_plan(w, **ckw)[1].info
    tiles, items = info.num_tiles * w.num_kv_heads, info.num_row_items * w.num_kv_heads
    assert tiles > 1280 if w.head_dim == 64 else tiles + items > 512
    assert info.row_blocks == (2 if "256 rows" in name else 1)
    check(w, ckw, name)
