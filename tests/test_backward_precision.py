"""Gradients of concentrated attention.  Where few rows see many keys and a handful of keys hold nearly all of a row's
weight, the elements of a gradient are much smaller than the terms they are summed from and much larger than the
tensor's root mean square: an error of half a bf16 step in the operands of a product (queries, keys, P, dS) shows as a
multiple of both.  Every element has to be right to half a step of its own plus what two-part operands and fp32 sums
allow (``operand`` in ``oracle/gradient_oracle.py``).

Over a tensor: a rounding to bf16 has a root mean square of at most 2^-8 / sqrt(3) = 0.00226 relative, the result's own;
operands add 2^-15 at most.  0.0023 of the 2-norm is allowed.
"""
import numpy as np
import pytest
import torch

from oracle import gradient_oracle as GO
from paper_2606_04302_amd import ops
from paper_2606_04302_amd import workloads as W
from tests.test_backward import arrays, cover_masks, make_plan, oracle_kw, shared

REL = 0.0023
OPERAND = 2.0 ** -15


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ops.lib()
    torch.cuda.init()


def louder(w, factor):
    """The workload with its queries multiplied: sharper scores."""
    w.q[...] = (w.q.astype(np.float32) * factor).astype(w.q.dtype)
    return w


def long_context(seed, hq, hkv, d, keys, rows, gap=0):
    """Some rows and their own keys behind many keys; with a gap no keys of their own, far from the others."""
    own = [] if gap else [(rows, keys)]
    return W.custom(seed, hq, hkv, d, 1.0e4, [dict(chunks=[("a", keys, 0), *own], q_len=rows, q_pos0=keys + gap)])


def gradients(w, ckw, dlse, seed=0, fill=3.0):
    """(dq, dk, dv) on the GPU, the oracle's gradients and their bounds."""
    cfg = ops.config_of(w, **ckw)
    dw = ops.upload(w)
    out, lse = ops.run_lazy(dw, cfg)
    gen = torch.Generator("cuda").manual_seed(seed)
    dout = torch.empty_like(dw.q).normal_(generator=gen)
    dl = torch.empty_like(lse).normal_(generator=gen) if dlse else None
    plan = ops.upload_backward_plan(ops.backward_plan(cfg, w.q_start, w.q_pos0, w.chunks, w.chunk_start))
    got = [torch.full_like(t, v) for t, v in ((dw.q, float("nan")), (dw.pool, fill), (dw.pool, fill))]
    ops.prefill_backward(cfg, dw.q, dw.q_start, dw.q_pos0, dw.pool, dw.pool, dw.chunks, dw.chunk_start, out, lse, dout,
                         plan, dlse=dl, dq=got[0], dk_pool=got[1], dv_pool=got[2])
    torch.cuda.synchronize()
    f64 = lambda t: t.float().cpu().numpy().astype(np.float64)  # noqa: E731
    ref, bound = GO.lazy_backward(w.q, w.q_start, w.q_pos0, w.pool, w.pool, w.chunks, w.chunk_start, w.num_q_heads,
                                  w.num_kv_heads, w.head_dim, w.rope_base, w.causal, f64(out), f64(lse), f64(dout),
                                  f64(dl) if dlse else None, operand=OPERAND, **oracle_kw(ckw))
    return [f64(t) for t in got], ref, bound


def check(w, ckw, tag, dlse=False, fill=3.0):
    got, ref, bound = gradients(w, ckw, dlse, fill=fill)
    masks = (np.ones(ref[0].shape, bool), *cover_masks(w))
    bad = []
    for name, x, r, b, m in zip(("dq", "dk", "dv"), got, ref, bound, masks):
        x = x.reshape(r.shape)
        assert name == "dq" or (x[~m] == fill).all(), f"{tag}: {name} written outside the records"
        x, r, b = x[m], r[m], b[m]
        assert np.isfinite(x).all(), f"{tag} {name}"
        err = np.abs(x - r)
        rms = np.sqrt(np.mean(r * r))
        worst, rel = (err / b).max(), np.linalg.norm(x - r) / np.linalg.norm(r)
        print(f"{tag} {name}: largest error {(err / np.maximum(np.abs(r), rms)).max():.5f} of max(element, rms), "
              f"{worst:.3f} of its bound; 2-norm {rel:.5f}", flush=True)
        if worst > 1.0 or rel > REL:
            bad.append((name, worst, rel))
    assert not bad, f"{tag}: {bad}"


IL, LOCAL, ALIBI = (dict(rope_style=ops.ROPE_INTERLEAVED), dict(key_positions=ops.KEYS_LOCAL),
                    dict(rope_style=ops.ALIBI))
CASES = {
    "alibi, 3 rows, 28000 keys": (lambda: long_context(60, 32, 8, 128, 28000, 3), ALIBI),
    "alibi d64, one row": (lambda: long_context(61, 8, 1, 64, 5000, 1), ALIBI),
    "alibi, far from its keys": (lambda: long_context(62, 8, 2, 128, 500, 4, gap=20000), ALIBI),
    "alibi, long question": (lambda: long_context(63, 8, 2, 128, 1500, 200), ALIBI),
    "peaked": (lambda: louder(long_context(64, 8, 2, 128, 3000, 3), 4), {}),
    "peaked d64": (lambda: louder(long_context(65, 8, 2, 64, 3000, 3), 4), {}),
    "peaked, interleaved": (lambda: louder(long_context(66, 4, 2, 128, 3000, 7), 4), IL),
    "peaked, interleaved local d64": (lambda: louder(long_context(67, 4, 2, 64, 3000, 7), 4), dict(IL, **LOCAL)),
    "peaked, local": (lambda: louder(long_context(68, 4, 2, 128, 3000, 2), 4), LOCAL),
    "peaked, prerotated": (lambda: louder(long_context(69, 8, 2, 128, 3000, 3), 4), dict(q_prerotated=True)),
    "peaked, shared chunks": (lambda: louder(shared(70, 8, 2, 128, [130, 64, 33, 700], [17, 40, 3]), 4), {}),
    "peaked, shared chunks d64": (lambda: louder(shared(71, 8, 2, 64, [130, 64, 33, 700], [17, 40, 3]), 4), {}),
    "peaked, parts": (lambda: louder(shared(72, 4, 1, 128, [64], [300, 301], reqs=5), 4), {}),
    "peaked, many tiles": (lambda: louder(shared(73, 32, 32, 128, [1030, 700, 517], [20, 33], reqs=2), 4), {}),
    "peaked, 256 rows": (lambda: louder(shared(74, 64, 16, 128, [1030, 700, 517, 2000], [128, 60], reqs=2), 4), {}),
    "peaked, many tiles d64": (lambda: louder(shared(75, 64, 64, 64, [1030, 700, 517, 500], [20, 33], reqs=2), 4), {}),
    "flat": (lambda: shared(76, 8, 2, 128, [1300, 640, 33], [64]), {}),
    "flat d64": (lambda: shared(77, 8, 2, 64, [1300, 640, 33], [64]), {}),
    "flat, not causal": (lambda: shared(78, 8, 2, 128, [130, 64], [64], causal=False), IL),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_gradients_to_half_a_step(gpu, name):
    make, ckw = CASES[name]
    check(make(), ckw, name, dlse="shared" in name or "far" in name)


def uneven(seed, hq, hkv, d, keys, rows):
    """One request with many keys, others with few."""
    return W.custom(seed, hq, hkv, d, 1.0e4, [dict(chunks=[(n, 0), (rows, n)], q_len=rows, q_pos0=n) for n in keys])


# Plans of each kind: (workload, options, rows of a workgroup, key splits of the requests).
PLANS = {
    "one split and several": (lambda: uneven(80, 8, 2, 128, [4000, 50, 700], 24), {}, 128, "both"),
    "one split and several, interleaved d64": (lambda: uneven(81, 8, 2, 64, [4000, 50, 700], 24), IL, 128, "both"),
    "256 rows, one split": (lambda: shared(82, 64, 16, 128, [180, 60], [64], reqs=40), {}, 256, "one"),
    "256 rows, one split, interleaved local": (lambda: shared(83, 64, 16, 128, [180, 60], [64], reqs=40),
                                               dict(IL, **LOCAL), 256, "one"),
    "256 rows, one split, alibi": (lambda: shared(84, 64, 16, 128, [180, 60], [64], reqs=40), ALIBI, 256, "one"),
    "256 rows, one split and several": (lambda: uneven(85, 64, 16, 128, [6000, 50] + [300] * 10, 64), {}, 256, "both"),
    "d64, many rows, one split": (lambda: shared(86, 32, 32, 64, [500, 130], [150], reqs=12), {}, 128, "one"),
    "d64 document": (lambda: W.custom(87, 4, 1, 64, 1.0e4, [dict(chunks=[(3001, 0)], q_len=3001, q_pos0=0)]), {}, 128,
                     None),
}


def splits_of(plan, w):
    rows = arrays(plan)[1]
    return {int(rows["splits"][rows["request"] == r][0]) for r in range(w.batch)}


@pytest.mark.parametrize("name", PLANS)
def test_plans_are_of_their_kind(name):
    make, ckw, rows, kind = PLANS[name]
    w = make()
    plan = make_plan(w, **ckw)[1]
    assert 128 * plan.info.row_blocks == rows
    got = splits_of(plan, w)
    assert kind is None or (got == {1} if kind == "one" else 1 in got and max(got) > 1), got


@pytest.mark.gpu
@pytest.mark.parametrize("name", PLANS)
def test_gradients_of_every_kind_of_plan(gpu, name):
    make, ckw, _, _ = PLANS[name]
    check(make(), ckw, name, dlse="interleaved" in name)


@pytest.mark.parametrize("room", [None, 0, 100])
@pytest.mark.parametrize("name", PLANS)
def test_plans_are_made_once(monkeypatch, name, room):
    """One run of the planner where the room guessed for the plan is enough, a second one where it is not; equal bytes."""
    make, ckw, _, _ = PLANS[name]
    w = make()
    library, codes = ops.lib(), []

    class Counting:
        def __getattr__(self, fn):
            real = getattr(library, fn)
            if fn != "lazy_attn_backward_plan":
                return real

            def call(*args):
                codes.append(real(*args))
                return codes[-1]
            return call

    want = make_plan(w, **ckw)[1]
    monkeypatch.setattr(ops, "lib", lambda: Counting())
    if room is not None:
        monkeypatch.setattr(ops, "_plan_room", lambda *a: room)
    plan = make_plan(w, **ckw)[1]
    assert codes == ([ops.LAZY_OK] if room is None else [ops.LAZY_EINVAL, ops.LAZY_OK])
    assert plan.data.size == plan.info.plan_bytes and np.array_equal(plan.data, want.data)


@pytest.mark.gpu
@pytest.mark.parametrize("d,ckw", [(64, {}), (128, IL), (128, ALIBI), (128, LOCAL)])
def test_products_of_hidden_pairs_may_overflow(gpu, d, ckw):
    """Large finite values of keys that a row does not see, times large finite gradients, are no number: nothing of them
    reaches a gradient."""
    w = W.custom(90, 4, 2, d, 1.0e4, [dict(chunks=[(90, 60)], q_len=30, q_pos0=90)])  # keys 60 to 89 lie past every row
    cfg, dw = ops.config_of(w, **ckw), ops.upload(w)
    out, lse = ops.run_lazy(dw, cfg)
    dout = torch.randn(w.q.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(torch.bfloat16) * 1e30
    plan = ops.upload_backward_plan(ops.backward_plan(cfg, w.q_start, w.q_pos0, w.chunks, w.chunk_start))

    def rows(pool, which):
        at, st = int(w.chunks[0][which + "_offset"]), int(w.chunks[0][which + "_stride"])
        return pool.view(-1)[at:at + 2 * st * d].view(2, st, d)

    got = []
    for large in (False, True):
        pool = dw.pool.clone()
        if large:
            rows(pool, "v")[:, 60:90] = 3.0e38
        got.append(ops.prefill_backward(cfg, dw.q, dw.q_start, dw.q_pos0, pool, pool.clone(), dw.chunks, dw.chunk_start,
                                        out, lse, dout, plan, dk_pool=torch.zeros_like(pool),
                                        dv_pool=torch.zeros_like(pool)))
    for a, b in zip(*got):
        assert torch.isfinite(b).all() and b.any() and torch.equal(a, b)
    for pool, which in ((got[1][1], "k"), (got[1][2], "v")):
        assert rows(pool, which)[:, :60].any() and not rows(pool, which)[:, 60:90].any()
