"""The calls around the attention itself: its gradients, and eviction from a cache by accumulated attention weight.

A case is one call, by its ``kind``:
  "backward"         ``ops.prefill_backward``: gradients of the queries and of the stored keys and values
  "prefill_weights"  ``ops.prefill_key_weights``: the attention weight that a prompt gave to each key
  "decode_weights"   ``ops.decode_key_weights``: the weight that one new token gives, added to the running sums
  "select"           ``ops.cache_select``: the heaviest keys of each request within its budget
  "compact"          ``ops.cache_compact``: the kept keys gathered into a record of the request's own

Other fields of a case:
  batch, hq, hkv, d, base   requests, query heads, KV heads, head dimension, RoPE base
  style     "half", "interleaved" (rotary pairing) or "alibi"
  keys      "nope" (keys stored unrotated) or "local" (keys stored at their local positions)
  prerot    True: queries arrive rotated
  causal    False: every query sees every key of its request
  prefix    keys of a prefix that every request shares (0: none)
  n_lo, n_hi, len_lo, len_hi   chunks per request and keys per chunk, uniform in the range
  pool      distinct stored chunks that the requests pick from without repetition; 0: private chunks
  q_lo, q_hi   question tokens (or tokens generated so far, of which the last one is the query), uniform in the range
  block     tokens per block of a paged store (0: chunks are contiguous)
  dlse      True: the loss depends on the log-sum-exps too
  budget, sink, recent   keys kept of a request, protected first and last ones
  rotate    True: kept keys are rotated to their positions in the copy
  decay     what the running sums are multiplied by before a token's weights are added
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_CHUNK = np.dtype([("k_offset", "<i8"), ("v_offset", "<i8"), ("len", "<i4"), ("pos_offset", "<i4"),
                   ("k_stride", "<i4"), ("v_stride", "<i4")])

_DEFAULTS = dict(batch=1, hq=32, hkv=8, d=128, base=5.0e5, style="half", keys="nope", prerot=False, causal=True,
                 prefix=0, n_lo=1, n_hi=1, len_lo=64, len_hi=64, pool=0, q_lo=1, q_hi=1, block=0, dlse=False,
                 budget=0, sink=0, recent=0, rotate=False, decay=1.0)


def _case(kind, **kw):
    assert set(kw) <= set(_DEFAULTS) | {"name"}
    return dict(_DEFAULTS, kind=kind, **kw)


def listed():
    return [
        # The smallest backward pass: a toy head layout, 272 keys, 16 question tokens.  Launch latency.
        _case("backward", name="tiny_backward", hq=2, hkv=1, d=64, base=1.0e4, n_lo=4, n_hi=4, len_lo=64, len_hi=64,
              q_lo=16, q_hi=16),
        # A training step's attention over retrieved chunks: eight requests that share a prefix and ten 512-key
        # chunks each from a pool of 64, 64 question tokens.
        _case("backward", name="rag_backward", batch=8, prefix=128, n_lo=10, n_hi=10, len_lo=512, len_hi=512, pool=64,
              q_lo=64, q_hi=64),
        # Whole documents as their own queries: three sequences of odd length, 64-wide interleaved heads, and a loss
        # that reads the log-sum-exps (partial attention that is merged later).
        _case("backward", name="document_backward", batch=3, hq=32, hkv=8, d=64, style="interleaved", n_lo=1, n_hi=1,
              len_lo=33, len_hi=33, q_lo=1501, q_hi=2048, dlse=True),
        # Ragged batch, the largest: skewed lengths, chunks of 128 to 2048 keys from a pool of 200, questions of 32 to
        # 256 tokens, seven query heads per KV head.
        _case("backward", name="varlen_backward", batch=16, hq=28, hkv=4, base=1.0e6, n_lo=8, n_hi=24, len_lo=128,
              len_hi=2048, pool=200, q_lo=32, q_hi=256),
        # What a question gave to each key of the retrieved chunks, to decide which of them stay.
        _case("prefill_weights", name="rag_prefill_weights", batch=8, prefix=128, n_lo=10, n_hi=10, len_lo=512,
              len_hi=512, pool=64, q_lo=64, q_hi=64),
        # The same for many-shot in-context learning: four requests, 128 exemplars each in their own order.
        _case("prefill_weights", name="icl_prefill_weights", batch=4, n_lo=128, n_hi=128, len_lo=256, len_hi=256,
              pool=128, q_lo=256, q_hi=256),
        # One user's decode step over a paged store: latency.
        _case("decode_weights", name="chat_decode_weights", keys="local", n_lo=5, n_hi=5, len_lo=301, len_hi=811,
              q_lo=37, q_hi=37, block=64),
        # A decode step of 64 requests, sixteen 1024-key chunks each from a pool of 256; older weight fades.
        _case("decode_weights", name="rag_decode_weights", batch=64, n_lo=16, n_hi=16, len_lo=1024, len_hi=1024,
              pool=256, q_lo=65, q_hi=65, decay=0.96875),
        # An eighth of four long contexts is kept.
        _case("select", name="icl_select", batch=4, n_lo=128, n_hi=128, len_lo=256, len_hi=256, pool=128, q_lo=300,
              q_hi=300, budget=4096, sink=4, recent=300),
        # One very long context, and a budget that is no round number.
        _case("select", name="long_select", n_lo=37, n_hi=37, len_lo=5000, len_hi=9000, q_lo=77, q_hi=77, budget=16001,
              sink=4, recent=128),
        # The kept keys of the 64 decoding requests, gathered for ordinary position-free decoding.
        _case("compact", name="rag_compact", batch=64, n_lo=16, n_hi=16, len_lo=1024, len_hi=1024, pool=256, q_lo=65,
              q_hi=65, budget=2048, sink=4, recent=65),
        # One user's paged context, kept keys rotated to their positions for attention over materialised keys.
        _case("compact", name="chat_compact", n_lo=5, n_hi=5, len_lo=301, len_hi=811, q_lo=37, q_hi=37, block=64,
              budget=701, sink=4, recent=37, rotate=True),
    ]


# ---------------------------------------------------------------------------------------------------------------
# Drawn cases.
# ---------------------------------------------------------------------------------------------------------------
_LIMIT = {"backward": 1.6e12, "prefill_weights": 2.9e11, "decode_weights": 2.1e9, "select": 2.6e5, "compact": 2.1e9}


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["backward", "backward", "prefill_weights", "decode_weights", "select", "compact"])
    hq, hkv, d = rng.choice([(32, 8, 128), (32, 8, 128), (28, 4, 128), (32, 8, 64), (8, 8, 128), (40, 8, 128),
                             (12, 2, 64), (16, 1, 128), (2, 1, 64)])
    style = rng.choice(["half", "half", "half", "interleaved", "alibi"])
    keys = "nope" if style == "alibi" else rng.choice(["nope", "nope", "local"])
    batch = _log(rng, 1, 64 if kind in ("decode_weights", "select", "compact") else 16)
    n_hi = _log(rng, 1, 128)
    len_hi = _log(rng, 20, 4096)
    q_hi = _log(rng, 1, 2000 if kind == "backward" else 400)
    ragged = rng.random() < 0.6
    shared = rng.random() < 0.6
    c = _case(kind, batch=batch, hq=hq, hkv=hkv, d=d, base=rng.choice([1.0e4, 5.0e5, 1.0e6]), style=style, keys=keys,
              prerot=style != "alibi" and rng.random() < 0.15, causal=rng.random() < 0.85,
              prefix=rng.choice([0, 0, 128, 77]), n_hi=n_hi, len_hi=len_hi, q_hi=q_hi,
              block=rng.choice([0, 0, 0, 64, 32]), dlse=rng.random() < 0.3,
              rotate=style != "alibi" and rng.random() < 0.4, decay=rng.choice([1.0, 1.0, 0.9, 0.0]))

    def keys_of(k):
        return k["prefix"] + k["n_hi"] * k["len_hi"] + k["q_hi"]

    # A drawn call costs no more than the largest listed one: shrink its longest ranges until it fits.
    def cost():
        kv = c["batch"] * keys_of(c)
        pairs = kv * c["q_hi"] * c["hq"] * c["d"]
        return {"backward": max(10.0 * pairs, 1.0e3 * kv * c["hkv"] * c["d"]), "prefill_weights": 2.0 * pairs,
                "decode_weights": 2.0 * kv * c["hkv"] * c["d"], "select": float(kv),
                "compact": 4.0 * kv * c["hkv"] * c["d"]}[kind]

    while cost() > _LIMIT[kind]:
        big = max(("batch", "n_hi"), key=lambda k: c[k]) if c["len_hi"] <= 256 else "len_hi"
        if c[big] <= 2:
            big = "q_hi"
        c[big] = max(1, int(c[big] * 0.71))
    c["n_lo"] = max(1, c["n_hi"] // 3) if ragged else c["n_hi"]
    c["len_lo"] = max(1, c["len_hi"] // 8) if ragged else c["len_hi"]
    c["q_lo"] = max(1, c["q_hi"] // 6) if ragged else c["q_hi"]
    c["pool"] = max(c["n_hi"], int(c["n_hi"] * rng.choice([1, 2, 6]))) if shared else 0
    c["budget"] = max(1, int(keys_of(c) * rng.uniform(0.02, 0.7)))
    c["sink"] = min(rng.choice([0, 1, 4]), c["budget"])
    c["recent"] = min(rng.choice([0, 1, 32, 100]), c["budget"] - c["sink"])
    return c


# ---------------------------------------------------------------------------------------------------------------
# Inputs: a chunk store, one table of records per request, queries.
# ---------------------------------------------------------------------------------------------------------------
def _tables(case, seed):
    """(records, chunk_start, q_lens, q_pos0, elements of the store): host tables.  The lengths belong to the case;
    which chunks a request picks, their order and the places of a paged store's blocks come from the seed."""
    rng = np.random.default_rng([int(seed), 29])
    lens = np.random.default_rng([case[k] for k in ("batch", "n_lo", "n_hi", "len_lo", "len_hi", "q_lo", "q_hi")])
    per_key = case["hkv"] * case["d"]
    bt = case["block"]
    size = 0

    def store(n):
        """Place a chunk of n keys: its blocks as (first key, keys, K offset, V offset, stride)."""
        nonlocal size
        got = []
        for first, keys, cap in [(0, n, n)] if not bt else [(b, min(bt, n - b), bt) for b in range(0, n, bt)]:
            got.append((first, keys, size, size + cap * per_key, cap))
            size += 2 * cap * per_key
        return n, got

    counts, want, q_lens = [], [], []
    for _ in range(case["batch"]):
        counts.append(int(lens.integers(case["n_lo"], case["n_hi"] + 1)))
        want.append(lens.integers(case["len_lo"], case["len_hi"] + 1, counts[-1]))
        q_lens.append(int(lens.integers(case["q_lo"], case["q_hi"] + 1)))
    prefix = store(case["prefix"]) if case["prefix"] else None
    pool = [store(int(n)) for n in lens.integers(case["len_lo"], case["len_hi"] + 1, case["pool"])]
    uses, q_pos0 = [], []
    for r in range(case["batch"]):
        if pool:  # the first picks of a request's share of the pool belong to the case, their order to the seed
            pick = np.random.default_rng([r, case["pool"], counts[r]]).choice(len(pool), counts[r], replace=False)
            mine = [pool[i] for i in rng.permutation(pick)]
        else:
            mine = [store(int(n)) for n in want[r]]
        uses.append(([prefix] if prefix else []) + mine)
    for u, n in zip(uses, q_lens):  # the question's (or the generated tokens') own keys
        q_pos0.append(sum(c[0] for c in u))
        u.append(store(n))
    if bt:  # a paged allocator's blocks lie in no particular order
        cap = 2 * bt * per_key
        where = rng.permutation(size // cap)
    recs, start = [], [0]
    for u in uses:
        pos = 0
        for n, blocks in u:
            for first, keys, ko, vo, cap_keys in blocks:
                if bt:
                    slot = int(where[ko // cap])
                    ko, vo = slot * cap, slot * cap + bt * per_key
                recs.append((ko, vo, keys, pos + first, cap_keys, cap_keys))
            pos += n
        start.append(len(recs))
    if case["kind"] != "backward" and case["kind"] != "prefill_weights":  # one new token: the last of its tail
        q_pos0 = [p + n - 1 for p, n in zip(q_pos0, q_lens)]
        q_lens = [1] * len(q_lens)
    return np.array(recs, dtype=_CHUNK), np.array(start, np.int32), q_lens, q_pos0, size


def _key_counts(recs, start):
    return [int(recs["len"][start[r]:start[r + 1]].sum()) for r in range(len(start) - 1)]


def _prefix_sum(v):
    return np.concatenate([[0], np.cumsum(np.asarray(v, np.int64))])


def _inputs(case, seed):
    """What the call is given: host tables, and on the GPU the store, queries, running weights and so on."""
    recs, start, q_lens, q_pos0, size = _tables(case, seed)
    kind = case["kind"]
    gen = torch.Generator("cuda").manual_seed(int(seed))
    n = _key_counts(recs, start)
    x = dict(recs=recs, start=start, q_lens=q_lens, q_pos0=q_pos0, size=size, n=n, key_start=_prefix_sum(n))
    if kind != "select":
        x["pool"] = torch.empty(size, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    if kind in ("backward", "prefill_weights", "decode_weights"):
        shape = (sum(q_lens), case["hq"], case["d"])
        x["q"] = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    if kind == "backward":
        x["dout"] = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
        x["dlse"] = torch.empty(shape[:2], device="cuda").normal_(generator=gen) if case["dlse"] else None
    if kind in ("decode_weights", "select", "compact"):
        # Accumulated weights: a few heavy keys over many light ones, some never attended to at all.
        w = torch.exp(2.0 * torch.empty(sum(n), device="cuda").normal_(generator=gen) - 3.0)
        x["weights"] = torch.where(torch.empty(sum(n), device="cuda").uniform_(generator=gen) < 0.1, 0.0, w)
    if kind in ("select", "compact"):
        x["kept_start"] = _prefix_sum([min(case["budget"], k) for k in n])
    if kind == "compact":
        # What select would keep: the protected keys and some of the others, ascending.
        kept = []
        for r, k in enumerate(n):
            b = min(case["budget"], k)
            score = torch.rand(k, device="cuda", generator=gen)
            _protect(score, case)
            kept.append(torch.sort(torch.topk(score, b).indices).values.to(torch.int32))
        x["kept"] = torch.cat(kept)
    return x


def _protect(score, case):
    n = score.shape[0]
    score[:min(case["sink"], n)] = math.inf
    score[n - min(case["recent"], n):] = math.inf


def prepare(case, seed):
    x = _inputs(case, seed)
    kind = case["kind"]
    dev = "cuda"

    def i32(v):
        return torch.tensor(np.asarray(v, np.int32), device=dev)

    s = dict(case=case, x=x, max_kv=max(x["n"]), key_start=i32(x["key_start"]))
    # Where each key of a request lies and sits: what the records say, one entry a key.
    if kind != "select":
        rep = x["recs"]["len"].astype(np.int64)
        first = np.repeat(_prefix_sum(rep)[:-1], rep)
        j = np.arange(int(rep.sum())) - first
        flat = {f: np.repeat(x["recs"][f].astype(np.int64), rep) for f in x["recs"].dtype.names}
        s["krow"] = torch.from_numpy(flat["k_offset"] // case["d"] + j).to(dev)
        s["vrow"] = torch.from_numpy(flat["v_offset"] // case["d"] + j).to(dev)
        s["stride"] = torch.from_numpy(flat["k_stride"]).to(dev)
        s["pos"] = torch.from_numpy(flat["pos_offset"] + j).to(dev)
        s["turn"] = s["pos"] if case["keys"] == "nope" else torch.from_numpy(flat["pos_offset"]).to(dev)
        s["local"] = torch.from_numpy(j).to(dev)
    if kind == "backward":  # the forward pass has run: its outputs, rounded as it stores them
        out, lse = _forward(s)
        s["out"], s["lse"] = out.to(torch.bfloat16), lse
        s["dq"] = torch.empty_like(x["q"])
        s["dpool"] = torch.zeros_like(x["pool"])  # gradients of keys that no request reads stay zero
    if kind in ("prefill_weights", "decode_weights"):
        s["lse"] = _forward(s)[1]
        s["weights"] = torch.empty(sum(x["n"]), device=dev)
    if kind in ("select", "compact"):
        s["kept_start"] = i32(x["kept_start"])
        s["max_kept"] = max(min(case["budget"], k) for k in x["n"])
    if kind == "select":
        s["kept"] = torch.empty(int(x["kept_start"][-1]), dtype=torch.int32, device=dev)
    if kind == "compact":  # a record of each request's own, with room for 32 more tokens
        per = case["hkv"] * case["d"]
        dst, at = [], 0
        for k in x["n"]:
            b = min(case["budget"], k)
            dst.append((at, at + (b + 32) * per, b, 0, b + 32, b + 32))
            at += 2 * (b + 32) * per
        s["dst"] = np.array(dst, dtype=_CHUNK)
        s["store"] = torch.zeros(at, dtype=torch.bfloat16, device=dev)
        s["weights_out"] = torch.empty(int(x["kept_start"][-1]), device=dev)
    if own:
        from paper_2606_04302_amd import ops

        s["ops"] = ops
        s["cfg"] = cfg = ops.Config(
            case["hq"], case["hkv"], case["d"], case["base"], causal=case["causal"],
            key_positions=ops.KEYS_LOCAL if case["keys"] == "local" else ops.KEYS_NOPE,
            rope_style={"half": ops.ROPE_HALF, "interleaved": ops.ROPE_INTERLEAVED, "alibi": ops.ALIBI}[case["style"]],
            q_prerotated=case["prerot"])
        s["chunks"] = torch.from_numpy(x["recs"].view(np.uint8).copy()).to(dev)
        s["chunk_start"] = i32(x["start"])
        q_start = _prefix_sum(x["q_lens"]).astype(np.int32)
        s["q_start"], s["q_pos0"], s["max_q"] = i32(q_start), i32(x["q_pos0"]), max(x["q_lens"])
        if kind == "backward":
            s["plan"] = ops.upload_backward_plan(
                ops.backward_plan(cfg, q_start, np.asarray(x["q_pos0"], np.int32), x["recs"], x["start"]), dev)
            nbytes = ops.backward_workspace_size(cfg, s["plan"])
        elif kind == "prefill_weights":
            nbytes = ops.prefill_key_weights_workspace_size(cfg, case["batch"], x["q"].shape[0], s["max_q"],
                                                            s["max_kv"], sum(x["n"]))
        elif kind == "decode_weights":
            nbytes = ops.decode_key_weights_workspace_size(cfg, case["batch"], s["max_kv"])
        elif kind == "select":
            nbytes = ops.cache_select_workspace_size(case["batch"], s["max_kv"])
        else:
            s["dst"] = torch.from_numpy(s["dst"].view(np.uint8).copy()).to(dev)
            nbytes = 0
        s["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    return s


# ---------------------------------------------------------------------------------------------------------------
# One call.
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    kind, x = s["case"]["kind"], s["x"]
    if not own:
        return {"backward": _backward, "prefill_weights": _weights, "decode_weights": _weights, "select": _select,
                "compact": _compact}[kind](s)
    ops, cfg = s["ops"], s["cfg"]
    if kind == "backward":
        ops.prefill_backward(cfg, x["q"], s["q_start"], s["q_pos0"], x["pool"], x["pool"], s["chunks"],
                             s["chunk_start"], s["out"], s["lse"], x["dout"], s["plan"], dlse=x["dlse"], dq=s["dq"],
                             dk_pool=s["dpool"], dv_pool=s["dpool"], workspace=s["workspace"])
        return s["dq"], s["dpool"]
    if kind == "prefill_weights":
        return ops.prefill_key_weights(cfg, x["q"], s["q_start"], s["q_pos0"], x["pool"], s["chunks"],
                                       s["chunk_start"], s["key_start"], s["max_q"], s["max_kv"], s["lse"],
                                       s["weights"], workspace=s["workspace"])
    if kind == "decode_weights":
        return ops.decode_key_weights(cfg, x["q"], s["q_pos0"], x["pool"], s["chunks"], s["chunk_start"],
                                      s["key_start"], s["max_kv"], s["lse"], s["weights"], weights_in=x["weights"],
                                      decay=s["case"]["decay"], workspace=s["workspace"])
    if kind == "select":
        return ops.cache_select(x["weights"], s["key_start"], s["kept_start"], s["max_kv"], s["kept"],
                                sink=s["case"]["sink"], recent=s["case"]["recent"], workspace=s["workspace"])
    ops.cache_compact(cfg, x["pool"], x["pool"], s["chunks"], s["chunk_start"], x["kept"], s["kept_start"],
                      s["max_kept"], s["dst"], s["store"], s["store"], rotate=s["case"]["rotate"],
                      key_start=s["key_start"], weights=x["weights"], weights_out=s["weights_out"])
    return s["store"], s["weights_out"]


# ---------------------------------------------------------------------------------------------------------------
# The plain forms: 32 bits (angles in 64), one request and KV head at a time.
# ---------------------------------------------------------------------------------------------------------------
def _turn(v, pos, case, back=False):
    """v [n, ..., d] (fp32) rotated at positions pos [n], or turned back by them."""
    d = case["d"]
    f = torch.exp(torch.arange(d // 2, dtype=torch.float64, device=v.device) * (-2.0 / d * math.log(case["base"])))
    a = pos.double().view(-1, *([1] * (v.dim() - 1))) * f
    c, s = torch.cos(a).float(), torch.sin(a).float()
    if back:
        s = -s
    out = torch.empty_like(v)
    one, two = (slice(0, None, 2), slice(1, None, 2)) if case["style"] == "interleaved" else \
        (slice(0, d // 2), slice(d // 2, None))
    out[..., one] = v[..., one] * c - v[..., two] * s
    out[..., two] = v[..., one] * s + v[..., two] * c
    return out


def _request(s, r, t0):
    """Request r's queries [tokens, hq, d] rotated, its tokens' positions and its keys' range in the flat arrays."""
    case, x = s["case"], s["x"]
    qpos = x["q_pos0"][r] + torch.arange(x["q_lens"][r], device="cuda")
    q = x["q"][t0:t0 + x["q_lens"][r]].float()
    if case["style"] != "alibi" and not case["prerot"]:
        q = _turn(q, qpos, case)
    return q, qpos, slice(int(x["key_start"][r]), int(x["key_start"][r + 1]))


def _head(s, q, qpos, keys, g):
    """Rotated queries [tokens * G, d] and keys of KV head g, and their scaled scores, -inf where hidden."""
    case = s["case"]
    G, d = case["hq"] // case["hkv"], case["d"]
    qg = q[:, g * G:(g + 1) * G].reshape(-1, d)
    k = s["x"]["pool"].view(-1, d)[s["krow"][keys] + g * s["stride"][keys]].float()
    if case["style"] != "alibi":
        k = _turn(k, s["turn"][keys], case)
    sc = (qg @ k.T).view(-1, G, k.shape[0]) / math.sqrt(d)
    pos = s["pos"][keys]
    if case["style"] == "alibi":
        h = torch.arange(g * G, (g + 1) * G, device="cuda")
        sc += (2.0 ** (-8.0 * (h + 1) / case["hq"]))[:, None] * (pos[None, :] - qpos[:, None])[:, None, :]
    if case["causal"]:
        sc.masked_fill_((pos[None, :] > qpos[:, None])[:, None, :], -math.inf)
    return qg, k, sc.view(-1, k.shape[0])


def _forward(s):
    case, x = s["case"], s["x"]
    G, d = case["hq"] // case["hkv"], case["d"]
    out = torch.zeros(x["q"].shape, device="cuda")
    lse = torch.empty(x["q"].shape[:2], device="cuda")
    t0 = 0
    for r, n in enumerate(x["q_lens"]):
        q, qpos, keys = _request(s, r, t0)
        for g in range(case["hkv"]):
            sc = _head(s, q, qpos, keys, g)[2]
            m = sc.amax(1, keepdim=True).clamp_min(-1.0e30)
            p = torch.exp(sc - m)
            z = p.sum(1, keepdim=True)
            v = x["pool"].view(-1, d)[s["vrow"][keys] + g * s["stride"][keys]].float()
            heads = slice(g * G, (g + 1) * G)
            if case["kind"] == "backward":
                out[t0:t0 + n, heads] = (p @ v / z.clamp_min(1.0e-30)).view(n, G, d)
            lse[t0:t0 + n, heads] = (m + torch.log(z)).view(n, G)
        t0 += n
    return out, lse


def _probabilities(sc, lse):
    return torch.where(torch.isinf(lse), 0.0, torch.exp(sc - lse))


def _backward(s):
    case, x = s["case"], s["x"]
    G, d = case["hq"] // case["hkv"], case["d"]
    scale = 1.0 / math.sqrt(d)
    delta = (x["dout"].float() * s["out"].float()).sum(-1)
    if x["dlse"] is not None:
        delta = delta - x["dlse"]
    dq = torch.empty(x["q"].shape, device="cuda")
    dpool = torch.zeros(x["size"], device="cuda").view(-1, d)
    t0 = 0
    for r, n in enumerate(x["q_lens"]):
        q, qpos, keys = _request(s, r, t0)
        rows = slice(t0, t0 + n)
        for g in range(case["hkv"]):
            heads = slice(g * G, (g + 1) * G)
            qg, k, sc = _head(s, q, qpos, keys, g)
            p = _probabilities(sc, s["lse"][rows, heads].reshape(-1, 1))
            do = x["dout"][rows, heads].float().reshape(-1, d)
            at = s["vrow"][keys] + g * s["stride"][keys]
            v = x["pool"].view(-1, d)[at].float()
            ds = p * (do @ v.T - delta[rows, heads].reshape(-1, 1)) * scale
            dpool.index_add_(0, at, p.T @ do)
            dk, dqg = ds.T @ qg, (ds @ k).view(n, G, d)
            if case["style"] != "alibi":
                dk = _turn(dk, s["turn"][keys], case, back=True)
                if not case["prerot"]:
                    dqg = _turn(dqg, qpos, case, back=True)
            dpool.index_add_(0, s["krow"][keys] + g * s["stride"][keys], dk)
            dq[rows, heads] = dqg
        t0 += n
    return dq.to(torch.bfloat16), dpool.view(-1).to(torch.bfloat16)


def _weights(s):
    case, x = s["case"], s["x"]
    G = case["hq"] // case["hkv"]
    w = x["weights"] * case["decay"] if "weights" in x else torch.zeros(sum(x["n"]), device="cuda")
    t0 = 0
    for r, n in enumerate(x["q_lens"]):
        q, qpos, keys = _request(s, r, t0)
        for g in range(case["hkv"]):
            sc = _head(s, q, qpos, keys, g)[2]
            lse = s["lse"][t0:t0 + n, g * G:(g + 1) * G].reshape(-1, 1)
            w[keys] += _probabilities(sc, lse).sum(0)
        t0 += n
    return w


def _select(s):
    case, x = s["case"], s["x"]
    kept = []
    for r, n in enumerate(x["n"]):
        score = x["weights"][int(x["key_start"][r]):int(x["key_start"][r + 1])].clone()
        _protect(score, case)
        first = torch.sort(score, descending=True, stable=True).indices[:min(case["budget"], n)]
        kept.append(torch.sort(first).values.to(torch.int32))
    return torch.cat(kept)


def _compact(s):
    case, x = s["case"], s["x"]
    d = case["d"]
    pool, store = x["pool"].view(-1, d), s["store"].view(-1, d)
    weights = torch.empty(int(x["kept_start"][-1]), device="cuda")
    for r, n in enumerate(x["n"]):
        mine = slice(int(x["kept_start"][r]), int(x["kept_start"][r + 1]))
        at = x["kept"][mine].long() + int(x["key_start"][r])
        weights[mine] = x["weights"][at]
        i = torch.arange(at.shape[0], device="cuda")
        dst = s["dst"][r]
        for g in range(case["hkv"]):
            k = pool[s["krow"][at] + g * s["stride"][at]]
            if case["rotate"]:
                k = _turn(k.float(), s["turn"][at], case).to(torch.bfloat16)
            elif case["keys"] == "local":
                k = _turn(k.float(), i - s["local"][at], case).to(torch.bfloat16)
            store[int(dst["k_offset"]) // d + g * int(dst["k_stride"]) + i] = k
            store[int(dst["v_offset"]) // d + g * int(dst["v_stride"]) + i] = pool[s["vrow"][at] + g * s["stride"][at]]
    return s["store"], weights


# ---------------------------------------------------------------------------------------------------------------
# What a call cannot do without, and what its outputs should be.
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    """Bytes: every stored key (and value) that some request reads, once, and every other input and output, once.
    FLOPs: the products over the visible (query, key) pairs, five for the backward pass and one for the weights."""
    recs, start, q_lens, _, _ = _tables(case, 0)
    d, hq, hkv, kind = case["d"], case["hq"], case["hkv"], case["kind"]
    n = _key_counts(recs, start)
    keys = float(sum(n))
    kept = float(sum(min(case["budget"], k) for k in n))
    distinct = {(int(k), int(v)): int(ln) for k, v, ln in zip(recs["k_offset"], recs["v_offset"], recs["len"])}
    stored = float(sum(distinct.values()))
    tokens = float(sum(q_lens))
    pairs = 0.0
    for k, t in zip(n, q_lens):
        # A prompt's own keys are the last of its table: token i does not see the t - 1 - i after it.
        pairs += t * k - (t * (t - 1) / 2 if case["causal"] and kind in ("backward", "prefill_weights") else 0)
    if kind == "backward":
        return {"bytes": 8.0 * hkv * d * stored + recs.nbytes + tokens * hq * (8.0 * d + 4 + 4 * case["dlse"]),
                "flops": 10.0 * d * hq * pairs}
    if kind == "prefill_weights":
        return {"bytes": 2.0 * hkv * d * stored + recs.nbytes + tokens * hq * (2.0 * d + 4) + 4 * keys,
                "flops": 2.0 * d * hq * pairs}
    if kind == "decode_weights":
        return {"bytes": 2.0 * hkv * d * stored + recs.nbytes + tokens * hq * (2.0 * d + 4) + 8 * keys,
                "flops": 2.0 * d * hq * pairs}
    if kind == "select":
        return {"bytes": 4 * keys + 4 * kept, "flops": keys}
    return {"bytes": 8.0 * hkv * d * kept + recs.nbytes + 12 * kept, "flops": 3.0 * hkv * d * kept * case["rotate"]}


def _spin(case, pos):
    """exp(i p theta_t) in 64 bits, [n, d/2] complex."""
    t = torch.arange(case["d"] // 2, dtype=torch.float64, device=pos.device)
    theta = torch.pow(torch.tensor(case["base"], dtype=torch.float64, device=pos.device), -2.0 * t / case["d"])
    a = pos.double()[:, None] * theta[None, :]
    return torch.polar(torch.ones_like(a), a)


def _as_pairs(case, v):
    v = v.double()
    if case["style"] == "interleaved":
        return torch.view_as_complex(v.reshape(*v.shape[:-1], -1, 2).contiguous())
    h = case["d"] // 2
    return torch.complex(v[..., :h].contiguous(), v[..., h:].contiguous())


def _from_pairs(case, z):
    if case["style"] == "interleaved":
        return torch.view_as_real(z.resolve_conj()).reshape(*z.shape[:-1], -1)
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    """The outputs in 64 bits: rotations as complex products, one query head at a time, keys looked up record by
    record."""
    kind = case["kind"]
    x = _inputs(case, seed)
    recs, start, d, hq, hkv = x["recs"], x["start"], case["d"], case["hq"], case["hkv"]
    G = hq // hkv
    dev = "cuda"
    rope = case["style"] != "alibi"
    if kind == "select":
        w = x["weights"].cpu().numpy()
        got = []
        for r, n in enumerate(x["n"]):
            b = min(case["budget"], n)
            mine = w[x["key_start"][r]:x["key_start"][r + 1]].astype(np.float64)
            j = np.arange(n)
            guarded = (j < case["sink"]) | (j >= n - case["recent"])
            rank = np.lexsort((j, -mine, ~guarded))
            got.append(np.sort(rank[:b]))
        return torch.from_numpy(np.concatenate(got).astype(np.int32))
    if kind == "compact":
        per = hkv * d
        rooms = [min(case["budget"], n) + 32 for n in x["n"]]
        store = torch.zeros(2 * sum(rooms) * per, dtype=torch.float64, device=dev)
        at = 0
        for r, room in enumerate(rooms):
            kept = x["kept"][int(x["kept_start"][r]):int(x["kept_start"][r + 1])].long()
            ks = store[at:at + room * per].view(hkv, room, d)
            vs = store[at + room * per:at + 2 * room * per].view(hkv, room, d)
            at += 2 * room * per
            first = 0
            for rec in recs[start[r]:start[r + 1]]:
                ko, vo, ln, pos, st, _ = (int(v) for v in rec)
                i = torch.nonzero((kept >= first) & (kept < first + ln)).view(-1)
                j = kept[i] - first
                first += ln
                k = x["pool"][ko:ko + st * per].view(hkv, st, d)[:, j].double()
                turn = None
                if case["rotate"]:
                    turn = pos + j if case["keys"] == "nope" else torch.full_like(j, pos)
                elif case["keys"] == "local":
                    turn = i - j
                if turn is not None:
                    k = _from_pairs(case, _as_pairs(case, k) * _spin(case, turn))
                ks[:, i] = k
                vs[:, i] = x["pool"][vo:vo + st * per].view(hkv, st, d)[:, j].double()
        out_w = [x["weights"].double()[x["kept"][int(x["kept_start"][r]):int(x["kept_start"][r + 1])].long() +
                                       int(x["key_start"][r])] for r in range(len(x["n"]))]
        return store, torch.cat(out_w)

    if 4.0 * d * hq * sum(k * t for k, t in zip(x["n"], x["q_lens"])) > 2.0e13:
        return None
    back = kind == "backward"
    if kind == "prefill_weights" or back:
        w = torch.zeros(sum(x["n"]), dtype=torch.float64, device=dev)
    else:
        w = x["weights"].double() * case["decay"]
    if back:
        dq = torch.zeros(x["q"].shape, dtype=torch.float64, device=dev)
        dpool = torch.zeros(x["size"], dtype=torch.float64, device=dev)
    t0 = 0
    for r, n in enumerate(x["q_lens"]):
        qpos = x["q_pos0"][r] + torch.arange(n, device=dev)
        spots = []
        for rec in recs[start[r]:start[r + 1]]:
            ko, vo, ln, pos, st, _ = (int(v) for v in rec)
            p = pos + torch.arange(ln, device=dev)
            spots.append((ko, vo, ln, st, p, p if case["keys"] == "nope" else torch.full_like(p, pos)))
        kpos = torch.cat([sp[4] for sp in spots])
        kspin = _spin(case, torch.cat([sp[5] for sp in spots])) if rope else None
        qspin = _spin(case, qpos) if rope and not case["prerot"] else None
        hidden = (kpos[None, :] > qpos[:, None]) if case["causal"] else None
        k0 = int(x["key_start"][r])
        for g in range(hkv):
            def stored(which):
                return torch.cat([x["pool"][sp[which]:sp[which] + hkv * sp[3] * d].view(hkv, sp[3], d)[g, :sp[2]]
                                  for sp in spots]).double()

            k, v = stored(0), stored(1) if back else None
            if rope:
                k = _from_pairs(case, _as_pairs(case, k) * kspin)
            kt = k.T.contiguous()
            dk, dv = torch.zeros_like(k), torch.zeros_like(k)
            for h in range(g * G, (g + 1) * G):
                q = x["q"][t0:t0 + n, h].double()
                if qspin is not None:
                    q = _from_pairs(case, _as_pairs(case, q) * qspin)
                sc = q @ kt / math.sqrt(d)
                if not rope:
                    sc += math.pow(2.0, -8.0 * (h + 1) / hq) * (kpos[None, :] - qpos[:, None]).double()
                if hidden is not None:
                    sc.masked_fill_(hidden, -math.inf)
                if not back:
                    w[k0:k0 + k.shape[0]] += torch.nan_to_num(torch.softmax(sc, -1), nan=0.0).sum(0)
                    continue
                # The call is given the forward pass's results, rounded to bf16 and fp32.
                lse = torch.logsumexp(sc, -1, keepdim=True)
                o = (torch.nan_to_num(torch.exp(sc - lse), nan=0.0) @ v).to(torch.bfloat16).double()
                lse = lse.float().double()
                p = torch.where(torch.isinf(lse), 0.0, torch.exp(sc - lse))
                do = x["dout"][t0:t0 + n, h].double()
                inner = (do * o).sum(-1, keepdim=True)
                if x["dlse"] is not None:
                    inner = inner - x["dlse"][t0:t0 + n, h, None].double()
                ds = p * (do @ v.T.contiguous() - inner) / math.sqrt(d)
                dv += p.T.contiguous() @ do
                dk += ds.T.contiguous() @ q
                dqh = ds @ k
                if qspin is not None:
                    dqh = _from_pairs(case, _as_pairs(case, dqh) * qspin.conj())
                dq[t0:t0 + n, h] = dqh
            if back:
                if rope:
                    dk = _from_pairs(case, _as_pairs(case, dk) * kspin.conj())
                j0 = 0
                for ko, vo, ln, st, _, _ in spots:
                    dpool[ko:ko + hkv * st * d].view(hkv, st, d)[g, :ln] += dk[j0:j0 + ln]
                    dpool[vo:vo + hkv * st * d].view(hkv, st, d)[g, :ln] += dv[j0:j0 + ln]
                    j0 += ln
        t0 += n
    return (dq, dpool) if back else w
