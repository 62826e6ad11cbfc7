"""What a decoder's step does beside its products and its attention, as measurable cases: norms before and after a block with its
gate and residual sum ("norm"), low-rank adapters of many requests beside the projections that they share ("adapt", and "group":
the step's rows by adapter), log probabilities of given tokens with entropy and top alternatives ("score").

    norm     s = skip x + scale act(gate) norm_y(y),  out = norm_x(s), a row of `width` elements at a time
    adapt    out[t] = y[t] + scale_a B_a (A_a x[t]) for each projection, a the adapter of row t's request (or none)
    group    the rows of every adapter in tiles of up to 64, in order; rows of no adapter behind them
    score    log p of tokens, -sum p log p, the `top` most probable tokens, p = softmax(scale logits), a row at a time
"""
import math

import numpy as np
import torch

own = False

TILE = 64                        # rows of a tile of one adapter


def listed():
    return [
        # One token, 7B shape, binary32 stream: the sum and the norm before the next block.  The smallest call: latency counts.
        dict(name="norm-7b-one", kind="norm", rows=1, width=4096, y="f32", x="f32", out="f16", norm_y=None, norm_x="rms", gate=None, act=None),
        # A tree of 16 drafted tokens, 65B shape, norms on both sides of the block, a learned gate for each channel.
        dict(name="norm-65b-tree16", kind="norm", rows=16, width=8192, y="f32", x="f32", out="f16", norm_y="rms", norm_x="rms", gate="channel", act=None),
        # Prompts, 33B shape, 16-bit stream and products, a gate for each token and channel out of a product of its own.
        dict(name="norm-prompts-gated", kind="norm", rows=4096, width=6656, y="f16", x="bf16", out="f16", norm_y="layer", norm_x="layer", gate="row", act="sigmoid"),
        # One request, one token, q, k and v of the 7B shape.
        dict(name="adapt-7b-one", kind="adapt", R=1, fresh=1, slots=8, width=4096, ms="4096,4096,4096", rank=16, mixed=False, dtype="f16", y="f32"),
        # Sixteen requests, an adapter each, of different ranks; gate and up of the 33B shape, 16-bit outputs.
        dict(name="adapt-33b-own16", kind="adapt", R=16, fresh=1, slots=24, width=6656, ms="17920,17920", rank=64, mixed=True, dtype="f16", y="f16"),
        # A hundred requests with short chains of drafted tokens on 37 adapters, 65B shape.
        dict(name="adapt-65b-chains", kind="adapt", R=100, fresh=5, slots=37, width=8192, ms="8192", rank=32, mixed=False, dtype="bf16", y="f32"),
        # Slices of prompts of nine requests on six adapters, grouped heads: most rows a call has.
        dict(name="adapt-prompts", kind="adapt", R=9, fresh=801, slots=6, width=8192, ms="8192,1024,1024", rank=64, mixed=True, dtype="f16", y="f32"),
        # The rows of 64 requests with a tree of 16 tokens each, by adapter.
        dict(name="group-trees", kind="group", R=64, fresh=16, slots=48, by_row=False),
        # 4096 rows with an adapter named for each.
        dict(name="group-rows", kind="group", R=4096, fresh=1, slots=200, by_row=True),
        # One row behind the head: the next token's alternatives.
        dict(name="score-one", kind="score", rows=1, vocab=32000, pitch=32000, dtype="f32", given=1, top=5, scale=1.0, masked=False),
        # Sixteen rows of a tree over a large vocabulary, tokens forbidden by a grammar, a temperature, the drafted children's probabilities.
        dict(name="score-tree16", kind="score", rows=16, vocab=128000, pitch=128000, dtype="f16", given=4, top=20, scale=1.4, masked=True),
        # The probabilities of a text's tokens, an odd vocabulary.
        dict(name="score-text", kind="score", rows=2048, vocab=65537, pitch=65537, dtype="bf16", given=1, top=10, scale=1.0, masked=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _odd_or_even(rng, n, step):
    """n, or a multiple of `step` near it."""
    return n if rng.random() < 0.4 else max(step, n // step * step)


def draw(rng):
    kind = rng.choice(["norm", "norm", "adapt", "adapt", "adapt", "score", "score", "score", "group"])
    types = ["f32", "f16", "bf16"]
    if kind == "norm":
        width = _odd_or_even(rng, _log_int(rng, 64, 24000), 64)
        gate = rng.choice([None, "channel", "row"])
        return dict(kind=kind, rows=max(1, min(_log_int(rng, 1, 8192), 27_000_000 // width)), width=width, y=rng.choice(types), x=rng.choice(types + [None]),
                    out=rng.choice(["f16", "bf16", "f32"]), norm_y=rng.choice([None, "rms", "layer"]), norm_x=rng.choice(["rms", "rms", "layer"]),
                    gate=gate, act=rng.choice([None, "silu", "sigmoid", "tanh"]) if gate else None)
    if kind == "score":
        vocab = _odd_or_even(rng, _log_int(rng, 500, 260000), 64)
        pitch = vocab + rng.choice([0, 0, 0, 64, 7])
        return dict(kind=kind, rows=max(1, min(_log_int(rng, 1, 3000), 130_000_000 // pitch)), vocab=vocab, pitch=pitch, dtype=rng.choice(types),
                    given=rng.choice([1, 1, 2, 5]), top=rng.choice([0, 1, 5, 10, 20, 50]), scale=rng.choice([1.0, 0.8, 2.5]),
                    masked=rng.choice([True, False]))
    if kind == "group":
        return dict(kind=kind, R=_log_int(rng, 1, 1000), fresh=_log_int(rng, 1, 64), slots=_log_int(rng, 1, 500), by_row=rng.choice([True, False]))
    c = dict(kind=kind, R=_log_int(rng, 1, 256), fresh=_log_int(rng, 1, 1000), slots=_log_int(rng, 1, 100),
             width=_odd_or_even(rng, _log_int(rng, 100, 16000), 32), rank=rng.choice([4, 8, 16, 16, 24, 32, 64, 128, 200]),
             mixed=rng.choice([True, False]), dtype=rng.choice(["f16", "bf16"]), y=rng.choice(types))
    if rng.random() < 0.4:
        c["fresh"] = 1
    ms = [_odd_or_even(rng, _log_int(rng, 100, 16000), 32)]
    if rng.random() < 0.5:
        ms += [_odd_or_even(rng, max(64, ms[0] // rng.choice([1, 2, 8])), 32)] * rng.choice([1, 2])
    c["ms"] = ",".join(map(str, ms))
    total = c["width"] + sum(ms)
    c["slots"] = max(1, min(c["slots"], 60_000_000 // (c["rank"] * total)))
    # as many rows a request as the largest listed case has elements of rows, and a sixth of its products
    most = min(40_000_000 // total, 1_200_000_000 // (c["rank"] * total))
    c["R"] = max(1, min(c["R"], most))
    c["fresh"] = max(1, min(c["fresh"], most // c["R"]))
    return c


# ---------------------------------------------------------------------------------------------------------------------
# Inputs.  Sizes, lengths and who has which adapter go by the case, contents by the seed.
# ---------------------------------------------------------------------------------------------------------------------
_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 7)
    return g


def _randn(shape, g, dtype, size=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(size).to(_TYPES[dtype])


def _int(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _ms(case):
    return [int(m) for m in case["ms"].split(",")]


def _requests(case):
    """New tokens and adapter of each request: spread between 1 and the most; one in seven has no adapter."""
    R, most, slots = case["R"], case["fresh"], case["slots"]
    fresh = [most if r == 0 else 1 + (389 * r + 101 * r * r) % most for r in range(R)]
    adapter = [-1 if r % 7 == 4 else (5 * r + 2 + r * r % 3) % slots for r in range(R)]
    return fresh, adapter


def _ranks(case):
    """Of each slot: the bank's, or spread below it."""
    top = case["rank"]
    return [top if not case["mixed"] or a % 4 == 0 else max(1, top * (1 + a % 4) // 5) for a in range(case["slots"])]


def prepare(case, seed):
    st = globals()["_prepare_" + case["kind"]](case, _generator(seed))
    st["case"] = case
    if own:                      # the handles that a program keeps: weights' addresses, sizes, the kernels' scratch, the step's plan
        import paper_2306_03078_amd.block_binding as K
        if case["kind"] == "norm":
            st["handle"] = K.SpQRResidualNorm(case["width"], norm_y=case["norm_y"], norm_x=case["norm_x"], act=case["act"],
                                              out_dtype=_TYPES[case["out"]], **{n: st[n] for n in ("y_weight", "y_bias", "x_weight", "x_bias", "eps", "skip", "scale")})
        elif case["kind"] == "score":
            st["handle"] = K.SpQRScores(case["rows"], case["vocab"], given=case["given"], top=case["top"])
        else:
            st["plan"] = K.SpQRAdapterPlan(st["rows"], case["slots"])
            if case["kind"] == "adapt":
                K.spqr_adapter_plan(st["plan"], st["adapter"], st["q_start"])
                st["handle"] = K.SpQRAdapters(st["A"], st["B"], rank=st["rank"], scale=st["scale"], rows=st["rows"])
    return st


def _prepare_norm(case, g):
    rows, n = case["rows"], case["width"]
    w = {}
    for side in ("y", "x"):
        kind = case["norm_" + side]
        w[side + "_weight"] = 1.0 + 0.2 * torch.randn(n, generator=g, device="cuda") if kind else None
        w[side + "_bias"] = 0.1 * torch.randn(n, generator=g, device="cuda") if kind == "layer" else None
    # a stream with a few channels far larger than the others, a product's rows of different sizes
    x = None
    if case["x"]:
        x = torch.randn((rows, n), generator=g, device="cuda")
        x[:, ::max(1, n // 5)] *= 40.0
        x = x.to(_TYPES[case["x"]])
    y = torch.randn((rows, n), generator=g, device="cuda")
    y *= 2.0 ** torch.randint(-3, 4, (rows, 1), generator=g, device="cuda")
    gate = None if case["gate"] is None else _randn((n,) if case["gate"] == "channel" else (rows, n), g, case["y"])
    return dict(x=x, y=y.to(_TYPES[case["y"]]), gate=gate, eps=1e-5, skip=0.9 if case["x"] else 1.0, scale=0.7, **w)


def _prepare_score(case, g):
    rows, vocab = case["rows"], case["vocab"]
    whole = torch.randn((rows, case["pitch"]), generator=g, device="cuda", dtype=_TYPES[case["dtype"]])
    logits = whole.mul_(3.0)[:, :vocab]
    tokens = torch.randint(0, vocab, (rows, case["given"]), generator=g, device="cuda", dtype=torch.int32)
    r = torch.arange(rows, device="cuda")
    logits[r, tokens[:, 0].long()] += 8.0                    # what a text has next is probable
    if case["masked"]:
        # a grammar forbids half of the tokens in some rows, all but seven in others
        half = torch.rand((rows, vocab), generator=g, device="cuda") < 0.5
        logits.masked_fill_(half & (r % 4 == 1)[:, None], -math.inf)
        few = torch.ones((rows, vocab), dtype=torch.bool, device="cuda")
        few[r[:, None], torch.randint(0, vocab, (rows, 7), generator=g, device="cuda")] = False
        logits.masked_fill_(few & (r % 16 == 6)[:, None], -math.inf)
    return dict(logits=logits, tokens=tokens)


def _prepare_group(case, g):
    fresh, adapter = _requests(case)
    # which request comes first goes by the seed
    turn = int(torch.randint(0, case["R"], (1,), generator=g, device="cuda"))
    fresh, adapter = fresh[turn:] + fresh[:turn], adapter[turn:] + adapter[:turn]
    q_start = None
    if case["by_row"]:
        adapter = [a for a, n in zip(adapter, fresh) for _ in range(n)]
    else:
        q_start = _int([0] + list(np.cumsum(fresh)))
    return dict(adapter=_int(adapter), q_start=q_start, rows=sum(fresh))


def _prepare_adapt(case, g):
    fresh, adapter = _requests(case)
    T, n, R, slots, ms = sum(fresh), case["width"], case["rank"], case["slots"], _ms(case)
    A = [torch.randn((slots, R, n), generator=g, device="cuda", dtype=_TYPES[case["dtype"]]).mul_(n ** -0.5) for _ in ms]
    B = [torch.randn((slots, m, R), generator=g, device="cuda", dtype=_TYPES[case["dtype"]]).mul_(R ** -0.5) for m in ms]
    # rows of each adapter in a table, -1 behind the last one: what the plain form goes by
    of_row = np.repeat(np.array(adapter), fresh)
    used = [a for a in range(slots) if (of_row == a).any()]
    table = np.full((len(used), max([1] + [int((of_row == a).sum()) for a in used])), -1)
    for i, a in enumerate(used):
        at = np.flatnonzero(of_row == a)
        table[i, :len(at)] = at
    return dict(A=A, B=B, rank=_int(_ranks(case)), scale=0.5 + torch.rand(slots, generator=g, device="cuda"), x=_randn((T, n), g, case["dtype"]),
                y=[_randn((T, m), g, case["y"]) for m in ms], adapter=_int(adapter), q_start=_int([0] + list(np.cumsum(fresh))), rows=T,
                used=_int(used, torch.int64), table=torch.from_numpy(table).cuda())


# ---------------------------------------------------------------------------------------------------------------------
# One pass.
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if not own:
        return globals()["_plain_" + kind](state)
    import paper_2306_03078_amd.block_binding as K
    if kind == "norm":
        total, out = K.spqr_residual_norm(state["handle"], state["x"], state["y"], state["gate"])
        return dict(out=out) if total is None else dict(sum=total, out=out)
    if kind == "score":
        s = K.spqr_token_logprobs(state["handle"], state["logits"], state["tokens"], scale=state["case"]["scale"])
        return dict(logprob=s.logprob, entropy=s.entropy, top_token=s.top_token, top_logprob=s.top_logprob)
    if kind == "group":
        p = K.spqr_adapter_plan(state["plan"], state["adapter"], state["q_start"])
        return dict(count=p.count, tile=p.tile, row=p.row)
    return K.spqr_adapters(state["handle"], state["plan"], state["x"], state["y"])


def _normed(v, kind, weight, bias, eps):
    if kind is None:
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(1, keepdim=True) + eps) * weight
    return v if bias is None else v + bias


def _plain_norm(st):
    case, x = st["case"], st["x"]
    u = _normed(st["y"].float(), case["norm_y"], st["y_weight"], st["y_bias"], st["eps"])
    if st["gate"] is not None:
        gate = st["gate"].float()
        if case["act"] == "tanh":
            gate = torch.tanh(gate)
        elif case["act"]:
            gate = (gate if case["act"] == "silu" else 1.0) / (1.0 + torch.exp(-gate))
        u = u * gate
    s = st["scale"] * u
    if x is not None:
        s = st["skip"] * x.float() + s
    out = _normed(s, case["norm_x"], st["x_weight"], st["x_bias"], st["eps"]).to(_TYPES[case["out"]])
    return dict(out=out) if x is None else dict(sum=s.to(x.dtype), out=out)


def _plain_adapt(st):
    rows, used = st["table"], st["used"]
    at = rows.clamp(min=0)
    rank = torch.arange(st["case"]["rank"], device="cuda") < st["rank"][used][:, None]     # [used, rank]
    factor = torch.where(rank, st["scale"][used][:, None], 0.0)
    X = st["x"][at].float()                                                                # [used, most, width]

    def one(A, B, y):
        v = torch.matmul(X, A[used].float().transpose(1, 2)) * factor[:, None]
        v = torch.matmul(v, B[used].float().transpose(1, 2))                               # [used, most, m]
        out = torch.cat([y, y[:1]])
        out[torch.where(rows < 0, y.shape[0], rows)] = (y[at].float() + v).to(y.dtype)
        return out[:-1]
    return [one(A, B, y) for A, B, y in zip(st["A"], st["B"], st["y"])]


def _plain_group(st):
    T, slots, adapter = st["rows"], st["case"]["slots"], st["adapter"].long()
    if st["q_start"] is not None:
        adapter = torch.repeat_interleave(adapter, st["q_start"].diff(), output_size=T)
    of_row = torch.where((adapter >= 0) & (adapter < slots), adapter, slots)               # `slots`: no adapter
    order = torch.argsort(of_row, stable=True)
    rows = torch.zeros(slots + 1, dtype=torch.int64, device="cuda").index_add_(0, of_row, torch.ones_like(of_row))
    tiles = (rows + TILE - 1) // TILE
    first_row, first_tile = rows.cumsum(0) - rows, tiles.cumsum(0) - tiles
    most = min(T, T // TILE + slots + 1)
    which = of_row[order]
    place = torch.arange(T, device="cuda") - first_row[which]
    row = torch.full((most, TILE), -1, dtype=torch.int32, device="cuda")
    row[first_tile[which] + place // TILE, place % TILE] = order.to(torch.int32)
    tile = torch.stack([torch.full((most,), -1, dtype=torch.int32, device="cuda"), (row >= 0).sum(1).to(torch.int32)], 1)
    tile[first_tile[which] + place // TILE, 0] = torch.where(which < slots, which, -1).to(torch.int32)
    return dict(count=tiles.sum(0, keepdim=True).to(torch.int32), tile=tile, row=row)


def _plain_score(st):
    case, logits, tokens = st["case"], st["logits"], st["tokens"].long()
    vocab, top = case["vocab"], case["top"]
    raw = logits.float()
    z = raw * case["scale"]
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    lse = torch.log(total)
    entropy = lse[:, 0] - (torch.where(e > 0, z, 0.0) * e).sum(1) / total[:, 0]
    logprob = torch.gather(z, 1, tokens) - lse
    # the largest logits, the lowest id among equal ones: one order of whole numbers
    bits = (raw + 0.0).view(torch.int32)
    key = ((bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32) | torch.arange(vocab - 1, -1, -1, device="cuda")
    best = torch.topk(key, top, dim=1).values
    token = vocab - 1 - (best & 0xFFFFFFFF)
    there = torch.gather(raw, 1, token) > -math.inf
    return dict(logprob=logprob, entropy=entropy, top_token=torch.where(there, token, -1).to(torch.int32),
                top_logprob=torch.gather(z, 1, token) - lse)


_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def work(case):
    if case["kind"] == "norm":
        rows, n = case["rows"], case["width"]
        size = _BYTES[case["y"]] + _BYTES[case["out"]] + (2 * _BYTES[case["x"]] if case["x"] else 0)
        vectors = sum({"rms": 1, "layer": 2, None: 0}[case["norm_" + s]] for s in ("y", "x"))
        gate = {None: 0, "channel": n, "row": rows * n}[case["gate"]] * _BYTES[case["y"]]
        return {"bytes": rows * n * size + gate + 4 * n * vectors, "flops": 12 * rows * n}
    if case["kind"] == "score":
        rows, vocab = case["rows"], case["vocab"]
        return {"bytes": rows * (vocab * _BYTES[case["dtype"]] + 8 * case["given"] + 4 + 8 * case["top"]), "flops": 8 * rows * vocab}
    fresh, adapter = _requests(case)
    T = sum(fresh)
    if case["kind"] == "group":
        most = min(T, T // TILE + case["slots"] + 1)
        return {"bytes": (4 * T if case["by_row"] else 8 * case["R"]) + most * (8 + 4 * TILE), "flops": 0}
    ranks, n = _ranks(case), case["width"]
    weights = sum(ranks[a] for a in set(adapter) if a >= 0)
    products = sum(f * ranks[a] for f, a in zip(fresh, adapter) if a >= 0)
    adapted = sum(f for f, a in zip(fresh, adapter) if a >= 0)
    return {"bytes": sum(2 * weights * (n + m) + 2 * T * m * _BYTES[case["y"]] for m in _ms(case)) + 2 * adapted * n,
            "flops": sum(2 * products * (n + m) for m in _ms(case))}


# ---------------------------------------------------------------------------------------------------------------------
# The same results in 64 bits, row by row or request by request.
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "group":
        return None              # whole numbers
    return globals()["_exact_" + case["kind"]](globals()["_prepare_" + case["kind"]](case, _generator(seed)), case)


def _exact_norm(st, case):
    def norm(v, side):
        kind = case["norm_" + side]
        if kind is None:
            return v
        mean = v.sum(1, keepdim=True) / v.shape[1] if kind == "layer" else 0.0
        spread = ((v - mean) ** 2).sum(1, keepdim=True) / v.shape[1]
        v = (v - mean) / (spread + st["eps"]).sqrt() * st[side + "_weight"].double()
        return v + st[side + "_bias"].double() if kind == "layer" else v

    outs, sums = [], []
    for a in range(0, case["rows"], 512):
        s = norm(st["y"][a:a + 512].double(), "y")
        if st["gate"] is not None:
            w = (st["gate"] if case["gate"] == "channel" else st["gate"][a:a + 512]).double()
            s = s * {None: w, "sigmoid": torch.sigmoid(w), "silu": w * torch.sigmoid(w), "tanh": torch.tanh(w)}[case["act"]]
        s = s * st["scale"]
        if st["x"] is not None:
            s = s + st["x"][a:a + 512].double() * st["skip"]
            sums.append(s)
        outs.append(norm(s, "x"))
    return dict(sum=torch.cat(sums), out=torch.cat(outs)) if sums else dict(out=torch.cat(outs))


def _exact_adapt(st, case):
    start, ranks = st["q_start"].tolist(), st["rank"].tolist()
    outs = [y.double() for y in st["y"]]
    for r, a in enumerate(st["adapter"].tolist()):
        if a < 0:
            continue
        x, k = st["x"][start[r]:start[r + 1]].double(), ranks[a]
        for A, B, out in zip(st["A"], st["B"], outs):
            out[start[r]:start[r + 1]] += st["scale"][a].double() * (x @ A[a, :k].double().T) @ B[a, :, :k].double().T
    return outs


def _exact_score(st, case):
    found = []
    for r in range(0, case["rows"], 64):
        z = st["logits"][r:r + 64].double() * case["scale"]
        lp = torch.log_softmax(z, 1)
        entropy = -torch.special.xlogy(lp.exp(), lp.exp()).sum(1)
        found.append((lp.gather(1, st["tokens"][r:r + 64].long()), entropy, lp.sort(1, descending=True).values[:, :case["top"]]))
    logprob, entropy, best = (torch.cat(f) for f in zip(*found))
    return dict(logprob=logprob, entropy=entropy, top_token=None, top_logprob=best)
