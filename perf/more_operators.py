"""Token ends and expert rows of a language model: the calls they are measured by, and what each has to give.

Every case is one pass on tensors that are already on the GPU, as a training
or answering program holds them.  ``listed()`` are fixed sizes, ``draw()`` gives
more of the same ranges.  Kinds of case:

``embed_fwd``     rows of a vocabulary shard's table for a batch of token ids, scaled
                  (``sb_embed_fwd``).  Ids outside the shard, and the negative ids of
                  padding, give zero rows.
``embed_step``    the same and the table's gradient (``sb_embed_bwd``): dy summed by id, fp32.
``experts_fwd``   a batch's slots sorted by expert (``sb_expert_sort``), the tokens' rows laid
                  out in that order (``sb_expert_gather``), and the experts' output rows
                  brought back with their weights (``sb_expert_combine``).  What the experts
                  make of the rows is given.
``experts_step``  the same and its gradients: of the output rows and the weights
                  (``sb_expert_combine_bwd``), and of the tokens (``sb_expert_combine``
                  without weights on the rows' gradient).
``logp_fwd``      log-probabilities of given tokens, entropies and the most likely
                  alternatives (``sb_token_logp_fwd``).  Negative targets are padding.
``logp_step``     the same and the logits' gradient (``sb_token_logp_bwd``).
``route``         the same calls as a router uses them: narrow rows, no targets, the
                  probabilities of the best experts and the gradient through them.

The plain forms are torch products, sums, comparisons and indexing in fp32.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # A few sequences answer one token each: launches count.
        dict(name="embed_fwd_few_bf16", kind="embed_fwd", dtype="bf16", tokens=8, vocab=32000, width=1024,
             shards=1, pad=False, scale=1.0),
        # A worker's quarter of a vocabulary in fp32, odd sizes, a padded batch.
        dict(name="embed_step_odd_f32", kind="embed_step", dtype="f32", tokens=4099, vocab=12501, width=741,
             shards=4, pad=True, scale=1.0),
        # The largest table on a large batch.
        dict(name="embed_step_large_bf16", kind="embed_step", dtype="bf16", tokens=65536, vocab=131072, width=2048,
             shards=1, pad=False, scale=32.0),
        # Sixteen sequences answer one token each through two of eight experts.
        dict(name="experts_fwd_few_bf16", kind="experts_fwd", dtype="bf16", tokens=16, top=2, experts=8, width=1024,
             shards=1),
        # fp32, odd sizes, half of the experts on another worker.
        dict(name="experts_step_odd_f32", kind="experts_step", dtype="f32", tokens=1777, top=3, experts=11, width=741,
             shards=2),
        # An ordinary training batch.
        dict(name="experts_step_bf16", kind="experts_step", dtype="bf16", tokens=8192, top=2, experts=8, width=2048,
             shards=1),
        # The largest: many small experts, eight for each token.
        dict(name="experts_step_large_bf16", kind="experts_step", dtype="bf16", tokens=32768, top=8, experts=128,
             width=2048, shards=1),
        # One sequence answers one token, its five best alternatives beside it.
        dict(name="logp_fwd_one_row_bf16", kind="logp_fwd", dtype="bf16", rows=1, classes=32000, top=5, masked=False),
        # Scoring of a batch in fp32, odd sizes, a part of the vocabulary ruled out.
        dict(name="logp_fwd_odd_f32", kind="logp_fwd", dtype="f32", rows=333, classes=50001, top=20, masked=True),
        # A training step on a padded batch.
        dict(name="logp_step_bf16", kind="logp_step", dtype="bf16", rows=2048, classes=32000, top=0, masked=False),
        # The largest vocabulary on a large batch, with alternatives.
        dict(name="logp_step_large_bf16", kind="logp_step", dtype="bf16", rows=4096, classes=131072, top=8,
             masked=False),
        # A router's rows in fp32: the best eight of 128 experts.
        dict(name="route_f32", kind="route", dtype="f32", rows=32768, classes=128, top=8, masked=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("embed_fwd", "embed_step", "experts_fwd", "experts_step", "logp_fwd", "logp_step", "route"))
    c = dict(kind=kind, dtype=rng.choice(("f32", "bf16")))
    e = SIZE[c["dtype"]]
    if kind in ("embed_fwd", "embed_step"):
        c["width"] = _log(rng, 64, 4096)
        if rng.random() < 0.6:                  # most widths are multiples of 64, the others anything
            c["width"] = c["width"] // 64 * 64
        c["tokens"] = _log(rng, 1, min(65536, 65536 * 2048 * 2 // (c["width"] * e)))
        c["vocab"] = _log(rng, 1000, min(131072, 131072 * 2048 // c["width"]))
        c["shards"], c["pad"], c["scale"] = rng.choice((1, 1, 2, 4)), rng.random() < 0.5, rng.choice((1.0, 32.0, 0.3))
    elif kind in ("experts_fwd", "experts_step"):
        c["width"] = _log(rng, 64, 4096)
        if rng.random() < 0.6:
            c["width"] = c["width"] // 64 * 64
        c["shards"] = rng.choice((1, 1, 2, 4))
        c["experts"] = _log(rng, 2, 256)
        c["top"] = rng.randint(1, min(8, c["experts"]))
        c["tokens"] = _log(rng, 1, min(32768, 32768 * 8 * 2048 * 2 // (c["top"] * c["width"] * e)))
    elif kind == "route":
        c["classes"] = rng.randint(4, 512)
        c["top"], c["masked"] = rng.randint(1, min(8, c["classes"])), False
        c["rows"] = _log(rng, 1, 32768)
    else:
        c["classes"] = _log(rng, 1000, 131072)
        c["top"], c["masked"] = rng.choice((0, 1, 5, 8, 20)), rng.random() < 0.3
        c["rows"] = _log(rng, 1, min(4096, 4096 * 131072 * 2 // (c["classes"] * e)))
    return c


# ------------------------------------------------------------------ embedding --
def _frequencies(case):
    """Of the ranks of a whole vocabulary: the n-th word in use falls off as 1 / n."""
    p = 1.0 / (torch.arange(case["vocab"] * case["shards"], dtype=torch.float64) + 2.7)
    return p / p.sum()


def _prepare_embed(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, v, d, dt = case["tokens"], case["vocab"], case["width"], TYPES[case["dtype"]]
    whole = v * case["shards"]
    first = v * (case["shards"] // 2)
    cdf = _frequencies(case).to(DEV).cumsum(0)
    rank = torch.searchsorted(cdf, torch.rand(n, generator=g, device=DEV, dtype=torch.float64)).clamp(max=whole - 1)
    ids = torch.randperm(whole, generator=g, device=DEV)[rank].to(torch.int32)
    if case["pad"]:                             # an eighth of the batch, at its end
        ids[n - n // 8:] = -1
    s = {"case": case, "ids": ids, "first": first,
         "table": torch.randn((v, d), generator=g, device=DEV).to(dt)}
    if case["kind"] == "embed_step":
        s["dy"] = torch.randn((n, d), generator=g, device=DEV).to(dt)
    if own:
        from paper_2112_15317_amd import sb
        s["desc"] = sb.embed_desc(n, v, d, sb.SB_BF16 if case["dtype"] == "bf16" else sb.SB_F32, first=first,
                                  scale=case["scale"])
        s["y"] = torch.empty((n, d), dtype=dt, device=DEV)
        if case["kind"] == "embed_step":
            s["dtable"] = torch.empty((v, d), dtype=torch.float32, device=DEV)
            s["ws"] = torch.empty((max(sb.sb_embed_workspace_bytes(s["desc"]), 256),), dtype=torch.uint8, device=DEV)
    return s


def _plain_embed(s):
    case, dt = s["case"], s["table"].dtype
    at = s["ids"].long() - s["first"]
    inside = (at >= 0) & (at < case["vocab"])
    at = torch.where(inside, at, 0)
    keep = inside[:, None].float()
    y = (s["table"][at].float() * case["scale"] * keep).to(dt)
    if case["kind"] == "embed_fwd":
        return {"y": y}
    dtable = torch.zeros((case["vocab"], case["width"]), device=DEV)
    dtable.index_add_(0, at, s["dy"].float() * keep)
    return {"y": y, "dtable": dtable * case["scale"]}


def _own_embed(s):
    from paper_2112_15317_amd import sb
    sb.sb_embed_fwd(s["desc"], s["table"], s["ids"], s["y"])
    if "dtable" not in s:
        return {"y": s["y"]}
    sb.sb_embed_bwd(s["desc"], s["ids"], s["dy"], s["dtable"], False, s["ws"])
    return {"y": s["y"], "dtable": s["dtable"]}


def _exact_embed(case, seed):
    s = _prepare_embed(case, seed)
    d = torch.float64
    v = case["vocab"]
    # One row more than the table has stands for every id that is not the shard's.
    at = s["ids"].long() - s["first"]
    at[(s["ids"].long() < s["first"]) | (s["ids"].long() >= s["first"] + v)] = v
    longer = torch.cat([s["table"], s["table"].new_zeros(1, case["width"])])
    y = longer.index_select(0, at).to(d) * case["scale"]
    if case["kind"] == "embed_fwd":
        return {"y": y}
    sums = torch.zeros((v + 1, case["width"]), dtype=d, device=DEV)
    sums.index_put_((at,), s["dy"].to(d) * case["scale"], accumulate=True)
    return {"y": y, "dtable": sums[:v]}


# -------------------------------------------------------------------- experts --
def _prepare_experts(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, k, e, d, dt = case["tokens"], case["top"], case["experts"], case["width"], TYPES[case["dtype"]]
    first = e * (case["shards"] // 2)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)
    # The router's scores: some experts are in demand more than others.
    score = normal(n, e * case["shards"]) + 0.5 * normal(e * case["shards"])
    best, ids = torch.topk(score, k, dim=1)
    s = {"case": case, "ids": ids.to(torch.int32).contiguous(), "first": first,
         "weights": torch.softmax(best, 1).contiguous(),
         "x": normal(n, d).to(dt), "ys": normal(n * k, d).to(dt)}
    if case["kind"] == "experts_step":
        s["dy"], s["dxs"] = normal(n, d).to(dt), normal(n * k, d).to(dt)
    if own:
        from paper_2112_15317_amd import sb
        i32 = dict(dtype=torch.int32, device=DEV)
        s["desc"] = sb.expert_desc(n, k, e, d, sb.SB_BF16 if case["dtype"] == "bf16" else sb.SB_F32, first=first)
        s["place"], s["offsets"] = torch.empty((n, k), **i32), torch.empty((e + 1,), **i32)
        s["y"] = torch.empty((n, d), dtype=dt, device=DEV)
        # Rows behind the last expert's stay as they are.
        s["xs"] = torch.zeros((n * k, d), dtype=dt, device=DEV)
        if case["kind"] == "experts_step":
            s["dys"] = torch.zeros((n * k, d), dtype=dt, device=DEV)
            s["dx"] = torch.empty((n, d), dtype=dt, device=DEV)
            s["dweights"] = torch.empty((n, k), dtype=torch.float32, device=DEV)
        s["ws"] = torch.empty((max(sb.sb_expert_workspace_bytes(s["desc"]), 256),), dtype=torch.uint8, device=DEV)
    return s


def _plain_experts(s):
    case, dt = s["case"], s["x"].dtype
    n, k, e = case["tokens"], case["top"], case["experts"]
    slot = s["ids"].reshape(-1).long() - s["first"]
    here = torch.arange(e, device=DEV)[:, None] == slot                       # [experts][slots]
    before = here.int().cumsum(1)                                             # of a slot's expert, up to it
    offsets = torch.zeros(e + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = before[:, -1].cumsum(0)
    place = ((before - 1 + offsets[:e, None]) * here).sum(0)
    inside = here.any(0)
    place = torch.where(inside, place, -1).int()
    got = {"place": place.view(n, k), "offsets": offsets}
    at, keep = place.clamp(min=0).long(), inside[:, None].float()
    spare = torch.where(inside, place, n * k).long()                          # a row more takes what is not kept

    def lay_out(rows):
        wide = torch.zeros((n * k + 1, case["width"]), dtype=dt, device=DEV)
        wide[spare] = rows
        return wide[:-1]
    got["xs"] = lay_out(s["x"][torch.arange(n * k, device=DEV) // k])
    rows = s["ys"][at].float() * keep
    w = s["weights"].reshape(-1, 1)
    got["y"] = (rows * w).view(n, k, -1).sum(1).to(dt)
    if case["kind"] == "experts_fwd":
        return got
    dy = s["dy"].float()[:, None, :]
    got["dys"] = lay_out((dy * w.view(n, k, 1)).reshape(n * k, -1).to(dt))
    got["dweights"] = (rows.view(n, k, -1) * dy).sum(2)
    got["dx"] = (s["dxs"][at].float() * keep).view(n, k, -1).sum(1).to(dt)
    return got


def _own_experts(s):
    from paper_2112_15317_amd import sb
    d = s["desc"]
    sb.sb_expert_sort(d, s["ids"], s["place"], s["offsets"], s["ws"])
    sb.sb_expert_gather(d, s["x"], s["place"], s["xs"])
    sb.sb_expert_combine(d, s["ys"], s["place"], s["weights"], s["y"])
    got = {"place": s["place"], "offsets": s["offsets"], "xs": s["xs"], "y": s["y"]}
    if "dys" in s:
        sb.sb_expert_combine_bwd(d, s["dy"], s["ys"], s["place"], s["weights"], s["dys"], s["dweights"])
        sb.sb_expert_combine(d, s["dxs"], s["place"], None, s["dx"])
        got.update(dys=s["dys"], dweights=s["dweights"], dx=s["dx"])
    return got


def _exact_experts(case, seed):
    s = _prepare_experts(case, seed)
    d = torch.float64
    n, k, e, first = case["tokens"], case["top"], case["experts"], s["first"]
    ids = s["ids"].reshape(-1).long()
    sorted_ids, order = torch.sort(ids, stable=True)
    bounds = torch.searchsorted(sorted_ids, torch.arange(first, first + e + 1, device=DEV))
    lo, hi = int(bounds[0]), int(bounds[-1])
    mine = order[lo:hi]                                                       # slot of each row
    place = torch.full((n * k,), -1, dtype=torch.int32, device=DEV)
    place[mine] = torch.arange(hi - lo, dtype=torch.int32, device=DEV)
    token = mine // k
    w = s["weights"].reshape(-1).to(d)[mine]
    xs = torch.zeros((n * k, case["width"]), dtype=d, device=DEV)
    xs[:hi - lo] = s["x"][token].to(d)
    y = torch.zeros((n, case["width"]), dtype=d, device=DEV)
    y.index_add_(0, token, s["ys"][:hi - lo].to(d) * w[:, None])
    got = {"place": place.view(n, k), "offsets": (bounds - lo).int(), "xs": xs, "y": y}
    if case["kind"] == "experts_fwd":
        return got
    rows_dy = s["dy"].to(d)[token]
    dys = torch.zeros_like(xs)
    dys[:hi - lo] = rows_dy * w[:, None]
    dweights = torch.zeros(n * k, dtype=d, device=DEV)
    dweights[mine] = torch.linalg.vecdot(rows_dy, s["ys"][:hi - lo].to(d))
    dx = torch.zeros_like(y)
    dx.index_add_(0, token, s["dxs"][:hi - lo].to(d))
    return {**got, "dys": dys, "dweights": dweights.view(n, k), "dx": dx}


# ---------------------------------------------------------- log-probabilities --
def _prepare_logp(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    m, v, k, dt = case["rows"], case["classes"], case["top"], TYPES[case["dtype"]]
    z = torch.randn((m, v), generator=g, device=DEV)
    if case["kind"] != "route":
        # Sure of some tokens, in doubt over others.
        z *= 1 + 2 * torch.rand((m, 1), generator=g, device=DEV)
    s = {"case": case, "targets": None}
    if case["kind"] != "route":
        t = torch.randint(0, v, (m,), generator=g, device=DEV)
        # Every second row puts its token ahead of the others.
        z[torch.arange(0, m, 2, device=DEV), t[::2]] += 12.0
        if case["masked"]:                      # classes that every row rules out, the targets apart
            out = torch.rand(v, generator=g, device=DEV) < 0.3
            out[t] = False
            z[:, out] = -math.inf
        s["targets"] = torch.where(torch.rand(m, generator=g, device=DEV) < 0.1, -1, t).to(torch.int32)
    s["z"] = z.to(dt)
    if case["kind"] == "logp_step":
        s["dlogp"] = torch.randn(m, generator=g, device=DEV) - 1.0
        s["dentropy"] = 0.1 * torch.randn(m, generator=g, device=DEV)
    if case["kind"] == "route":
        s["dtop"] = torch.randn((m, k), generator=g, device=DEV)
    if own:
        from paper_2112_15317_amd import sb
        f32 = dict(dtype=torch.float32, device=DEV)
        s["desc"] = sb.token_logp_desc(m, v, k, sb.SB_BF16 if case["dtype"] == "bf16" else sb.SB_F32,
                                       probs=case["kind"] == "route")
        s["logp"] = None if case["kind"] == "route" else torch.empty((m,), **f32)
        s["entropy"] = None if case["kind"] == "route" else torch.empty((m,), **f32)
        s["stats"] = torch.empty((m, 2), **f32)
        s["top_ids"] = torch.empty((m, k), dtype=torch.int32, device=DEV) if k else None
        s["top"] = torch.empty((m, k), **f32) if k else None
        s["dz"] = None if case["kind"] == "logp_fwd" else torch.empty_like(s["z"])
        s["ws"] = torch.empty((max(sb.sb_token_logp_workspace_bytes(s["desc"]), 256),), dtype=torch.uint8, device=DEV)
    return s


def _plain_logp(s):
    case, k = s["case"], s["case"]["top"]
    z = s["z"].float()
    most = z.amax(1, keepdim=True)
    p = torch.exp(z - most)
    total = p.sum(1, keepdim=True)
    lsum = torch.log(total)
    p /= total
    logp = z - most - lsum
    got = {"stats": torch.cat([most, lsum], 1)}
    if k:
        # Larger values first, then lower indices: both in one whole number.
        bits = (z + 0.0).view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() << 32
        key |= 0x7fffffff - torch.arange(case["classes"], device=DEV)
        ids = 0x7fffffff - (torch.topk(key, k, dim=1).values & 0x7fffffff)
        del key, bits
        got["top_ids"] = ids.int()
        got["top"] = (p if case["kind"] == "route" else logp).gather(1, ids)
    if case["kind"] == "route":
        g = s["dtop"] * got["top"]
        return {**got, "dz": (-p * g.sum(1, keepdim=True)).scatter_add_(1, ids, g).to(s["z"].dtype)}
    t = s["targets"].long()[:, None]
    valid = t >= 0
    t = t.clamp(min=0)
    got["logp"] = torch.where(valid, logp.gather(1, t), 0.0)[:, 0]
    surprise = torch.where(p > 0, logp, 0.0)
    h = -(p * surprise).sum(1, keepdim=True)
    got["entropy"] = h[:, 0]
    if case["kind"] == "logp_fwd":
        return got
    g = torch.where(valid, s["dlogp"][:, None], 0.0)
    dz = -p * (g + s["dentropy"][:, None] * (surprise + h))
    return {**got, "dz": dz.scatter_add_(1, t, g).to(s["z"].dtype)}


def _own_logp(s):
    from paper_2112_15317_amd import sb
    sb.sb_token_logp_fwd(s["desc"], s["z"], s["targets"], s["logp"], s["entropy"], s["stats"], s["top_ids"], s["top"],
                         s["ws"])
    got = {"stats": s["stats"]}
    if s["top"] is not None:
        got.update(top_ids=s["top_ids"], top=s["top"])
    if s["logp"] is not None:
        got.update(logp=s["logp"], entropy=s["entropy"])
    if s["dz"] is not None:
        sb.sb_token_logp_bwd(s["desc"], s["z"], s["stats"], s["targets"], s.get("dlogp"), s["entropy"],
                             s.get("dentropy"), s["top_ids"], s["top"], s.get("dtop"), s["dz"])
        got["dz"] = s["dz"]
    return got


def _exact_logp(case, seed):
    s = _prepare_logp(case, seed)
    k = case["top"]
    z = s["z"].to(torch.float64)
    rows = torch.arange(case["rows"], device=DEV)
    most = z.max(1).values
    lsum = torch.logsumexp(z, 1) - most
    got = {"stats": torch.stack([most, lsum], 1)}
    lp = torch.log_softmax(z, 1)
    p = torch.softmax(z, 1)
    if k:
        ids = torch.sort(s["z"], dim=1, descending=True, stable=True).indices[:, :k]
        got["top_ids"] = ids.int()
        got["top"] = (p if case["kind"] == "route" else lp)[rows[:, None], ids]
    # What reaches the log-probabilities, then through them the logits.
    grad = torch.zeros_like(z)
    if case["kind"] == "route":
        grad[rows[:, None], ids] = s["dtop"].to(grad) * got["top"]
    else:
        real = rows[s["targets"] >= 0]
        t = s["targets"][real].long()
        got["logp"] = torch.zeros_like(most)
        got["logp"][real] = lp[real, t]
        got["entropy"] = torch.special.entr(p).sum(1)
        if case["kind"] == "logp_fwd":
            return got
        grad[real, t] = s["dlogp"][real].to(grad)
        grad += s["dentropy"].to(grad)[:, None] * (torch.special.entr(p) - p)
    grad -= p * grad.sum(1, keepdim=True)
    return {**got, "dz": grad}


# --------------------------------------------------------------------- the file --
def _of(case, embed, experts, logp):
    return embed if case["kind"][:5] == "embed" else experts if case["kind"][:7] == "experts" else logp


def prepare(case, seed):
    return _of(case, _prepare_embed, _prepare_experts, _prepare_logp)(case, seed)


def run(state):
    if own:
        return _of(state["case"], _own_embed, _own_experts, _own_logp)(state)
    return _of(state["case"], _plain_embed, _plain_experts, _plain_logp)(state)


def exact(case, seed):
    return _of(case, _exact_embed, _exact_experts, _exact_logp)(case, seed)


def _work_embed(case):
    n, d, e = case["tokens"], case["width"], SIZE[case["dtype"]]
    used = n - (n // 8 if case["pad"] else 0)
    # Rows of the table that such a batch names, on average: each is read once.
    rows = float((1 - torch.exp(used * torch.log1p(-_frequencies(case)))).sum()) / case["shards"]
    fwd = 4 * n + e * d * (rows + n)
    if case["kind"] == "embed_fwd":
        return {"bytes": int(fwd), "flops": n * d}
    # dy of the shard's ids, every row of the gradient.
    return {"bytes": int(fwd + e * d * used / case["shards"] + 4 * case["vocab"] * d), "flops": 3 * n * d}


def _work_experts(case):
    n, k, d, e = case["tokens"], case["top"], case["width"], SIZE[case["dtype"]]
    rows = n * k // case["shards"]              # of the experts that are here, on average
    # ids in, places out; x in, xs out; ys and weights in, y out.
    fwd = 12 * n * k + e * d * (2 * n + 2 * rows)
    if case["kind"] == "experts_fwd":
        return {"bytes": fwd, "flops": 2 * rows * d}
    # dy in, dys out, dweights out (ys is read above); dxs in, dx out.
    return {"bytes": fwd + 4 * n * k + e * d * (2 * n + 2 * rows), "flops": 6 * rows * d}


def _work_logp(case):
    m, v, k, e = case["rows"], case["classes"], case["top"], SIZE[case["dtype"]]
    fwd = e * m * v + m * (8 * k + 8)
    if case["kind"] == "logp_fwd":
        return {"bytes": fwd + 12 * m, "flops": 6 * m * v}
    return {"bytes": fwd + e * m * v + 4 * m * (k if case["kind"] == "route" else 5), "flops": 12 * m * v}


def work(case):
    return _of(case, _work_embed, _work_experts, _work_logp)(case)
