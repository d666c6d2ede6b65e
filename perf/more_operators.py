"""Performance cases of further calls around a verification: attention of draft trees whose requests share a long prefix, log
probabilities of what was emitted, the attention weight that cached positions gather, and the eviction of those that gather little.

A case is a dict of plain values; "kind" names the operator:
  "prefix"    mpv_prefix_attention  B trees (K chains of L2 nodes behind a trunk of L1), H query heads on KV cache heads of D values; G prefixes
                                    of plo to phi tokens (spare: some trees have none), contexts of lo to hi tokens of a tree's own behind
                                    it, pages of `page` tokens, window and sinks (0: none); own_shapes: a parent array for each tree,
                                    ragged: trees of fewer nodes in the batch; lse: the logarithms of the sums are wanted, too
  "logprobs"  mpv_token_logprobs    paths: of the emitted tokens of B trees, otherwise of a token for each of N rows of a request;
                                    logits over V tokens, `top` alternatives
  "scores"    mpv_score_positions   what the accepted nodes of B trees (paths of up to `deep`) give to contexts of lo to hi positions, in
                                    `layers` layers; per_head: a score for each cache head
  "evict"     mpv_evict_positions   requests with more than `trigger` positions are cut down to `budget`

Where `own` is false, run() computes the same with elementary torch operations.
"""

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _prefix(B, K, L1, L2, H, KV, D, dtype, G, plo, phi, lo, hi, page, window=0, sinks=0, spare=False, own_shapes=False, ragged=False,
            lse=False, name=None):
    c = dict(kind="prefix", B=B, K=K, L1=L1, L2=L2, H=H, KV=KV, D=D, dtype=dtype, G=G, plo=plo, phi=phi, lo=lo, hi=hi, page=page,
             window=window, sinks=sinks, spare=spare, own_shapes=own_shapes, ragged=ragged, lse=lse)
    return dict(c, name=name) if name else c


def _logprobs(B, N, V, dtype, top, paths, temperature=1.0, name=None):
    c = dict(kind="logprobs", B=B, N=N, V=V, dtype=dtype, top=top, paths=paths, temperature=temperature)
    return dict(c, name=name) if name else c


def _scores(layers, B, deep, H, KV, D, dtype, lo, hi, page, per_head, name=None):
    c = dict(kind="scores", layers=layers, B=B, deep=deep, H=H, KV=KV, D=D, dtype=dtype, lo=lo, hi=hi, page=page, per_head=per_head)
    return dict(c, name=name) if name else c


def _evict(layers, B, KV, D, dtype, lo, hi, page, budget, trigger, sinks, recent, per_head, name=None):
    c = dict(kind="evict", layers=layers, B=B, KV=KV, D=D, dtype=dtype, lo=lo, hi=hi, page=page, budget=budget, trigger=trigger, sinks=sinks,
             recent=recent, per_head=per_head)
    return dict(c, name=name) if name else c


def listed():
    return [
        # two requests with a short chain each behind one system prompt: latency
        _prefix(2, 1, 0, 3, 32, 8, 128, "bf16", 1, 1000, 1000, 1, 100, 16, name="prefix_two_requests"),
        # a serving batch of single tokens behind one long document
        _prefix(64, 1, 0, 0, 32, 8, 128, "bf16", 1, 8192, 8192, 16, 1024, 64, name="prefix_single_tokens"),
        # the benchmark batch's trees, 41 nodes each, behind four system prompts; the weights are asked for afterwards
        _prefix(256, 8, 0, 5, 32, 8, 128, "bf16", 4, 512, 2048, 64, 1024, 64, lse=True, name="prefix_v152k_root"),
        # odd sizes: a sliding window with sinks, prefixes of all lengths and requests without one, trees of different shapes and sizes
        _prefix(48, 4, 1, 3, 16, 4, 96, "f16", 5, 1, 2900, 0, 700, 24, window=2000, sinks=4, spare=True, own_shapes=True, ragged=True, lse=True,
                name="prefix_window_ragged"),
        # one request's emitted tokens, a small vocabulary: latency
        _logprobs(1, 7, 32000, "bf16", 5, True, name="logprobs_one_request"),
        # the benchmark batch's emitted tokens: the rows of the accepted paths among all rows
        _logprobs(256, 41, 151936, "bf16", 8, True, name="logprobs_v152k_root"),
        # prompts that are scored token by token, float32 rows at odd addresses, many alternatives
        _logprobs(16, 64, 128257, "f32", 20, False, temperature=0.7, name="logprobs_prompts_odd_f32"),
        # a single token of one request, one layer: latency
        _scores(1, 1, 0, 32, 8, 128, "bf16", 900, 900, 16, True, name="scores_one_token"),
        # after a verification, all layers of a model at once
        _scores(16, 16, 5, 32, 8, 128, "bf16", 500, 8192, 64, True, name="scores_all_layers"),
        # a few positions too many of one request: latency
        _evict(4, 1, 8, 128, "bf16", 1100, 1100, 16, 1000, 1000, 4, 64, True, name="evict_one_request"),
        # a batch that has outgrown its budget, a set of positions for each cache head
        _evict(8, 16, 8, 128, "bf16", 2048, 6000, 64, 2048, 2560, 4, 512, True, name="evict_batch"),
        # whole slots in float32, odd sizes, requests of all lengths
        _evict(8, 24, 3, 80, "f32", 0, 2500, 24, 700, 701, 3, 100, False, name="evict_slots_odd_f32"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _tree(rng, most):
    K, L1, L2 = rng.randint(1, 8), rng.choice([0, 0, 1, 2, 3]), rng.randint(1, 5)
    if rng.random() < 0.3:
        return 1, 0, 0                             # a single token
    while 1 + L1 + K * L2 > most:
        K -= 1
    return K, L1, L2


def draw(rng):
    kind = rng.choices(["prefix", "logprobs", "scores", "evict"], [5, 3, 3, 3])[0]
    dtype = rng.choices(["bf16", "f16", "f32"], [4, 2, 1])[0]
    KV, group, D = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 80, 96, 128, 192, 256])
    page = rng.choice([1, 16, 24, 32, 64, 128])
    row = KV * D * _BYTES[dtype]
    if kind == "prefix":
        K, L1, L2 = _tree(rng, 60)
        N = 1 + L1 + K * L2
        phi, hi = _spread(rng, 8, 16384), _spread(rng, 1, 4096)
        window = rng.choice([0, 0, 0, 128, 1000, 4096])
        # no more values gathered for the plain form, and no more multiplications, than the largest listed case has
        gathered = 2 * (phi + hi) * KV * D * 4
        flops = 4 * N * KV * group * D * (phi + hi + N) * (8 if dtype == "f32" else 1)
        B = _spread(rng, 1, max(1, min(256, 5_000_000_000 // gathered, 400_000_000_000 // flops)))
        return _prefix(B, K, L1, L2, KV * group, KV, D, dtype, rng.randint(1, max(1, min(8, B // 2))), rng.choice([0, 1, phi // 2, phi]), phi,
                       rng.choice([0, 1, hi // 4, hi]), hi, page, window, rng.choice([0, 1, 4, 16]) if window else 0, rng.random() < 0.3,
                       rng.random() < 0.3, rng.random() < 0.3, rng.random() < 0.5)
    if kind == "logprobs":
        V = _spread(rng, 1000, 262144)
        paths = rng.random() < 0.6
        N = rng.randint(1, 41) if paths else _spread(rng, 1, 64)
        B = _spread(rng, 1, max(1, min(256, 400_000_000 // (N * V))))
        return _logprobs(B, N, V, dtype, rng.choice([0, 1, 5, 8, 20, 64]), paths, rng.choice([1.0, 0.7, 1.3]))
    layers = rng.choice([1, 4, 16])
    hi = _spread(rng, 16, min(32768, 2_000_000_000 // (layers * row)))
    lo, per_head = rng.choice([0, 1, hi // 4, hi]), rng.random() < 0.7
    if kind == "scores":
        deep = rng.choice([0, 0, 1, 3, 5, 8])
        cost = layers * hi * max(row, 2 * KV * group * (deep + 1) * (8 if dtype == "f32" else 1))
        return _scores(layers, _spread(rng, 1, max(1, min(128, 3_000_000_000 // cost))), deep, KV * group, KV, D, dtype, lo, hi, page, per_head)
    budget = _spread(rng, 1, hi)
    sinks = rng.randint(0, min(4, budget))
    return _evict(layers, _spread(rng, 1, max(1, min(128, 800_000_000 // (layers * hi * row)))), KV, D, dtype, lo, hi, page, budget,
                  budget + rng.choice([0, 0, 1, budget // 4]), sinks, rng.randint(0, budget - sinks), per_head)


# ---------------------------------------------------------------- inputs


def _parents(case):
    parent, last = [-1], 0
    for _ in range(case["L1"]):
        parent.append(last)
        last = len(parent) - 1
    for _ in range(case["K"]):
        prev = last
        for _ in range(case["L2"]):
            parent.append(prev)
            prev = len(parent) - 1
    return parent


def _between(lo, hi, shape, gen, dev):
    return torch.randint(lo, hi + 1, shape, generator=gen, device=dev)


def _normal(gen, dev, t, *shape):
    return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32).to(t)


def _prepare_prefix(case, gen, dev):
    B, H, KV, D, G, page, t = case["B"], case["H"], case["KV"], case["D"], case["G"], case["page"], _DTYPES[case["dtype"]]
    parent = _parents(case)
    N = len(parent)
    context = _between(case["lo"], case["hi"], (B,), gen, dev)
    context[0] = case["hi"]
    length = _between(case["plo"], case["phi"], (G,), gen, dev)
    length[0] = case["phi"]
    # requests are ordered by their prefix, as a scheduler that shares them has them
    which = torch.sort(_between(-1 if case["spare"] else 0, G - 1, (B,), gen, dev))[0]
    pages, many = -(-case["hi"] // page) + 1, -(-case["phi"] // page)
    order = torch.randperm(B * pages + G * many, generator=gen, device=dev).to(torch.int32)
    rows = torch.tensor(parent, device=dev, dtype=torch.int32).repeat(B, 1)
    if case["own_shapes"] and N > 1:               # some nodes hang under an earlier node than the shared shape says
        other = (torch.rand(B, N, generator=gen, device=dev) * torch.arange(N, device=dev)).long().to(torch.int32)
        move = torch.rand(B, N, generator=gen, device=dev) < 0.2
        move[:, 0] = False
        rows = torch.where(move, other, rows)
    nodes = _between(1, N, (B,), gen, dev) if case["ragged"] else torch.full((B,), N, device=dev)
    qkv = _normal(gen, dev, t, B, N, H + 2 * KV, D)
    q = qkv[:, :, :H]                              # views of one projection's output, as a model has them
    q *= 1.5
    return dict(case=case, parent=parent, tree_parent=rows, num_nodes=nodes.to(torch.int32), context=context.to(torch.int32),
                table=order[:B * pages].view(B, pages), prefix_table=order[B * pages:].view(G, many), prefix_len=length.to(torch.int32),
                prefix_of=which.to(torch.int32), q=q, tree_k=qkv[:, :, H:H + KV], tree_v=qkv[:, :, H + KV:],
                cache_k=_normal(gen, dev, t, order.shape[0], page, KV, D), cache_v=_normal(gen, dev, t, order.shape[0], page, KV, D),
                out=torch.zeros(B, N, H, D, device=dev, dtype=t), lse=torch.zeros(B, N, H, device=dev) if case["lse"] else None, result=None)


def _prepare_logprobs(case, gen, dev):
    B, N, V, t = case["B"], case["N"], case["V"], _DTYPES[case["dtype"]]
    logits = torch.empty(B, N, V, device=dev, dtype=t)
    for n in range(N):                             # a row's logits: noise, and a few tokens that stand out
        z = torch.randn(B, V, generator=gen, device=dev) * 2.5
        z += 6.0 * (torch.rand(B, V, generator=gen, device=dev) < 20.0 / V)
        logits[:, n] = z.to(t)
    s = dict(case=case, logits=logits, result=None)
    if not case["paths"]:
        likely = logits.argmax(dim=-1)
        other = _between(0, V - 1, (B, N), gen, dev)
        s["tokens"] = torch.where(torch.rand(B, N, generator=gen, device=dev) < 0.7, likely, other).to(torch.int32)
        return s
    deep = max(1, min(5, N - 1))
    accepted = _between(0, min(deep, N - 1), (B,), gen, dev)
    step = torch.arange(deep, device=dev)
    # ascending nodes, as a path has them
    path = torch.rand(B, max(deep, N - 1), generator=gen, device=dev).argsort(dim=1)[:, :deep].sort(dim=1)[0] + 1
    at = torch.cat([torch.zeros(B, 1, device=dev, dtype=torch.int64), path], dim=1).clamp(max=N - 1)
    likely = logits[torch.arange(B, device=dev)[:, None], at].argmax(dim=-1)
    other = _between(0, V - 1, (B, deep + 1), gen, dev)
    tokens = torch.where(torch.rand(B, deep + 1, generator=gen, device=dev) < 0.7, likely, other)
    taken = step < accepted[:, None]
    return dict(s, accepted=accepted.to(torch.int32), path=torch.where(taken, path, -1).to(torch.int32),
                tokens=torch.where(taken, tokens[:, :deep], -1).to(torch.int32),
                bonus=tokens.gather(1, accepted[:, None])[:, 0].contiguous().to(torch.int32))


def _prepare_scores(case, gen, dev):
    layers, B, deep, H, KV, D, page, t = (case[k] for k in ("layers", "B", "deep", "H", "KV", "D", "page", "dtype"))
    t = _DTYPES[t]
    N = 2 * deep + 1                               # two chains from the root, of which one was accepted in part
    context = _between(case["lo"], case["hi"], (B,), gen, dev)
    context[0] = case["hi"]
    pages = -(-(case["hi"] + deep + 1) // page)
    accepted = _between(0, deep, (B,), gen, dev)
    step = torch.arange(max(1, deep), device=dev)
    path = 1 + deep * _between(0, 1, (B, 1), gen, dev) + step
    path = torch.where(step < accepted[:, None], path, -1)
    q = _normal(gen, dev, t, layers, B, N, H, D)
    q *= 1.5
    # what the attention of such queries finds: the keys are normal numbers, so the products are, too
    lse = torch.log(context + 1.0).view(1, B, 1, 1) + q.float().square().sum(dim=-1) / (2 * D)
    scores = torch.rand(layers, B, KV if case["per_head"] else 1, pages * page, generator=gen, device=dev)
    return dict(case=case, q=q, tree_k=_normal(gen, dev, t, layers, B, N, KV, D), cache_k=_normal(gen, dev, t, layers, B * pages, page, KV, D),
                table=torch.randperm(B * pages, generator=gen, device=dev).view(B, pages).to(torch.int32), context=context.to(torch.int32),
                lse=lse, scores=scores, accepted=accepted.to(torch.int32), path=path.to(torch.int32))


def _prepare_evict(case, gen, dev):
    layers, B, KV, D, page, t = case["layers"], case["B"], case["KV"], case["D"], case["page"], _DTYPES[case["dtype"]]
    context = _between(case["lo"], case["hi"], (B,), gen, dev)
    context[0] = case["hi"]
    width = -(-case["hi"] // page)
    total = B * width + 5
    order = torch.randperm(total, generator=gen, device=dev).to(torch.int32)
    free = torch.full((total,), -1, device=dev, dtype=torch.int32)
    free[:5] = order[B * width:]
    heads = KV if case["per_head"] else 1
    # few positions gather most of the weight; some have none at all
    scores = torch.exp(2.0 * torch.randn(layers, B, heads, width * page, generator=gen, device=dev))
    scores *= torch.rand(layers, B, heads, width * page, generator=gen, device=dev) > 0.05
    return dict(case=case, cache_k=_normal(gen, dev, t, layers, total, page, KV, D), cache_v=_normal(gen, dev, t, layers, total, page, KV, D),
                table=order[:B * width].view(B, width), context=context.to(torch.int32), scores=scores, free=free,
                free_count=torch.tensor([5], device=dev, dtype=torch.int32), scores_out=torch.zeros_like(scores), result=None)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    return globals()["_prepare_" + case["kind"]](case, gen, dev)


# ---------------------------------------------------------------- plain forms


def _closure(rows):
    """[B,N,N]: node m is node n or an ancestor of it."""
    N = rows.shape[1]
    nodes = torch.arange(N, device=rows.device)
    up = ((rows[:, :, None] == nodes) | (nodes[:, None] == nodes)).float()
    for _ in range(6):                             # squares reach 64 steps up
        up = (up @ up).clamp(max=1.0)
    return up > 0.5


def _plain_prefix(s):
    case = s["case"]
    page, KV, window, sinks = case["page"], case["KV"], case["window"], case["sinks"]
    B, N, H, D = s["q"].shape
    dev = s["q"].device
    L, P = case["hi"], case["phi"]
    up = _closure(s["tree_parent"])
    which = s["prefix_of"].long()
    before = torch.where(which >= 0, s["prefix_len"].long()[which.clamp(min=0)], 0)
    first, where = torch.arange(P, device=dev), torch.arange(L, device=dev)
    shared = s["prefix_table"].long()[which.clamp(min=0)][:, first // page] * page + first % page
    slot = torch.cat([shared, s["table"].long()[:, where // page] * page + where % page], dim=1)
    keys = torch.cat([s["cache_k"].view(-1, KV, D)[slot].float(), s["tree_k"].float()], dim=1).permute(0, 2, 1, 3)
    values = torch.cat([s["cache_v"].view(-1, KV, D)[slot].float(), s["tree_v"].float()], dim=1).permute(0, 2, 1, 3)
    context = s["context"].long()[:, None]
    at = before[:, None] + context + up.sum(dim=-1) - 1                           # a node's position
    place = torch.cat([first.expand(B, P), before[:, None] + where, at], dim=1)   # a key's
    cached = torch.cat([first < before[:, None], where < context], dim=1)
    there = torch.cat([cached[:, None].expand(B, N, P + L), up], dim=2)
    near = (place[:, None] > at[:, :, None] - window) | (place[:, None] < sinks) if window else torch.ones_like(there)
    seen = (there & near)[:, None, :, None]                                       # [B,1,N,1,P+L+N]
    q = s["q"].float().view(B, N, KV, H // KV, D).permute(0, 2, 1, 3, 4).reshape(B, KV, -1, D)
    score = (q @ keys.transpose(2, 3)).view(B, KV, N, H // KV, P + L + N) * D ** -0.5
    score = score.masked_fill(~seen, -math.inf)
    most = score.amax(dim=-1, keepdim=True)
    weight = torch.exp(score - most)
    total = weight.sum(dim=-1, keepdim=True)
    weight = weight / total
    out = weight.view(B, KV, -1, P + L + N) @ values
    out = out.view(B, KV, N, H // KV, D).permute(0, 2, 1, 3, 4).reshape(B, N, H, D).to(s["q"].dtype)
    real = torch.arange(N, device=dev) < s["num_nodes"][:, None]
    answer = {"out": torch.where(real[:, :, None, None], out, s["out"])}
    if case["lse"]:
        lse = (most + torch.log(total)).view(B, KV, N, H // KV).permute(0, 2, 1, 3).reshape(B, N, H)
        answer["lse"] = torch.where(real[:, :, None], lse, s["lse"])
    return answer


def _plain_logprobs(s):
    case = s["case"]
    B, N, V = s["logits"].shape
    dev = s["logits"].device
    top = case["top"]
    tree = torch.arange(B, device=dev)[:, None]
    if case["paths"]:
        width = s["path"].shape[1] + 1
        index = torch.arange(width, device=dev)
        length = s["accepted"].long()[:, None]
        real = index <= length
        node = torch.cat([torch.zeros(B, 1, device=dev, dtype=torch.int64), s["path"].long()], dim=1).clamp(min=0)
        token = torch.cat([s["tokens"].long(), s["bonus"].long()[:, None]], dim=1)
        token = torch.where(index == length, s["bonus"].long()[:, None], token)
    else:
        width = N
        real = torch.ones(B, N, device=dev, dtype=torch.bool)
        node = torch.arange(N, device=dev).expand(B, N)
        token = s["tokens"].long()
    raw = s["logits"][tree, node]
    token = token.clamp(min=0)[:, :, None]
    z = raw.float() / case["temperature"]
    z = z - z.amax(dim=-1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(dim=-1, dtype=torch.float64)
    entropy = torch.log(total) - (e * z).sum(dim=-1, dtype=torch.float64) / total
    shift = torch.log(total)[:, :, None]
    logprob = (z.gather(2, token) - shift)[:, :, 0]
    mine = raw.gather(2, token)
    better = (raw > mine) | ((raw == mine) & (torch.arange(V, device=dev) < token))
    answer = {"logprob": torch.where(real, logprob, 0.0).float(), "entropy": torch.where(real, entropy, 0.0).float(),
              "rank": torch.where(real, 1 + better.sum(dim=-1), -1).to(torch.int32)}
    if top:
        # (topk may take any of several equal logits: a stable sort does not)
        best = torch.sort(raw, dim=-1, descending=True, stable=True)[1][:, :, :top]
        chosen = z.gather(2, best) - shift
        answer["top_tokens"] = torch.where(real[:, :, None], best, -1).to(torch.int32)
        answer["top_logprobs"] = torch.where(real[:, :, None], chosen, -math.inf).float()
    return answer


def _plain_scores(s):
    case = s["case"]
    page, KV, H, D = case["page"], case["KV"], case["H"], case["D"]
    layers, B = s["q"].shape[:2]
    dev = s["q"].device
    L, W, group = case["hi"], s["scores"].shape[3], H // KV
    context, accepted = s["context"].long(), s["accepted"].long()
    node = torch.cat([torch.zeros(B, 1, device=dev, dtype=torch.int64), s["path"].long()], dim=1).clamp(min=0)
    R = node.shape[1]
    tree, row = torch.arange(B, device=dev)[:, None], torch.arange(R, device=dev)
    where = torch.arange(L, device=dev)
    slot = s["table"].long()[:, where // page] * page + where % page
    keys = torch.cat([s["cache_k"].view(layers, -1, KV, D)[:, slot].float(), s["tree_k"][:, tree, node].float()], dim=2)
    q = s["q"][:, tree, node].float().view(layers, B, R, KV, group, D).permute(0, 1, 3, 2, 4, 5).reshape(layers, B, KV, R * group, D)
    score = (q @ keys.permute(0, 1, 3, 4, 2)).view(layers, B, KV, R, group, L + R) * D ** -0.5
    lse = s["lse"][:, tree, node].view(layers, B, R, KV, group).permute(0, 1, 3, 2, 4)
    seen = torch.cat([(where < context[:, None])[:, None].expand(B, R, L), (row <= row[:, None]).expand(B, R, R)], dim=2)
    seen = seen & (row <= accepted[:, None])[:, :, None]
    weight = torch.exp(score - lse[..., None]).masked_fill(~seen[None, :, None, :, None], 0.0)
    given = weight.sum(dim=(3, 4))                                                # [layers,B,KV,L+R]
    if not case["per_head"]:
        given = given.sum(dim=2, keepdim=True)
    place = torch.arange(W, device=dev)
    behind = place - context[:, None]                                             # of a position: its place in the path
    index = torch.where(behind < 0, place.clamp(max=max(0, L - 1)), L + behind.clamp(0, R - 1))
    added = given.gather(3, index[None, :, None].expand(layers, B, given.shape[2], W))
    new = (behind >= 0)[None, :, None]
    kept = torch.where(new, 0.0, 0.95 * s["scores"]) + added
    s["scores"].copy_(torch.where((behind <= accepted[:, None])[None, :, None], kept, s["scores"]))
    return s["scores"]


def _plain_evict(s):
    case = s["case"]
    page, budget, sinks, recent = case["page"], case["budget"], case["sinks"], case["recent"]
    layers, total, _, KV, D = s["cache_k"].shape
    B, W = s["scores"].shape[1], s["scores"].shape[3]
    heads = s["scores"].shape[2]
    dev = s["scores"].device
    context = s["context"].long()
    cut = context > case["trigger"]
    place = torch.arange(W, device=dev)
    safe = (place < sinks) | (place >= context[:, None] - recent)
    order = s["scores"].masked_fill(safe[None, :, None], math.inf)
    order = order.masked_fill((place >= context[:, None])[None, :, None], -math.inf)
    take = min(budget, W)
    best = torch.sort(order, dim=-1, descending=True, stable=True)[1][..., :take].sort(dim=-1)[0]     # [layers,B,heads,take]
    kept = torch.full((layers, B, heads, budget), -1, device=dev, dtype=torch.int32)
    kept[..., :take] = torch.where(cut[None, :, None, None], best, -1).to(torch.int32)
    # a request that is not cut down keeps everything where it is
    real = (place < torch.where(cut, budget, context)[:, None])[None, :, None]
    source = place.expand(layers, B, heads, W).clone()
    source[..., :take] = torch.where(cut[None, :, None, None], best, source[..., :take])
    s["scores_out"].copy_(torch.where(real, s["scores"].gather(3, source), s["scores_out"]))
    tree = torch.arange(B, device=dev).view(1, B, 1, 1)
    request, to = (cut[:, None] & (place < budget)).nonzero(as_tuple=True)
    layer = torch.arange(layers, device=dev).view(layers, 1, 1)
    head = torch.arange(KV, device=dev).view(1, 1, KV)
    origin = source[:, request, :, to].permute(1, 0, 2).expand(layers, request.shape[0], KV)         # [layers,moved,KV]
    old = s["table"].long()[request[None, :, None], origin // page] * page + origin % page
    new = (s["table"].long()[request, to // page] * page + to % page)[None, :, None]
    for cache in (s["cache_k"], s["cache_v"]):
        flat = cache.view(layers, total * page, KV, D)
        flat[layer, new, head] = flat[layer, old, head]
    column = torch.arange(s["table"].shape[1], device=dev)
    left = cut[:, None] & (column >= -(-budget // page)) & (column < -(-context // page)[:, None])
    count = s["free_count"].long()
    back = (count + left.flatten().cumsum(0) - 1).masked_fill(~left.flatten(), total)
    free = torch.cat([s["free"], s["free"][:1]]).scatter(0, back, s["table"].flatten())[:total]
    return {"cache_k": s["cache_k"], "cache_v": s["cache_v"], "scores": s["scores_out"], "kept": kept, "free_pages": free,
            "free_count": (count + left.sum()).to(torch.int32), "context_len": torch.where(cut, budget, context).to(torch.int32)}


# ---------------------------------------------------------------- the framework's calls


def _own_prefix(s):
    import paper_2602_16994_amd as mpv
    case = s["case"]
    if s["result"] is None:
        s["result"] = mpv.PrefixAttentionResult(out=s["out"], lse=s["lse"])
    r = s["result"]
    mpv.mpv_prefix_attention(s["parent"], s["q"], s["tree_k"], s["tree_v"], s["cache_k"], s["cache_v"], s["table"], s["context"],
                             s["prefix_of"], s["prefix_table"], s["prefix_len"], window=case["window"], sinks=case["sinks"],
                             num_nodes=s["num_nodes"] if case["ragged"] else None,
                             tree_parent=s["tree_parent"] if case["own_shapes"] else None, out=r)
    return {"out": r.out, "lse": r.lse} if case["lse"] else {"out": r.out}


def _own_logprobs(s):
    import paper_2602_16994_amd as mpv
    case = s["case"]
    if case["paths"]:
        s["result"] = mpv.mpv_token_logprobs(s["logits"], s["tokens"], temperature=case["temperature"], top=case["top"],
                                             accept_len=s["accepted"], path_nodes=s["path"], bonus_token=s["bonus"], out=s["result"])
    else:
        s["result"] = mpv.mpv_token_logprobs(s["logits"], s["tokens"], temperature=case["temperature"], top=case["top"], out=s["result"])
    r = s["result"]
    answer = {"logprob": r.logprob, "entropy": r.entropy, "rank": r.rank}
    return dict(answer, top_tokens=r.top_tokens, top_logprobs=r.top_logprobs) if case["top"] else answer


def _own_scores(s):
    import paper_2602_16994_amd as mpv
    mpv.mpv_score_positions(s["q"], s["tree_k"], s["cache_k"], s["table"], s["context"], s["lse"], s["scores"], accept_len=s["accepted"],
                            path_nodes=s["path"], decay=0.95)
    return s["scores"]


def _own_evict(s):
    import paper_2602_16994_amd as mpv
    case = s["case"]
    if s["result"] is None:
        s["result"] = mpv.EvictResult(scores=s["scores_out"])
    r = mpv.mpv_evict_positions(s["cache_k"], s["cache_v"], s["table"], s["context"], s["scores"], s["free"], s["free_count"], case["budget"],
                                trigger=case["trigger"], sinks=case["sinks"], recent=case["recent"], out=s["result"])
    return {"cache_k": s["cache_k"], "cache_v": s["cache_v"], "scores": r.scores, "kept": r.kept, "free_pages": s["free"],
            "free_count": r.free_count, "context_len": r.context_len}


_PLAIN = {"prefix": _plain_prefix, "logprobs": _plain_logprobs, "scores": _plain_scores, "evict": _plain_evict}
_OWN = {"prefix": _own_prefix, "logprobs": _own_logprobs, "scores": _own_scores, "evict": _own_evict}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    kind, B, e = case["kind"], case["B"], _BYTES[case["dtype"]]
    if kind == "logprobs":
        rows = B * (1 + max(1, min(5, case["N"] - 1)) / 2 if case["paths"] and case["N"] > 1 else 1 if case["paths"] else case["N"])
        return {"bytes": rows * (case["V"] * e + 8 * case["top"] + 16), "flops": 5.0 * rows * case["V"]}
    row = case["KV"] * case["D"]
    mean = case["lo"] + (case["hi"] - case["lo"]) / 2
    mean = (mean * (B - 1) + case["hi"]) / B                       # the first context is the longest one
    if kind == "prefix":
        N, G = 1 + case["L1"] + case["K"] * case["L2"], case["G"]
        prefix = case["plo"] + (case["phi"] - case["plo"]) / 2
        prefix = (prefix * (G - 1) + case["phi"]) / G
        share = G / (G + 1) if case["spare"] else 1.0              # of the trees, those that have a prefix
        near = case["window"] + case["sinks"] if case["window"] else prefix + mean
        seen = min(mean, near)
        ahead = min(prefix, near - seen)
        used = min(G, B * share)
        nodes = (N + 1) / 2 if case["ragged"] else N
        deep = case["L1"] + case["L2"] / 2 + 1
        return {"bytes": e * (2 * row * (used * ahead + B * (seen + nodes)) + 2 * B * nodes * case["H"] * case["D"])
                + (4 * B * nodes * case["H"] if case["lse"] else 0),
                "flops": 4.0 * B * nodes * case["H"] * case["D"] * (share * ahead + seen + deep)}
    heads = case["KV"] if case["per_head"] else 1
    if kind == "scores":
        rows = case["layers"] * B * (1 + case["deep"] / 2)
        return {"bytes": case["layers"] * B * mean * (row * e + 8 * heads) + rows * (case["H"] * (case["D"] * e + 4) + row * e),
                "flops": 2.0 * rows * mean * case["H"] * case["D"]}
    # requests longer than the trigger: their scores are read, and about the kept rows move
    span = max(1, case["hi"] - case["lo"] + 1)
    over = min(1.0, max(0, case["hi"] - case["trigger"]) / span)
    cut = (1 if case["hi"] > case["trigger"] else 0) + (B - 1) * over
    return {"bytes": case["layers"] * (cut * max(0, case["budget"] - case["sinks"]) * (4 * row * e + 8 * heads) + 4 * B * mean * heads) + 64,
            "flops": 0.0}


# ---------------------------------------------------------------- the definitions in 64 bits


def _exact_prefix(case, s):
    page, KV, window, sinks = case["page"], case["KV"], case["window"], case["sinks"]
    B, N, H, D = s["q"].shape
    group = H // KV
    out = s["out"].double()
    lse = s["lse"].double() if case["lse"] else None
    lengths, nodes, rows = s["context"].tolist(), s["num_nodes"].tolist(), s["tree_parent"].tolist()
    which, ahead = s["prefix_of"].tolist(), s["prefix_len"].tolist()
    for b in range(B):
        P = ahead[which[b]] if which[b] >= 0 else 0
        L = lengths[b]
        n_nodes = nodes[b]
        chain = [[0]]
        for n in range(1, n_nodes):
            chain.append(chain[rows[b][n]] + [n])
        use = torch.zeros(n_nodes, P + L + n_nodes, dtype=torch.bool)
        for n in range(n_nodes):
            lo = max(0, P + L + len(chain[n]) - window) if window else 0
            use[n, min(lo, P + L):P + L] = True
            use[n, :min(sinks, P + L)] = True
            for d, a in enumerate(chain[n]):
                if P + L + d >= lo or P + L + d < sinks:
                    use[n, P + L + a] = True
        use = use.to(s["q"].device).repeat_interleave(group, dim=0)
        own_pages = s["table"][b, : -(-L // page)].long()
        first_pages = s["prefix_table"][max(0, which[b]), : -(-P // page)].long()
        for h in range(KV):
            both = [torch.cat([cache[first_pages, :, h].reshape(-1, D)[:P], cache[own_pages, :, h].reshape(-1, D)[:L], nodes_of[b, :n_nodes, h]]).double()
                    for cache, nodes_of in ((s["cache_k"], s["tree_k"]), (s["cache_v"], s["tree_v"]))]
            q = s["q"][b, :n_nodes, h * group:(h + 1) * group].reshape(-1, D).double()
            x = torch.mm(q, both[0].t().contiguous()) / math.sqrt(D)
            x[~use] = -math.inf
            out[b, :n_nodes, h * group:(h + 1) * group] = torch.mm(torch.softmax(x, dim=1), both[1]).view(n_nodes, group, D)
            if lse is not None:
                lse[b, :n_nodes, h * group:(h + 1) * group] = torch.logsumexp(x, dim=1).view(n_nodes, group)
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _exact_logprobs(case, s):
    B, N, V = s["logits"].shape
    top, dev = case["top"], s["logits"].device
    width = s["path"].shape[1] + 1 if case["paths"] else N
    answer = {"logprob": torch.zeros(B, width, device=dev, dtype=torch.float64), "entropy": torch.zeros(B, width, device=dev, dtype=torch.float64),
              "rank": None}
    if top:
        answer["top_tokens"] = None
        answer["top_logprobs"] = torch.full((B, width, top), -math.inf, device=dev, dtype=torch.float64)
    tokens = s["tokens"].tolist()
    accepted = s["accepted"].tolist() if case["paths"] else [N - 1] * B
    path = s["path"].tolist() if case["paths"] else [list(range(1, N))] * B
    if case["paths"]:
        for b, x in enumerate(s["bonus"].tolist()):
            tokens[b] = tokens[b][:accepted[b]] + [x]
    for b in range(B):
        nodes = [0] + path[b][:accepted[b]]
        logp = torch.log_softmax(s["logits"][b, nodes].double() / case["temperature"], dim=1)
        at = torch.tensor(tokens[b][:len(nodes)], device=dev)
        answer["logprob"][b, :len(nodes)] = logp[torch.arange(len(nodes), device=dev), at]
        answer["entropy"][b, :len(nodes)] = -(logp.exp() * logp).sum(dim=1)
        if top:
            answer["top_logprobs"][b, :len(nodes), :min(top, V)] = torch.topk(logp, min(top, V), dim=1)[0]
    return answer


def _exact_scores(case, s):
    page, KV, D = case["page"], case["KV"], case["D"]
    group = case["H"] // KV
    scores = s["scores"].double()
    context, accepted, path = s["context"].tolist(), s["accepted"].tolist(), s["path"].tolist()
    for b in range(case["B"]):
        L, nodes = context[b], [0] + path[b][:accepted[b]]
        n = len(nodes)
        scores[:, b, :, :L] *= 0.95
        scores[:, b, :, L:L + n] = 0.0
        pages = s["table"][b, : -(-L // page)].long()
        hidden = torch.ones(n, L + n, dtype=torch.bool, device=scores.device).triu(L + 1).repeat_interleave(group, dim=0)
        for layer in range(case["layers"]):
            for h in range(KV):
                k = torch.cat([s["cache_k"][layer, pages, :, h].reshape(-1, D)[:L], s["tree_k"][layer, b, nodes, h]]).double()
                q = s["q"][layer, b, nodes, h * group:(h + 1) * group].reshape(-1, D).double()
                x = torch.mm(q, k.t().contiguous()) / math.sqrt(D) - s["lse"][layer, b, nodes, h * group:(h + 1) * group].reshape(-1, 1).double()
                w = torch.exp(x)
                w[hidden] = 0.0
                scores[layer, b, h if case["per_head"] else 0, :L + n] += w.sum(dim=0)
    return scores


def _exact_evict(case, s):
    page, budget, KV = case["page"], case["budget"], case["KV"]
    heads = s["scores"].shape[2]
    scores = s["scores_out"].double()
    cache = [s["cache_k"], s["cache_v"]]
    width = KV // heads
    for b, L in enumerate(s["context"].tolist()):
        if L <= case["trigger"]:
            scores[:, b, :, :L] = s["scores"][:, b, :, :L].double()
            continue
        slots = (s["table"][b].long()[:, None] * page + torch.arange(page, device=scores.device)).flatten()
        middle = budget - case["sinks"] - case["recent"]
        for layer in range(case["layers"]):
            for h in range(heads):
                row = s["scores"][layer, b, h, :L]
                # (numpy's and torch's stable sorts agree: the lowest index of equal scores comes first)
                inner = torch.sort(-row[case["sinks"]:L - case["recent"]], stable=True)[1][:middle] + case["sinks"]
                keep = torch.cat([torch.arange(case["sinks"], device=row.device), torch.sort(inner)[0],
                                  torch.arange(L - case["recent"], L, device=row.device)])
                scores[layer, b, h, :budget] = row[keep].double()
                for c in cache:
                    flat = c[layer].view(-1, KV, c.shape[-1])
                    mine = flat[:, h * width:(h + 1) * width]
                    mine[slots[:budget]] = mine[slots[keep]]
    return {"cache_k": cache[0], "cache_v": cache[1], "scores": scores, "kept": None, "free_pages": None, "free_count": None, "context_len": None}


def exact(case, seed):
    return globals()["_exact_" + case["kind"]](case, prepare(case, seed))
