"""Performance cases of the operators that stand around a verification in a serving loop: the attention of draft trees over a
paged cache, the verification of drafted chains from probabilities, block tables and slot maps, and the move of accepted rows
into the cache.

A case is a dict of plain values; "kind" names the operator:
  "attention"  mpv_tree_attention   B trees (K chains of L2 nodes behind a trunk of L1), H query heads on KV cache heads of D
                                    values, contexts of lo to hi tokens in pages of `page` tokens, window and sinks (0: none);
                                    own_shapes: a parent array for each tree, ragged: trees of fewer nodes in the batch
  "chains"     mpv_verify_chains    B chains of up to N - 1 drafted tokens over V tokens; draft: with the draft's distribution
  "tables"     mpv_extend_tables    B requests, new lengths of lo to hi tokens, contexts up to `context`; packed slot map or rows
  "append"     mpv_append_paths     the accepted paths of B trees into a cache of `layers` layers

Where `own` is false, run() computes the same with elementary torch operations.
"""

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _attention(B, K, L1, L2, H, KV, D, dtype, lo, hi, page, window=0, sinks=0, own_shapes=False, ragged=False, name=None):
    c = dict(kind="attention", B=B, K=K, L1=L1, L2=L2, H=H, KV=KV, D=D, dtype=dtype, lo=lo, hi=hi, page=page, window=window,
             sinks=sinks, own_shapes=own_shapes, ragged=ragged)
    return dict(c, name=name) if name else c


def _chains(B, N, V, dtype, draft, ragged, name=None):
    c = dict(kind="chains", B=B, N=N, V=V, dtype=dtype, draft=draft, ragged=ragged)
    return dict(c, name=name) if name else c


def _tables(B, lo, hi, context, page, packed, name=None):
    c = dict(kind="tables", B=B, lo=lo, hi=hi, context=context, page=page, packed=packed)
    return dict(c, name=name) if name else c


def _append(B, K, L1, L2, layers, KV, D, dtype, page, name=None):
    c = dict(kind="append", B=B, K=K, L1=L1, L2=L2, layers=layers, KV=KV, D=D, dtype=dtype, page=page)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one interactive request with a small tree: latency
        _attention(1, 2, 0, 3, 32, 8, 128, "bf16", 900, 900, 16, name="attention_one_request"),
        # single tokens (a step without a draft) against long contexts
        _attention(8, 1, 0, 0, 32, 8, 128, "bf16", 20000, 131072, 64, name="attention_single_token_long"),
        # a serving batch with a sliding window and sinks, wide heads, trees of distinct contexts of different sizes
        _attention(32, 8, 3, 3, 16, 4, 256, "f16", 1, 16384, 32, window=1024, sinks=4, own_shapes=True, ragged=True,
                   name="attention_window_sinks"),
        # float32 and odd sizes throughout: one query head a cache head, pages that are no power of two
        _attention(5, 4, 1, 3, 12, 12, 80, "f32", 0, 2500, 24, name="attention_odd_f32"),
        # the benchmark batch's trees: 41 nodes each, ordinary contexts
        _attention(256, 8, 0, 5, 32, 8, 128, "bf16", 512, 4096, 64, name="attention_v152k_root"),
        # one request, a few drafted tokens of a small vocabulary: latency
        _chains(1, 5, 32000, "f32", True, False, name="chains_one_request"),
        # a serving batch with a draft model
        _chains(64, 6, 128256, "f32", True, True, name="chains_v128k"),
        # a large batch with drafts looked up in the prompt (no draft distribution), an odd vocabulary in bf16
        _chains(256, 9, 151937, "bf16", False, True, name="chains_lookup_v152k"),
        # after a verification: one to a few tokens for each request of a batch, some requests finished
        _tables(64, 0, 5, 4096, 16, False, name="tables_after_verification"),
        # prompts enter: thousands of tokens for each request, one packed slot map
        _tables(300, 1, 8192, 1, 64, True, name="tables_prompts"),
        # accepted paths of a small batch, and of the benchmark batch, over the layers of a model
        _append(4, 4, 2, 3, 32, 8, 128, "bf16", 16, name="append_small"),
        _append(256, 8, 0, 5, 16, 8, 128, "bf16", 64, name="append_v152k_root"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _tree(rng, most):
    K, L1, L2 = rng.randint(1, 8), rng.choice([0, 0, 1, 2, 3]), rng.randint(1, 5)
    if rng.random() < 0.2:
        return 1, 0, 0                             # a single token
    while 1 + L1 + K * L2 > most:
        K -= 1
    return K, L1, L2


def draw(rng):
    kind = rng.choices(["attention", "chains", "tables", "append"], [5, 3, 2, 2])[0]
    dtype = rng.choices(["bf16", "f16", "f32"], [4, 2, 1])[0]
    if kind == "attention":
        K, L1, L2 = _tree(rng, 60)
        N = 1 + L1 + K * L2
        KV, group, D = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 80, 96, 128, 192, 256])
        hi = _spread(rng, 16, 65536)
        window = rng.choice([0, 0, 128, 1000, 4096])
        # no more cached values, and no more multiplications, than the largest listed case has
        cached = 2 * hi * KV * D * _BYTES[dtype]
        flops = 4 * N * KV * group * D * (hi + N) * (8 if dtype == "f32" else 1)
        B = _spread(rng, 1, max(1, min(256, 4_000_000_000 // cached, 600_000_000_000 // flops)))
        return _attention(B, K, L1, L2, KV * group, KV, D, dtype, rng.choice([0, 1, hi // 4, hi]), hi, rng.choice([1, 16, 24, 32, 64, 128]),
                          window, rng.choice([0, 1, 4, 16]) if window else 0, rng.random() < 0.3, rng.random() < 0.3)
    if kind == "chains":
        V = _spread(rng, 1000, 262144)
        return _chains(_spread(rng, 1, min(256, max(1, 400_000_000 // (9 * V)))), rng.randint(1, 9), V, dtype, rng.random() < 0.6,
                       rng.random() < 0.5)
    if kind == "tables":
        packed = rng.random() < 0.5
        return _tables(_spread(rng, 1, 512), 0, _spread(rng, 16, 4096) if packed else rng.randint(1, 16), _spread(rng, 1, 8192),
                       rng.choice([1, 16, 24, 64, 128]), packed)
    K, L1, L2 = _tree(rng, 60)
    return _append(_spread(rng, 1, 256), K, L1, L2, rng.choice([1, 8, 16]), rng.choice([1, 2, 8]), rng.choice([64, 80, 128]), dtype,
                   rng.choice([16, 24, 64]))


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


def _prepare_attention(case, gen, dev):
    B, H, KV, D, page, t = case["B"], case["H"], case["KV"], case["D"], case["page"], _DTYPES[case["dtype"]]
    parent = _parents(case)
    N = len(parent)
    context = _between(case["lo"], case["hi"], (B,), gen, dev)
    context[0] = case["hi"]
    pages = -(-case["hi"] // page) + 1             # the row of a block table has room for what the step will add
    table = torch.randperm(B * pages, generator=gen, device=dev).view(B, pages).to(torch.int32)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev).to(t)

    rows = torch.tensor(parent, device=dev, dtype=torch.int32).repeat(B, 1)
    if case["own_shapes"] and N > 1:               # some nodes hang under an earlier node than the shared shape says
        other = (torch.rand(B, N, generator=gen, device=dev) * torch.arange(N, device=dev)).long().to(torch.int32)
        move = torch.rand(B, N, generator=gen, device=dev) < 0.2
        move[:, 0] = False
        rows = torch.where(move, other, rows)
    nodes = _between(1, N, (B,), gen, dev) if case["ragged"] else torch.full((B,), N, device=dev)
    # queries lean towards some of the keys: a few tokens of a context carry most of the weight
    qkv = normal(B, N, H + 2 * KV, D)
    q = qkv[:, :, :H]                              # views of one projection's output, as a model has them
    q *= 1.5
    return dict(case=case, parent=parent, tree_parent=rows, num_nodes=nodes.to(torch.int32), context=context.to(torch.int32),
                table=table, q=q, tree_k=qkv[:, :, H:H + KV], tree_v=qkv[:, :, H + KV:],
                cache_k=normal(B * pages, page, KV, D), cache_v=normal(B * pages, page, KV, D),
                out=torch.zeros(B, N, H, D, device=dev, dtype=t), result=None)


def _prepare_chains(case, gen, dev):
    B, N, V, t = case["B"], case["N"], case["V"], _DTYPES[case["dtype"]]
    target = torch.empty(B, N, V, device=dev, dtype=t)
    draft = torch.empty(B, N, V, device=dev, dtype=t) if case["draft"] else None
    tokens = torch.zeros(B, N, device=dev, dtype=torch.int32)
    for n in range(N):
        z = torch.randn(B, V, generator=gen, device=dev) * 2.5
        z += 5.0 * (torch.rand(B, V, generator=gen, device=dev) < 20.0 / V)
        target[:, n] = torch.softmax(z + 0.8 * torch.randn(B, V, generator=gen, device=dev), dim=-1).to(t)
        q = torch.softmax(z, dim=-1)
        if case["draft"]:
            draft[:, n] = q.to(t)
            q = draft[:, n].float()
        if n + 1 < N:                              # the drafted token after node n; a lookup proposes likely ones
            q = q if case["draft"] else q ** 1.5
            tokens[:, n + 1] = torch.multinomial(q, 1, generator=gen).squeeze(1).to(torch.int32)
    nodes = _between(1, N, (B,), gen, dev) if case["ragged"] else torch.full((B,), N, device=dev)
    return dict(case=case, target=target, draft=draft, tokens=tokens, num_nodes=nodes.to(torch.int32),
                uniforms=torch.rand(B, N, generator=gen, device=dev), result=None)


def _prepare_tables(case, gen, dev):
    B, page = case["B"], case["page"]
    context = _between(0, case["context"], (B,), gen, dev)
    new = _between(case["lo"], case["hi"], (B,), gen, dev)
    new[torch.rand(B, generator=gen, device=dev) < 0.05] = -1      # finished requests
    width = -(-(case["context"] + case["hi"] + 1) // page)
    have = -(-context // page)
    # pages for all but the last few requests of a full cache: those have to wait (the others are held by other requests)
    total, held = B * width, int(have.sum())
    order = torch.randperm(total, generator=gen, device=dev).to(torch.int32)
    free_count = min(total - held, max(1, int(0.97 * int((new.clamp(min=0) // page + 1).sum()))))
    table = torch.full((B, width), -1, device=dev, dtype=torch.int32)
    used = torch.arange(width, device=dev) < have[:, None]
    table[used] = order[total - held:]
    free = torch.full((total,), -1, device=dev, dtype=torch.int32)
    free[:free_count] = order[:free_count]
    most = case["hi"] + 1
    slots = torch.full((B * most,) if case["packed"] else (B, most), -1, device=dev, dtype=torch.int64)
    return dict(case=case, table=table, context=context.to(torch.int32), new=new.to(torch.int32), free=free,
                free_count=torch.tensor([free_count], device=dev, dtype=torch.int32), slots=slots, result=None)


def _prepare_append(case, gen, dev):
    B, layers, KV, D, page, t = case["B"], case["layers"], case["KV"], case["D"], case["page"], _DTYPES[case["dtype"]]
    parent = _parents(case)
    N, depth = len(parent), case["L1"] + case["L2"]
    most = max(1, depth)
    pages = -(-B * (most + 1) // page) + 8

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32).to(t)

    accepted = _between(0, depth, (B,), gen, dev)
    chain = _between(0, case["K"] - 1, (B, 1), gen, dev)           # the chain that was accepted behind the trunk
    step = torch.arange(most, device=dev)
    path = torch.where(step < case["L1"], step + 1, 1 + case["L1"] + chain * case["L2"] + step - case["L1"])
    path = torch.where(step < accepted[:, None], path, -1)
    slots = torch.randperm(pages * page, generator=gen, device=dev)[:B * (most + 1)].view(B, most + 1).clone()
    slots[torch.arange(most + 1, device=dev) > accepted[:, None]] = -1
    return dict(case=case, tree_k=normal(layers, B, N, KV, D), tree_v=normal(layers, B, N, KV, D),
                cache_k=normal(layers, pages, page, KV, D), cache_v=normal(layers, pages, page, KV, D), slots=slots,
                accepted=accepted.to(torch.int32), path=path.to(torch.int32))


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


def _plain_attention(s):
    case = s["case"]
    page, KV, window, sinks = case["page"], case["KV"], case["window"], case["sinks"]
    B, N, H, D = s["q"].shape
    dev = s["q"].device
    L = case["hi"]
    up = _closure(s["tree_parent"])
    where = torch.arange(L, device=dev)
    slot = s["table"].long()[:, where // page] * page + where % page
    keys = torch.cat([s["cache_k"].view(-1, KV, D)[slot].float(), s["tree_k"].float()], dim=1).permute(0, 2, 1, 3)
    values = torch.cat([s["cache_v"].view(-1, KV, D)[slot].float(), s["tree_v"].float()], dim=1).permute(0, 2, 1, 3)
    at = s["context"].long()[:, None] + up.sum(dim=-1) - 1                        # a node's position
    place = torch.cat([where.expand(B, L), at], dim=1)                            # a key's
    there = torch.cat([(where < s["context"][:, None])[:, None].expand(B, N, L), up], dim=2)
    near = (place[:, None] > at[:, :, None] - window) | (place[:, None] < sinks) if window else torch.ones_like(there)
    seen = (there & near)[:, None, :, None]                                       # [B,1,N,1,L+N]
    q = s["q"].float().view(B, N, KV, H // KV, D).permute(0, 2, 1, 3, 4).reshape(B, KV, -1, D)
    score = (q @ keys.transpose(2, 3)).view(B, KV, N, H // KV, L + N) * D ** -0.5
    score = score.masked_fill(~seen, -math.inf)
    weight = torch.exp(score - score.amax(dim=-1, keepdim=True))
    weight = weight / weight.sum(dim=-1, keepdim=True)
    read = there.any(dim=1)[:, None, :, None]
    out = weight.view(B, KV, -1, L + N) @ values.masked_fill(~read, 0.0)
    out = out.view(B, KV, N, H // KV, D).permute(0, 2, 1, 3, 4).reshape(B, N, H, D).to(s["q"].dtype)
    real = torch.arange(N, device=dev) < s["num_nodes"][:, None]
    return torch.where(real[:, :, None, None], out, s["out"])


def _plain_chains(s):
    B, N, V = s["target"].shape
    dev = s["target"].device
    deep, tree = max(1, N - 1), torch.arange(B, device=dev)
    tokens, u = s["tokens"].long(), s["uniforms"].double()
    step = torch.arange(1, N, device=dev)
    drafted = tokens[:, 1:]
    p = s["target"][:, :-1].gather(2, drafted[:, :, None])[:, :, 0].double()
    q = s["draft"][:, :-1].gather(2, drafted[:, :, None])[:, :, 0].double() if s["draft"] is not None else torch.ones_like(p)
    passed = (u[:, 1:] * q < p) & (step < s["num_nodes"][:, None])
    length = passed.long().cumprod(dim=1).sum(dim=1)
    row = s["target"][tree, length].double()
    stopped = (length + 1 < s["num_nodes"])[:, None]
    next_token = tokens[tree, (length + 1).clamp(max=N - 1)]
    if s["draft"] is not None:
        away = s["draft"][tree, length].double()
    else:
        away = torch.zeros_like(row).scatter(1, next_token[:, None], math.inf)
    rest = (row - away).clamp(min=0.0)
    mass = torch.where(stopped & (rest.sum(dim=1, keepdim=True) > 0.0), rest, row)
    total = mass.cumsum(dim=1)
    bonus = (total <= u[:, :1] * total[:, -1:]).sum(dim=1)
    taken = torch.arange(1, deep + 1, device=dev) <= length[:, None]
    nodes = torch.where(taken, torch.arange(1, deep + 1, device=dev), -1)
    return {"accept_len": length.to(torch.int32), "path_nodes": nodes.to(torch.int32),
            "path_tokens": torch.where(taken, tokens.gather(1, nodes.clamp(min=0)), -1).to(torch.int32),
            "bonus_token": bonus.to(torch.int32)}


def _plain_tables(s):
    page = s["case"]["page"]
    B, width = s["table"].shape
    dev = s["table"].device
    pages = s["free"].shape[0]
    packed = s["slots"].dim() == 1
    old, new, table = s["context"].long(), s["new"].long(), s["table"].long()
    done = new < 0
    n = torch.where(done, 0, new + 1)
    have = -(-old // page)
    back = (torch.arange(width, device=dev) < have[:, None]) & done[:, None]
    at = (s["free_count"].long() + back.flatten().cumsum(0) - 1).masked_fill(~back.flatten(), pages)
    free = torch.cat([s["free"], s["free"][:1]]).scatter(0, at, s["table"].flatten())[:pages]
    count = s["free_count"].long() + back.sum()
    want = -(-(old + n) // page)
    never = done | (want > width)
    if not packed:
        never = never | (n > s["slots"].shape[1])
    need = (want - have).masked_fill(never, 0)
    asked = need.cumsum(0)
    granted = ~never & ((need == 0) | (asked <= count))
    if packed:
        granted = granted & (n.masked_fill(never, 0).cumsum(0) <= s["slots"].shape[0])
    given = torch.where(granted, n, torch.where(done, 0, -1))
    first = asked - need
    column = torch.arange(width, device=dev)
    fresh = (count - 1 - first[:, None] - (column - have[:, None])).clamp(0, pages - 1)
    is_new = granted[:, None] & (column >= have[:, None]) & (column < want[:, None])
    table = torch.where(is_new, free[fresh].long(), table)
    tokens = given.clamp(min=0)
    if packed:
        begin = torch.cat([tokens.new_zeros(1), tokens.cumsum(0)])
        index = torch.arange(s["slots"].shape[0], device=dev)
        row = torch.searchsorted(begin[1:], index, right=True).clamp(max=B - 1)
        where = old[row] + index - begin[row]
        slots = table[row, (where // page).clamp(max=width - 1)] * page + where % page
        slots = torch.where(index < begin[-1], slots, s["slots"])
    else:
        index = torch.arange(s["slots"].shape[1], device=dev)
        where = old[:, None] + index
        slots = table.gather(1, (where // page).clamp(max=width - 1)) * page + where % page
        slots = torch.where(index < tokens[:, None], slots, -1)
    answer = {"block_table": table.to(torch.int32), "context_len": torch.where(done, 0, old + tokens).to(torch.int32),
              "free_pages": free, "free_count": (count - need.masked_fill(~granted, 0).sum()).view(1).to(torch.int32),
              "granted": given.to(torch.int32), "slot_map": slots}
    if packed:
        answer["offsets"] = begin.to(torch.int32)
    return answer


def _plain_append(s):
    case = s["case"]
    layers, B, N, KV, D = s["tree_k"].shape
    most = s["slots"].shape[1]
    dev = s["slots"].device
    node = torch.cat([torch.zeros(B, 1, device=dev, dtype=torch.int64), s["path"].long()], dim=1)[:, :most]
    valid = (torch.arange(most, device=dev) <= s["accepted"][:, None]) & (s["slots"] >= 0)
    tree, step = valid.nonzero(as_tuple=True)
    slot, node = s["slots"][tree, step], node[tree, step]
    s["cache_k"].view(layers, -1, KV, D)[:, slot] = s["tree_k"][:, tree, node]
    s["cache_v"].view(layers, -1, KV, D)[:, slot] = s["tree_v"][:, tree, node]
    return {"cache_k": s["cache_k"], "cache_v": s["cache_v"]}


# ---------------------------------------------------------------- the framework's calls


def _own_attention(s):
    import paper_2602_16994_amd as mpv
    case = s["case"]
    if s["result"] is None:
        s["result"] = mpv.TreeAttentionResult(out=s["out"])
    mpv.mpv_tree_attention(s["parent"], s["q"], s["tree_k"], s["tree_v"], s["cache_k"], s["cache_v"], s["table"], s["context"],
                           window=case["window"], sinks=case["sinks"], num_nodes=s["num_nodes"] if case["ragged"] else None,
                           tree_parent=s["tree_parent"] if case["own_shapes"] else None, out=s["result"])
    return s["result"].out


def _own_chains(s):
    import paper_2602_16994_amd as mpv
    s["result"] = mpv.mpv_verify_chains(s["tokens"], s["target"], s["draft"], s["uniforms"],
                                        num_nodes=s["num_nodes"] if s["case"]["ragged"] else None, out=s["result"])
    r = s["result"]
    return {"accept_len": r.accept_len, "path_nodes": r.path_nodes, "path_tokens": r.path_tokens, "bonus_token": r.bonus_token}


def _own_tables(s):
    import paper_2602_16994_amd as mpv
    s["result"] = mpv.mpv_extend_tables(s["table"], s["context"], s["new"], s["free"], s["free_count"], s["case"]["page"], s["slots"],
                                        extra=1, out=s["result"])
    r = s["result"]
    answer = {"block_table": s["table"], "context_len": r.context_len, "free_pages": s["free"], "free_count": r.free_count,
              "granted": r.granted, "slot_map": s["slots"]}
    if s["slots"].dim() == 1:
        answer["offsets"] = r.offsets
    return answer


def _own_append(s):
    import paper_2602_16994_amd as mpv
    mpv.mpv_append_paths(s["tree_k"], s["tree_v"], s["cache_k"], s["cache_v"], s["slots"], s["accepted"], path_nodes=s["path"])
    return {"cache_k": s["cache_k"], "cache_v": s["cache_v"]}


_PLAIN = {"attention": _plain_attention, "chains": _plain_chains, "tables": _plain_tables, "append": _plain_append}
_OWN = {"attention": _own_attention, "chains": _own_chains, "tables": _own_tables, "append": _own_append}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    kind, B = case["kind"], case["B"]
    if kind == "attention":
        N = 1 + case["L1"] + case["K"] * case["L2"]
        mean = case["lo"] + (case["hi"] - case["lo"]) / 2
        mean = (mean * (B - 1) + case["hi"]) / B                   # the first context is the longest one
        seen = min(mean, case["window"] + case["sinks"]) if case["window"] else mean
        nodes = (N + 1) / 2 if case["ragged"] else N
        row, e = case["KV"] * case["D"], _BYTES[case["dtype"]]
        deep = case["L1"] + case["L2"] / 2 + 1
        return {"bytes": B * e * (2 * row * (seen + nodes) + 2 * nodes * case["H"] * case["D"]),
                "flops": 4.0 * B * nodes * case["H"] * case["D"] * (seen + deep)}
    if kind == "chains":
        rows = 2 if case["draft"] else 1
        return {"bytes": B * case["V"] * _BYTES[case["dtype"]] * rows, "flops": 2.0 * B * case["V"] * rows}
    if kind == "tables":
        tokens = B * (1 + (case["lo"] + case["hi"]) / 2)
        return {"bytes": 8 * tokens + 8 * tokens / case["page"] + 24 * B, "flops": 4.0 * tokens}
    rows = B * (1 + (case["L1"] + case["L2"]) / 2) * case["layers"] * 2
    return {"bytes": 2 * rows * case["KV"] * case["D"] * _BYTES[case["dtype"]], "flops": 0.0}


# ---------------------------------------------------------------- the definitions in 64 bits


def _exact_attention(case, s):
    page, KV, window, sinks = case["page"], case["KV"], case["window"], case["sinks"]
    B, N, H, D = s["q"].shape
    group = H // KV
    out = s["out"].double()
    lengths, nodes, rows = s["context"].tolist(), s["num_nodes"].tolist(), s["tree_parent"].tolist()
    for b in range(B):
        L = lengths[b]
        chain = [[0]]
        for n in range(1, nodes[b]):
            chain.append(chain[rows[b][n]] + [n])
        use = torch.zeros(nodes[b], L + nodes[b], dtype=torch.bool)
        for n in range(nodes[b]):
            p = L + len(chain[n]) - 1
            lo = max(0, p - window + 1) if window else 0
            use[n, min(lo, L):L] = True
            use[n, :min(sinks, L)] = True
            for d, a in enumerate(chain[n]):
                if L + d >= lo or L + d < sinks:
                    use[n, L + a] = True
        use = use.to(s["q"].device).repeat_interleave(group, dim=0)
        pages = s["table"][b, : -(-L // page)].long()
        for h in range(KV):
            k = torch.cat([s["cache_k"][pages, :, h].reshape(-1, D)[:L], s["tree_k"][b, :nodes[b], h]]).double()
            v = torch.cat([s["cache_v"][pages, :, h].reshape(-1, D)[:L], s["tree_v"][b, :nodes[b], h]]).double()
            q = s["q"][b, :nodes[b], h * group:(h + 1) * group].reshape(-1, D).double()
            e = torch.mm(q, k.t().contiguous()) / math.sqrt(D)
            e[~use] = -math.inf
            w = torch.softmax(e, dim=1)
            out[b, :nodes[b], h * group:(h + 1) * group] = torch.mm(w, v).view(nodes[b], group, D)
    return out


def _exact_chains(case, s):
    B, N = s["tokens"].shape
    tokens, u, nodes = s["tokens"].tolist(), s["uniforms"].double().cpu(), s["num_nodes"].tolist()
    deep = max(1, N - 1)
    length, path_nodes, path_tokens, bonus = [], [], [], []
    for b in range(B):
        a = 0
        while a + 1 < nodes[b]:
            x = tokens[b][a + 1]
            p = float(s["target"][b, a, x])
            q = float(s["draft"][b, a, x]) if case["draft"] else 1.0
            if not float(u[b, a + 1]) * q < p:
                break
            a += 1
        row = s["target"][b, a].double()
        if a + 1 < nodes[b]:
            rest = row.clone()
            if case["draft"]:
                rest = torch.relu(rest - s["draft"][b, a].double())
            else:
                rest[tokens[b][a + 1]] = 0.0
            row = rest if float(rest.sum()) > 0.0 else row
        c = torch.cumsum(row, 0)
        bonus.append(int(torch.searchsorted(c, c[-1:] * float(u[b, 0]), right=True)))
        length.append(a)
        path_nodes.append(list(range(1, a + 1)) + [-1] * (deep - a))
        path_tokens.append(tokens[b][1:a + 1] + [-1] * (deep - a))
    dev = s["tokens"].device

    def whole(x):
        return torch.tensor(x, device=dev, dtype=torch.int32)

    return {"accept_len": whole(length), "path_nodes": whole(path_nodes), "path_tokens": whole(path_tokens), "bonus_token": whole(bonus)}


def _exact_append(case, s):
    page = case["page"]
    path, slots = s["path"].tolist(), s["slots"].tolist()
    for b, accepted in enumerate(s["accepted"].tolist()):
        for i, n in enumerate(([0] + path[b])[:accepted + 1]):
            at = slots[b][i]
            s["cache_k"][:, at // page, at % page] = s["tree_k"][:, b, n]
            s["cache_v"][:, at // page, at % page] = s["tree_v"][:, b, n]
    return {"cache_k": s["cache_k"].double(), "cache_v": s["cache_v"].double()}


def exact(case, seed):
    if case["kind"] == "attention":
        return _exact_attention(case, prepare(case, seed))
    if case["kind"] == "chains":
        return _exact_chains(case, prepare(case, seed))
    if case["kind"] == "append":
        return _exact_append(case, prepare(case, seed))
    return None                                    # whole numbers: nothing is computed that could be rounded
