"""mpv_extend_tables and mpv_append_paths against their definitions, and a run of all the calls around a verification as a serving
loop makes them (needs an MI355X).  Whole numbers and moved rows: everything has to be equal."""

import numpy as np
import pytest
import torch

import paper_2602_16994_amd as mpv
import workloads
from oracle import serving_oracle as so

pytestmark = pytest.mark.gpu


def gpu(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def make(B, width, size, context, free_share, seed, total=None):
    rng = np.random.default_rng(seed)
    have = [-(-max(c, 0) // size) for c in context]
    total = sum(min(h, width) for h in have) + free_share if total is None else total
    order = rng.permutation(total)
    table = np.full((B, width), -1)
    at = 0
    for b, h in enumerate(have):
        h = min(h, width)
        table[b, :h] = order[at:at + h]
        at += h
    free = np.full(total, -9)
    free[:total - at] = order[at:]
    return table, free, total - at


def check(table, context, new_len, free, count, size, slot_width, extra, packed, res=None, inplace=False):
    B = len(context)
    dev = dict(table=gpu(table), context=gpu(context), new=gpu(new_len), free=gpu(free), count=gpu([count]))
    slots = torch.full((slot_width,) if packed else (B, slot_width), -77, dtype=torch.int64, device="cuda")
    res = mpv.mpv_extend_tables(dev["table"], dev["context"], dev["new"], dev["free"], dev["count"], size, slots, extra=extra,
                                inplace=inplace, out=res)
    torch.cuda.synchronize()
    t, after, free2, count2, granted, rows, offsets = so.extend_tables(table, context, new_len, free, count, size, slot_width, extra, packed)
    assert np.array_equal(dev["table"].cpu().numpy(), t)
    assert res.context_len.tolist() == after.tolist() and res.granted.tolist() == granted.tolist()
    assert res.free_count.tolist() == [count2] and res.offsets.tolist() == offsets.tolist()
    got = dev["free"].cpu().numpy()
    assert got[:len(free2)].tolist() == free2 and np.array_equal(got[len(free2):], np.asarray(free)[len(free2):])
    pages = len(free)
    for b, row in enumerate(rows):
        want = [p * size + s if 0 <= p < pages else -1 for p, s in row]
        if packed:
            assert slots[int(offsets[b]):int(offsets[b + 1])].tolist() == want, b
        else:
            assert slots[b].tolist() == want + [-1] * (slot_width - len(want)), b
    if packed:
        assert (slots[int(offsets[-1]):] == -77).all()
    if inplace:
        assert res.context_len.data_ptr() == dev["context"].data_ptr() and dev["context"].tolist() == after.tolist()
        assert dev["count"].tolist() == [count2]
    else:
        assert dev["context"].tolist() == list(context) and dev["count"].tolist() == [count]
    return res


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("size", [1, 3, 16, 64])
@pytest.mark.parametrize("B,most", [(1, 1), (5, 4), (64, 6), (1100, 9), (2500, 3)])
def test_growth(B, most, size, packed):
    print("[case] growth", B, most, size, packed, flush=True)
    rng = np.random.default_rng(B + size)
    context = rng.integers(0, 40, B).tolist()
    new = rng.integers(0, most + 1, B).tolist()
    for b in rng.integers(0, B, max(1, B // 10)):
        new[b] = -1
    width = -(-60 // size)
    for share in (0, B // 2, 3 * B):               # pages for nobody, for some, for all
        table, free, count = make(B, width, size, context, share, seed=share + 1)
        check(table, context, new, free, count, size, B * (most + 1) if packed else most + 1, 1, packed)


@pytest.mark.parametrize("packed", [False, True])
def test_prompts(packed):
    print("[case] prompts", packed, flush=True)
    rng = np.random.default_rng(7)
    new = rng.integers(1, 3000, 40).tolist()
    new[3], new[11] = 0, -1
    context = [0] * 40
    context[11] = 500
    table, free, count = make(40, 200, 16, context, 40 * 190, seed=2)
    check(table, context, new, free, count, 16, sum(max(n, 0) for n in new) if packed else 3000, 0, packed)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("most", [50, 204, 205, 300, 819, 820, 5000])
def test_slot_maps_of_all_sizes(most, packed):
    """Filled by one workgroup or by many, with one slot, four or more of a thread."""
    print("[case] slot maps", most, packed, flush=True)
    rng = np.random.default_rng(most)
    new = rng.integers(most // 2, most + 1, 5).tolist()
    new[4] = most
    context = rng.integers(0, 100, 5).tolist()
    table, free, count = make(5, -(-(most + 100) // 24), 24, context, 5 * (most // 24 + 2), seed=most)
    check(table, context, new, free, count, 24, 5 * most if packed else most, 0, packed)


@pytest.mark.parametrize("packed", [False, True])
def test_many_requests_and_no_slots(packed):
    print("[case] no slots", packed, flush=True)
    new = [-1 if b % 7 == 0 else 0 for b in range(2000)]
    context = [b % 40 for b in range(2000)]
    table, free, count = make(2000, 3, 16, context, 5, seed=8)
    check(table, context, new, free, count, 16, 0, 0, packed)


def test_a_slot_map_that_is_too_small():
    print("[case] small map", flush=True)
    table, free, count = make(6, 10, 4, [0, 3, 4, 8, 1, 0], 50, seed=3)
    check(table, [0, 3, 4, 8, 1, 0], [5, 2, 7, 0, 3, 0], free, count, 4, 14, 0, True)      # request 2 fits exactly, request 4 does not
    table, free, count = make(6, 10, 4, [0, 3, 4, 8, 1, 0], 50, seed=3)
    check(table, [0, 3, 4, 8, 1, 0], [5, 2, 7, 0, 3, 0], free, count, 4, 5, 0, False)      # request 2 exceeds its row
    table, free, count = make(2, 10, 4, [0, 3], 50, seed=3)
    check(table, [0, 3], [0, -1], free, count, 4, 0, 0, True)                              # nothing to place


@pytest.mark.parametrize("packed", [False, True])
def test_numbers_out_of_range(packed):
    print("[case] out of range", packed, flush=True)
    context = [-3, 10 ** 6, 2 ** 31 - 1, 7, 10 ** 6]
    new = [3, 2, 5, 2 ** 31 - 1, -1]
    table, free, count = make(5, 4, 8, [0, 32, 32, 7, 32], 6, seed=4)
    check(table, context, new, free, count, 8, 40, 1, packed)
    table, free, count = make(3, 4, 8, [9, 9, 9], 6, seed=5)
    table[0, 1], table[1, 1] = -1, 10 ** 6         # a last page that cannot be: its slots are -1
    check(table, [9, 9, 9], [3, 10, 2], free, count, 8, 40, 0, packed)
    table, free, count = make(3, 4, 8, [9, 9, 9], 6, seed=6)
    check(table, [9, 9, 9], [3, 10, 2], free, 10 ** 6, 8, 40, 0, packed) if len(free) == count else None
    table, free, count = make(3, 4, 8, [9, 9, 9], 6, seed=6)
    check(table, [9, 9, 9], [20, 10, 2], free, -4, 8, 40, 0, packed)


def test_in_place_step_after_step():
    print("[case] in place", flush=True)
    rng = np.random.default_rng(8)
    B, size, width = 30, 16, 40
    context = rng.integers(0, 100, B).tolist()
    table, free, count = make(B, width, size, context, 120, seed=9)
    res = None
    for step in range(6):
        new = rng.integers(-1, 30, B).tolist()
        res = check(table, context, new, free, count, size, 31, 1, False, res=res, inplace=True)
        t, after, free2, count2, *_ = so.extend_tables(table, context, new, free, count, size, 31, 1, False)
        free[:len(free2)] = free2
        table, context, count = t, after.tolist(), count2
    assert len(set(free[:count]) | {int(p) for b in range(B) for p in table[b, :-(-context[b] // size)]}) \
        == count + sum(-(-c // size) for c in context)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("layers,B,N,KV,D,size", [(1, 1, 1, 1, 8, 1), (3, 5, 15, 2, 64, 16), (17, 4, 7, 1, 72, 24), (2, 40, 41, 8, 128, 64)])
def test_append(layers, B, N, KV, D, size, dtype):
    print("[case] append", layers, B, N, KV, D, size, dtype, flush=True)
    rng = np.random.default_rng(N)
    pages = B + 2
    deep = min(6, max(1, N - 1))
    accepted = rng.integers(0, min(deep, N - 1) + 1, B)
    path = np.full((B, deep), -1)
    for b in range(B):
        path[b, :accepted[b]] = np.sort(rng.choice(np.arange(1, N), accepted[b], replace=False))
    slots = rng.permutation(max(pages * size, B * (deep + 1)))[:B * (deep + 1)].reshape(B, deep + 1)
    slots[slots >= pages * size] = -1
    if B > 3:
        slots[1] = -1                              # a refused request
        slots[2, 0] = pages * size                 # behind the cache
        path[3, 0] = N                             # no such node
        accepted[3] = max(accepted[3], 1)
    for strided in (False, True):
        if strided:                                # slices of a projection; keys and values in one tensor
            tree = torch.randn(layers, B, N, 2 * KV, D, device="cuda").to(dtype)
            tk, tv = tree[:, :, :, :KV], tree[:, :, :, KV:]
            cache = torch.randn(layers, pages, 2, size, KV, D, device="cuda").to(dtype)
            ck, cv = cache[:, :, 0], cache[:, :, 1]
        else:
            tk, tv = torch.randn(2, layers, B, N, KV, D, device="cuda").to(dtype)
            ck, cv = torch.randn(2, layers, pages, size, KV, D, device="cuda").to(dtype)
        want_k, want_v = ck.clone(), cv.clone()
        for b in range(B):
            for i in range(int(accepted[b]) + 1):
                n, at = 0 if i == 0 else int(path[b, i - 1]), int(slots[b, i])
                if 0 <= at < pages * size and 0 <= n < N:
                    want_k[:, at // size, at % size] = tk[:, b, n]
                    want_v[:, at // size, at % size] = tv[:, b, n]
        args = (gpu(slots, torch.int64), gpu(accepted))
        if layers == 1 and strided:
            mpv.mpv_append_paths(tk[0], tv[0], ck[0], cv[0], *args, path_nodes=gpu(path))
        else:
            mpv.mpv_append_paths(tk, tv, ck, cv, *args, path_nodes=gpu(path))
        torch.cuda.synchronize()
        assert torch.equal(ck, want_k) and torch.equal(cv, want_v)


def test_append_of_chains():
    print("[case] append chains", flush=True)
    tk, tv = torch.randn(2, 2, 3, 4, 2, 8, device="cuda")
    ck, cv = torch.zeros(2, 2, 5, 4, 2, 8, device="cuda")
    slots = torch.tensor([[3, 4, 5, 6], [0, 1, -1, -1], [19, 18, 17, -1]], device="cuda")
    mpv.mpv_append_paths(tk, tv, ck, cv, slots, gpu([9, 1, 2]))     # longer than the chain: its four rows
    torch.cuda.synchronize()
    flat = ck.view(2, 20, 2, 8)
    for b, row in enumerate(slots.tolist()):
        for i, s in enumerate(row):
            if s >= 0:
                assert torch.equal(flat[:, s], tk[:, b, i])
    assert (flat[:, 7:17] == 0).all() and (flat[:, 2] == 0).all()


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("kind", ["trees", "chains"])
def test_a_serving_loop(kind, graph):
    """Steps of a loop over a two-layer model whose logits come from the attention's output: attention, verification, room in the cache,
    accepted rows.  After every step the cache holds, for each request, the keys and values of the tokens emitted so far, and the
    attention of the last one over it is that of the definition."""
    print("[case] loop", kind, graph, flush=True)
    torch.manual_seed(3)
    B, layers, H, KV, D, V, size, steps = 6, 2, 4, 2, 64, 97, 8, 5
    parent = mpv.delayed_tree(2, 1, 2) if kind == "trees" else [-1, 0, 1, 2]
    N, depth = len(parent), 3
    width = 8
    dev = "cuda"
    ck, cv = torch.zeros(2, layers, B * width, size, KV, D, device=dev, dtype=torch.bfloat16)
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    free = torch.randperm(B * width, device=dev).to(torch.int32)
    count = torch.tensor([B * width], dtype=torch.int32, device=dev)
    context = torch.zeros(B, dtype=torch.int32, device=dev)
    slots = torch.full((B, depth + 1), -1, dtype=torch.int64, device=dev)
    q = torch.empty(layers, B, N, H, D, device=dev, dtype=torch.bfloat16)
    tk, tv = torch.empty(2, layers, B, N, KV, D, device=dev, dtype=torch.bfloat16)
    head = torch.randn(H * D, V, device=dev)
    draft = torch.empty(B, N, V, device=dev)
    target = torch.empty(B, N, V, device=dev)
    tokens = torch.empty(B, N, dtype=torch.int32, device=dev)
    u = torch.empty(B, N, device=dev)
    held = {}

    def step():
        for layer in range(layers):
            held[layer] = mpv.mpv_tree_attention(parent, q[layer], tk[layer], tv[layer], ck[layer], cv[layer], table, context,
                                                 window=20, sinks=2, out=held.get(layer))
        if kind == "trees":
            held["res"] = mpv.mpv_verify(parent, tokens, target, draft, 1.0, u, mpv.MPV_METHOD_TRAVERSAL, out=held.get("res"))
        else:
            held["res"] = mpv.mpv_verify_chains(tokens, target, draft, u, out=held.get("res"))
        r = held["res"]
        held["tables"] = mpv.mpv_extend_tables(table, context, r.accept_len, free, count, size, slots, extra=1, inplace=True,
                                               out=held.get("tables"))
        mpv.mpv_append_paths(tk, tv, ck, cv, slots, r.accept_len, path_nodes=r.path_nodes)

    kept_k = [[] for _ in range(B)]
    kept_v = [[] for _ in range(B)]
    g = None
    for t in range(steps):
        for x in (q, tk, tv):
            x.normal_()
        target.normal_(); draft.copy_(target + 0.3 * torch.randn_like(target))
        q_draft = torch.softmax(draft, -1)
        for n in range(1, N):
            tokens[:, n] = torch.multinomial(q_draft[:, parent[n]], 1).squeeze(1).to(torch.int32)
        tokens[:, 0] = 0
        if kind == "chains":
            target.copy_(torch.softmax(target, -1)); draft.copy_(q_draft)
        u.uniform_()
        before = context.tolist()
        if graph and t == 1:                       # the buffers exist after the first step
            state = [x.clone() for x in (table, free, count, context, slots, ck, cv)]
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            for x, y in zip((table, free, count, context, slots, ck, cv), state):
                assert torch.equal(x, y)           # capturing ran nothing
        if g is not None:
            g.replay()
        else:
            step()
        torch.cuda.synchronize()
        r = held["res"]
        if kind == "trees":
            r.raise_on_timeout()
        for layer in range(layers):
            got = held[layer].out.double().cpu().numpy()
            f = [x.double().cpu().numpy() for x in (q[layer], tk[layer], tv[layer])]
            for b in range(B):
                k0 = np.array([k[layer] for k in kept_k[b]]).reshape(1, -1, KV, D)
                v0 = np.array([v[layer] for v in kept_v[b]]).reshape(1, -1, KV, D)
                want, A, *_ = so.tree_attention(f[0][b:b + 1], f[1][b:b + 1], f[2][b:b + 1], k0, v0, np.zeros((1, 1), int), [before[b]], [parent],
                                                [N], 20, 2, D ** -0.5) if before[b] else \
                    so.tree_attention(f[0][b:b + 1], f[1][b:b + 1], f[2][b:b + 1], np.zeros((0, 1, KV, D)), np.zeros((0, 1, KV, D)),
                                      np.zeros((1, 0), int), [0], [parent], [N], 20, 2, D ** -0.5)
                assert (np.abs(got[b] - want[0]) <= 2.0 ** -8 * np.abs(want[0]) + (2.0 ** -8 + 2.0 ** -12) * A[0]).all()
        for b in range(B):
            a = int(r.accept_len[b])
            path = [0] + r.path_nodes[b, :a].tolist()
            kept_k[b] += [tk[:, b, n].double().cpu().numpy() for n in path]
            kept_v[b] += [tv[:, b, n].double().cpu().numpy() for n in path]
            assert int(context[b]) == before[b] + a + 1 == len(kept_k[b])
            for j in range(len(kept_k[b])):
                page = int(table[b, j // size])
                assert np.array_equal(ck[:, page, j % size].double().cpu().numpy(), kept_k[b][j])
                assert np.array_equal(cv[:, page, j % size].double().cpu().numpy(), kept_v[b][j])
