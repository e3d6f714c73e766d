"""The serving calls together: a server's loop of single-token steps over one page pool, with
requests that end and arrive, and a verification round whose targets are sampled."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps
from oracle.walk import walk_arrays

from test_gpu_decode import bound

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def host(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_server_loop(dtype):
    """Prompts are appended, then every step reserves a row, appends the new token's K and V,
    attends over the cache and samples the next token; requests end and new ones take their
    pages.  Pages, caches and tokens follow the oracle, which keeps plain Python lists."""
    B, Hq, Hkv, hd, pr, V, width, pages = 4, 8, 2, 64, 32, 600, 6, 14
    code = taps.BF16 if dtype == BF else taps.FP32
    g = torch.Generator(device="cuda").manual_seed(1)
    rng = np.random.default_rng(1)
    emb = torch.randn(V, (Hq + 2 * Hkv) * hd, generator=g, device="cuda").to(dtype)
    head = torch.randn(Hq * hd, V, generator=g, device="cuda") * 0.3
    T, top_p = np.float32([0.7, 0.0, 1.1, 1.0]), np.float32([0.9, 1.0, 1.0, 0.5])
    top_k = [0, 0, 30, 0]
    res = taps.PagedKVReserve(B, width, pages, pr, 40)
    app = taps.PagedKVAppend(Hkv, hd, pr, dtype=code)
    att = taps.PagedDecodeAttention(B, Hq, Hkv, hd, width * pr, pr, dtype=code)
    smp = taps.TokenSampler(B, 1, V, dtype=taps.FP32)
    Kp = torch.full((pages, pr, Hkv, hd), float("nan"), dtype=dtype, device="cuda")
    Vp = torch.full_like(Kp, float("nan"))
    table, held = np.zeros((B, width), np.int32), np.zeros(B, np.int32)
    free, n_free = rng.permutation(pages).astype(np.int32), pages
    t_dev, f_dev, h_dev, n_dev = i32(table), i32(free), i32(held), i32([n_free])
    rows = [[] for _ in range(B)]                 # each request's cached tokens
    prompt = [list(rng.integers(0, V, n)) for n in (40, 1, 33, 7)]
    todo = list(prompt)                           # tokens to append next
    ends = {3: 0, 5: 2, 6: 3}                     # step: request that ends after it
    for step in range(9):
        new = [len(x) for x in todo]
        ctx = [len(x) for x in rows]
        want = oracle.kv_reserve_paged(table, held, ctx, new, free, n_free, pr, 40)
        h_dev, n_dev, short, slots = res(t_dev, h_dev, i32(ctx), i32(new), f_dev, n_dev)
        table, held, free, n_free = want[0], want[1], want[2], want[3]
        np.testing.assert_array_equal(t_dev.cpu().numpy(), table)
        np.testing.assert_array_equal(f_dev.cpu().numpy(), free)
        np.testing.assert_array_equal(slots.cpu().numpy(), want[5])
        assert h_dev.tolist() == held.tolist() and n_dev.tolist() == [n_free]
        assert short.tolist() == [0] and want[4] == 0
        tok = np.zeros((B, 40), np.int64)
        for b in range(B):
            tok[b, :new[b]] = todo[b]
            rows[b] = rows[b] + todo[b]
        x = emb[torch.from_numpy(tok).cuda().view(-1)]
        k = x[:, Hq * hd:(Hq + Hkv) * hd].unflatten(1, (Hkv, hd))
        v = x[:, (Hq + Hkv) * hd:].unflatten(1, (Hkv, hd))
        app(k, v, slots, Kp, Vp)
        lens = np.array([len(r) for r in rows])
        last = [r[-1] if r else 0 for r in rows]
        q = emb[torch.tensor(last, device="cuda")][:, :Hq * hd].unflatten(1, (Hq, hd))
        O = att(q, Kp, Vp, t_dev, i32(lens))
        # the same attention over the token lists, without pages
        flat = torch.zeros(B, width * pr, 2 * Hkv, hd, dtype=dtype, device="cuda")
        for b, r in enumerate(rows):
            if r:
                flat[b, :len(r)] = emb[torch.tensor(r, device="cuda")][:, Hq * hd:].unflatten(1, (2 * Hkv, hd))
        ident = np.arange(B)[:, None]
        ref, A, D = oracle.decode_attention_paged(host(q), host(flat[:, :, :Hkv]), host(flat[:, :, Hkv:]),
                                                  ident.repeat(1, 1), lens, att.scale)
        assert (np.abs(host(O) - ref) <= bound(ref, A, D, lens, hd, att.scale, dtype)).all(), step
        logits = (O.float().flatten(1) @ head).view(B, 1, V)
        u = rng.random((B, 1)).astype(np.float32)
        got, probs = smp(logits, torch.from_numpy(u).cuda(), temperature=torch.from_numpy(T).cuda(),
                         top_k=i32(top_k), top_p=torch.from_numpy(top_p).cuda())
        wt, wp = oracle.sample(host(logits), u, None, T, top_k, top_p)
        np.testing.assert_array_equal(got.cpu().numpy(), wt)
        assert (np.abs(host(probs) - wp) <= 2.0 ** -24 * wp + 2.0 ** -40).all()
        todo = [[int(t)] for t in wt[:, 0]]
        if step in ends:
            rows[ends[step]], todo[ends[step]] = [], []
        for b in range(B):                        # a free slot takes a prompt two steps later
            if not rows[b] and step - 2 in ends and ends[step - 2] == b:
                todo[b] = list(rng.integers(0, V, 39))
            elif not rows[b]:
                todo[b] = []


def test_round_with_sampled_targets():
    """Selection, targets sampled from the nodes' logits, walk and paged commit, then pages for
    the next round: the walk follows the oracle on the oracle's samples."""
    B, D, V, K, N, Hkv, hd, pr = 3, 6, 3000, 4, 24, 2, 128, 32
    g = torch.Generator(device="cuda").manual_seed(2)
    rng = np.random.default_rng(2)
    marg = (torch.randn(B, D, V, generator=g, device="cuda") * 2).to(BF)
    tree = taps.Selector(B, D, V, K, N)(marg)
    # the target agrees with the draft now and then: its logits raise the children's tokens
    logits = torch.randn(B, N, V, generator=g, device="cuda").to(BF)
    par, tok, n = tree.parent.cpu().numpy(), tree.token.cpu().numpy(), tree.n_nodes.cpu().numpy()
    for b in range(B):
        for i in range(1, n[b]):
            logits[b, par[b, i], tok[b, i]] += 9.0
    u = rng.random((B, N)).astype(np.float32)
    T, top_p = np.float32([1.0, 0.7, 0.0]), np.float32([1.0, 0.95, 1.0])
    smp = taps.TokenSampler(B, N, V)
    target, _ = smp(logits, torch.from_numpy(u).cuda(), tree.n_nodes,
                    temperature=torch.from_numpy(T).cuda(), top_p=torch.from_numpy(top_p).cuda())
    wt, _ = oracle.sample(host(logits), u, n, T, None, top_p)
    np.testing.assert_array_equal(target.cpu().numpy(), wt)
    path, plen, bonus = taps.AcceptWalk(B, N, D)(tree, target)
    accepted = 0
    for b in range(B):
        arr, ln, bn = walk_arrays(*oracle.accept_walk(par[b], tok[b], n[b], wt[b]), D)
        assert path[b].tolist() == arr.tolist() and int(plen[b]) == ln and int(bonus[b]) == bn
        accepted += ln - 1
    assert accepted > 0
    # the committed rows, and pages for the next round's tree
    ctx = np.array([70, 5, 31])
    held = -(-(ctx + N) // pr)
    width = 6
    ids = rng.permutation(40)
    table = np.zeros((B, width), np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    free = np.zeros(40, np.int32)
    free[:40 - at] = ids[at:]
    Kp = torch.randn(40, pr, Hkv, hd, generator=g, device="cuda").to(BF)
    Vp = torch.randn(40, pr, Hkv, hd, generator=g, device="cuda").to(BF)
    com = taps.PagedKVCommit(B, N, D, Hkv, hd, 100, pr)
    t_dev = i32(table)
    new_ctx, _, m = com(Kp, Vp, t_dev, i32(ctx), tree, path, plen, bonus)
    f_dev = i32(free)
    res = taps.PagedKVReserve(B, width, 40, pr, N, slot_map=False)
    h, nf, short, _ = res(t_dev, i32(held), new_ctx, i32([N] * B), f_dev, i32([40 - at]))
    nc = new_ctx.cpu().numpy()
    assert (nc == ctx + m.cpu().numpy()).all()
    want = oracle.kv_reserve_paged(table, held, nc, [N] * B, free, 40 - at, pr, N)
    np.testing.assert_array_equal(t_dev.cpu().numpy(), want[0])
    assert h.tolist() == want[1].tolist() and nf.tolist() == [want[3]] and short.tolist() == [0]


def test_captured_step():
    """One decoding step (reserve, append, attention, sampling, lengths) captured once and
    replayed per token: the same pages, caches and tokens as the step run eagerly, also where
    requests end in between and eager work runs beside the replays."""
    B, Hq, Hkv, hd, pr, width, pages = 5, 8, 2, 64, 32, 20, 60
    V = Hq * hd                                   # the attention's output serves as logits
    g = torch.Generator(device="cuda").manual_seed(7)
    emb = torch.randn(V, (Hq + 2 * Hkv) * hd, generator=g, device="cuda") * 2
    T, top_p, top_k = (torch.tensor(a, device="cuda") for a in (
        [0.3, 1.0, 0.0, 0.5, 0.8], [0.9, 1.0, 1.0, 0.8, 0.95], [0, 0, 0, 20, 300]))
    top_k = top_k.int()
    u = torch.rand(64, B, 1, generator=g, device="cuda")
    res = taps.PagedKVReserve(B, width, pages, pr, 1)
    app = taps.PagedKVAppend(Hkv, hd, pr, dtype=taps.FP32)
    att = taps.PagedDecodeAttention(B, Hq, Hkv, hd, width * pr, pr, dtype=taps.FP32)
    smp = taps.TokenSampler(B, 1, V, dtype=taps.FP32)

    def state():
        return dict(table=torch.zeros(B, width, dtype=torch.int32, device="cuda"),
                    held=i32([0] * B), ctx=i32([0] * B), new=i32([1] * B),
                    free=i32(range(pages)), n_free=i32([pages]), tok=i32([[b] for b in range(B)]),
                    K=torch.zeros(pages, pr, Hkv, hd, device="cuda"),
                    V=torch.zeros(pages, pr, Hkv, hd, device="cuda"), u=u[0].clone())

    def step(s):
        held, n_free, _, slots = res(s["table"], s["held"], s["ctx"], s["new"], s["free"], s["n_free"])
        x = emb.index_select(0, s["tok"].view(-1)).unflatten(1, (Hq + 2 * Hkv, hd))
        app(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], slots, s["K"], s["V"])
        s["ctx"].add_(s["new"])
        O = att(x[:, :Hq], s["K"], s["V"], s["table"], s["ctx"])
        tok, _ = smp(O.view(B, 1, V), s["u"], temperature=T, top_p=top_p, top_k=top_k)
        s["tok"].copy_(tok), s["held"].copy_(held), s["n_free"].copy_(n_free)

    eager, caught = state(), state()
    warm = state()
    step(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caught)
    torch.cuda.synchronize()
    for t in range(64):
        for s in (eager, caught):
            s["u"].copy_(u[t])
            if t in (20, 41):                     # a request ends, and starts again as a new one
                s["ctx"][t % B] = 0
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        for k in eager:
            assert torch.equal(eager[k], caught[k]), (t, k)
    assert int(eager["held"].sum()) + int(eager["n_free"]) == pages
    assert eager["ctx"].tolist() == [64 - 20, 64 - 41, 64, 64, 64]


def test_empty_batches():
    """A batch of no requests: nothing is taken, and the stack's length is passed on."""
    e = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    held, n_free, short, slots = taps.PagedKVReserve(0, 4, 8, 32, 3)(
        e(0, 4), e(0), e(0), e(0), i32(range(8)), i32([5]))
    assert held.shape == (0,) and n_free.tolist() == [5] and short.tolist() == [0]
    assert slots.shape == (0, 3)
    pool = torch.ones(8, 32, 2, 64, dtype=BF, device="cuda")
    row = torch.empty(0, 2, 64, dtype=BF, device="cuda")
    taps.PagedKVAppend(2, 64, 32)(row, row, torch.empty(0, dtype=torch.int64, device="cuda"), pool, pool.clone())
    assert taps.PagedDecodeAttention(0, 4, 2, 64, 128, 32)(
        torch.empty(0, 4, 64, dtype=BF, device="cuda"), pool, pool, e(0, 4), e(0)).shape == (0, 4, 64)
    tok, probs = taps.TokenSampler(0, 3, 50)(torch.empty(0, 3, 50, dtype=BF, device="cuda"),
                                            torch.empty(0, 3, device="cuda"))
    assert tok.shape == (0, 3) and probs.shape == (0, 3)
