"""Prompts over the paged cache in bf16 with heads of 128, as servers run them: the calls chained,
each against 64 bits on what the one before it left."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps
from test_gpu_chunk import BF, bound
from test_gpu_rope import f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,window,chunk", [(8, 2, 0, 256), (32, 8, 0, 100), (4, 4, 200, 311)])
def test_prompts_in_chunks_then_decoding(Hq, Hkv, window, chunk):
    hd, PR, hid, vocab, dev = 128, 32, 256, 5003, "cuda"
    lens = [700, 300, 77, 1]
    B, width = len(lens), 23
    pages = sum(-(-(n + 1) // PR) for n in lens) + 1
    g = torch.Generator(device=dev).manual_seed(Hq)
    r = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    emb, Wqkv = r(vocab, hid).to(BF), (r(hid, (Hq + 2 * Hkv) * hd) * hid ** -0.5).to(BF)
    Wo = (r(Hq * hd, vocab) * 0.1).to(BF)
    qn, kn = (1 + 0.2 * r(hd)).to(BF), (1 + 0.2 * r(hd)).to(BF)
    prompts = [torch.randint(0, vocab, (n + 1,), generator=g, device=dev) for n in lens]
    freq, m = taps.rope_frequencies(hd, 1e6, scaling="yarn", factor=4.0, trained_len=256)
    table = torch.zeros(B, width, dtype=torch.int32, device=dev)
    held, ctx = (torch.zeros(B, dtype=torch.int32, device=dev) for _ in range(2))
    free = torch.randperm(pages, generator=g, device=dev).int()
    n_free = torch.tensor([pages], dtype=torch.int32, device=dev)
    K, V = (torch.full((pages, PR, Hkv, hd), float("nan"), dtype=BF, device=dev) for _ in range(2))
    reserve = taps.PagedKVReserve(B, width, pages, PR, chunk)
    rope = taps.PagedQKRope(Hq, Hkv, hd, PR, freq, mscale=m)
    att = taps.PagedChunkAttention(B, B * chunk, Hq, Hkv, hd, width * PR, PR, window=window)
    dec = taps.PagedDecodeAttention(B, Hq, Hkv, hd, width * PR, PR)
    q_in, k_in, v_in, q_out, o_out = ([[] for _ in range(B)] for _ in range(5))
    at, decoded = 0, False
    while not decoded:
        decoded = at >= max(lens)                          # the last: a token of every request
        new = [1] * B if decoded else [max(0, min(chunk, n - at)) for n in lens]
        toks = [prompts[b][lens[b]:] if decoded else prompts[b][at:at + n] for b, n in enumerate(new)]
        n_new = torch.tensor(new, dtype=torch.int32, device=dev)
        held, n_free, short, slots = reserve(table, held, ctx, n_new, free, n_free)
        assert int(short) == 0
        q, k, v = (emb[torch.cat(toks)] @ Wqkv).split([Hq * hd, Hkv * hd, Hkv * hd], dim=1)
        q, k, v = q.unflatten(1, (Hq, hd)), k.unflatten(1, (Hkv, hd)), v.unflatten(1, (Hkv, hd))
        inside = torch.arange(chunk, device=dev) < n_new[:, None]
        pos = (ctx[:, None] + torch.arange(chunk, device=dev, dtype=torch.int32))[inside]
        Q = rope(q, k, v, pos, slots[inside], K, V, qn, kn)
        start = torch.cat((n_new.new_zeros(1), n_new.cumsum(0).int()))
        ctx = ctx + n_new
        O = att(Q, K, V, table, start, ctx)
        for b in range(B):
            s = slice(int(start[b]), int(start[b + 1]))
            for dst, t in ((q_in, q), (k_in, k), (v_in, v), (q_out, Q), (o_out, O)):
                dst[b].append(t[s])
        if decoded and window == 0:
            Od = dec(Q, K, V, table, ctx)
        at += chunk
    Kc, Vc, tab = f64(K), f64(V), table.cpu().numpy()
    for b, n in enumerate(lens):
        n += 1
        qi, ki, vi, qo, oo = (f64(torch.cat(t[b])) for t in (q_in, k_in, v_in, q_out, o_out))
        rows = tab[b, np.arange(n) // PR] * PR + np.arange(n) % PR
        kc, vc = (x.reshape(-1, Hkv, hd)[rows] for x in (Kc, Vc))
        # norm, rotation and cache write: half a step, and 2^-19 of the pair (17 fp32 roundings)
        zero = np.zeros((-(-n // PR), PR, Hkv, hd))
        Qr, Kr, _, Qm, Km = oracle.qk_rope_paged(qi, ki, vi, np.arange(n), np.arange(n), f64(freq), m,
                                                 False, f64(qn), f64(kn), 1e-6, zero, zero)
        Kr, Km = (x.reshape(-1, Hkv, hd)[:n] for x in (Kr, Km))
        assert (np.abs(qo - Qr) <= np.abs(Qr) * 2.0 ** -8 + m * Qm * 2.0 ** -19).all()
        assert (np.abs(kc - Kr) <= np.abs(Kr) * 2.0 ** -8 + m * Km * 2.0 ** -19).all()
        assert np.array_equal(vc, vi)
        # attention over the pools as they are
        ref, A, D, N = oracle.chunk_attention_paged(qo, Kc, Vc, tab[b:b + 1], [0, n], [n], hd ** -0.5,
                                                    window)
        lim = bound(ref, A, D, N, hd, hd ** -0.5, BF)
        assert (np.abs(oo - ref) <= lim).all()
        if window == 0:
            assert (np.abs(f64(Od)[b] - ref[-1]) <= lim[-1]).all()
        # log probabilities of the prompt's next tokens from these outputs
        logits = torch.cat(o_out[b]).flatten(1) @ Wo
        for i0 in range(0, n - 1, 512):
            part, nxt = logits[i0:min(i0 + 512, n - 1)][None], prompts[b][i0 + 1:i0 + 513].int()[None]
            lp, ent, rank, idx, tlp = (t[0].cpu().numpy() for t in taps.TokenLogProbs(
                1, part.shape[1], vocab, top=3)(part, nxt))
            assert (lp <= 0).all() and (ent >= 0).all()
            rel = (vocab / 512 + 43) * 2.0 ** -24
            for i in range(0, part.shape[1], 7):
                w = oracle.logprobs_row(f64(part[0, i]), int(nxt[0, i]), 3)
                assert rank[i] == w[2] and np.array_equal(idx[i], w[3])
                assert abs(lp[i] - w[0]) <= rel + abs(w[0]) * 2.0 ** -24
                assert (np.abs(tlp[i] - w[4]) <= rel + np.abs(w[4]) * 2.0 ** -24).all()
                assert abs(ent[i] - w[1]) <= rel * (1 + w[5] + 12) + abs(w[1]) * 2.0 ** -24
