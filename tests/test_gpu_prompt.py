"""A prompt over the paged cache in chunks, then a decoding step and the prompt's log
probabilities: the calls together, against the same in 64 bits."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu

B, HQ, HKV, HD, PR, HID, VOCAB = 3, 8, 2, 64, 32, 256, 1003


def test_prompt_in_chunks_then_decoding():
    """fp32: tokens -> projections -> pages -> norm, rotation and cache write -> attention -> logits
    -> log probabilities.  Chunks of 50, 1 and 23 tokens a request (fewer where the prompt ends)."""
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    emb, Wqkv = r(VOCAB, HID), r((HQ + 2 * HKV) * HD, HID) * HID ** -0.5
    Wo, qn, kn = r(VOCAB, HQ * HD) * 0.1, 1 + 0.2 * r(HD), 1 + 0.2 * r(HD)
    lens = [74, 51, 13]
    prompts = [torch.randint(0, VOCAB, (n,), generator=g, device=dev) for n in lens]
    freq, m = taps.rope_frequencies(32, 1e4, scaling="yarn", factor=4.0, trained_len=64)
    width, pages = 4, 12
    table = torch.zeros(B, width, dtype=torch.int32, device=dev)
    held, ctx = (torch.zeros(B, dtype=torch.int32, device=dev) for _ in range(2))
    free = torch.randperm(pages, generator=g, device=dev).int()
    n_free = torch.tensor([pages], dtype=torch.int32, device=dev)
    K, V = (torch.full((pages, PR, HKV, HD), float("nan"), device=dev) for _ in range(2))
    rope = taps.PagedQKRope(HQ, HKV, HD, PR, freq, dtype=taps.FP32, mscale=m)
    att = taps.PagedChunkAttention(B, B * 50, HQ, HKV, HD, width * PR, PR, dtype=taps.FP32)
    outs, at = [[] for _ in range(B)], 0
    for step in (50, 1, 23, 1):                            # the last: a decoding step
        new = [max(0, min(step, n - at)) for n in lens] if at < max(lens) else [1] * B
        toks = [prompts[b][at:at + n] if at < max(lens) else prompts[b][:1] for b, n in enumerate(new)]
        n_new = torch.tensor(new, dtype=torch.int32, device=dev)
        res = taps.PagedKVReserve(B, width, pages, PR, 50)
        held, n_free, short, slots = res(table, held, ctx, n_new, free, n_free)
        assert int(short) == 0
        x = emb[torch.cat(toks)] @ Wqkv.T
        q, k, v = x.split([HQ * HD, HKV * HD, HKV * HD], dim=1)
        inside = torch.arange(50, device=dev) < n_new[:, None]
        pos = (ctx[:, None] + torch.arange(50, device=dev, dtype=torch.int32))[inside]
        Q = rope(q.unflatten(1, (HQ, HD)), k.unflatten(1, (HKV, HD)), v.unflatten(1, (HKV, HD)),
                 pos, slots[inside], K, V, qn, kn)
        start = torch.cat((n_new.new_zeros(1), n_new.cumsum(0).int()))
        ctx = ctx + n_new
        O = att(Q, K, V, table, start, ctx)
        for b in range(B):
            outs[b].append(O[start[b]:start[b + 1]])
        if at < max(lens):
            at += step
        else:
            dec = taps.PagedDecodeAttention(B, HQ, HKV, HD, width * PR, PR, dtype=taps.FP32)
            assert torch.allclose(dec(Q, K, V, table, ctx), O, rtol=0, atol=2e-6)
    # the same in 64 bits, each prompt and its decoding step whole
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    for b in range(B):
        tok = torch.cat((prompts[b], prompts[b][:1]))
        n = len(tok)
        x = f64(emb[tok]) @ f64(Wqkv).T
        q, k, v = np.split(x, [HQ * HD, (HQ + HKV) * HD], axis=1)
        Kp, Vp = np.zeros((2, width, PR, HKV, HD))
        Qr, Kp, Vp, _, _ = oracle.qk_rope_paged(
            q.reshape(n, HQ, HD), k.reshape(n, HKV, HD), v.reshape(n, HKV, HD), np.arange(n),
            np.arange(n), *oracle.rope_frequencies(32, 1e4, "yarn", 4.0, 64), False, f64(qn),
            f64(kn), 1e-6, Kp, Vp)
        ref, A, D, N = oracle.chunk_attention_paged(Qr, Kp, Vp, np.arange(width)[None], [0, n], [n],
                                                    HD ** -0.5)
        got = f64(torch.cat(outs[b]))
        # inputs of the attention carry the projection's error (HID products, twice through the
        # norm) and the rotation's, 2^-19: about 2^-15 of the scores' magnitude, twice, and of |v|
        lim = A * (2 * HD ** -0.5 * D[..., None] * 2.0 ** -14 + 2.0 ** -14) + 1e-30
        assert (np.abs(got - ref) <= lim).all()
        # log probabilities of the prompt's next tokens from these outputs
        logits = (torch.cat(outs[b]).flatten(1) @ Wo.T)[None, :n - 1]
        nxt = tok[1:].int()[None]
        lp, ent, rank, idx, tlp = taps.TokenLogProbs(1, n - 1, VOCAB, top=3, dtype=taps.FP32)(
            logits, nxt)
        for i in range(n - 1):
            w = oracle.logprobs_row(f64(logits[0, i]), int(nxt[0, i]), 3)
            assert int(rank[0, i]) == w[2] and idx[0, i].tolist() == w[3].tolist()
            assert math.isclose(float(lp[0, i]), w[0], rel_tol=2 ** -23, abs_tol=4e-6)
