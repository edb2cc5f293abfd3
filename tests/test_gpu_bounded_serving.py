"""The serving operators together: drafted tokens attended, verified, weighed and evicted, step after step."""
import math

import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from oracle import bounded as ob
from oracle import cache4 as o4
from tests.gpu_util import need_gpu, say
from tests.op_util import DT

pytestmark = pytest.mark.gpu


def test_drafting_over_a_bounded_cache():
    """Every step's weights, kept tokens and lengths against the oracle on the pool's bytes as they were."""
    need_gpu()
    say("bounded serving")
    B, K, H, Hq, d, page, V, budget, columns = 3, 3, 2, 4, 64, 32, 211, 40, 4
    g = torch.Generator("cuda").manual_seed(5)
    cache = cq.Cache4(B * columns + 1, H, d, page_size=page)
    pages = (torch.randperm(B * columns, generator=g, device="cuda").int() + 1).view(B, columns).contiguous()
    lengths = torch.tensor([50, 7, 31], dtype=torch.int32, device="cuda")
    W = torch.full((B, H, columns * page), math.nan, device="cuda")
    batch = cq.CacheBatch(pages, lengths)  # its lengths change in place

    def rows(n, heads):
        return torch.randn(B, n, heads, d, generator=g, device="cuda").to(DT["bf16"])

    # prompts: all their rows, of which a shorter sequence's first ones lie before position 0
    cq.cqsa_cache_write(cache, batch, rows(50, H), rows(50, H))
    out = torch.zeros(B, K + 1, dtype=torch.int32, device="cuda")
    n_out = torch.zeros(B, dtype=torch.int32, device="cuda")
    kept_lengths = torch.zeros_like(lengths)
    q = rows(50, Hq)
    lse = torch.zeros(B, Hq, 50, device="cuda")
    cq.cqsa_cache_attend(cache, batch, q, torch.empty_like(q), lse)
    cq.cqsa_cache_weigh(cache, batch, q, lse, W)
    for step in range(12):
        lengths += K + 1
        q = rows(K + 1, Hq)
        cq.cqsa_cache_write(cache, batch, rows(K + 1, H), rows(K + 1, H))
        lse = torch.zeros(B, Hq, K + 1, device="cuda")
        cq.cqsa_cache_attend(cache, batch, q, torch.empty_like(q), lse)
        p = torch.softmax(2 * torch.randn(B, K + 1, V, generator=g, device="cuda"), -1)
        f = torch.softmax(p[:, :K].log() + 0.5 * torch.randn(B, K, V, generator=g, device="cuda"), -1)
        tokens = torch.multinomial(f.view(-1, V), 1, generator=g).view(B, K).int()
        u = torch.rand(B, K + 1, generator=g, device="cuda")
        cq.cqsa_draft_verify(p, f, tokens, u, out, n_out, lengths=lengths, new_lengths=kept_lengths)
        before = W.clone()
        cq.cqsa_cache_weigh(cache, batch, q, lse, W, prior=W, decay=0.9, counts=n_out)
        torch.cuda.synchronize()
        data, table, lens = cache.data.cpu().numpy(), pages.cpu().numpy(), lengths.tolist()
        for b in range(B):
            o, n, _, _ = ob.verify(p[b].double().cpu().numpy(), f[b].double().cpu().numpy(), tokens[b].cpu().numpy(), K,
                                   u[b].double().cpu().numpy())
            assert out[b].tolist() == o.tolist() and n_out[b].item() == n
            assert kept_lengths[b].item() == lens[b] - (K - (n - 1))
            t = np.arange(lens[b])
            k, _ = o4.read(data, page, H, d, table[b, t // page], t % page)
            want, big = ob.weigh(q[b].double().cpu().numpy(), k, lse[b].double().cpu().numpy().T, np.ones(lens[b], bool),
                                 lens[b], n, True, 1 / math.sqrt(d), before[b].double().cpu().numpy(), float(np.float32(0.9)))
            got = W[b, :, :lens[b]].double().cpu().numpy()
            assert (np.abs(got - want) <= want * 2.0 ** -24 * ((d + 8) * big + 32) + 1e-36).all()
        lengths.copy_(kept_lengths)
        if step % 3 == 2:
            w = W.cpu().numpy()
            lens = lengths.tolist()
            kept = torch.zeros(B, H, budget, dtype=torch.int32, device="cuda")
            cq.cqsa_cache_evict(cache, batch, W, lengths, budget, first=2, recent=6, kept=kept)
            for b in range(B):
                for h in range(H):
                    k = ob.keep(w[b, h], np.ones(lens[b], bool), lens[b], budget, 2, 6)
                    assert kept[b, h, :len(k)].tolist() == k and lengths[b].item() == min(lens[b], budget)
                    assert np.array_equal(W[b, h, :len(k)].cpu().numpy(), w[b, h, k])
    assert max(lengths.tolist()) <= budget + 3 * (K + 1)
