"""The verification loop: the operators together, step after step, against the whole sequences computed anew in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _forward(loop, tokens):
    """Logits of the verifier behind every token of one sequence, in 64 bits from the rounded weights, with the roundings of the path
    (queries, keys, values, the attention's output and the residual stream are bfloat16) where it has them."""
    b = lambda t: t.bfloat16().double()
    x = loop.embed.cpu().double()[tokens]
    qkv = b((x @ loop.w_qkv.cpu().double()).float()).view(len(tokens), -1, loop.D)
    q, k, v = qkv.split([loop.Hq, loop.Hk, loop.Hk], 1)
    ang = torch.arange(len(tokens), dtype=torch.float64)[:, None, None] * loop.inv_freq.cpu()
    c, s, h = torch.cos(ang), torch.sin(ang), loop.D // 2

    def turn(t):
        return b(torch.cat([t[..., :h] * c - t[..., h:] * s, t[..., h:] * c + t[..., :h] * s], -1).float())
    q, k = turn(q), turn(k).repeat_interleave(loop.Hq // loop.Hk, 1)
    v = v.repeat_interleave(loop.Hq // loop.Hk, 1)
    out = torch.zeros(len(tokens), loop.Hq, loop.D, dtype=torch.float64)
    late = torch.triu(torch.ones(len(tokens), len(tokens), dtype=torch.bool), 1)
    for i in range(loop.Hq):
        w = torch.softmax((q[:, i] @ k[:, i].T / math.sqrt(loop.D)).masked_fill(late, -math.inf), -1)
        out[:, i] = w @ v[:, i]
    y = b(out.float()).view(len(tokens), -1) @ loop.w_out.cpu().double()
    return (x + y) @ loop.w_logits.cpu().double()


@pytest.mark.parametrize("requests,window,page", [(1, 1, 16), (5, 4, 16), (3, 8, 32)])
def test_the_loop_says_what_the_whole_sequences_say(requests, window, page):
    import paper_2603_25463_amd as ciar
    from paper_2603_25463_amd.verification import VerificationLoop
    assert torch.cuda.is_available()
    ciar.lib()
    loop = VerificationLoop(requests, window, vocab=200, heads=4, kv_heads=2, head_dim=32, page_size=page, max_len=130, seed=window)
    said = [[int(t)] for t in loop.last]
    for step in range(12):
        o = loop.step()
        torch.cuda.synchronize()
        print("step", step, o["accept_len"].tolist(), flush=True)
        ids = o["ids"].view(requests, window).tolist()
        for r in range(requests):
            seen = said[r] + ids[r][:-1]
            want = _forward(loop, torch.tensor(seen))[-window:]
            got = o["logits"].view(requests, window, -1)[r].double().cpu()
            # the weights' and the last product's roundings to bfloat16: half a step of the residual stream and of the logits, in a
            # row of E products, by their root mean square (4 sigma), and the weights' of the attention
            tol = 2.0 ** -8 * (want.abs() + 4 * math.sqrt(want.pow(2).mean()) + 1.0)
            assert bool(((got - want).abs() <= 4 * tol).all()), (step, r, float(((got - want).abs() / tol).max()))
            # what was adjusted, by the rules in plain words
            row = o["adjusted"].view(requests, window, -1)[r].double().cpu()
            for j in range(window):
                x, heard = got[j].clone(), said[r] + ids[r][:j]
                for t in set(heard):
                    n = heard.count(t)
                    x[t] = (x[t] / 1.1 if x[t] > 0 else x[t] * 1.1) - 0.05 * n - 0.1
                gone = torch.arange(200) % 16 == 0
                assert bool((row[j][gone] == -math.inf).all())
                assert bool(((row[j] - x)[~gone].abs() <= 8 * 2.0 ** -24 * (x[~gone].abs() + 1 + len(heard))).all())
            assert o["left"].view(requests, window)[r].tolist() == [200 - 13] * window
            a = int(o["accept_len"][r])
            said[r] += ids[r][:a] + ([int(o["resampled_id"][r])] if a < window else [])
            assert int(loop.last[r]) == said[r][-1]
            n = int(loop.count[r])
            assert loop.said[r, :n].tolist() == said[r]
        assert (loop.plan["lengths"] + loop.kept).tolist() == [len(s) - 1 for s in said]
    pages = [int(loop.table[r, c]) for r in range(requests) for c in range(int(loop.held[r]))]
    head, tail = loop.ring_state.tolist()
    pages += [int(loop.ring[i % loop.ring.numel()]) for i in range(head, tail)]
    assert sorted(pages) == list(range(loop.ring.numel()))
