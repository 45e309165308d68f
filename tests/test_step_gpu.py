"""The verification step's operators on the GPU against plain 64-bit implementations on the CPU.

Tolerances, from the roundings counted (half a step is 2^-24 of a float32, 2^-8 of a bfloat16 value):
  rotary     the result's own rounding, and 8 x 2^-24 of m (|a| + |b|): sine and cosine 3 (argument, polynomial, times m), the two
             products and their sum 3, two to spare for the argument of angles near pi / 2
  attention  a score is D exact products summed in 32 bits: off by at most eps = 2^-24 (D + 4) scale sum |q k|, so a weight by a
             factor 1 + 2 eps (its own and the sum's); weights are rounded to bfloat16 for the second product (2^-8 of sum p |v|);
             exponentials (2^-22) and sums over L tokens in 32 bits (L 2^-24 at most); the result's rounding 2^-8 |out|
  logits     up to six operations in 32 bits, each half a step of the largest intermediate; the result's own rounding
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

H32, H16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def ciar():
    import paper_2603_25463_amd as m
    m.lib()
    assert torch.cuda.is_available()
    return m


def say(*a):
    print(*a, flush=True)


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


# ---- cache plan -----------------------------------------------------------------------------------------------

def plan_reference(lengths, kept, new, held, ring, state, table, page, T):
    """The plan request by request; ring and table are changed in place (numpy, int64)."""
    R, (width, P) = len(lengths), (table.shape[1], len(ring))
    head, tail = state
    old_ring, free, asked = ring.copy(), state[1] - state[0], 0
    out = dict(lengths=[], kv_len=[], cu_new=[0], held=[], granted=[], slots=[-1] * T, positions=[0] * T, requests=[-1] * T)
    at = 0
    for r in range(R):
        length = lengths[r] + kept[r]
        pages = -(-(length + new[r]) // page)
        fits = pages <= width and at + new[r] <= T
        need = max(pages - held[r], 0) if fits else 0
        asked += need
        granted = fits and (need == 0 or asked <= free)
        if granted:
            for c in range(held[r], held[r] + need):
                table[r, c] = old_ring[head % P]
                head += 1
            for c in range(pages, held[r]):
                ring[tail % P] = table[r, c]
                tail += 1
        for j in range(new[r]):
            if at + j < T:
                p = length + j
                out["positions"][at + j], out["requests"][at + j] = p, r
                if granted:
                    out["slots"][at + j] = table[r, p // page] * page + p % page
        at += new[r]
        out["lengths"].append(length)
        out["kv_len"].append(length + new[r] if granted else 0)
        out["cu_new"].append(min(at, T))
        out["held"].append(pages if granted else held[r])
        out["granted"].append(int(granted))
    out["ring_state"] = [head, tail]
    return out


def plan_case(seed, R, most_new, context, page, spare, width=None, tokens=None):
    rng = np.random.default_rng(seed)
    lengths = rng.integers(0, context + 1, R)
    kept = rng.integers(0, most_new + 1, R)
    new = rng.choice([0, 1, most_new, max(0, most_new - 1)], R)
    held = -(-(lengths + most_new) // page)
    width = int(width or (-(-(context + 3 * most_new + page) // page)))
    held = np.minimum(held, width)
    used = int(held.sum())
    P = used + spare
    order = rng.permutation(P)
    table = np.full((R, width), -1, dtype=np.int64)
    at = 0
    for r in range(R):
        table[r, :held[r]] = order[at:at + held[r]]
        at += held[r]
    head = int(rng.integers(0, 1 << 40))
    ring = np.full(P, -7, dtype=np.int64)
    for j in range(spare):
        ring[(head + j) % P] = order[at + j]
    return (lengths, kept, new, held, ring, [head, head + spare], table), page, int(tokens if tokens is not None else new.sum() + 3)


PLANS = {  # R, most new, context, page, spare pages
    "one": (1, 1, 1, 16, 4), "one_empty": (1, 0, 0, 16, 1), "window": (8, 8, 600, 16, 40), "short_of_pages": (40, 30, 200, 16, 9),
    "no_free_page": (17, 20, 50, 32, 0), "narrow_table": (30, 16, 300, 16, 100, 12), "few_places": (30, 16, 300, 16, 100, None, 50),
    "256": (256, 5, 100, 64, 30), "257": (257, 33, 1000, 16, 600), "fleet": (1025, 64, 2000, 16, 3000), "chunks": (2500, 9, 70, 16, 700),
    "long_prompt": (2, 5000, 100, 16, 900), "no_places": (5, 4, 40, 16, 20, None, 0),
}


@pytest.mark.parametrize("name", list(PLANS))
@pytest.mark.parametrize("with_kept", [True, False])
def test_cache_plan(ciar, name, with_kept):
    (lengths, kept, new, held, ring, state, table), page, T = plan_case(len(name) + 100 * with_kept, *PLANS[name])
    say("[plan]", name, "R", len(lengths), "T", T)
    if not with_kept:
        kept = np.zeros_like(kept)
    wide = torch.full((len(lengths), table.shape[1] + 3), -9, dtype=torch.int32, device="cuda")   # a stride beyond the width
    wide[:, :table.shape[1]] = i32(table)
    g_table, g_ring = wide[:, :table.shape[1]], i32(ring)
    o = ciar.cache_plan(i32(lengths), i32(new), i32(held), g_ring, torch.tensor(state, device="cuda"), g_table, T, page_size=page,
                        kept=i32(kept) if with_kept else None)
    torch.cuda.synchronize()
    want = plan_reference(lengths, kept, new, held, ring, state, table, page, T)
    for k, v in want.items():
        assert o[k].tolist() == [int(x) for x in v], k
    assert np.array_equal(g_table.cpu().numpy(), table) and np.array_equal(g_ring.cpu().numpy(), ring)
    assert bool((wide[:, table.shape[1]:] == -9).all())


def test_cache_plan_without_requests(ciar):
    e = i32([])
    state = torch.tensor([5, 9], device="cuda")
    o = ciar.cache_plan(e, e, e, i32(range(8)), state, torch.empty((0, 4), dtype=torch.int32, device="cuda"), 3, page_size=16)
    assert o["cu_new"].tolist() == [0] and o["slots"].tolist() == [-1] * 3 and o["requests"].tolist() == [-1] * 3
    assert o["ring_state"].tolist() == [5, 9]


def test_cache_plan_steps_follow_each_other(ciar):
    """Twenty steps of drafting and verifying, planned from each other's outputs: no page is ever in two places."""
    rng = np.random.default_rng(3)
    R, page, K, P, width = 12, 16, 8, 90, 14
    table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    ring, state = i32(rng.permutation(P)), torch.tensor([0, P], device="cuda")
    lengths, held = i32(np.zeros(R)), i32(np.zeros(R))
    kept = i32(np.zeros(R))
    for step in range(20):
        new = rng.integers(0, K + 1, R)
        o = ciar.cache_plan(lengths, i32(new), held, ring, state, table, R * K, page_size=page, kept=kept)
        lengths, held, state = o["lengths"], o["held"], o["ring_state"]
        owned = [int(table[r, c]) for r in range(R) for c in range(int(held[r]))]
        s = state.tolist()
        free = [int(ring[i % P]) for i in range(s[0], s[1])]
        assert sorted(owned + free) == list(range(P)), step
        slots = o["slots"][o["slots"] >= 0].tolist()
        assert len(set(slots)) == len(slots)
        kept = torch.where(o["granted"] != 0, torch.minimum(i32(rng.integers(0, K + 1, R)), i32(new)), 0).int()


# ---- rotary positions -----------------------------------------------------------------------------------------

def rotary_reference(x, pos, freq, layout, m, inverse):
    x = x.double().cpu()
    n = 2 * freq.numel()
    ang = pos.double().cpu()[:, None, None] * freq.double().cpu() * (-1 if inverse else 1)
    c, s = torch.cos(ang) * m, torch.sin(ang) * m
    y, size = x.clone(), torch.zeros_like(x)
    one = torch.arange(0, n, 2) if layout == "interleaved" else torch.arange(n // 2)
    two = one + 1 if layout == "interleaved" else one + n // 2
    a, b = x[..., one], x[..., two]
    y[..., one], y[..., two] = a * c - b * s, b * c + a * s
    size[..., one] = size[..., two] = abs(m) * (a.abs() + b.abs())
    return y, size


def check_rotary(got, want, size, dtype):
    tol = (H16 if dtype == torch.bfloat16 else H32) * want.abs() + 8 * H32 * size + (H16 * 8 * H32 * size)
    err = (got.double().cpu() - want).abs()
    assert bool((err <= tol).all()), float((err / tol.clamp(min=1e-300)).max())


def freqs(n, slow=1.0):
    return (10000.0 ** (-torch.arange(n // 2, dtype=torch.float64) / (n // 2)) * slow).cuda()


ROTARY = [  # T, q heads, kv heads, D, rotary_dim, far, dtype
    (1, 1, 1, 2, 2, 5, torch.float32), (1, 8, 2, 64, 64, 199999, torch.bfloat16), (3, 5, 5, 34, 22, 1000, torch.bfloat16),
    (17, 4, 1, 80, 80, 4099, torch.float32), (33, 7, 1, 129, 74, 2 ** 31 - 100, torch.float32), (65, 8, 8, 96, 10, 300, torch.bfloat16),
    (130, 32, 8, 128, 128, 150000, torch.bfloat16), (40, 3, 3, 192, 190, 77, torch.bfloat16), (64, 2, 1, 256, 256, 8000, torch.float32),
    (19, 4, 4, 6, 4, 100, torch.float32), (1000, 2, 2, 32, 16, 5000, torch.bfloat16),
]


@pytest.mark.parametrize("T,Hq,Hk,D,n,far,dtype", ROTARY)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary_dense(ciar, T, Hq, Hk, D, n, far, dtype, layout, inverse):
    say("[rotary]", T, Hq, Hk, D, n, far, dtype, layout, inverse)
    g = torch.Generator().manual_seed(T + D + n)
    qkv = torch.randn((T, Hq + Hk, D), generator=g).to(dtype).cuda()
    q, k = qkv[:, :Hq], qkv[:, Hq:]
    pos = torch.randint(0, far, (T,), generator=g, dtype=torch.int32).cuda()
    f, m = freqs(n, 0.7), 1.25
    o = ciar.rotary(q, k, pos, f, layout=layout, inverse=inverse, magnitude=m)
    for got, x in ((o["q"], q), (o["k"], k)):
        want, size = rotary_reference(x, pos, f, layout, m, inverse)
        check_rotary(got, want, size, dtype)
        assert torch.equal(got[..., n:], x[..., n:])


@pytest.mark.parametrize("T,Hq,Hk,D,n,page,start", [(1, 8, 2, 64, 64, 16, 3), (16, 4, 4, 96, 50, 16, 0), (33, 3, 1, 32, 32, 32, 5),
                                                    (200, 7, 1, 128, 100, 64, 61), (77, 4, 2, 256, 256, 32, 15), (50, 2, 2, 8, 8, 16, 9)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("order", ["chunk", "scattered"])
def test_rotary_into_the_cache(ciar, T, Hq, Hk, D, n, page, start, layout, order):
    say("[rotary cache]", T, Hq, Hk, D, n, page, start, layout, order)
    g = torch.Generator().manual_seed(T + D)
    wide = torch.randn((T, Hq + 2 * Hk, D + 3), generator=g).bfloat16().cuda()[..., 1:D + 1]      # rows at odd places
    q, k, v = wide[:, :Hq], wide[:, Hq:Hq + Hk], wide[:, Hq + Hk:]
    pages = (T + start) // page + 3
    ks, vs = ciar.cache_shapes(pages, Hk, D, page)
    kc, vc = torch.full(ks, 9.0).bfloat16().cuda(), torch.full(vs, -9.0).bfloat16().cuda()
    own = torch.randperm(pages, generator=g)
    i = torch.arange(T) + start
    slots = own[i // page] * page + i % page
    if order == "scattered":
        slots = slots[torch.randperm(T, generator=g)]
    slots[T // 2] = -1 if T > 1 else slots[0]                     # a token without a place
    if T > 4:
        slots[3] = pages * page                                   # and one beyond the cache
    pos = (torch.arange(T, dtype=torch.int32) + 120000).cuda()
    f = freqs(n)
    o = ciar.rotary(q, k, pos, f, layout=layout, v=v, k_cache=kc, v_cache=vc, slots=slots.int().cuda())
    torch.cuda.synchronize()
    assert set(o) == {"q"}
    want, size = rotary_reference(q, pos, f, layout, 1.0, False)
    check_rotary(o["q"], want, size, torch.bfloat16)
    rows_k = kc.permute(0, 2, 4, 1, 3, 5).reshape(pages * page, Hk, D).cpu()
    rows_v = vc.permute(0, 2, 3, 5, 1, 4).reshape(pages * page, Hk, D).cpu()
    ok = (slots >= 0) & (slots < pages * page)
    want, size = rotary_reference(k, pos, f, layout, 1.0, False)
    check_rotary(rows_k[slots[ok]], want[ok], size[ok], torch.bfloat16)
    assert torch.equal(rows_v[slots[ok]], v.cpu()[ok])
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[slots[ok]] = False
    assert bool((rows_k[rest] == 9.0).all()) and bool((rows_v[rest] == -9.0).all())


@pytest.mark.parametrize("T,Hq,Hk,D,n,page", [(1024, 2, 1, 128, 128, 16), (1500, 1, 3, 96, 34, 32), (3001, 4, 2, 64, 64, 48), (1203, 1, 1, 256, 200, 64),
                                              (1100, 3, 2, 264, 16, 16), (2000, 1, 1, 16, 16, 16), (1031, 2, 5, 40, 40, 32)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("order", ["chunk", "requests", "scattered"])
def test_rotary_of_many_tokens_into_the_cache(ciar, T, Hq, Hk, D, n, page, layout, order):
    """Sixteen tokens at a time: one long run of slots from an odd place, runs of one to forty tokens, every slot for itself; some have none."""
    say("[rotary cache, many]", T, Hq, Hk, D, n, page, layout, order)
    g = torch.Generator().manual_seed(T + D)
    x = torch.randn((T, Hq + 2 * Hk, D), generator=g).bfloat16().cuda()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    pages = (2 * T + 5) // page + 3
    ks, vs = ciar.cache_shapes(pages, Hk, D, page)
    kc, vc = torch.full(ks, 9.0).bfloat16().cuda(), torch.full(vs, -9.0).bfloat16().cuda()
    own = torch.randperm(pages, generator=g)
    i = torch.arange(T) + 5
    if order == "requests":                                       # (a gap behind every run)
        cut = torch.cumsum(torch.randint(1, 41, (T,), generator=g), 0)
        i = i + torch.cumsum(torch.randint(0, 2, (T,), generator=g), 0)[torch.searchsorted(cut, torch.arange(T), right=True)]
    slots = own[i // page] * page + i % page
    if order == "scattered":
        slots = slots[torch.randperm(T, generator=g)]
    slots[torch.randint(0, T, (T // 50,), generator=g)] = -1
    pos = torch.randint(0, 100000, (T,), generator=g, dtype=torch.int32).cuda()
    f = freqs(n)
    o = ciar.rotary(q, k, pos, f, layout=layout, v=v, k_cache=kc, v_cache=vc, slots=slots.int().cuda())
    torch.cuda.synchronize()
    want, size = rotary_reference(q, pos, f, layout, 1.0, False)
    check_rotary(o["q"], want, size, torch.bfloat16)
    rows_k = kc.permute(0, 2, 4, 1, 3, 5).reshape(pages * page, Hk, D).cpu()
    rows_v = vc.permute(0, 2, 3, 5, 1, 4).reshape(pages * page, Hk, D).cpu()
    ok = slots >= 0
    want, size = rotary_reference(k, pos, f, layout, 1.0, False)
    check_rotary(rows_k[slots[ok]], want[ok], size[ok], torch.bfloat16)
    assert torch.equal(rows_v[slots[ok]], v.cpu()[ok])
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[slots[ok]] = False
    assert bool((rows_k[rest] == 9.0).all()) and bool((rows_v[rest] == -9.0).all())


@pytest.mark.parametrize("new,tokens", [(3, 100), (150, 400)])
def test_offsets_beyond_32_bits(ciar, new, tokens):
    """Caches of 5 GB each, used at their far end, and rows of q and out 2^31 elements apart."""
    Hq, Hk, D, page = 4, 8, 128, 64
    pages = 40000
    ks, vs = ciar.cache_shapes(pages, Hk, D, page)
    kc, vc = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in (ks, vs))
    assert kc.numel() > 1 << 31
    g = torch.Generator().manual_seed(new)
    need = -(-tokens // page)
    own = pages - 1 - torch.randperm(need, generator=g)
    i = torch.arange(tokens)
    slots = (own[i // page] * page + i % page).int().cuda()
    k, v = (torch.randn((tokens, Hk, D), generator=g).bfloat16() for _ in range(2))
    still = torch.zeros(tokens, dtype=torch.int32, device="cuda")
    ciar.rotary(torch.zeros((tokens, 1, D)).bfloat16().cuda(), k.cuda(), still, freqs(D), v=v.cuda(), k_cache=kc, v_cache=vc, slots=slots)
    apart = (1 << 31) // new + 8
    qs, ys = (torch.empty(apart * (new - 1) + 2 * Hq * D, dtype=torch.bfloat16, device="cuda").as_strided((new, Hq * 2, D), (apart, D, 1)) for _ in range(2))
    assert apart * (new - 1) * 2 > 1 << 31
    x = torch.randn((new, 2 * Hq, D), generator=g).bfloat16()
    qs.copy_(x)
    table = own.int()[None].cuda()
    o = ciar.paged_attention(qs, kc, vc, table, i32([0, new]), i32([tokens]), new, tokens, out={"out": ys})
    check_attention({"out": ys, "lse": o["lse"]}, x, [(k.double(), v.double())], [new], [0], 1 / math.sqrt(D), 1)
    turned = ciar.rotary(qs, qs, still[:new], freqs(D), out={"q": ys})
    assert torch.equal(turned["k"].cpu(), x) and torch.equal(ys.cpu(), x)


def test_logit_rows_beyond_32_bits(ciar):
    V, apart = 5000, (1 << 31) + 64
    rows = torch.empty(2 * apart + V, dtype=torch.bfloat16, device="cuda").as_strided((3, V), (apart, 1))
    x = torch.randn((3, V), generator=torch.Generator().manual_seed(2)).bfloat16()
    rows.copy_(x)
    words = torch.full((1, -(-V // 32)), 0x55555555, dtype=torch.int32, device="cuda")
    o = ciar.adjust_logits(rows, ciar.Params(window=3), allowed=words, allowed_row=i32([0, -1, 0]), out={"logits": rows})
    want = x.clone()
    want[0, 1::2] = want[2, 1::2] = -math.inf
    assert torch.equal(rows.cpu(), want) and o["left"].tolist() == [V // 2, V, V // 2]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_gradient(ciar, layout):
    """The inverse turn is the gradient: against autograd of the formula in 64 bits, and against differences."""
    T, H, D, n = 9, 3, 20, 14
    g = torch.Generator().manual_seed(8)
    q, k = torch.randn((T, H, D), generator=g), torch.randn((T, 1, D), generator=g)
    gq, gk = torch.randn((T, H, D), generator=g), torch.randn((T, 1, D), generator=g)
    pos, f, m = torch.randint(0, 5000, (T,), generator=g, dtype=torch.int32), freqs(n), 1.1
    o = ciar.rotary(gq.cuda(), gk.cuda(), pos.cuda(), f, layout=layout, inverse=True, magnitude=m)
    ang = pos.double()[:, None, None] * f.cpu()
    for x, gx, got in ((q, gq, o["q"]), (k, gk, o["k"])):
        z = x.double().requires_grad_(True)
        one = slice(0, n, 2) if layout == "interleaved" else slice(0, n // 2)
        two = slice(1, n, 2) if layout == "interleaved" else slice(n // 2, n)
        a, b, c, s = z[..., one], z[..., two], torch.cos(ang) * m, torch.sin(ang) * m
        G = gx.double()
        total = (G[..., one] * (a * c - b * s)).sum() + (G[..., two] * (b * c + a * s)).sum() + (G[..., n:] * z[..., n:]).sum()
        total.backward()
        _, size = rotary_reference(gx, pos, f, layout, m, True)
        assert bool(((got.double().cpu() - z.grad).abs() <= H32 * z.grad.abs() + 8 * H32 * size).all())
    # differences of the forward kernel itself along a direction: the turn is linear, so they are exact up to roundings
    d = torch.randn((T, H, D), generator=g)
    y1 = ciar.rotary((q + d).cuda(), k.cuda(), pos.cuda(), f, layout=layout, magnitude=m)["q"]
    y0 = ciar.rotary((q - d).cuda(), k.cuda(), pos.cuda(), f, layout=layout, magnitude=m)["q"]
    slope = ((y1.double() - y0.double()).cpu() / 2 * gq.double()).sum()
    want = (o["q"].double().cpu() * d.double()).sum()
    scale = 4 * m * (gq.double().abs() * (q.abs() + d.abs()).double()).sum()
    assert abs(float(slope - want)) <= 16 * H32 * 2 * float(scale)


# ---- attention ------------------------------------------------------------------------------------------------

def make_cache(ciar, lens, Hk, D, page, seed, extra=2):
    """Pages in random order; every slot that no request owns holds NaN."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    pages, width = sum(need) + extra, max(need + [1]) + 1
    ks, vs = ciar.cache_shapes(pages, Hk, D, page)
    rows_k = torch.full((pages * page, Hk, D), float("nan"))
    rows_v = torch.full((pages * page, Hk, D), float("nan"))
    order, table, at = torch.randperm(pages, generator=g), torch.full((max(len(lens), 1), width), -1, dtype=torch.int32), 0
    kv = []
    for r, n in enumerate(lens):
        own = order[at:at + need[r]]
        at += need[r]
        table[r, :need[r]] = own.int()
        i = torch.arange(n)
        slots = own[i // page] * page + i % page if n else i
        k, v = torch.randn((n, Hk, D), generator=g).bfloat16().float(), torch.randn((n, Hk, D), generator=g).bfloat16().float()
        rows_k[slots], rows_v[slots] = k, v
        kv.append((k.double(), v.double()))
    A = page // 16
    kc = rows_k.view(pages, A, 16, Hk, D // 8, 8).permute(0, 3, 1, 4, 2, 5).contiguous().bfloat16().cuda()
    vc = rows_v.view(pages, A, 2, 8, Hk, D).permute(0, 4, 1, 2, 5, 3).contiguous().bfloat16().cuda()
    assert kc.shape == ks and vc.shape == vs
    return kc, vc, table.cuda(), kv


def check_attention(o, q, kv, news, starts, scale, g):
    """out and lse of every request's rows against the formula in 64 bits, row by row."""
    T, Hq, D = q.shape
    out, lse, q = o["out"].double().cpu(), o["lse"].double().cpu(), q.double().cpu()
    claimed = torch.zeros(T, dtype=torch.bool)
    for (k, v), n, b in zip(kv, news, starts):
        L = k.shape[0]
        claimed[b:b + n] = True
        for h in range(Hq):
            kh, vh, qh = k[:, h // g], v[:, h // g], q[b:b + n, h]
            s = qh @ kh.T * scale
            size = (qh.abs() @ kh.abs().T * abs(scale)).amax(1, keepdim=True) if L else torch.zeros((n, 1), dtype=torch.float64)
            late = torch.arange(L) > (L - n + torch.arange(n))[:, None]
            s = s.masked_fill(late, -math.inf)
            want_lse = torch.logsumexp(s, -1) if L else torch.full((n,), -math.inf, dtype=torch.float64)
            p = torch.where(late, 0.0, torch.exp(s - torch.where(want_lse == -math.inf, 0.0, want_lse)[:, None]))
            want = p @ torch.where(torch.isfinite(vh), vh, 0.0)
            eps = H32 * (D + 4) * size
            rel = 2 * eps + 2.0 ** -21 + (L + 8) * H32
            tol = (H16 * (1 + rel) + rel) * (p @ torch.where(torch.isfinite(vh), vh, 0.0).abs()) + H16 * want.abs() * (1 + H16) + 1e-30
            err = (out[b:b + n, h] - want).abs()
            assert bool((err <= tol).all()), (h, float((err / tol).max()))
            gone = want_lse == -math.inf
            assert bool((lse[b:b + n, h][gone] == -math.inf).all()) and bool((out[b:b + n, h][gone] == 0).all())
            e = (lse[b:b + n, h] - want_lse)[~gone].abs()
            assert bool((e <= (eps[:, 0] + 2.0 ** -21 + (L / 8 + 8) * H32 + 4 * H32 * want_lse.abs())[~gone]).all()), float(e.max())
    assert bool((out[~claimed] == 0).all()) and bool((lse[~claimed] == -math.inf).all())


ATTENTION = {  # [(tokens in the cache, new)], q heads, kv heads, D, page
    "one_token": ([(1, 1)], 1, 1, 64, 16), "two": ([(2, 1)], 2, 1, 32, 16), "first": ([(40, 8)], 8, 8, 64, 16),
    "prompt_only": ([(33, 33)], 4, 4, 96, 32), "single_tokens": ([(100, 1), (1, 1), (333, 1), (16, 1), (17, 1)], 8, 2, 128, 16),
    "group_of_seven": ([(50, 3), (260, 5)], 7, 1, 64, 32), "group_of_eight": ([(130, 8), (129, 7), (128, 1)], 16, 2, 128, 64),
    "empty_requests": ([(0, 0), (64, 0), (0, 3), (31, 4), (0, 0)], 4, 2, 64, 16), "none_granted": ([(0, 2), (0, 1)], 4, 2, 128, 16),
    "chunk": ([(300, 130), (200, 200)], 4, 2, 128, 64), "chunk_192": ([(257, 70)], 5, 5, 192, 16),
    "chunk_256": ([(500, 65), (64, 64)], 4, 1, 256, 32), "d160": ([(70, 9)], 3, 1, 160, 16), "d224": ([(48, 48)], 2, 2, 224, 48),
    "long": ([(5003, 1)], 16, 2, 128, 64), "long_window": ([(3001, 8), (47, 8)], 8, 2, 64, 16),
    "long_chunk": ([(2100, 300)], 6, 2, 128, 16), "ragged": ([(n, min(n, 1 + n % 17)) for n in (1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 500)], 12, 4, 64, 16),
    "few_rows_long_256": ([(4000, 3)], 8, 4, 256, 64), "wide_group": ([(90, 5)], 40, 1, 128, 16),
}


@pytest.mark.parametrize("name", list(ATTENTION))
def test_paged_attention(ciar, name):
    reqs, Hq, Hk, D, page = ATTENTION[name]
    say("[attention]", name)
    lens, news = [a for a, _ in reqs], [b for _, b in reqs]
    kc, vc, table, kv = make_cache(ciar, lens, Hk, D, page, seed=len(name))
    first, spare = (2, 3) if name == "ragged" else (0, 2 if name == "none_granted" else 0)      # rows that belong to no request
    cu = [first]
    for n in news:
        cu.append(cu[-1] + n)
    T = cu[-1] + spare
    g = torch.Generator().manual_seed(5)
    sharp = 0.5 + 2.5 * torch.rand((1, Hq, 1), generator=g)
    q = (torch.randn((T, Hq, D), generator=g) * sharp).bfloat16()
    scale = 1.0 / math.sqrt(D)
    out = {"out": torch.full((T, Hq, D), 7.0).bfloat16().cuda(), "lse": torch.full((T, Hq), 7.0).cuda()}
    o = ciar.paged_attention(q.cuda(), kc, vc, table, i32(cu), i32(lens), max(news), max(lens), out=out)
    torch.cuda.synchronize()
    check_attention(o, q, kv, news, cu, scale, Hq // Hk)


def test_attention_of_strided_rows(ciar):
    """q and out with their heads outermost and at odd places; max_new and max_len larger than any request's; another scale."""
    lens, news, Hq, Hk, D, page = [77, 300], [5, 20], 6, 3, 64, 16
    kc, vc, table, kv = make_cache(ciar, lens, Hk, D, page, seed=9)
    T, g = sum(news), torch.Generator().manual_seed(6)
    q = torch.randn((Hq, T, D + 1), generator=g).bfloat16().cuda()[..., 1:].permute(1, 0, 2)
    y = torch.full((Hq, T, D + 5), 3.0).bfloat16().cuda()
    o = ciar.paged_attention(q, kc, vc, table, i32([0, 5, 25]), i32(lens), 1000, 100000, scale=-0.21,
                             out={"out": y[..., 3:D + 3].permute(1, 0, 2)})
    check_attention(o, q.cpu(), kv, news, [0, 5], -0.21, 2)
    assert bool((y[..., :3] == 3.0).all()) and bool((y[..., D + 3:] == 3.0).all())


@pytest.mark.parametrize("reqs,Hq,Hk,D", [([(100, 20)], 4, 2, 64), ([(70, 8), (40, 40)], 8, 1, 128), ([(300, 150)], 2, 2, 128),
                                          ([(1500, 4)], 8, 2, 128), ([(90, 40)], 2, 1, 256), ([(300, 200)], 4, 2, 96),
                                          ([(2000, 300)], 2, 1, 96), ([(700, 260)], 2, 1, 192), ([(100, 3), (90, 70)], 2, 2, 160),
                                          ([(1000, 400)], 1, 1, 224), ([(2500, 500)], 4, 1, 64)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_attention_keeps_what_a_row_does_not_see_out_of_it(ciar, reqs, Hq, Hk, D, bad):
    """The last new token's key and value are not finite: rows before it are as if they were not there."""
    lens, news = [a for a, _ in reqs], [b for _, b in reqs]
    kc, vc, table, kv = make_cache(ciar, lens, Hk, D, 16, seed=3)
    last = lens[0] - 1
    page, off = int(table[0, last // 16]), last % 16
    kc[page, :, 0, :, off] = bad
    vc[page, :, 0, off // 8, :, off % 8] = bad
    cu = [0]
    for n in news:
        cu.append(cu[-1] + n)
    q = torch.randn((cu[-1], Hq, D), generator=torch.Generator().manual_seed(2)).bfloat16()
    o = ciar.paged_attention(q.cuda(), kc, vc, table, i32(cu), i32(lens), max(news), max(lens))
    skip = news[0] - 1
    own = {k: torch.cat([v[:skip], v[news[0]:]]) for k, v in o.items()}
    # the first request without its last token
    kv = [(kv[0][0][:-1], kv[0][1][:-1])] + kv[1:]
    check_attention(own, torch.cat([q[:skip], q[news[0]:]]), kv, [skip] + news[1:], [0] + [c - 1 for c in cu[1:-1]], 1 / math.sqrt(D),
                    Hq // Hk)
    assert bool(torch.isnan(o["out"][skip]).any())


def test_attention_takes_pages_outside_the_cache_without_harm(ciar):
    """Broken tables and lengths give numbers of some kind for the requests concerned, and the others theirs."""
    lens, news, Hq, Hk, D = [200, 100, 150], [3, 4, 5], 4, 2, 64
    kc, vc, table, kv = make_cache(ciar, lens, Hk, D, 16, seed=13)
    kc.nan_to_num_(0.0)
    vc.nan_to_num_(0.0)
    table[1, 2], table[1, 4] = 1 << 30, -5
    q = torch.randn((12, Hq, D), generator=torch.Generator().manual_seed(2)).bfloat16()
    o = ciar.paged_attention(q.cuda(), kc, vc, table, i32([0, 3, 7, 12]), i32(lens), 5, 200)
    pick = [0, 1, 2, 7, 8, 9, 10, 11]
    check_attention({k: v[pick] for k, v in o.items()}, q[pick], [kv[0], kv[2]], [3, 5], [0, 3], 1 / math.sqrt(D), 2)
    o = ciar.paged_attention(q.cuda(), kc, vc, table, i32([0, 3, 7, 90000]), i32([200, -4, 1 << 30]), 5, 200)
    torch.cuda.synchronize()
    check_attention({k: v[:7] for k, v in o.items()}, q[:7], [kv[0], (kv[1][0][:0], kv[1][1][:0])], [3, 4], [0, 3], 1 / math.sqrt(D), 2)


TOLD = {  # [(tokens in the cache, new)], q heads, kv heads, D, page
    "one_long": ([(20, 1)] * 5 + [(9000, 1)] + [(33, 1)] * 6, 8, 2, 64, 16),
    "beyond_64": ([(7, 1)] * 70 + [(6000, 1)] + [(40, 1)] * 75 + [(3000, 1)], 4, 1, 64, 16),
    "windows": ([(5000, 8), (100, 8), (64, 7), (0, 3), (33, 8), (8, 8)], 8, 1, 128, 32),
    "wide_parts": ([(14000, 2), (1, 1), (17, 2), (0, 0)], 4, 4, 128, 16),
    "chunks": ([(3500, 90), (100, 100), (90, 17), (64, 1)], 8, 1, 128, 64), "chunks_192": ([(40, 30), (2500, 140)], 4, 2, 192, 16),
    "d256": ([(4000, 1), (30, 2), (0, 2)], 2, 1, 256, 48),
}


@pytest.mark.parametrize("name", list(TOLD))
def test_attention_of_contexts_that_differ(ciar, name):
    """Told how many tokens there are in all, the work is divided by the lengths on the GPU: every row is held to the formula."""
    reqs, Hq, Hk, D, page = TOLD[name]
    lens, news = [a for a, _ in reqs], [b for _, b in reqs]
    say("[attention told]", name, len(reqs))
    kc, vc, table, kv = make_cache(ciar, lens, Hk, D, page, seed=3 + len(name))
    T = sum(news)
    starts = [sum(news[:i]) for i in range(len(news))]
    q = torch.randn((T, Hq, D), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    cu, kl = i32(starts + [T]), i32(lens)
    scale = 1 / math.sqrt(D)
    for total in (sum(lens), sum(lens) + 500):
        args = (q, kc, vc, table, cu, kl, max(news), max(lens))
        assert ciar.attention_workspace_bytes(q, kc, table, max(news), max(lens), total) > 0      # (so that parts are what is tested)
        o = ciar.paged_attention(*args, total_len=total)
        check_attention(o, q, kv, news, starts, scale, Hq // Hk)
        p = ciar.paged_attention(*args, total_len=total)
        assert torch.equal(o["out"], p["out"]) and torch.equal(o["lse"], p["lse"])


def test_calls_without_tokens(ciar):
    """Nothing to do: no launch, no complaint about lists that have no address."""
    kc, vc, table, _ = make_cache(ciar, [4], 2, 64, 16, seed=1)
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    o = ciar.rotary(none, none, i32([]), freqs(64), v=none, k_cache=kc, v_cache=vc, slots=i32([]))
    assert o["q"].shape == (0, 2, 64)
    assert ciar.rotary(none, none, i32([]), freqs(64))["k"].shape == (0, 2, 64)
    o = ciar.paged_attention(none, kc, vc, table, i32([0, 0]), i32([4]), 0, 4)
    assert o["out"].shape == (0, 2, 64) and o["lse"].shape == (0, 2)
    e = torch.empty(0, device="cuda")
    o = ciar.adjust_logits(torch.empty((0, 40), device="cuda"), ciar.Params(window=4), history_start=torch.zeros(1, dtype=torch.int64, device="cuda"),
                           history=i32([]), drafted=i32([]), repetition=e, allowed=torch.zeros((1, 2), dtype=torch.int32, device="cuda"),
                           allowed_row=i32([]))
    assert o["logits"].shape == (0, 40) and o["left"].numel() == 0
    x = torch.randn((3, 40), device="cuda")
    zeros = torch.zeros(2, dtype=torch.int64, device="cuda")
    o = ciar.adjust_logits(x, ciar.Params(window=4), history_start=zeros, history=i32([]), prompt_len=i32([0]), bias_start=zeros, bias_ids=i32([]),
                           bias_values=e)
    assert torch.equal(o["logits"], x)


def test_attention_without_requests(ciar):
    kc, vc, table, _ = make_cache(ciar, [4], 1, 64, 16, seed=1)
    q = torch.randn((3, 2, 64)).bfloat16().cuda()
    o = ciar.paged_attention(q, kc, vc, table[:0], i32([0]), i32([]), 0, 0)
    assert bool((o["out"] == 0).all()) and bool((o["lse"] == -math.inf).all())


# ---- the logits' adjustments ----------------------------------------------------------------------------------

def adjust_reference(x, K, a):
    """In 64 bits; returns the values, the sum of the magnitudes they went through, and the finite count."""
    x = x.double().cpu()
    N, V = x.shape
    size = x.abs().nan_to_num(0.0, 0.0, 0.0)
    a = {k: v.cpu() for k, v in a.items()}
    for n in range(N):
        r = n // K
        said, seen = torch.zeros(V, dtype=torch.int64), torch.zeros(V, dtype=torch.bool)
        if "history" in a:
            lo, hi = int(a["history_start"][r]), int(a["history_start"][r + 1])
            h = a["history"][lo:hi].long()
            p = int(a["prompt_len"][r]) if "prompt_len" in a else 0
            ok = (h >= 0) & (h < V)
            seen[h[ok]] = True
            said += torch.bincount(h[ok & (torch.arange(len(h)) >= p)], minlength=V)
        if "drafted" in a:
            d = a["drafted"][r * K:n].long()
            d = d[(d >= 0) & (d < V)]
            seen[d] = True
            said += torch.bincount(d, minlength=V)
        y = x[n]
        if "repetition" in a:
            th = float(a["repetition"][r])
            y = torch.where(seen, torch.where(y > 0, y / th, y * th), y)
            size[n] = torch.maximum(size[n], y.abs().nan_to_num(0.0, 0.0, 0.0))
        if "frequency" in a:
            y = y - float(a["frequency"][r]) * said
            size[n] += abs(float(a["frequency"][r])) * said
        if "presence" in a:
            y = y - float(a["presence"][r]) * (said > 0)
            size[n] += abs(float(a["presence"][r])) * (said > 0)
        if "bias_ids" in a:
            lo, hi = int(a["bias_start"][r]), int(a["bias_start"][r + 1])
            for t, b in zip(a["bias_ids"][lo:hi].tolist(), a["bias_values"][lo:hi].tolist()):
                if 0 <= t < V:
                    y[t] += b
                    size[n, t] += abs(b)
        if "allowed" in a and int(a["allowed_row"][n]) >= 0:
            t = torch.arange(V)
            bits = (a["allowed"][int(a["allowed_row"][n])][t // 32] >> (t % 32)) & 1
            y = torch.where(bits != 0, y, -math.inf)
        x[n] = y
    return x, size, torch.isfinite(x).sum(1)


def adjust_case(N, V, K, dtype, seed, groups):
    g = torch.Generator().manual_seed(seed)
    per = 4 if dtype == torch.float32 else 8
    x = (torch.randn((N, -(-V // per) * per + per), generator=g) * 3).to(dtype)[:, :V]
    x[0, V // 2], x[-1, 0] = -math.inf, 0.0
    W = -(-N // K)
    a = {}

    def ids(n):
        return (V * torch.rand(n, generator=g) ** 2).int().clamp(max=V - 1)

    if "history" in groups:
        lens = torch.randint(0, 90, (W,), generator=g)
        a["history_start"] = torch.nn.functional.pad(torch.cumsum(lens, 0), (1, 0)) + 2
        a["history"] = torch.cat([ids(int(lens.sum()) + 2), torch.tensor([-1, V, 1 << 30], dtype=torch.int32)])
        a["history_start"][-1] += 3                                            # the last window's: three that are no tokens
        a["prompt_len"] = (lens // 3).int()
    if "drafted" in groups:
        a["drafted"] = ids(N)
        a["drafted"][N // 2] = -1
    if "penalties" in groups:
        a["repetition"] = 0.8 + torch.rand(W, generator=g)
        a["presence"], a["frequency"] = torch.rand(W, generator=g), torch.rand(W, generator=g) - 0.3
    if "bias" in groups:
        lens = torch.randint(0, 12, (W,), generator=g)
        a["bias_start"] = torch.nn.functional.pad(torch.cumsum(lens, 0), (1, 0))
        a["bias_ids"] = torch.cat([ids(int(n)).sort()[0] for n in lens] + [torch.zeros(0, dtype=torch.int32)])
        a["bias_values"] = torch.randn(int(lens.sum()), generator=g) * 3
    if "masks" in groups:
        words = (V + 31) // 32
        a["allowed"] = torch.randint(-(1 << 31), 1 << 31, (3, words + 1), generator=g, dtype=torch.int64).int()
        a["allowed"][1] = 0                                                    # nothing is left
        a["allowed_row"] = torch.randint(-1, 3, (N,), generator=g, dtype=torch.int32)
    return x, a


ALL = ("history", "drafted", "penalties", "bias", "masks")
ADJUST = [  # rows, vocabulary, window, dtype, groups
    (1, 1, 1, torch.float32, ALL), (3, 37, 2, torch.float32, ALL), (8, 1000, 8, torch.bfloat16, ALL), (17, 2049, 4, torch.float32, ALL),
    (21, 4099, 5, torch.bfloat16, ALL), (9, 16384, 8, torch.float32, ALL), (6, 65536, 3, torch.bfloat16, ALL), (70, 300, 100, torch.float32, ALL),
    (40, 5000, 40, torch.bfloat16, ALL), (5, 32768, 1, torch.float32, ALL), (10, 700, 4, torch.float32, ()), (10, 700, 4, torch.bfloat16, ("masks",)),
    (10, 700, 4, torch.bfloat16, ("bias",)), (10, 700, 4, torch.float32, ("history", "penalties")),
    (10, 700, 4, torch.float32, ("drafted", "penalties")), (10, 700, 4, torch.float32, ("history", "drafted")),
]


def check_adjust(o, x, K, a):
    want, size, left = adjust_reference(x, K, a)
    got = o["logits"].double().cpu()
    assert torch.equal(o["left"].cpu().long(), left)
    gone = want == -math.inf
    assert bool((got[gone] == -math.inf).all())
    tol = (H16 if x.dtype == torch.bfloat16 else H32) * want.abs() + 6 * H32 * size * (1 + H16) + 1e-38
    err = torch.where(gone, 0.0, (got - want).abs())
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("N,V,K,dtype,groups", ADJUST)
@pytest.mark.parametrize("place", ["new", "in_place", "wider"])
def test_adjust_logits(ciar, N, V, K, dtype, groups, place):
    say("[adjust]", N, V, K, dtype, groups, place)
    x, a = adjust_case(N, V, K, dtype, N + V, groups)
    stride = x.stride(0)
    whole = torch.full((N, stride), 5.0, dtype=dtype, device="cuda")
    gx = whole[:, :V]
    gx.copy_(x)
    out = None
    if place == "in_place":
        out = {"logits": gx}
    elif place == "wider":
        wide = torch.full((N, stride + 16), 6.0, dtype=dtype, device="cuda")
        out = {"logits": wide[:, :V]}
    o = ciar.adjust_logits(gx, ciar.Params(window=K), out=out, **{k: v.cuda() for k, v in a.items()})
    torch.cuda.synchronize()
    check_adjust(o, x, K, a)
    assert bool((whole[:, V:] == 5.0).all())
    if place == "wider":
        assert bool((wide[:, V:] == 6.0).all())


def test_adjust_logits_of_values_that_are_no_numbers(ciar):
    """Infinities and NaN stay what the formula makes of them, under a mask they are -inf, and `left` does not count them."""
    V, x = 64, torch.zeros((2, 64))
    x[:, 1], x[:, 2], x[:, 3], x[:, 4] = math.inf, -math.inf, math.nan, torch.finfo(torch.float32).min
    allowed = torch.full((1, 2), -1, dtype=torch.int32)
    allowed[0, 0] = ~0b1010
    o = ciar.adjust_logits(x.cuda(), ciar.Params(window=2), allowed=allowed.cuda(), allowed_row=i32([-1, 0]))
    y = o["logits"].cpu()
    assert y[0, 1] == math.inf and y[0, 2] == -math.inf and torch.isnan(y[0, 3]) and y[0, 4] == x[0, 4]
    assert y[1, 1] == -math.inf and y[1, 3] == -math.inf and y[1, 4] == x[0, 4]
    assert o["left"].tolist() == [61, 61]


# ---- together, on other streams, in a graph -------------------------------------------------------------------

def _step(ciar, s):
    o = ciar.cache_plan(s["lengths"], s["new"], s["held"], s["ring"], s["state"], s["table"], s["T"], page_size=16, kept=s["kept"],
                        out=s["plan"])
    r = ciar.rotary(s["q"], s["k"], o["positions"], s["freq"], v=s["v"], k_cache=s["kc"], v_cache=s["vc"], slots=o["slots"],
                    out=s["turned"])
    a = ciar.paged_attention(r["q"], s["kc"], s["vc"], s["table"], o["cu_new"], o["kv_len"], s["most"], s["width"] * 16,
                             out=s["attn"], workspace=s["aws"])
    y = ciar.adjust_logits(s["logits"], ciar.Params(window=8), drafted=s["drafted"], repetition=s["theta"], allowed=s["allowed"],
                           allowed_row=s["rows"], out=s["adj"], workspace=s["lws"])
    return {**{"plan." + k: v for k, v in o.items()}, "q": r["q"], **a, **y, "table": s["table"], "ring": s["ring"], "kc": s["kc"],
            "vc": s["vc"]}


def _state(ciar, seed, R=6, Hq=8, Hk=2, D=64, K=8, width=80):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, P = R * K, R * width + 8
    lengths = torch.randint(0, (width - 2) * 16, (R,), generator=g, device="cuda", dtype=torch.int32)
    held = (lengths + 15) // 16
    order = torch.randperm(P, generator=g, device="cuda").int()
    table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r in range(R):
        n = int(held[r])
        table[r, :n] = order[at:at + n]
        at += n
    ring = torch.zeros(P, dtype=torch.int32, device="cuda")
    ring[:P - at] = order[at:]
    ks, vs = ciar.cache_shapes(P, Hk, D, 16)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    qkv = rnd(T, Hq + 2 * Hk, D).bfloat16()
    e = lambda n, dt=torch.int32: torch.empty(n, dtype=dt, device="cuda")
    s = dict(lengths=lengths, held=held.int(), ring=ring, state=torch.tensor([0, P - at], device="cuda"), table=table, T=T, most=K,
             width=width, kept=torch.zeros(R, dtype=torch.int32, device="cuda"),
             new=torch.randint(0, K + 1, (R,), generator=g, device="cuda", dtype=torch.int32), q=qkv[:, :Hq],
             k=qkv[:, Hq:Hq + Hk], v=qkv[:, Hq + Hk:], freq=freqs(D), kc=rnd(*ks).bfloat16(), vc=rnd(*vs).bfloat16(),
             logits=rnd(T, 5000).bfloat16(), drafted=torch.randint(0, 5000, (T,), generator=g, device="cuda", dtype=torch.int32),
             theta=1 + torch.rand(R, generator=g, device="cuda"),
             allowed=torch.randint(-(1 << 31), 1 << 31, (R, 157), generator=g, device="cuda").int(),
             rows=(torch.arange(T, device="cuda") // 8).int(), turned={"q": e((T, Hq, D), torch.bfloat16)},
             plan={"lengths": e(R), "kv_len": e(R), "cu_new": e(R + 1), "held": e(R), "granted": e(R, torch.uint8),
                   "ring_state": e(2, torch.int64), "slots": e(T), "positions": e(T), "requests": e(T)},
             attn={"out": e((T, Hq, D), torch.bfloat16), "lse": e((T, Hq), torch.float32)},
             adj={"logits": e((T, 5000), torch.bfloat16), "left": e(T)})
    s["aws"] = e(max(16, ciar.attention_workspace_bytes(s["turned"]["q"], s["kc"], table, K, width * 16)), torch.uint8)
    s["lws"] = e(ciar.adjust_workspace_bytes(T), torch.uint8)
    return s


def test_step_twice_and_on_another_stream(ciar):
    """The same inputs give the same bits, also on a stream that is not the current one."""
    say("[step] streams")
    one, two, three = (_state(ciar, 4) for _ in range(3))
    a, b = _step(ciar, one), _step(ciar, two)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c = _step(ciar, three)
    torch.cuda.synchronize()
    for k in a:
        assert torch.equal(a[k], b[k]) and torch.equal(a[k], c[k]), k


def test_calls_on_a_given_stream(ciar):
    """A stream handed to the calls: outputs and workspaces that they allocate stay theirs until that stream is through."""
    say("[step] given stream")
    lens, news, Hq, Hk, D = [9000, 5000], [1, 1], 8, 2, 128
    kc, vc, table, kv = make_cache(ciar, lens, Hk, D, 16, seed=5)
    q = torch.randn((2, Hq, D), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    x, a = adjust_case(40, 5000, 40, torch.bfloat16, 3, ALL)
    x, a = x.cuda(), {k: v.cuda() for k, v in a.items()}
    cu, kl = i32([0, 1, 2]), i32(lens)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                                # the calls below wait for this
    o = ciar.paged_attention(q, kc, vc, table, cu, kl, 1, 9000, stream=side)
    y = ciar.adjust_logits(x, ciar.Params(window=40), stream=side, **a)
    trash = [torch.full((1 << 18,), 255, dtype=torch.uint8, device="cuda") for _ in range(32)]      # on the current stream, at once
    torch.cuda.synchronize()
    check_attention(o, q.cpu(), kv, news, [0, 1], 1 / math.sqrt(D), Hq // Hk)
    check_adjust(y, x.cpu(), 40, a)
    del trash


def test_step_in_a_graph(ciar):
    """Captured once, replayed on new inputs several times, with eager steps between the replays."""
    say("[step] graph")
    s = _state(ciar, 11)
    _step(ciar, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(ciar, s)
    for seed in (21, 22, 23, 24):
        fresh, eager = _state(ciar, seed), _state(ciar, seed)
        for k in ("lengths", "held", "ring", "state", "table", "kept", "new", "q", "k", "v", "kc", "vc", "logits", "drafted", "theta",
                  "allowed", "rows"):
            s[k].copy_(fresh[k])
        graph.replay()
        want = _step(ciar, eager)
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(got[k], want[k]), (seed, k)


@pytest.mark.parametrize("step", [3.0, 40.0])
@pytest.mark.parametrize("new,D", [(1, 64), (8, 128), (40, 64), (200, 128), (40, 256)])
def test_attention_of_scores_that_climb(ciar, step, new, D):
    """Scores that grow from token to token by far more than the range of 32 bits between the first and the last: the softmax's
    reference is found again (values large enough to overflow where it is not)."""
    L, Hq, Hk, page = 700, 4, 2, 16
    kc, vc, table, kv = make_cache(ciar, [L], Hk, D, page, seed=17)
    for i in range(L):
        p, off = int(table[0, i // page]), i % page
        for cache, rows, x in ((kc, kv[0][0], step * (i // 8)), (vc, kv[0][1], 1e33 if i % 2 else -2e33)):
            rows[i, :, :] = torch.tensor(x).bfloat16().double()
    rows_k, rows_v = kv[0]
    i = torch.arange(L)
    page_of, off = table[0].cpu()[i // page].long(), i % page
    kc[page_of.cuda(), :, 0, :, off.cuda()] = rows_k.bfloat16().cuda().view(L, Hk, D // 8, 8)
    vc[page_of.cuda(), :, 0, (off // 8).cuda(), :, (off % 8).cuda()] = rows_v.bfloat16().cuda()
    q = torch.full((new, Hq, D), 1.0 / D).bfloat16()
    o = ciar.paged_attention(q.cuda(), kc, vc, table, i32([0, new]), i32([L]), new, L, scale=1.0)
    assert bool(torch.isfinite(o["out"].float()).all())
    check_attention(o, q, kv, [new], [0], 1.0, Hq // Hk)


MANY_ROWS = [  # D, [(tokens in the cache, new)], q heads, kv heads, page: what the matrix cores' kernel takes, 128 and 256 rows, whole and in parts
    (32, [(600, 50), (599, 33), (310, 49), (64, 50)], 128, 64, 16), (32, [(130, 100), (129, 99), (100, 100), (128, 65)], 128, 32, 16),
    (64, [(300, 33), (299, 32), (40, 33)], 128, 64, 32), (64, [(2000, 100), (1501, 99), (100, 100), (1999, 3)], 16, 16, 16),
    (64, [(130, 130), (129, 100), (130, 77), (16, 16)], 64, 16, 16), (64, [(1500, 130), (1400, 130), (131, 129)], 32, 32, 16),
    (96, [(130, 50), (129, 49), (50, 50)], 128, 64, 16), (96, [(2000, 33), (1999, 32), (33, 33), (700, 31)], 16, 8, 48),
    (96, [(130, 130), (129, 129), (130, 1), (64, 64)], 32, 8, 16), (96, [(2000, 130), (1300, 130), (129, 65), (130, 130)], 8, 8, 16),
    (128, [(130, 33), (129, 32), (64, 33)], 128, 64, 16), (128, [(2000, 33), (1999, 32), (33, 33), (700, 31)], 16, 8, 64),
    (128, [(130, 130), (129, 129), (130, 5), (130, 64)], 32, 8, 32), (128, [(2000, 130), (1300, 130), (129, 65), (130, 130)], 8, 8, 16),
    (160, [(130, 33), (129, 33), (40, 31)], 64, 32, 16), (160, [(1500, 33), (1499, 32), (33, 33)], 16, 16, 32),
    (192, [(130, 33), (129, 33), (40, 31)], 64, 32, 16), (192, [(1000, 33), (999, 32), (33, 33), (512, 33)], 16, 16, 64),
    (224, [(130, 33), (129, 33), (40, 31)], 32, 32, 16), (224, [(1000, 33), (999, 32), (33, 33), (512, 33)], 8, 8, 16),
    (256, [(130, 33), (129, 33), (40, 31)], 32, 32, 48), (256, [(1000, 33), (999, 32), (33, 33), (512, 33)], 8, 8, 16),
]


FEW_ROWS = [  # the same, for the kernel of few rows: 16, 32 and 64 rows, in one part, a few, many
    *((D, [(L, n)], h, 1, 16) for D in range(32, 257, 32) for h, n in ((3, 3), (4, 5)) for L in (40, 1000, 2000)),
    (32, [(1000, 12), (999, 11), (33, 12)] * 6, 48, 16, 16), (64, [(1000, 24), (31, 20)] * 8, 24, 8, 16), (64, [(4000, 40), (3333, 39), (64, 1), (40, 40)], 8, 1, 64),
    (96, [(40, 24), (39, 23)] * 8, 24, 8, 16), (96, [(4000, 12), (130, 12), (12, 9), (0, 3)] * 4, 6, 2, 48), (128, [(40, 24), (25, 24)] * 8, 24, 8, 16),
    (128, [(2000, 40), (1025, 33)] * 8, 2, 2, 16), (128, [(4000, 40), (129, 40), (2222, 20), (40, 40)], 8, 1, 32),
]


def attention_case(ciar, case, kind, seed):
    """plain; the first request's last key and value not finite, which only its last row sees; scores of the first request that climb out of
    range; the tokens in all told."""
    D, reqs, Hq, Hk, page = case
    say("[attention]", kind, case)
    lens, news = [a for a, _ in reqs], [b for _, b in reqs]
    kc, vc, table, kv = make_cache(ciar, lens, Hk, D, page, seed=seed)
    starts, T, L = [sum(news[:i]) for i in range(len(news))], sum(news), lens[0]
    i = torch.arange(L)
    pages, atom, t = table[0].cpu()[i // page].long().cuda(), (i % page // 16).cuda(), (i % 16).cuda()
    q = torch.randn((T, Hq, D), generator=torch.Generator().manual_seed(seed)).bfloat16()
    if kind in ("inf", "nan"):
        kc[pages[-1], :, atom[-1], :, t[-1]] = vc[pages[-1], :, atom[-1], t[-1] // 8, :, t[-1] % 8] = float(kind)
    if kind == "climb":
        q[:news[0]] = 1.0 / D
        kv[0][0][:] = (3.0 * (i // 8)).bfloat16().double()[:, None, None]
        kv[0][1][:] = torch.where(i % 2 == 0, -2e33, 1e33).bfloat16().double()[:, None, None]
        kc[pages, :, atom, :, t] = kv[0][0].bfloat16().cuda().view(L, Hk, D // 8, 8)
        vc[pages, :, atom, t // 8, :, t % 8] = kv[0][1].bfloat16().cuda()
    scale = 1.0 if kind == "climb" else 1 / math.sqrt(D)
    o = ciar.paged_attention(q.cuda(), kc, vc, table, i32(starts + [T]), i32(lens), max(news), max(lens), scale=scale,
                             total_len=sum(lens) if kind == "told" else None)
    torch.cuda.synchronize()
    if kind in ("inf", "nan"):
        n = news[0] - 1
        assert bool(torch.isnan(o["out"][n]).any())
        o, q = {k: torch.cat([v[:n], v[n + 1:]]) for k, v in o.items()}, torch.cat([q[:n], q[n + 1:]])
        kv, news, starts = [(kv[0][0][:-1], kv[0][1][:-1])] + kv[1:], [n] + news[1:], [0] + [b - 1 for b in starts[1:]]
    check_attention(o, q, kv, news, starts, scale, Hq // Hk)


@pytest.mark.parametrize("case", range(len(MANY_ROWS)))
@pytest.mark.parametrize("kind", ["plain", "inf", "nan", "climb", "told"])
def test_attention_of_many_rows(ciar, case, kind):
    attention_case(ciar, MANY_ROWS[case], kind, case)


@pytest.mark.parametrize("case", range(len(FEW_ROWS)))
@pytest.mark.parametrize("kind", ["plain", "nan", "climb", "told"])
def test_attention_of_few_rows(ciar, case, kind):
    attention_case(ciar, FEW_ROWS[case], kind, case)
