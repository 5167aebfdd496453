"""The operators on a paged key/value cache (include/attn.h): the append with its rotation, and the attention over the cache, with and
without a shared prefix, against plain evaluations in 64 bits.

Tolerance of the attention, element by element.  The kernel keeps logits, statistics and sums in fp32 and rounds twice: the weights to
the input type before the second product (relative u = 2^-11 binary16, 2^-8 bfloat16; binary16 weights below 2^-14 lose up to 2^-25 each,
and the sum of weights is at least 1 because the reference never exceeds the row's maximum), and the result.  fp32 logits are sums of D
products and one multiplication: off by at most (D + 2) 2^-24 scale sum |q| |k|, below 2^-16 z with z = scale |q| . |k| at its largest; the sum
of weights, the exponential and the division add less than 2e-5 relative for the lengths here.  With A = sum_j w_j |v_j|:
    |o - ref| <= (u + 2^-16 z + 2e-5) A + 2^-25 sum_j |v_j| [binary16] + u |ref| + 2^-25
    |lse - ref| <= 2^-16 z + 2e-5 max(1, |ref|)
"""
import math

import pytest
import torch

import paper_2501_08071_amd as P

pytestmark = pytest.mark.gpu

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
F16, BF16 = torch.float16, torch.bfloat16


def make(new, kv, Hq, Hk, D, page, dtype, prefix=0, seed=0, mul=1.0, interleave=False, spare=3, nan=True, width=None):
    """A batch: pages in random order, everything that is no key NaN, table entries past a sequence's end no page at all."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-max(0, n) // page) for n in kv]
    pn = -(-prefix // page)
    n_pages = sum(need) + pn + spare
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    W = max(1, max(need, default=1)) if width is None else width
    table = torch.full((len(kv), W), 2 ** 30, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (n_pages, Hk, page, D)
    fill = float("nan") if nan else 1.0
    if interleave:
        both = torch.full((n_pages, 2, Hk, page, D), fill, dtype=dtype)
        kc, vc = both[:, 0], both[:, 1]
    else:
        kc, vc = torch.full(shape, fill, dtype=dtype), torch.full(shape, fill, dtype=dtype)
    for pages, n in [(table[b, :need[b]], kv[b]) for b in range(len(kv))] + [(order[at:at + pn], prefix)]:
        for c in (kc, vc):
            for j, pg in enumerate(pages.tolist()):
                m = min(page, n - j * page)
                c[pg, :, :m] = (torch.randn(Hk, m, D, generator=g) * (mul if c is kc else 1.0)).to(dtype)
    T = sum(new)
    q = (torch.randn(T, Hq * D + 2 * Hk * D, generator=g) * mul).to(dtype)
    if interleave:
        both = both.cuda()
        kc, vc = both[:, 0], both[:, 1]
    cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32)
    return {"q": q.cuda()[:, :Hq * D].view(T, Hq, D), "k_cache": kc.cuda(), "v_cache": vc.cuda(), "page_table": table.cuda(), "cu_q": cu.cuda(),
            "kv_len": torch.tensor(kv, dtype=torch.int32).cuda(), "prefix_table": order[at:at + pn].cuda() if prefix else None,
            "prefix_len": prefix}


def reference(s, scale):
    """o, lse, and what the tolerances need, in 64 bits on the CPU, row by row of the definition."""
    q, kc, vc = (s[n].cpu().double() for n in ("q", "k_cache", "v_cache"))
    table, cu, kv = s["page_table"].cpu(), s["cu_q"].tolist(), s["kv_len"].tolist()
    T, Hq, D = q.shape
    Hk, page = kc.shape[1], kc.shape[2]
    G, pre = Hq // Hk, s["prefix_len"]

    def keys(c, pages, n):
        return c[pages[:-(-n // page)].long()].transpose(0, 1).reshape(Hk, -1, D)[:, :n]

    o, lse = torch.zeros(T, Hq, D, dtype=torch.float64), torch.full((T, Hq), -math.inf, dtype=torch.float64)
    A, V, z = torch.zeros_like(o), torch.zeros_like(o), torch.zeros_like(lse)
    for b in range(len(kv)):
        n, L = cu[b + 1] - cu[b], max(0, kv[b])
        k, v = keys(kc, table[b], L), keys(vc, table[b], L)
        if pre:
            k, v = (torch.cat((keys(c, s["prefix_table"].cpu(), pre), x), 1) for c, x in ((kc, k), (vc, v)))
        for i in range(n):
            m = pre + max(0, min(L, kv[b] - n + i + 1))
            if m == 0:
                continue
            t = cu[b] + i
            for h in range(Hk):
                qq = q[t, h * G:(h + 1) * G]
                x = scale * qq @ k[h, :m].T
                w = torch.softmax(x, 1)
                sl = slice(h * G, (h + 1) * G)
                o[t, sl], lse[t, sl] = w @ v[h, :m], torch.logsumexp(x, 1)
                A[t, sl], V[t, sl] = w @ v[h, :m].abs(), v[h, :m].abs().sum(0)
                z[t, sl] = abs(scale) * (qq.abs() @ k[h, :m].abs().T).amax(1)
    return o, lse, A, V, z


def check(got, ref, dtype):
    o, lse, A, V, z = ref
    u = U[dtype]
    go, gl = got[0].double().cpu(), got[1].double().cpu()
    assert torch.equal(torch.isinf(gl), torch.isinf(lse)) and not torch.isnan(gl).any() and torch.isfinite(go).all()
    tol = (u + 2.0 ** -16 * z[..., None] + 2e-5) * A + (2.0 ** -25 * V if dtype == F16 else 0) + u * o.abs() + 2.0 ** -25
    worst = ((go - o).abs() / tol).max().item() if o.numel() else 0.0
    assert worst <= 1.0, f"o is {worst:.2f} times the tolerance off"
    fine = torch.isfinite(lse)
    tol = 2.0 ** -16 * z + 2e-5 * lse.abs().clamp(min=1.0)
    assert ((gl - lse).abs()[fine] <= tol[fine]).all()
    assert (go[~fine] == 0).all()


def attend(s, scale, **kw):
    if "max_q" not in kw:
        kw["max_q"] = int((s["cu_q"][1:] - s["cu_q"][:-1]).max()) if s["cu_q"].numel() > 1 else 0
    return P.attn_paged_fwd(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["cu_q"], s["kv_len"], scale, prefix_table=s["prefix_table"],
                            prefix_len=s["prefix_len"], **kw)


# new tokens and keys of every sequence: one token, lengths around blocks and pages, none at all, fewer keys than tokens, no new token
BATCHES = {
    "one key": ([1], [1]),
    "edges": ([1] * 9, [1, 15, 16, 17, 31, 32, 33, 64, 65]),
    "empty ones": ([1, 0, 2, 1, 3], [0, 50, 1, 7, 0]),
    "drafts": ([1, 5, 2, 7], [200, 129, 2, 300]),
    "chunks": ([40, 1, 0, 33], [40, 90, 12, 257]),
    "more tokens than keys": ([6, 3], [2, 3]),
    "longer": ([1, 2], [1500, 700]),
}


@pytest.mark.parametrize("hint", ["short", "long"])     # whole tiles to a workgroup, keys shared out
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("Hq,Hk,D,page,dtype", [(8, 2, 128, 16, BF16), (3, 3, 64, 32, F16), (10, 2, 32, 8, BF16), (20, 1, 128, 64, F16)])
def test_attention(Hq, Hk, D, page, dtype, batch, hint):
    new, kv = BATCHES[batch]
    s = make(new, kv, Hq, Hk, D, page, dtype, seed=len(batch))
    scale = 1.0 / math.sqrt(D)
    check(attend(s, scale, max_kv=1 if hint == "short" else 1 << 20), reference(s, scale), dtype)


@pytest.mark.parametrize("prefix", [1, 31, 100, 777])
@pytest.mark.parametrize("batch", ["one key", "empty ones", "drafts", "chunks", "longer"])
@pytest.mark.parametrize("Hq,Hk,D,page,dtype", [(8, 2, 128, 16, BF16), (6, 6, 64, 32, F16), (16, 2, 32, 8, F16)])
def test_shared_prefix(Hq, Hk, D, page, dtype, batch, prefix):
    new, kv = BATCHES[batch]
    s = make(new, kv, Hq, Hk, D, page, dtype, prefix=prefix, seed=prefix)
    check(attend(s, D ** -0.5), reference(s, D ** -0.5), dtype)


@pytest.mark.parametrize("page", [1, 2, 4, 16, 128, 512])
def test_page_sizes_and_interleaved_pages(page):
    s = make([1, 4, 2], [77, 130, 513], 4, 2, 64, page, BF16, prefix=45, seed=page, interleave=True)
    assert s["k_cache"].stride(0) == 2 * 2 * page * 64
    check(attend(s, 0.125), reference(s, 0.125), BF16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_scales(dtype, scale):
    s = make([1, 3], [300, 65], 4, 1, 64, 16, dtype, prefix=33, seed=7)
    check(attend(s, scale), reference(s, scale), dtype)


@pytest.mark.parametrize("rising", [True, False])
def test_references_that_move(rising):
    """Keys whose logits rise (or fall) all along the sequence, by far more than the weights' range."""
    s = make([1, 2], [900, 400], 2, 1, 64, 16, F16, prefix=100, seed=3)
    n = s["k_cache"].shape[0]
    for b, pages in enumerate([s["page_table"][0][:57], s["page_table"][1][:25], s["prefix_table"]]):
        f = torch.linspace(0.1, 8.0, len(pages), device="cuda")
        f = f if rising else f.flip(0)
        base = s["q"][0, 0].float()
        s["k_cache"][pages.long()] = (f[:, None, None, None] * base + 0.01 * torch.randn(len(pages), 1, 16, 64, device="cuda")).to(F16)
    assert n == s["k_cache"].shape[0]
    check(attend(s, 0.5), reference(s, 0.5), F16)


def test_many_sequences_of_few_keys():
    new = [1 + i % 2 for i in range(700)]
    kv = [n + i % 40 for i, n in enumerate(new)]
    s = make(new, kv, 2, 1, 32, 16, BF16, seed=5)
    ref = reference(s, 0.2)
    check(attend(s, 0.2, max_kv=41), ref, BF16)
    check(attend(s, 0.2), ref, BF16)


@pytest.mark.parametrize("D,Hq,Hk", [(128, 8, 2), (64, 20, 1), (32, 64, 1), (64, 6, 2)])
def test_a_hint_that_is_too_small(D, Hq, Hk):
    """Keys past max_kv are not lost where the work is shared out by it."""
    s = make([1, 2, 1, 1], [3000, 1200, 5, 0], Hq, Hk, D, 16, BF16, prefix=40, seed=D)
    ref = reference(s, D ** -0.5)
    for hint in (1050, 1300, 2999):
        check(attend(s, D ** -0.5, max_kv=hint), ref, BF16)


def test_hints_that_are_far_too_large():
    s = make([1, 2, 1, 3], [300, 120, 5, 0], 8, 2, 64, 16, F16, prefix=40, seed=21)
    ref, top = reference(s, 0.125), 2 ** 31 - 1
    for max_kv in (300, 5000, top):
        want = attend(s, 0.125, max_q=7, max_kv=max_kv)
        check(want, ref, F16)
        got = attend(s, 0.125, max_q=top, max_kv=max_kv)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("rising", [True, False])
def test_many_rows_whose_references_move(rising):
    """128-row tiles: keys whose logits rise or fall all along the sequence, a row's own limit inside the last blocks."""
    s = make([70, 3], [400, 130], 4, 1, 128, 16, F16, prefix=200, seed=13)
    for pages in (s["page_table"][0][:25], s["page_table"][1][:9], s["prefix_table"]):
        f = torch.linspace(0.1, 8.0, len(pages), device="cuda")
        f = f if rising else f.flip(0)
        s["k_cache"][pages.long()] = (f[:, None, None, None] * s["q"][0, 0].float() + 0.01 * torch.randn(len(pages), 1, 16, 128, device="cuda")).to(F16)
    ref = reference(s, 0.3)
    check(attend(s, 0.3), ref, F16)
    check(attend(s, 0.3, max_kv=1 << 20), ref, F16)


def test_rows_that_no_sequence_owns_and_rows_past_max_q():
    s = make([2, 1], [40, 30], 2, 1, 64, 16, F16, seed=1)
    ref = reference(s, 0.125)
    q = torch.cat((s["q"], s["q"][:2]))
    o = torch.full((5, 2, 64), 7.0, dtype=F16, device="cuda")
    lse = torch.full((5, 2), 7.0, device="cuda")
    P.attn_paged_fwd(q, s["k_cache"], s["v_cache"], s["page_table"], s["cu_q"], s["kv_len"], 0.125, max_q=2, o=o, lse=lse)
    check((o[:3], lse[:3]), ref, F16)
    assert (o[3:] == 7.0).all() and (lse[3:] == 7.0).all()
    o.fill_(7.0)
    P.attn_paged_fwd(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["cu_q"], s["kv_len"], 0.125, max_q=1, o=o[:3])
    assert (o[1] == 7.0).all() and torch.equal(o[0], P.attn_paged_fwd(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["cu_q"], s["kv_len"], 0.125)[0][0])


def test_lengths_that_make_no_sense_touch_nothing_else():
    """Offsets out of order or past T, negative and huge lengths: no index leaves its buffer, the sequences that make sense are right."""
    s = make([1, 1, 1], [50, 60, 70], 4, 2, 64, 16, BF16, seed=2)
    good = attend(s, 0.125)[0]
    s["kv_len"][0], s["cu_q"][3] = -5, 1000
    s["kv_len"][2] = 2 ** 31 - 1
    for hint in (1, 1 << 20):
        o, _ = attend(s, 0.125, max_q=3, max_kv=hint)
        assert torch.equal(o[1], good[1]) or (o[1].float() - good[1].float()).abs().max() <= 2.0 ** -6
        assert (o[0] == 0).all()
    s["cu_q"][1] = -7
    attend(s, 0.125, max_q=3)
    k = torch.zeros(3, 2, 64, dtype=BF16, device="cuda")
    before = s["k_cache"].clone()
    P.attn_kv_append(None, k, k, s["k_cache"], s["v_cache"], s["page_table"], s["cu_q"], s["kv_len"])
    torch.cuda.synchronize()
    assert ((s["k_cache"] == before) | before.isnan() | (s["k_cache"] == 0)).all()


def test_a_cache_past_32_bits_and_a_long_sequence():
    """Pages that begin beyond 2^32 elements, and 70001 keys."""
    page, Hk, D, L = 64, 2, 64, 70001
    n_pages, stride = 1300, 4 * 1024 * 1024
    buf = torch.empty(n_pages * stride, dtype=BF16, device="cuda")
    assert buf.numel() > 2 ** 32
    kc = buf.as_strided((n_pages, Hk, page, D), (stride, page * D, D, 1))
    vc = buf.as_strided((n_pages, Hk, page, D), (stride, page * D, D, 1), storage_offset=Hk * page * D)
    g = torch.Generator(device="cuda").manual_seed(1)
    order = torch.randperm(n_pages, generator=g, device="cuda")[:-(-L // page)].to(torch.int32)
    k = torch.randn(len(order), Hk, page, D, generator=g, device="cuda").to(BF16)
    v = torch.randn(len(order), Hk, page, D, generator=g, device="cuda").to(BF16)
    kc[order.long()], vc[order.long()] = k, v
    q = torch.randn(2, 8, D, generator=g, device="cuda").to(BF16)
    cu, kv = torch.tensor([0, 2], dtype=torch.int32).cuda(), torch.tensor([L], dtype=torch.int32).cuda()
    o, lse = P.attn_paged_fwd(q, kc, vc, order[None], cu, kv, 0.125, max_q=2)
    kd, vd = (x.transpose(0, 1).reshape(Hk, -1, D)[:, :L].double() for x in (k, v))
    for t in range(2):
        m = L - 1 + t
        for h in range(Hk):
            x = 0.125 * q[t, 4 * h:4 * h + 4].double() @ kd[h, :m].T
            w = torch.softmax(x, 1)
            ref, A = w @ vd[h, :m], w @ vd[h, :m].abs()
            assert ((o[t, 4 * h:4 * h + 4].double() - ref).abs() <= (2.0 ** -8 + 1e-3) * A + 2.0 ** -8 * ref.abs()).all()
            assert ((lse[t, 4 * h:4 * h + 4].double() - torch.logsumexp(x, 1)).abs() <= 1e-3).all()


@pytest.mark.parametrize("D,Hq", [(128, 4), (64, 2)])
def test_a_page_past_32_bits(D, Hq):
    """A page of more than 2^31 bytes: what is stored past its first 2^31 is what is read back, by one token, by some, as a prefix.  The keys in
    front are zeros, with logit 0 and value 0; those at the end have logits around 30, and outweigh them."""
    front, n, dtype = 2 ** 32 // (2 * D), 40, BF16             # keys of 2^32 bytes
    page = 2 * front
    g = torch.Generator(device="cuda").manual_seed(D)
    kc, vc = (torch.zeros(1, 1, page, D, dtype=dtype, device="cuda") for _ in range(2))
    scale = D ** -0.5
    q = (1.0 + 0.3 * torch.randn(n, Hq, D, device="cuda", generator=g)).to(dtype)
    k = (30.0 / (scale * D) + 0.3 * torch.randn(n, 1, D, device="cuda", generator=g)).to(dtype)
    v = torch.randn(n, 1, D, device="cuda", generator=g).to(dtype)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    P.attn_kv_append(None, k, v, kc, vc, table, i32(0, n), i32(front + n))
    assert torch.equal(kc[0, 0, front:front + n], k[:, 0]) and torch.equal(vc[0, 0, front:front + n], v[:, 0])

    def expected(rows, sees):
        """Rows of q, the first of the keys at the end that each sees."""
        z = scale * q[rows].double() @ k[:, 0].double().T
        hidden = torch.arange(n, device="cuda")[None, None, :] >= torch.tensor(sees, device="cuda")[:, None, None]
        w = z.masked_fill(hidden, -math.inf).exp()
        total = w.sum(-1) + front
        vd = v[:, 0].double()
        size = scale * (q[rows].double().abs() @ k[:, 0].double().abs().T).amax(-1)
        return [t.cpu() for t in (w @ vd / total[..., None], total.log(), w @ vd.abs() / total[..., None], torch.zeros(len(rows), Hq, D), size)]

    last = list(range(n - 1, n))
    got = P.attn_paged_fwd(q[last], kc, vc, table, i32(0, 1), i32(front + n), scale, max_q=1)
    check(got, expected(last, [n]), dtype)
    got = P.attn_paged_fwd(q, kc, vc, table, i32(0, n), i32(front + n), scale, max_q=n)
    check(got, expected(list(range(n)), [i + 1 for i in range(n)]), dtype)
    for rows in (last, list(range(n))):
        got = P.attn_paged_fwd(q[rows], kc, vc, table, i32(0, len(rows)), i32(0), scale, max_q=len(rows), prefix_table=table[0], prefix_len=front + n)
        check(got, expected(rows, [n] * len(rows)), dtype)


def test_what_non_finite_values_do():
    """A NaN key, an infinite value: in the rows that see them and no others of other sequences; rows that repeat bit for bit."""
    s = make([1, 1, 1], [100, 100, 100], 2, 1, 64, 16, BF16, seed=9)
    pages = s["page_table"].long()
    s["k_cache"][pages[0, 2], 0, 5] = float("nan")
    s["v_cache"][pages[1, 3], 0, 2, 7] = float("inf")
    o, lse = attend(s, 0.125)
    assert torch.isnan(o[0]).all() and torch.isnan(lse[0]).all()
    assert torch.isinf(o[1, :, 7]).all() and torch.isfinite(o[1, :, :7]).all() and torch.isfinite(lse[1:]).all()
    assert torch.isfinite(o[2]).all()
    again, _ = attend(s, 0.125)
    assert torch.equal(again.view(torch.int16), o.view(torch.int16))


@pytest.mark.parametrize("n,bad", [(5, 3), (70, 40)])       # 16- and 128-row tiles
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_key_that_a_row_does_not_see_may_hold_anything(n, bad, value):
    """A new token's key that is not finite: the tokens before it are as right as without."""
    for D, dtype in ((64, F16), (128, BF16)):
        s = make([n], [n + 30], 2, 1, D, 16, dtype, seed=n)
        ref, at = reference(s, 0.125), 30 + bad
        s["k_cache"][s["page_table"][0, at // 16].long(), 0, at % 16] = value
        for max_kv in (n + 30, 1 << 20):
            o, lse = attend(s, 0.125, max_kv=max_kv)
            check((o[:bad], lse[:bad]), tuple(t[:bad] for t in ref), dtype)
            assert value == value or (torch.isnan(o[bad:]).all() and torch.isnan(lse[bad:]).all())


def test_pages_that_do_not_exist_are_absent_keys():
    s = make([1], [160], 2, 1, 64, 16, F16, seed=2)
    t = s["page_table"]
    t[0, 3], t[0, 7] = -5, 1 << 20
    got = attend(s, 0.125)
    keep = [j for j in range(160) if j // 16 not in (3, 7)]
    pages = t[0].long()
    k, v = (torch.cat([c[pages[j // 16], 0, j % 16][None] for j in keep]).double() for c in (s["k_cache"], s["v_cache"]))
    x = 0.125 * s["q"][0].double() @ k.T
    w = torch.softmax(x, 1)
    assert (got[0][0].double() - w @ v).abs().max() <= 4 * 2.0 ** -11 and (got[1][0].double() - torch.logsumexp(x, 1)).abs().max() <= 1e-4


def test_streams_graphs_outputs_and_workspaces():
    s = make([1, 4, 1], [900, 77, 2000], 8, 2, 128, 16, BF16, prefix=300, seed=4)
    want, want_lse = attend(s, 0.09)
    T, Hq, D = s["q"].shape
    o, lse = torch.empty(T, Hq, D, dtype=BF16, device="cuda"), torch.empty(T, Hq, device="cuda")
    size = P.attn_paged_workspace(3, T, Hq, 2, D, 4, 2048, 300)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    got = attend(s, 0.09, o=o, lse=lse, workspace=ws, max_kv=2048)
    assert got[0] is o and got[1] is lse and torch.equal(o, want)
    assert attend(s, 0.09, want_lse=False)[1] is None
    with pytest.raises(P.AttnError) as e:
        attend(s, 0.09, workspace=ws[:size - 16], max_kv=2048)
    assert e.value.status == -8
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, _ = attend(s, 0.09, stream=side)
    with torch.cuda.stream(side):
        b, _ = attend(s, 0.09)
    side.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attend(s, 0.09, o=o, lse=lse, max_q=4)
    for n in (2000, 1999, 900, 1):
        s["kv_len"][2] = n
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        ref, ref_lse = attend(s, 0.09, max_q=4)
        assert torch.equal(o, ref) and torch.equal(lse, ref_lse)


# ---- append

def turned(x, angle_cos, angle_sin, interleaved):
    h = angle_cos.shape[1]
    y = x.clone()
    for j in range(h):
        u, v = (2 * j, 2 * j + 1) if interleaved else (j, j + h)
        c, n = angle_cos[:, None, j], angle_sin[:, None, j]
        y[..., u], y[..., v] = x[..., u] * c - x[..., v] * n, x[..., v] * c + x[..., u] * n
    return y


@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("Hq,Hk,D,page,rot,interleaved,dtype", [(8, 2, 128, 16, 128, False, BF16), (3, 3, 64, 32, 32, True, F16),
                                                               (10, 2, 32, 8, 16, False, F16), (1, 1, 128, 1, 64, False, F16),
                                                               (70, 20, 32, 64, 32, True, BF16), (4, 1, 64, 16, 0, False, BF16)])
def test_append(Hq, Hk, D, page, rot, interleaved, dtype, batch):
    """Every element: rotated ones within fp32's rounding of two products and one rounding to the type, the rest bit for bit, and nothing
    outside the new tokens' slots."""
    new, kv = BATCHES[batch]
    s = make(new, kv, Hq, Hk, D, page, dtype, seed=11, interleave=True, nan=False)
    T, offset = sum(new), 5
    qkv = torch.randn(T, (Hq + 2 * Hk) * D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(dtype)
    q, k, v = qkv[:, :Hq * D].view(T, Hq, D), qkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D), qkv[:, (Hq + Hk) * D:].view(T, Hk, D)
    cos = sin = None
    if rot:
        angle = torch.randn(2000, rot // 2, dtype=torch.float64)
        cos, sin = angle.cos().float().cuda(), angle.sin().float().cuda()
    before = [s["k_cache"].cpu().double(), s["v_cache"].cpu().double()]
    out = P.attn_kv_append(q, k, v, s["k_cache"], s["v_cache"], s["page_table"], s["cu_q"], s["kv_len"], cos=cos, sin=sin,
                           interleaved=interleaved, pos_offset=offset)
    owner = [b for b in range(len(new)) for _ in range(new[b])]
    place = [kv[b] - new[b] + i for b in range(len(new)) for i in range(new[b])]
    qd, kd, vd = (t.cpu().double() for t in (q, k, v))
    mag_q, mag_k = torch.zeros_like(qd), torch.zeros_like(kd)
    if rot:
        at = torch.tensor([max(0, p + offset) for p in place])
        c, n = cos.cpu().double()[at], sin.cpu().double()[at]
        mag_q[..., :rot] = turned(qd.abs(), c.abs(), -n.abs(), interleaved)[..., :rot].abs() + turned(qd.abs(), c.abs(), n.abs(), interleaved)[..., :rot].abs()
        mag_k[..., :rot] = turned(kd.abs(), c.abs(), -n.abs(), interleaved)[..., :rot].abs() + turned(kd.abs(), c.abs(), n.abs(), interleaved)[..., :rot].abs()
        qd, kd = turned(qd, c, n, interleaved), turned(kd, c, n, interleaved)
    tol = lambda ref, mag: torch.where(mag > 0, U[dtype] * ref.abs() + 2.0 ** -22 * mag + 2.0 ** -25, 0.0)  # noqa: E731
    stored = torch.tensor([p >= 0 for p in place], dtype=torch.bool)
    assert ((out.cpu().double() - qd).abs() <= tol(qd, mag_q)).all()
    table = s["page_table"].cpu()
    want_k, want_v, off = before[0].clone(), before[1].clone(), torch.zeros_like(before[0])
    for t, (b, p) in enumerate(zip(owner, place)):
        if p >= 0:
            pg = int(table[b, p // page])
            want_k[pg, :, p % page], want_v[pg, :, p % page] = kd[t], vd[t]
            off[pg, :, p % page] = tol(kd[t], mag_k[t])
    assert ((s["k_cache"].cpu().double() - want_k).abs() <= off).all() and torch.equal(s["v_cache"].cpu().double(), want_v)
    assert stored.sum() == sum(1 for p in place if p >= 0)


def test_append_forms():
    """In place on contiguous queries, keys and values alone, many tokens, more tokens than sequences own, positions past the angles."""
    T, Hq, Hk, D, page = 5000, 4, 2, 64, 16
    g = torch.Generator(device="cuda").manual_seed(8)
    q, k, v = (torch.randn(T, h, D, device="cuda", generator=g).to(F16) for h in (Hq, Hk, Hk))
    W = -(-T // page)
    kc, vc = torch.zeros(W, Hk, page, D, dtype=F16, device="cuda"), torch.zeros(W, Hk, page, D, dtype=F16, device="cuda")
    table = torch.arange(W, dtype=torch.int32, device="cuda")[None]
    cu, kv = torch.tensor([0, T - 7], dtype=torch.int32).cuda(), torch.tensor([T - 7], dtype=torch.int32).cuda()
    cos, sin = torch.full((100, D // 2), 0.0, device="cuda"), torch.full((100, D // 2), 1.0, device="cuda")
    qq = q.clone()
    assert P.attn_kv_append(qq, k, v, kc, vc, table, cu, kv, cos=cos, sin=sin, q_out=qq) is qq
    assert torch.equal(qq[:T - 7], torch.cat((-q[..., D // 2:], q[..., :D // 2]), -1)[:T - 7])     # a quarter turn, all positions alike
    flat = vc.transpose(1, 2).reshape(-1, Hk, D)
    assert torch.equal(flat[:T - 7], v[:T - 7]) and (flat[T - 7:] == 0).all()
    kc2 = torch.zeros_like(kc)
    assert P.attn_kv_append(None, k, v, kc2, vc, table, cu, kv, cos=cos, sin=sin) is None
    assert torch.equal(kc2, kc)
    # a page that is not there: the others are stored, nothing else is touched
    table[0, 1] = -1
    kc3 = torch.zeros_like(kc)
    P.attn_kv_append(None, k, v, kc3, torch.zeros_like(vc), table, cu, kv, cos=cos, sin=sin)
    assert (kc3[1] == 0).all() and torch.equal(kc3[0], kc[0]) and torch.equal(kc3[2:], kc[2:])


def test_append_then_attend():
    """A sequence built token by token, in one piece, and as a prefix with a rest gives the same answers."""
    Hq, Hk, D, page, n = 4, 2, 64, 16, 50
    g = torch.Generator(device="cuda").manual_seed(6)
    q, k, v = (torch.randn(n, h, D, device="cuda", generator=g).to(BF16) for h in (Hq, Hk, Hk))
    angle = torch.arange(200, device="cuda")[:, None] * 10000.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2))
    cos, sin = angle.cos(), angle.sin()
    table = torch.tensor([[5, 2, 7, 0]], dtype=torch.int32, device="cuda")
    cache = lambda: torch.full((8, Hk, page, D), float("nan"), dtype=BF16, device="cuda")  # noqa: E731
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kc, vc = cache(), cache()
    qr = P.attn_kv_append(q, k, v, kc, vc, table, i32(0, n), i32(n), cos=cos, sin=sin)
    once, lse = P.attn_paged_fwd(qr, kc, vc, table, i32(0, n), i32(n), 0.125)
    k1, v1 = cache(), cache()
    for t in range(n):
        q1 = P.attn_kv_append(q[t:t + 1], k[t:t + 1], v[t:t + 1], k1, v1, table, i32(0, 1), i32(t + 1), cos=cos, sin=sin)
        assert torch.equal(q1[0], qr[t])
        o1, l1 = P.attn_paged_fwd(q1, k1, v1, table, i32(0, 1), i32(t + 1), 0.125)
        assert (o1[0].float() - once[t].float()).abs().max() <= 4 * 2.0 ** -8 and (l1[0] - lse[t]).abs().max() <= 1e-4
    pre = 35
    k2, v2 = cache(), cache()
    P.attn_kv_append(None, k[:pre], v[:pre], k2, v2, table, i32(0, pre), i32(pre), cos=cos, sin=sin)
    own = torch.tensor([[1], [3]], dtype=torch.int32, device="cuda")
    rest = n - pre
    two = lambda x: torch.cat((x[pre:], x[pre:])).contiguous()  # noqa: E731
    q2 = P.attn_kv_append(two(q), two(k), two(v), k2, v2, own, i32(0, rest, 2 * rest), i32(rest, rest), cos=cos, sin=sin, pos_offset=pre)
    o2, l2 = P.attn_paged_fwd(q2, k2, v2, own, i32(0, rest, 2 * rest), i32(rest, rest), 0.125, max_q=rest, prefix_table=table[0], prefix_len=pre)
    for half in (o2[:rest], o2[rest:]):
        assert (half.float() - once[pre:].float()).abs().max() <= 4 * 2.0 ** -8
    assert (l2[:rest] - lse[pre:]).abs().max() <= 1e-4 and torch.equal(l2[:rest], l2[rest:])


# ---- what is refused

@pytest.fixture(params=["short", "long"])
def way(request, monkeypatch):
    from paper_2501_08071_amd import binding
    if request.param == "long":
        class Never:
            def __getattr__(self, name):
                return lambda *a: None
        monkeypatch.setattr(binding, "_fast", Never())
    return request.param


def test_both_ways_agree_and_what_is_refused(way):
    s = make([1, 3], [40, 90], 4, 2, 64, 16, F16, prefix=20, seed=1)
    check(attend(s, 0.125), reference(s, 0.125), F16)
    q, kc, vc, t, cu, kv = (s[n] for n in ("q", "k_cache", "v_cache", "page_table", "cu_q", "kv_len"))
    fwd = lambda **x: P.attn_paged_fwd(*[x.get(n, d) for n, d in zip("q kc vc t cu kv scale".split(), (q, kc, vc, t, cu, kv, 0.125))],  # noqa: E731
                                       **{n: v for n, v in x.items() if n not in "q kc vc t cu kv scale".split()})
    none = torch.empty(0, 4, 64, dtype=F16, device="cuda")
    assert fwd(q=none, cu=torch.zeros(3, dtype=torch.int32, device="cuda"))[0].shape == (0, 4, 64)
    bad = [(TypeError, dict(q=q.bfloat16())), (TypeError, dict(kc=kc.float(), vc=vc.float())), (ValueError, dict(kc=kc.cpu(), vc=vc.cpu())),
           (ValueError, dict(vc=vc[:, :, :8])), (ValueError, dict(kc=kc.transpose(2, 3).contiguous().transpose(2, 3))), (ValueError, dict(q=q[:, :3])),
           (ValueError, dict(q=q[0])), (ValueError, dict(q=q.transpose(1, 2).contiguous().transpose(1, 2))), (ValueError, dict(t=t.long())), (ValueError, dict(t=t[:1])),
           (ValueError, dict(cu=cu[:2])), (ValueError, dict(kv=kv.float())), (ValueError, dict(o=torch.empty(4, 4, 64, device="cuda"))),
           (ValueError, dict(lse=torch.empty(4, 5, device="cuda"))), (ValueError, dict(prefix_len=20)),
           (ValueError, dict(prefix_len=200, prefix_table=s["prefix_table"])), (P.AttnError, dict(scale=float("nan"))), (P.AttnError, dict(max_q=-1)),
           (ValueError, dict(workspace=torch.empty(10, device="cuda")))]
    for kind, x in bad:
        with pytest.raises(kind):
            fwd(**x)
    k, v = (torch.randn(4, 2, 64, device="cuda").to(F16) for _ in range(2))
    cos = torch.ones(100, 32, device="cuda")
    app = lambda **x: P.attn_kv_append(*[x.get(n, d) for n, d in zip("q k v kc vc t cu kv".split(), (q, k, v, kc, vc, t, cu, kv))],  # noqa: E731
                                       **{n: y for n, y in x.items() if n not in "q k v kc vc t cu kv".split()})
    assert app(cos=cos, sin=cos).shape == q.shape
    bad = [(TypeError, dict(k=k.float())), (ValueError, dict(k=k[:3])), (ValueError, dict(v=v[:, :1])), (ValueError, dict(cos=cos)), (TypeError, dict(cos=cos.half(), sin=cos.half())),
           (ValueError, dict(cos=cos, sin=cos[:, :16])), (P.AttnError, dict(cos=cos[:, :20].contiguous(), sin=cos[:, :20].contiguous())),
           (ValueError, dict(q_out=torch.empty(4, 4, 32, dtype=F16, device="cuda"))), (ValueError, dict(q=q[:, :, :32])), (ValueError, dict(kv=kv[:1])),
           (P.AttnError, dict(cos=torch.ones(9, 64, device="cuda"), sin=torch.ones(9, 64, device="cuda")))]
    for kind, x in bad:
        with pytest.raises(kind):
            app(**x)
    page3 = torch.zeros(2, 2, 12, 64, dtype=F16, device="cuda")
    with pytest.raises(P.AttnError):
        fwd(kc=page3, vc=page3)
    torch.cuda.synchronize()


def test_numbers_past_32_bits_are_refused(way):
    s = make([1, 3], [40, 90], 4, 2, 64, 16, F16, prefix=20, seed=1)
    k, v = (torch.randn(4, 2, 64, device="cuda").to(F16) for _ in range(2))
    cos = torch.ones(200, 32, device="cuda")
    for far in (2 ** 32, 2 ** 32 + 3, -2 ** 32 + 3, 2 ** 31, 2 ** 40):
        for x in ("max_q", "max_kv"):
            with pytest.raises(ValueError):
                attend(s, 0.125, **{x: far})
        with pytest.raises(ValueError):
            attend({**s, "prefix_len": far}, 0.125)
        with pytest.raises(ValueError):
            P.attn_kv_append(s["q"], k, v, s["k_cache"], s["v_cache"], s["page_table"], s["cu_q"], s["kv_len"], cos=cos, sin=cos, pos_offset=far)
    torch.cuda.synchronize()
