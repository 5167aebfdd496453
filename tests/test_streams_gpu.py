"""Calls on another stream than the current one: memory that an entry point allocates for itself (results, a workspace) belongs to the stream that
writes it.

Memory that is free in the current stream's pool may still be written by work under way on the current stream, for which the other stream does not
wait.  Here such work is: a queue of additions, and behind it bytes of 255 into tensors that are given up at once.  The other way round, a
result that is given up while the current stream is still to read it must not be handed to the other stream's next allocation.  Results
are compared bit for bit with those of a call on the current stream.
"""
import pytest
import torch

import paper_2501_08071_amd as P

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def rows(n=8192, d=2048):
    g = torch.Generator(device="cuda").manual_seed(n)
    return torch.randn(n, d, generator=g, device="cuda").to(BF16)


def row_calls():
    x, r, w = rows(), rows().flip(0).contiguous(), rows(1).view(-1)
    return {"softmax": lambda **k: (P.softmax_rows_fwd(x, **k),), "rmsnorm": lambda **k: (P.rmsnorm_fwd(x, w, 1e-6, **k),),
            "residual norm": lambda **k: P.residual_rmsnorm_fwd(x, r, w, 1e-6, **k),
            "residual norm, 8 bits": lambda **k: P.residual_rmsnorm_fwd_fp8(x, r, w, 1e-6, group=128, **k)}


def gemm_call():
    a, b = rows(4096, 64), rows(64, 4096)
    return lambda **k: (P.gemm_leakyrelu_fwd(a, b, 0.01, **k),)


def attn_call():
    q, k, v = (rows(4096 * 8 + i, 128)[:4096 * 8].view(1, 8, 4096, 128).contiguous() for i in range(3))
    return lambda **kw: P.attn_fwd(q, k, v, True, 0.09, **kw)


def paged_calls():
    """Keys shared out, behind a prefix: the workspace holds parts, what joins them, and the prefix's sums."""
    T, Hq, Hk, D, page = 4096, 16, 2, 128, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)  # noqa: E731
    q, k, v, kc, vc = r(T, Hq, D), r(T, Hk, D), r(T, Hk, D), r(80, Hk, page, D), r(80, Hk, page, D)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, prefix = torch.arange(64, dtype=torch.int32, device="cuda")[None], torch.arange(64, 80, dtype=torch.int32, device="cuda")
    cos, sin = torch.ones(T, D // 2, device="cuda"), torch.zeros(T, D // 2, device="cuda")
    cu, kv = i32(0, T), i32(T)
    assert P.attn_paged_workspace(1, T, Hq, Hk, D, T, T, 1000) > 1 << 26
    return {"append": lambda **kw: (P.attn_kv_append(q, k, v, kc, vc, table, cu, kv, cos=cos, sin=sin, **kw),),
            "paged": lambda **kw: P.attn_paged_fwd(q, kc, vc, table, cu, kv, 0.09, prefix_table=prefix, prefix_len=1000, **kw)}, [
            P.attn_paged_workspace(1, T, Hq, Hk, D, T, T, 1000)]


@pytest.fixture(params=["short", "long"])
def way(request, monkeypatch):
    from paper_2501_08071_amd import binding
    if request.param == "long":
        class Never:
            def __getattr__(self, name):
                return lambda *a: None
        monkeypatch.setattr(binding, "_fast", Never())
    return request.param


@pytest.mark.parametrize("name", ["softmax", "rmsnorm", "residual norm", "residual norm, 8 bits", "gemm", "attn", "append", "paged"])
def test_memory_belongs_to_the_stream_that_writes_it(name, way):
    more = []
    if name == "gemm":
        call = gemm_call()
    elif name == "attn":
        call = attn_call()
    elif name in ("append", "paged"):
        calls, more = paged_calls()
        call = calls[name]
    else:
        call = row_calls()[name]
    bits = lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    want = [bits(t).clone() for t in call()]
    busy = torch.zeros(1 << 28, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    given_up = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in [w.numel() for w in want] + more for _ in range(2)]
    torch.cuda.synchronize()

    def queue():
        for _ in range(60):
            busy.add_(1.0)

    queue()
    for t in given_up:
        t.fill_(255)
    del given_up, t
    got = call(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(bits(a), b) for a, b in zip(got, want))
    # given up while the current stream is still to read it
    torch.cuda.current_stream().wait_stream(side)
    queue()
    copies = [bits(t).clone() for t in got]
    del got
    with torch.cuda.stream(side):
        other = [torch.empty(w.numel(), dtype=torch.uint8, device="cuda").fill_(255) for w in want for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(copies, want)) and len(other) == 2 * len(want)
