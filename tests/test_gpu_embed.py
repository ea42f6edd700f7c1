"""Embedding lookup and its gradient against plain 64-bit forms.

Tolerances.  Lookup: one fp32 product, one rounding - the bits are compared.  Gradient: a sum of n fp32 terms in any order is
off by at most e = (n - 1) u / (1 - (n - 1) u) of the sum of magnitudes (u = 2^-24), the product with the scale adds u.
Rounding is monotone, so an output lies between round(exact - e) and round(exact + e) in its own type."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2203_17063_b200 import binding as ec

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make_rows(n, d, dtype, stride, seed, std=1.0, offset=0):
    """[n][d] view into a larger allocation: rows `stride` apart, starting `offset` elements in, NaN everywhere else."""
    g = torch.Generator().manual_seed(seed)
    big = torch.full((offset + max(n, 1) * stride + 16,), float("nan"), dtype=dtype)
    view = big[offset:offset + max(n, 1) * stride].view(max(n, 1), stride)[:n, :d]
    view.copy_(torch.randn(n, d, generator=g, dtype=torch.float64) * std)
    big = big.cuda()
    return big, big[offset:offset + max(n, 1) * stride].view(max(n, 1), stride)[:n, :d]


def untouched(big, view, stride, offset=0):
    """Everything of `big` outside the rows is still NaN."""
    keep = torch.ones(big.numel(), dtype=torch.bool, device="cuda")
    n, d = view.shape
    if n:
        keep[offset:offset + n * stride].view(n, stride)[:, :d] = False
    return bool(torch.isnan(big[keep]).all())


def make_tokens(kind, T, V, index, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "uniform":
        t = torch.randint(-1, V + 2, (T,), generator=g)                    # some outside on either side
    elif kind == "one":
        t = torch.full((T,), V // 2)
    elif kind == "none":
        t = torch.where(torch.arange(T) % 2 == 0, torch.tensor(-1), torch.tensor(V))
    elif kind == "zipf":
        t = (torch.exp(torch.rand(T, generator=g, dtype=torch.float64) * np.log(V + 1.0)) - 1).long().clamp(0, V - 1)
    elif kind == "extremes":
        lim = torch.iinfo(index)
        t = torch.tensor([0, V - 1, V, lim.min, lim.max, -1])[torch.arange(T) % 6]
    else:
        t = torch.arange(T) % V
    return t.to(index).cuda()


SHAPES = [  # T, V, D
    (0, 5, 8), (1, 1, 1), (1, 7, 33), (2, 3, 8), (33, 1, 64), (64, 1000, 4), (300, 17, 129), (1000, 511, 64), (777, 512, 256),
    (5000, 513, 40), (4097, 70000, 16), (2049, 300, 1000), (513, 65, 2056), (100, 4, 4100), (20000, 50, 72), (300, 600000, 8),
]


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_lookup_bits(cuda_device, T, V, D, src, dst):
    for k, (kind, index, pad, off) in enumerate([("uniform", torch.int64, 0, 0), ("extremes", torch.int32, 8, 8), ("zipf", torch.int32, 3, 1)]):
        _, table = make_rows(V, D, DT[src], D + pad, 1 + k, offset=off)
        tokens = make_tokens(kind, T, V, index, 2 + k)
        out_all, out = make_rows(T, D, DT[dst], D + pad, 3, offset=off)
        out.fill_(7.0)
        scale = 2.718281828
        ec.embed_lookup(table, tokens, out, scale)
        torch.cuda.synchronize()
        inside = (tokens >= 0) & (tokens < V)
        want = table[tokens.long().clamp(0, V - 1)].float() * torch.tensor(scale, dtype=torch.float32, device="cuda")
        want = torch.where(inside[:, None], want, torch.zeros_like(want)).to(DT[dst])
        assert torch.equal(out, want)
        assert untouched(out_all, out, D + pad, off)


def reference_grad(dout, tokens, V, scale, skip, old):
    """(gradient, bound of the fp32 error) in 64 bits; old: what is accumulated onto, or None."""
    x = dout.double()
    t = tokens.long()
    use = (t >= 0) & (t < V) & (t != skip)
    g = torch.zeros(V, x.shape[1], dtype=torch.float64, device="cuda")
    m = torch.zeros_like(g)
    g.index_add_(0, t[use], x[use])
    m.index_add_(0, t[use], x[use].abs())
    n = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, t[use], torch.ones(int(use.sum()), dtype=torch.float64, device="cuda"))
    s = float(torch.tensor(scale, dtype=torch.float32))
    bound = (n[:, None] + 2) * 2.0 ** -24 * 1.01 * m * abs(s)
    g = g * s
    if old is not None:
        g = g + old.double()
        bound = bound + 2.0 ** -24 * (g.abs() + bound)                     # one more addition
        bound = torch.where((n > 0)[:, None], bound, torch.zeros_like(bound))
    return g, bound, n


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_grad(cuda_device, T, V, D, accumulate, src, dst):
    for k, (kind, index, pad, off, skip) in enumerate([("uniform", torch.int32, 0, 0, -1), ("one", torch.int64, 8, 8, -1),
                                                       ("zipf", torch.int64, 5, 3, 0), ("none", torch.int32, 0, 0, -1)]):
        _, dout = make_rows(T, D, DT[src], D + pad, 11 + k, offset=off)
        tokens = make_tokens(kind, T, V, index, 12 + k)
        g_all, grad = make_rows(V, D, DT[dst], D + pad, 13 + k, offset=off)
        if not accumulate:
            grad.fill_(float("nan"))                                       # must not be read
        before = grad.clone()
        ws = torch.full((ec.embed_grad_workspace_bytes(T, V, D),), 0xA5, dtype=torch.uint8, device="cuda")
        ec.embed_grad(dout, tokens, grad, ws, -1.7, skip, accumulate)
        torch.cuda.synchronize()
        want, bound, n = reference_grad(dout, tokens, V, -1.7, skip, before if accumulate else None)
        low, high = (want - bound).float().to(DT[dst]), (want + bound).float().to(DT[dst])
        assert bool(((low <= grad) & (grad <= high)).all()), f"{kind}: off by {(grad.double() - want).abs().max().item():g}"
        assert torch.equal(grad[n == 0], before[n == 0] if accumulate else torch.zeros_like(grad[n == 0]))
        assert untouched(g_all, grad, D + pad, off)
        again = before.clone().contiguous()
        ec.embed_grad(dout, tokens, again, ws, -1.7, skip, accumulate)     # dirty workspace, same bits
        torch.cuda.synchronize()
        if pad == 0:                                                       # (the same path: rows aligned alike)
            assert torch.equal(again, grad)


@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("off", [0, 1, 2, 3, 5, 7])
@pytest.mark.parametrize("T,V,D", [(1, 4, 1), (9, 1003, 5), (250, 1000, 1024), (251, 1003, 1001), (900, 5000, 33)])
def test_grad_of_few_tokens_without_gaps(cuda_device, T, V, D, off, dst):
    """Rows that follow each other without gaps from any element on: nothing before or behind them is written."""
    _, dout = make_rows(T, D, torch.float32, D, 41, offset=off)
    g_all, grad = make_rows(V, D, DT[dst], D, 42, offset=off)
    grad.fill_(float("inf"))
    tokens = make_tokens("zipf", T, V, torch.int32, 43)
    ws = torch.full((ec.embed_grad_workspace_bytes(T, V, D),), 0xA5, dtype=torch.uint8, device="cuda")
    ec.embed_grad(dout, tokens, grad, ws, 0.5, -1, False)
    torch.cuda.synchronize()
    want, bound, _ = reference_grad(dout, tokens, V, 0.5, -1, None)
    low, high = (want - bound).float().to(DT[dst]), (want + bound).float().to(DT[dst])
    assert bool(((low <= grad) & (grad <= high)).all())
    assert untouched(g_all, grad, D, off)


@pytest.mark.parametrize("T,V,D,index", [(40000, 1000, 16, torch.int32), (65536, 70000, 8, torch.int64), (65537, 300, 24, torch.int64),
                                         (200001, 600000, 4, torch.int32), (150000, 3, 33, torch.int64)])
def test_grad_of_many_tokens(cuda_device, T, V, D, index):
    """One cluster sorts up to 65536 tokens, several launches more; both keep a row's positions in ascending order."""
    for k, kind in enumerate(["zipf", "uniform", "one"]):
        _, dout = make_rows(T, D, torch.float32, D, 40 + k)
        tokens = make_tokens(kind, T, V, index, 41 + k)
        ws = torch.full((ec.embed_grad_workspace_bytes(T, V, D),), 0x5A, dtype=torch.uint8, device="cuda")
        outs = []
        for _ in range(2):
            grad = torch.full((V, D), float("nan"), device="cuda")
            ec.embed_grad(dout, tokens, grad, ws, 0.5, 1)
            outs.append(grad)
        torch.cuda.synchronize()
        want, bound, _ = reference_grad(dout, tokens, V, 0.5, 1, None)
        assert bool(((outs[0].double() - want).abs() <= bound).all())
        assert torch.equal(outs[0], outs[1])


def test_grad_is_the_derivative_of_the_lookup(cuda_device):
    """f(table) = <lookup(table), dout> is linear: f(table + delta) - f(table) = <delta, grad>; integers, so exact."""
    T, V, D = 700, 90, 24
    g = torch.Generator().manual_seed(5)
    table = torch.randint(-8, 9, (V, D), generator=g).float().cuda()
    delta = torch.randint(-8, 9, (V, D), generator=g).float().cuda()
    dout = torch.randint(-8, 9, (T, D), generator=g).float().cuda()
    tokens = make_tokens("uniform", T, V, torch.int64, 6)
    out0, out1 = torch.empty(T, D, device="cuda"), torch.empty(T, D, device="cuda")
    ec.embed_lookup(table, tokens, out0, 4.0)
    ec.embed_lookup(table + delta, tokens, out1, 4.0)
    grad = torch.empty(V, D, device="cuda")
    ws = torch.empty(ec.embed_grad_workspace_bytes(T, V, D), dtype=torch.uint8, device="cuda")
    ec.embed_grad(dout, tokens, grad, ws, 4.0)
    torch.cuda.synchronize()
    left = ((out1 - out0).double() * dout.double()).sum()
    right = (delta.double() * grad.double()).sum()
    assert left.item() == right.item()


def test_what_gives_nothing_may_hold_anything(cuda_device):
    """Rows of dropped tokens are NaN or infinite, and so are table rows that no token names."""
    T, V, D = 900, 40, 36
    tokens = make_tokens("uniform", T, V, torch.int64, 8)
    tokens[::5] = 7
    dout = torch.randn(T, D, device="cuda")
    clean, dirty = torch.empty(V, D, device="cuda"), torch.empty(V, D, device="cuda")
    ws = torch.empty(ec.embed_grad_workspace_bytes(T, V, D), dtype=torch.uint8, device="cuda")
    ec.embed_grad(dout, tokens, clean, ws, 1.5, 7)
    gone = (tokens < 0) | (tokens >= V) | (tokens == 7)
    dout[gone] = float("nan")
    dout[torch.nonzero(gone)[0]] = float("inf")
    ec.embed_grad(dout, tokens, dirty, ws, 1.5, 7)
    table = torch.full((V, D), float("nan"), device="cuda")
    table[3] = 2.0
    out = torch.empty(3, D, device="cuda")
    ec.embed_lookup(table, torch.tensor([3, -1, V], device="cuda"), out, 0.5)
    torch.cuda.synchronize()
    assert torch.equal(clean, dirty) and not clean[7].any()
    assert bool((out[0] == 1).all()) and not out[1:].any()


def test_two_streams_two_workspaces(cuda_device):
    """Calls on other streams than the tensors' own, running side by side, end where they end alone."""
    T, V, D = 30000, 5000, 256
    jobs = []
    for k in range(2):
        dout = torch.randn(T, D, device="cuda")
        tokens = make_tokens("zipf", T, V, torch.int64, 20 + k)
        ws = torch.empty(ec.embed_grad_workspace_bytes(T, V, D), dtype=torch.uint8, device="cuda")
        alone = torch.empty(V, D, device="cuda")
        ec.embed_grad(dout, tokens, alone, ws)
        jobs.append((dout, tokens, ws, alone, torch.full((V, D), float("nan"), device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for dout, tokens, ws, _, grad, st in jobs:
            ec.embed_grad(dout, tokens, grad, ws, stream=st)
    torch.cuda.synchronize()
    for _, _, _, alone, grad, _ in jobs:
        assert torch.equal(alone, grad)


def test_offsets_past_32_bits(cuda_device):
    """A table of more than 2^32 elements: the last rows are looked up, and their gradient is accumulated."""
    V, D = (1 << 21) + 3, 2048 + 8
    table = torch.empty(V, D, dtype=torch.bfloat16, device="cuda")
    table[-3:] = torch.arange(3 * D, device="cuda").view(3, D).to(torch.bfloat16)
    tokens = torch.tensor([V - 1, V - 3, V, V - 1], device="cuda")
    out = torch.empty(4, D, dtype=torch.bfloat16, device="cuda")
    ec.embed_lookup(table, tokens, out, 2.0)
    torch.cuda.synchronize()
    assert torch.equal(out[0], (table[V - 1].float() * 2).bfloat16()) and torch.equal(out[1], (table[V - 3].float() * 2).bfloat16())
    assert not out[2].any() and torch.equal(out[3], out[0])
    table[-3:] = 1.0
    ws = torch.empty(ec.embed_grad_workspace_bytes(4, V, D), dtype=torch.uint8, device="cuda")
    ec.embed_grad(torch.ones(4, D, device="cuda"), tokens, table, ws, 1.0, accumulate=True)
    torch.cuda.synchronize()
    assert bool((table[V - 1] == 3).all()) and bool((table[V - 3] == 2).all()) and bool((table[V - 2] == 1).all())


def test_binding_refuses(cuda_device):
    table, tok = torch.zeros(8, 16, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    out = torch.zeros(4, 16, device="cuda")
    ws = torch.zeros(ec.embed_grad_workspace_bytes(4, 8, 16), dtype=torch.uint8, device="cuda")
    bad = [
        (lambda: ec.embed_lookup(table.half(), tok, out), ec.ERR_UNSUPPORTED),
        (lambda: ec.embed_lookup(table, tok.float(), out), ec.ERR_UNSUPPORTED),
        (lambda: ec.embed_lookup(table, tok, out[:3]), ec.ERR_INVALID),
        (lambda: ec.embed_lookup(table, tok, out[:, :8]), ec.ERR_INVALID),
        (lambda: ec.embed_lookup(table.t(), tok, out), ec.ERR_INVALID),
        (lambda: ec.embed_lookup(table.cpu(), tok, out), ec.ERR_INVALID),
        (lambda: ec.embed_grad(out, tok, table, ws[:-1]), ec.ERR_CAPACITY),
        (lambda: ec.embed_grad(out, tok, table[:, :8], ws), ec.ERR_INVALID),
        (lambda: ec.embed_grad(out, tok[::2], table, ws), ec.ERR_INVALID),
    ]
    for call, code in bad:
        with pytest.raises(ec.EcError) as err:
            call()
        assert err.value.code == code
