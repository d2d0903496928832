"""Low-rank adapters on the GPU against 64-bit arithmetic.

A row's bound.  t is a sum of K products in fp32, each addition taken as truncating (2^-23): off by (K + 64) * 2^-23 of the sum of
magnitudes, joins among it.  It meets B as two bf16, of which the second is off by 2^-9 of 2^-8: less than 2^-16 with the factor's product.
The sum over 2 * rank terms and the addition to out: (2 * rank + 8) * 2^-23 of the sum of magnitudes.  The result is rounded to bf16:
half a step, 2^-8 of it."""
import pytest
import torch

from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu


def _case(seed, M, K, widths, rank, adapters, kind="mixed", gap=0):
    g = torch.Generator().manual_seed(seed)
    N, R = sum(widths), rank * len(widths)
    bf16 = lambda *shape: torch.randn(*shape, generator=g).to(torch.bfloat16)
    ids = torch.randint(-1, adapters, (M,), generator=g)
    if kind == "grouped":
        ids = ids.sort().values
    elif kind == "one":
        ids[:] = adapters - 1
    elif kind == "distinct":
        ids = torch.randperm(max(M, adapters), generator=g)[:M]                 # those from `adapters` on are none's
    elif kind == "none":
        ids = torch.where(ids < 0, adapters, -1 - ids)
    return dict(x=bf16(M, K + gap)[:, :K], a=bf16(adapters, R, K) * K ** -0.5, b=bf16(adapters, N, rank) * rank ** -0.5,
                factors=torch.randn(adapters, generator=g), ids=ids.to(torch.int32), out=bf16(M, N + gap)[:, :N], widths=widths)


def _on(case):
    return {k: v.cuda() if torch.is_tensor(v) else v for k, v in case.items()}


def _ends(widths):
    return tuple(sum(widths[:i + 1]) for i in range(len(widths)))


def _call(dev, out=None, workspace=None):
    M, K = dev["x"].shape
    N, (adapters, _, rank) = sum(dev["widths"]), dev["b"].shape
    if workspace is None:
        workspace = eq.alloc_adapters_workspace(M, N, K, rank, len(dev["widths"]), adapters)
        workspace.fill_(0xFF)                                               # NaN wherever it is read before it is written
    out = dev["out"] if out is None else out
    eq.equarx_adapters(dev["x"], dev["a"], dev["b"], dev["factors"], dev["ids"], out, _ends(dev["widths"]), workspace)
    return out


def _want(case, device="cpu"):
    """Results and how far they may be off."""
    c = {k: v.to(device) if torch.is_tensor(v) else v for k, v in case.items()}
    out, bound = c["out"].double(), torch.zeros(c["out"].shape, dtype=torch.float64, device=device)
    rank, K = c["b"].shape[2], c["x"].shape[1]
    for i in range(c["b"].shape[0]):
        rows = (c["ids"] == i).nonzero().flatten()
        if rows.numel() == 0:
            continue
        x, a, f = c["x"][rows].double(), c["a"][i].double(), float(c["factors"][i])
        t, mass = x @ a.T, x.abs() @ a.abs().T
        begin = 0
        for s, width in enumerate(c["widths"]):
            b = c["b"][i, begin:begin + width].double()
            ts, ms = (v[:, s * rank:(s + 1) * rank] for v in (t, mass))
            out[rows, begin:begin + width] += f * (ts @ b.T)
            size = ts.abs() @ b.abs().T
            bound[rows, begin:begin + width] = abs(f) * ((K + 64) * 2.0 ** -23 * (ms @ b.abs().T) + (2.0 ** -16 + (2 * rank + 8) * 2.0 ** -23) * size)
            begin += width
    changed = ((c["ids"] >= 0) & (c["ids"] < c["b"].shape[0]))[:, None]
    return out, torch.where(changed, 2.0 ** -8 * out.abs() + 1.01 * bound + 2.0 ** -23 * c["out"].double().abs(), 0.0)


def _check(case, got, device="cpu"):
    want, bound = _want(case, device)
    off = (got.double().to(device) - want).abs()
    assert (off <= bound).all(), float((off - bound).max())


SIZES = [(1, 8, (8,), 8, 1), (1, 4096, (4096, 2048, 2048), 16, 32), (3, 1, (1,), 8, 2), (2, 7, (3, 5), 8, 3), (16, 64, (64,), 16, 4),
         (17, 65, (65, 63), 24, 5), (33, 255, (257,), 32, 40), (64, 5376, (512, 256, 256), 16, 32), (65, 1511, (1001, 1500), 24, 7),
         (100, 300, (31, 1, 900, 70), 64, 9), (31, 1024, (129,), 128, 6), (128, 333, (400, 1), 128, 2), (200, 2049, (333,), 40, 64),
         (333, 130, (1000,), 8, 5), (700, 96, (90,), 16, 300), (1000, 777, (300, 200), 56, 3), (4096, 256, (128,), 64, 4),
         (2111, 515, (77, 300, 5), 72, 8000), (200, 700, (300, 20), 16, 130), (256, 264, (70,), 48, 300), (64, 3, (7,), 128, 64), (2048, 90, (6,), 16, 2),
         (5000, 8, (9, 8), 8, 20), (1024, 700, (70, 40), 32, 64), (1030, 1200, (100, 30, 9), 128, 3), (1500, 513, (77,), 72, 90)]


@pytest.mark.parametrize("kind", ("mixed", "grouped", "one", "distinct", "none"))
@pytest.mark.parametrize("M,K,widths,rank,adapters", SIZES)
def test_rows_of_every_kind(M, K, widths, rank, adapters, kind):
    if adapters > 1000:
        K, widths, rank = 40, (30, 8), 8
    case = _case(M + K, M, K, widths, rank, adapters, kind, gap=(M + K) % 4)
    dev = _on(case)
    wide = torch.full((M, sum(widths) + 7), 9.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :sum(widths)] = dev["out"]
    _call(dev, wide[:, :sum(widths)])
    assert (wide[:, sum(widths):] == 9.0).all()
    _check(case, wide[:, :sum(widths)].cpu())


# Where a call goes over from one way of finding an item's rows to another, and the most and the fewest of each way.
EDGES = [(24, 3), (25, 2), (25, 5), (48, 8), (64, 10), (64, 11), (65, 32), (65, 33), (256, 127), (256, 128), (257, 3), (511, 5), (512, 1024), (513, 1023),
         (513, 1025), (2047, 1), (4095, 120), (4096, 127), (4096, 130), (4096, 1024), (2048, 64), (2048, 30), (2500, 24), (3900, 3), (4097, 4), (4097, 200), (6001, 1), (8192, 4), (8192, 100), (8193, 4)]


@pytest.mark.parametrize("kind", ("mixed", "grouped", "one", "none"))
@pytest.mark.parametrize("M,adapters", EDGES)
def test_every_row_is_found(M, adapters, kind):
    case = _case(M + adapters, M, 1100 if M * adapters < 10000 else 40, (30, 8), 8, adapters, kind)
    case["ids"][::37] = torch.tensor([-2 ** 31, 2 ** 31 - 1, adapters, 1 << 16])[torch.arange(len(case["ids"][::37])) % 4]
    _check(case, _call(_on(case)).cpu())


@pytest.mark.parametrize("rank", (8, 24, 32, 40, 64, 72, 128))
def test_many_rows_and_columns(rank):
    """Rows by 64, the last ones of an adapter fewer; outputs that go past the caches."""
    case = _on(_case(rank, 2300, 200, (5003, 4200, 1), rank, 3))
    start = case["out"].clone()
    got = _call(case).clone()
    case["out"] = start
    _check(case, got, "cuda")


@pytest.mark.parametrize("M,widths,rank,adapters", ((2600, (8001, 100), 16, 300), (2600, (8001, 100), 64, 300), (2600, (8001, 100), 128, 300),
                                                   ((20 << 20) // 5, (5,), 8, 3)))
def test_many_rows_of_many_adapters(M, widths, rank, adapters):
    """Rows by sixteen with outputs that go past the caches; and so many rows of fewer than eight columns."""
    case = _on(_case(rank, M, 72, widths, rank, adapters))
    start = case["out"].clone()
    got = _call(case).clone()
    case["out"] = start
    _check(case, got, "cuda")


def test_the_largest_products():
    case = _on(_case(1, 4096, 5376, (5376,), 64, 4, "grouped"))
    start = case["out"].clone()
    got = _call(case).clone()
    case["out"] = start
    _check(case, got, "cuda")


@pytest.mark.parametrize("M,adapters", ((50, 6), (500, 6), (3000, 3), (3000, 600)))
def test_a_row_does_not_depend_on_its_place(M, adapters):
    """The same rows in another order: the same bits."""
    dev = _on(_case(5, M, 515, (200, 90), 24, adapters))
    order = torch.randperm(M, generator=torch.Generator().manual_seed(1)).cuda()
    other = {**dev, **{k: dev[k][order].contiguous() for k in ("x", "ids", "out")}}
    a, b = _call(dev), _call(other)
    assert torch.equal(a[order], b)


@pytest.mark.parametrize("M", (40, 400, 2000))
@pytest.mark.parametrize("bad", (float("nan"), float("inf")))
def test_what_is_not_finite_stays_where_it_is(M, bad):
    """In a row of x, in an adapter and its factor: nobody else's rows change, down to the last bit."""
    adapters = 4
    dev = _on(_case(6, M, 200, (96, 50), 16, adapters))
    start, clean = dev["out"].clone(), None
    clean = _call(dev, dev["out"].clone())
    for where in ("x", "a", "b", "factors"):
        other = {k: v.clone() if torch.is_tensor(v) else v for k, v in dev.items()}
        touched = torch.zeros(M, dtype=torch.bool, device="cuda")
        if where == "x":
            row = int((dev["ids"] == 1).nonzero()[0])
            other["x"][row, 77] = bad
            touched[row] = True
        else:
            touched = dev["ids"] == 2
            if where == "a":
                other["a"][2, 3, 199] = bad
            elif where == "b":
                other["b"][2, 40, 15] = bad
            else:
                other["factors"][2] = bad
        other["out"] = start.clone()
        got = _call(other)
        assert torch.equal(got[~touched], clean[~touched]), where
        assert not got[touched].isfinite().all(dim=1).any(), where


def test_rows_past_32_bits():
    M, N = 40000, 65537
    x, a, b = torch.randn(M, 16, device="cuda").to(torch.bfloat16), torch.randn(2, 8, 16, device="cuda").to(torch.bfloat16), \
        torch.randn(2, N, 8, device="cuda").to(torch.bfloat16)
    ids = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    ids[39990:] = torch.arange(10, device="cuda") % 3 - 1
    out = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    factors = torch.tensor([0.5, -2.0], device="cuda")
    eq.equarx_adapters(x, a, b, factors, ids, out, None, eq.alloc_adapters_workspace(M, N, 16, 8, 1, 2))
    case = dict(x=x[-10:], a=a, b=b, factors=factors, ids=ids[-10:], out=torch.zeros(10, N, dtype=torch.bfloat16, device="cuda"), widths=(N,))
    _check(case, out[-10:], "cuda")
    assert not out[:39990].any()


def test_a_workspace_for_calls_of_fewer_rows():
    for N, K, rank, slices, adapters in ((256, 5376, 16, 3, 32), (5376, 4096, 64, 1, 4), (100, 300, 8, 4, 8000), (70, 40, 128, 4, 1)):
        needs = [int(eq.load().equarx_adapters_workspace_bytes(m, N, K, rank, slices, adapters)) for m in [*range(1, 700), 1000, 4096, 5000, 1 << 17]]
        assert needs == sorted(needs)


def test_a_captured_call_reads_its_ids_anew():
    case = _case(9, 64, 640, (256, 128), 16, 8)
    dev = _on(case)
    start, work = dev["out"].clone(), eq.alloc_adapters_workspace(64, 384, 640, 16, 2, 8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _call(dev, None, work)
    for step in range(4):
        ids = torch.randint(-1, 8, (64,), generator=torch.Generator().manual_seed(step)).to(torch.int32)
        if step == 2:
            ids[:] = 3
        dev["ids"].copy_(ids)
        dev["out"].copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        eager = _call({**dev, "out": start.clone()})
        assert torch.equal(dev["out"], eager)
        _check({**case, "ids": ids}, dev["out"].cpu())


def test_another_stream():
    case = _case(10, 90, 300, (100,), 16, 5)
    dev = _on(case)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = _call(dev)
    side.synchronize()
    _check(case, out.cpu())


def test_nothing_to_do():
    case = _on(_case(11, 5, 16, (8,), 8, 2))
    start = case["out"].clone()
    empty = dict(case, x=case["x"][:, :0], a=case["a"][:, :, :0].contiguous())
    assert torch.equal(_call(empty), start)
    none = {**case, **{k: case[k][:0] for k in ("x", "ids", "out")}}
    _call(none)
