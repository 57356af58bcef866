"""Dropout: bit by bit the definition, since nothing but the product with the factor and the result rounds."""
import math

import pytest
import torch

import step_defn as defn

pytestmark = pytest.mark.gpu
BF, H, F = torch.bfloat16, torch.float16, torch.float32


def definition(x, p, seed, offset, first_row=0):
    m = defn.mask(*x.shape, p, seed, offset, first_row).to(x.device)
    return torch.where(m == 0, 0.0, x.float() * m.float()).to(x.dtype)


@pytest.mark.parametrize("dtype", [BF, H, F])
@pytest.mark.parametrize("rows,cols,p,seed,offset", [(1, 1, 0.5, 0, 0), (1, 8, 0.1, 1, 2), (3, 1001, 0.25, 2 ** 64 - 1, 2 ** 40 + 5), (700, 64, 0.9, -3, 7),
                                                     (5, 4096, 0.0, 1, 1), (33, 17, 1e-9, 4, 4), (2, 16, 0.9999999, 5, -1), (0, 8, 0.1, 1, 1), (8, 0, 0.1, 1, 1)])
def test_dropout(rows, cols, p, seed, offset, dtype):
    from paper_2608_11034_b200 import step
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dtype)
    want = definition(x, p, seed % 2 ** 64, offset % 2 ** 64)
    got = step.dropout(x, p, seed=seed, offset=offset)
    assert got.dtype == dtype and torch.equal(got, want)
    wide = torch.full((rows, cols + 9), math.nan, dtype=dtype, device="cuda")
    wide[:, 1:cols + 1] = x
    assert torch.equal(step.dropout(wide[:, 1:cols + 1], p, seed=seed, offset=offset), want)
    at = torch.tensor([offset], device="cuda")
    assert torch.equal(step.dropout(x, p, seed=seed, offset=at), want)


def test_what_is_dropped_is_zero_whatever_it_was():
    from paper_2608_11034_b200 import step
    x = torch.full((40, 100), math.nan, device="cuda")
    got = step.dropout(x, 0.5, seed=1, offset=2)
    kept = defn.mask(40, 100, 0.5, 1, 2).cuda() > 0
    assert torch.equal(got.isnan(), kept) and (got[~kept] == 0).all()


def test_rows_are_told_apart_past_the_first_launch():
    """More eights than one launch takes: later launches go on with their own rows."""
    from paper_2608_11034_b200 import step
    if torch.cuda.mem_get_info()[0] < 110 << 30:
        pytest.skip("not enough free memory")
    rows, cols = (1 << 23) + 3, 2056                     # 257 eights a row: 8,355,967 rows a launch
    x = torch.ones(rows, cols, dtype=BF, device="cuda")
    y = step.dropout(x, 0.5, seed=11, offset=12)
    for first in (0, 8355960, rows - 5):
        part = slice(first, first + 5)
        assert torch.equal(y[part], definition(x[part], 0.5, 11, 12, first))
    for first in (8355965,):
        part = slice(first, first + 5)
        assert torch.equal(y[part], definition(x[part], 0.5, 11, 12, first))


def test_a_captured_call_drops_other_places_when_its_counter_moves():
    from paper_2608_11034_b200 import step
    x, at = torch.randn(64, 256, device="cuda"), torch.tensor([5], device="cuda")
    step.dropout(x, 0.3, seed=9, offset=at)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step.dropout(x, 0.3, seed=9, offset=at)
    for n in (5, 6, 2 ** 40):
        at.fill_(n)
        graph.replay()
        assert torch.equal(y, definition(x, 0.3, 9, n))


def test_refusals():
    from paper_2608_11034_b200 import step
    x = torch.zeros(4, 8, device="cuda")
    for bad in (lambda: step.dropout(x, 1.0, seed=1), lambda: step.dropout(x, -0.1, seed=1), lambda: step.dropout(x, math.nan, seed=1),
                lambda: step.dropout(x.t(), 0.1, seed=1), lambda: step.dropout(x[0], 0.1, seed=1), lambda: step.dropout(x.double(), 0.1, seed=1),
                lambda: step.dropout(x.cpu(), 0.1, seed=1), lambda: step.dropout(x.clone().requires_grad_(), 0.1, seed=1),
                lambda: step.dropout(x, 0.1, seed=1, offset=torch.zeros(2, dtype=torch.int64, device="cuda")),
                lambda: step.dropout(x, 0.1, seed=1, offset=torch.zeros(1, dtype=torch.int32, device="cuda")),
                lambda: step.dropout(x, 0.1, seed=1, offset=torch.zeros(1, dtype=torch.int64))):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("dtype", [BF, H, F])
@pytest.mark.parametrize("rows,cols", [(1, 65), (3, 67), (40, 71), (513, 101), (7, 1001), (2, 4095), (77, 255), (1000, 1027), (5, 100001)])
def test_rows_one_behind_the_other_of_any_length(rows, cols, dtype):
    """Taken as one long row: the bits of rows that lie apart, and nothing behind the last element is written."""
    from paper_2608_11034_b200 import binding as b
    from paper_2608_11034_b200 import step
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dtype)
    want = definition(x, 0.3, 5, 6)
    assert torch.equal(step.dropout(x, 0.3, seed=5, offset=6), want)
    wide = torch.full((rows, cols + 2), math.nan, dtype=dtype, device="cuda")
    wide[:, :cols] = x
    assert torch.equal(step.dropout(wide[:, :cols], 0.3, seed=5, offset=6), want)
    room = torch.full((rows * cols + 64,), 7.0, dtype=dtype, device="cuda")
    code = {BF: b.DT_BF16, H: b.DT_F16, F: b.DT_F32}[dtype]
    b.scout_dropout(code, rows, cols, x.data_ptr(), cols, room.data_ptr(), cols, 0.3, 5, 6, 0, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(room[:rows * cols].view(rows, cols), want) and (room[rows * cols:] == 7.0).all()
