"""Sizes of the embedding, norms and head losses that pass the integers of the C entry points are refused by the binding:
they would arrive as their lower halves, 2^32 + 8 as 8. On tensors without memory; nothing here needs a GPU."""
import pytest
import torch

import paper_2607_21291_amd as P

BIG = (1 << 32) + 8
SIGNED = 1 << 31


def _meta(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("V,d", [(BIG, 8), (8, BIG), (SIGNED, 8), (8, SIGNED)])
def test_tables_past_32_bits(V, d):
    tok, table, rows = _meta(3, dtype=torch.int32), _meta(V, d), _meta(3, d)
    calls = [lambda: P.embed_forward(tok, table, rows), lambda: P.embed_backward(tok, rows, table),
             lambda: P.head_cross_entropy(rows, table, tok, row_loss=_meta(3, dtype=torch.float32)),
             lambda: P.head_distill(rows, table, _meta(3, 2, dtype=torch.int32), _meta(3, 2, dtype=torch.float32), dh=rows)]
    for call in calls:
        with pytest.raises(ValueError, match="2\\^31"):
            call()


@pytest.mark.parametrize("d", [BIG, SIGNED])
def test_rows_past_32_bits(d):
    x, w = _meta(3, d), _meta(d)
    for call in (lambda: P.norm_forward(x, w, x), lambda: P.norm_backward(x, x, w, x)):
        with pytest.raises(ValueError, match="2\\^31"):
            call()


def test_lists_past_32_bits():
    rows, table = _meta(1, 8), _meta(9, 8)
    with pytest.raises(ValueError, match="2\\^31"):
        P.head_distill(rows, table, _meta(1, BIG, dtype=torch.int32), _meta(1, BIG, dtype=torch.float32), dh=rows)


@pytest.mark.parametrize("big", [BIG, SIGNED, -BIG])
def test_workspace_sizes_past_32_bits(big):
    for call in (lambda: P.embed_backward_workspace_size(10, big, 100), lambda: P.embed_backward_workspace_size(10, 64, big),
                 lambda: P.norm_backward_workspace_size(10, big), lambda: P.head_workspace_size(P.BF16, 10, big, 100),
                 lambda: P.head_workspace_size(P.BF16, 10, 64, big),
                 lambda: P.head_workspace_size(P.BF16, 10, 64, 100, top=big)):
        with pytest.raises(ValueError, match="2\\^31"):
            call()


def test_a_gradient_scale_that_overflows_with_the_temperature_is_refused():
    """dz is scaled by grad_scale x temperature in fp32: infinity there would make NaN of every gradient that is 0."""
    def call(scale, T, dh):
        at = 0x100000  # never dereferenced: refused before the device is looked for
        return P.lib().dsf_head_distill(at, at, P.BF16, 10, 64, 100, at, at, 8, T, None, scale, 0, at, at, dh, None, P.BF16, at,
                                        1 << 45, None)
    for scale in (3e38, -3e38, 4e32):
        assert call(scale, 1e6, 0x100000) == 1 and "grad_scale" in P.last_error()


@pytest.mark.parametrize("dtype,nbytes", [(P.F32, 4), (P.BF16, 2)])
def test_partial_sums_bound_a_piece(dtype, nbytes):
    """Few classes and wide rows: dh's partial sums, not the logits, are what a piece's rows are bounded by: 4 GiB of
    each, beside the copy of the rows, dW's sum and some values a row."""
    n, d, V = 1 << 20, 4096, 1000
    size = P.head_workspace_size(dtype, n, d, V)
    assert 0 < size <= n * d * nbytes + (4 << 30) + (4 << 30) + V * d * 4 + n * 64 + (1 << 20)


def test_workspaces_for_gradients_do_for_losses_alone():
    g = torch.Generator().manual_seed(0)
    log = lambda lo, hi: int(lo * (hi / lo) ** float(torch.rand((), generator=g)))  # noqa: E731
    for _ in range(3000):
        n, d, V, top = log(1, 1 << 24), 8 * log(1, 2048), log(1, 1 << 21), log(1, 1025) - 1
        for dtype in (P.F32, P.BF16):
            alone, every = (P.head_workspace_size(dtype, n, d, V, top=top, gradients=x) for x in (False, True))
            assert 0 < alone <= every, (dtype, n, d, V, top)
