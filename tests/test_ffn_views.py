"""CPU-only: views that the binding of the casts cannot describe to the library are refused before anything is enqueued.  The library's
entry points are replaced by ones that note what would have been called."""
import pytest
import torch

from paper_2406_06858_amd import ffn

ROWS, K = 40, 100
Q, S = ffn.flux_mx4_row_bytes(K), ffn.flux_mx4_scale_row_bytes(K)


@pytest.fixture
def calls(monkeypatch):
    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: made.append((name, args)) or 0

    monkeypatch.setattr(ffn, "lib", Library)
    monkeypatch.setattr(ffn, "_stream", lambda s: 0)
    return made


def _cast(name, wide, q, scales):
    if name == "quantize":
        ffn.flux_mx4_quantize(wide, q, scales)
    else:
        ffn.flux_mx4_dequantize(q, scales, wide)


def _bytes(rows, width):
    return torch.zeros(rows, width, dtype=torch.uint8)


@pytest.mark.parametrize("name", ["quantize", "dequantize"])
@pytest.mark.parametrize("wide", [
    torch.zeros(1, K).expand(ROWS, K), torch.zeros(K).expand(ROWS, K), torch.zeros(K + ROWS).as_strided((ROWS, K), (1, 1)), torch.zeros(1, 1).expand(ROWS, K),
    torch.zeros(K, ROWS).t(), torch.zeros(ROWS, 2 * K)[:, ::2],
])
def test_rows_that_overlap_or_are_no_runs_are_refused(calls, name, wide):
    assert wide.shape == (ROWS, K)
    with pytest.raises(ValueError):
        _cast(name, wide, _bytes(ROWS, Q), _bytes(ROWS, S))
    assert calls == []


def test_one_column_of_one_number_is_refused(calls):
    with pytest.raises(ValueError):
        ffn.flux_mx4_quantize(torch.zeros(1, 1).expand(ROWS, 1), _bytes(ROWS, 16), _bytes(ROWS, 16))
    assert calls == []


@pytest.mark.parametrize("name", ["quantize", "dequantize"])
@pytest.mark.parametrize("q,scales", [
    (_bytes(ROWS, Q + 16)[:, :Q], _bytes(ROWS, S)), (_bytes(ROWS, Q), _bytes(ROWS, S + 16)[:, 16:]), (_bytes(1, Q).expand(ROWS, Q), _bytes(ROWS, S)),
    (_bytes(ROWS, Q), _bytes(1, S).expand(ROWS, S)), (_bytes(Q, ROWS).t(), _bytes(ROWS, S)), (_bytes(2 * ROWS, Q)[::2], _bytes(ROWS, S)),
    (_bytes(ROWS, Q - 1), _bytes(ROWS, S)), (_bytes(ROWS - 1, Q), _bytes(ROWS, S)), (_bytes(ROWS, Q), _bytes(ROWS, S - 16)), (_bytes(ROWS, Q), _bytes(ROWS, 4)),
])
def test_blocks_that_are_not_packed_or_too_small_are_refused(calls, name, q, scales):
    with pytest.raises(ValueError):
        _cast(name, torch.zeros(ROWS, K), q, scales)
    assert calls == []


@pytest.mark.parametrize("name", ["quantize", "dequantize"])
@pytest.mark.parametrize("wide,rows,ld", [
    (torch.zeros(ROWS, K), ROWS, K), (torch.zeros(ROWS, K + 7)[:, 3:K + 3], ROWS, K + 7), (torch.zeros(2 * ROWS, K)[::2], ROWS, 2 * K), (torch.zeros(1, K), 1, 0),
    (torch.zeros(ROWS, 1).t(), 1, 0), (torch.zeros(5, ROWS)[:, 2:3], 5, ROWS),
])
def test_what_the_library_is_told(calls, name, wide, rows, ld):
    """Rows of any pitch from their length on; buffers that are larger than they have to be, of any element."""
    k = wide.shape[1]
    _cast(name, wide, torch.zeros(4 * ROWS, Q, dtype=torch.uint8), torch.zeros(ROWS * S, dtype=torch.int32))
    (called, args), = calls
    assert called == f"flux_mx4_{name}" and args[:2] == (rows, k) and ld in args[2:]
    assert args[4 if name == "quantize" else 6] == ld
