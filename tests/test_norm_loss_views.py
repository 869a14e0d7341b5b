"""CPU-only: tensors whose numbers do not lie where the problem says are refused before anything is enqueued, and every view that does lie so is taken.  The
library's entry points are replaced by ones that note what would have been called."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2406_06858_amd import loss, norm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
M, K, V = 6, 64, 40
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture
def calls(monkeypatch):
    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: made.append((name, args)) or 0

    for module in (norm, loss):
        monkeypatch.setattr(module, "lib", Library)
        monkeypatch.setattr(module, "_stream", lambda s: 0)
        monkeypatch.setattr(module, "_device", lambda: -1)
    return made


def z(*shape, dtype=BF16):
    return torch.zeros(shape, dtype=dtype)


WS = dict(workspace=z(64, dtype=torch.uint8))
CALLS = {
    "norm": (norm.flux_norm, lambda **kw: norm.norm_problem(M, K, **kw), dict(X=z(M, K), R=z(M, K), W=z(K), S=z(M, K), Y=z(M, K), rstd=z(M, dtype=F32))),
    "norm_bwd": (norm.flux_norm_backward, lambda **kw: norm.norm_problem(M, K, **kw),
                 dict(dY=z(M, K), S=z(M, K), W=z(K), rstd=z(M, dtype=F32), dS=z(M, K), dR=z(M, K), dX=z(M, K), dW=z(K, dtype=F32), **WS)),
    "loss": (loss.flux_loss, lambda **kw: loss.loss_problem(M, V, K, **kw),
             dict(X=z(M, K), W=z(V, K), target=z(M, dtype=torch.int64), lse=z(M, dtype=F32), logit=z(M, dtype=F32), loss=z(M, dtype=F32), **WS)),
    "loss_bwd": (loss.flux_loss_backward, lambda **kw: loss.loss_problem(M, V, K, **kw),
                 dict(X=z(M, K), W=z(V, K), target=z(M, dtype=torch.int64), lse=z(M, dtype=F32), dloss=z(M, dtype=F32), dX=z(M, K), dW=z(V, K), **WS)),
}
MATRICES = [(c, n) for c, (_, _, t) in CALLS.items() for n, v in t.items() if v.dim() == 2]
VECTORS = [(c, n) for c, (_, _, t) in CALLS.items() for n, v in t.items() if v.dim() == 1 and n != "workspace"]


def _call(name, problem={}, **other):
    function, problem_of, tensors = CALLS[name]
    function(problem_of(**problem), **{**tensors, **other})


@pytest.mark.parametrize("name", CALLS)
def test_taken_as_they_are(calls, name):
    _call(name)
    assert len(calls) == 1


@pytest.mark.parametrize("name,what", MATRICES)
@pytest.mark.parametrize("view", [
    lambda t: z(*t.shape[::-1], dtype=t.dtype).t(), lambda t: z(t.shape[0], 2 * t.shape[1], dtype=t.dtype)[:, ::2], lambda t: t[:1].expand(t.shape), lambda t: t[:-1],
    lambda t: t[:, :-8], lambda t: z(t.shape[0], t.shape[1] + 8, dtype=t.dtype), lambda t: z(t.shape[0], t.shape[1] + 8, dtype=t.dtype)[:, :-8],
    lambda t: z(2 * t.shape[0], t.shape[1], dtype=t.dtype)[::2], lambda t: t.view(-1)[:-1], lambda t: z(2, t.shape[0], t.shape[1] // 2 + 4, dtype=t.dtype),
    lambda t: z(t.shape[0], 2, t.shape[1], dtype=t.dtype)[:, 0],
])
def test_matrices_that_lie_elsewhere_are_refused(calls, name, what, view):
    with pytest.raises(ValueError, match=rf"^{what} has to be"):
        _call(name, **{what: view(CALLS[name][2][what])})
    assert calls == []


@pytest.mark.parametrize("name,what", VECTORS)
@pytest.mark.parametrize("view", [lambda t: z(2 * len(t), dtype=t.dtype)[::2], lambda t: t[:1].expand(t.shape), lambda t: z(len(t), 3, dtype=t.dtype)[:, 1], lambda t: t[:-1]])
def test_vectors_that_lie_elsewhere_are_refused(calls, name, what, view):
    with pytest.raises(ValueError, match=rf"^{what} has to be"):
        _call(name, **{what: view(CALLS[name][2][what])})
    assert calls == []


@pytest.mark.parametrize("name", ["norm_bwd", "loss", "loss_bwd"])
def test_a_workspace_is_one_piece(calls, name):
    for bad in (z(128, dtype=torch.uint8)[::2], z(8, 8, dtype=torch.uint8).t()):
        with pytest.raises(ValueError, match="workspace has to be"):
            _call(name, workspace=bad)
    assert calls == []


@pytest.mark.parametrize("name", CALLS)
def test_pitches(calls, name):
    """Rows as far apart as the problem says and no others; what is behind them is nobody's business."""
    pitches = dict(ldx=K + 8, lds=K + 16, ldy=K + 24) if name.startswith("norm") else dict(ldx=K + 8, ldw=K + 16)
    of = dict(X="ldx", dX="ldx", R="lds", S="lds", dS="lds", dR="lds", Y="ldy", dY="ldy") if name.startswith("norm") else dict(X="ldx", dX="ldx", W="ldw", dW="ldw")
    right, flat, whole = {}, {}, {}
    for what, ld in of.items():
        t = CALLS[name][2].get(what)
        if t is None:
            continue
        right[what] = z(t.shape[0] + 1, pitches[ld], dtype=t.dtype)[:, :K]
        whole[what] = z(t.shape[0], pitches[ld], dtype=t.dtype)
        flat[what] = z((t.shape[0] - 1) * pitches[ld] + K, dtype=t.dtype)
    for views in (right, whole, flat):
        _call(name, pitches, **views)
    assert len(calls) == 3
    for what in right:
        for bad in (CALLS[name][2][what], flat[what][:-1], z(right[what].shape[0], K + 32, dtype=BF16)[:, :K]):
            with pytest.raises(ValueError, match=rf"^{what} has to be"):
                _call(name, pitches, **{**right, what: bad})
    assert len(calls) == 3


def test_other_shapes_of_whole_matrices(calls):
    """A batch of sequences, more rows than the problem has, one row of any stride."""
    _call("loss", X=z(2, 3, K), W=z(V + 3, K), target=z(2, 3, dtype=torch.int64), lse=z(M + 1, dtype=F32))
    _call("norm", X=z(2, 3, K), Y=z(M * K), S=z(3, 2, K))
    norm.flux_norm(norm.norm_problem(1, K), z(5, 2 * K)[2:3, :K], None, z(K), None, z(K))
    norm.flux_norm(norm.norm_problem(M, 1), z(M, 1), None, z(1), None, z(1, M).t())
    assert len(calls) == 4
    with pytest.raises(ValueError):
        _call("loss", X=z(2, 3, K + 8))


@pytest.mark.parametrize("out,row", [("mx4", 16), ("mx8", 32)])
def test_blocks(calls, out, row):
    p = norm.norm_problem(M, 40, out=out)
    u8 = lambda *shape: z(*shape, dtype=torch.uint8)      # noqa: E731
    X, W = z(M, 40), z(40)
    norm.flux_norm(p, X, None, W, None, u8(M + 1, 2 * row), u8(M, 16))
    assert len(calls) == 1
    for q, scales in ((u8(M, 2 * row - 1), u8(M, 16)), (u8(M, 4 * row)[:, ::2], u8(M, 16)), (u8(M, 2 * row), u8(M, 15)), (u8(M, 2 * row), u8(M, 32)[:, :16]),
                      (u8(M, 2 * row + 16)[:, :2 * row], u8(M, 16))):
        with pytest.raises(ValueError):
            norm.flux_norm(p, X, None, W, None, q, scales)
    assert len(calls) == 1


def test_join(calls):
    p, v = loss.loss_problem(M, V, K), z(M, dtype=F32)
    t = z(M, dtype=torch.int64)
    loss.flux_loss_join(p, [v, v], [v, v], t, v, None, v)
    assert len(calls) == 1
    odd = z(M, 2, dtype=F32)[:, 0]
    for args in (([v, odd], [v, v], t, v, v, v), ([v, v], [v, v[:-1]], t, v, v, v), ([v], [v], z(M, 2, dtype=torch.int64)[:, 0], v, v, v), ([v], [v], t[1:], v, v, v),
                 ([v], [v], t, odd, v, v), ([v], [v], t, v, odd, v), ([v], [v], t, v, v, v[2:])):
        with pytest.raises(ValueError):
            loss.flux_loss_join(p, *args)
    assert len(calls) == 1


def test_one_dloss_for_all_rows(calls):
    one = torch.zeros(1)
    _call("loss_bwd", dict(dloss_one=1), dloss=one)
    _call("loss_bwd", dict(dloss_one=1), dloss=torch.zeros(()))
    with pytest.raises(ValueError):
        _call("loss_bwd", dloss=one)
    assert len(calls) == 2


@pytest.mark.parametrize("module", ["norm", "loss", "ffn"])
def test_a_torch_without_gpu_can_import(module):
    """As `ffn`: what only a build of torch for GPUs has is looked for when a call is made."""
    code = f"import torch; del torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream; import paper_2406_06858_amd.{module} as m; assert m.lib"
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-500:]
