"""The cross entropy of a vocabulary projection on the GPU against the oracle in 64 bits.

Bounds, with U = 2^-24 (a half step of fp32; of bf16 2^-8).  A logit is a sum of K products in fp32, 32 at a time, the accumulator of the matrix
units truncating at worst: off by (K / 16 + 16) 2 U of the sum of magnitudes, z_off.  lse is off by the largest of those of its row, by what exp and the sums
are: |Z - max| + 2 roundings a term, V / 256 + 64 of sums, and by the roundings of the logarithm and the last sum.
"""
import numpy as np
import pytest
import torch

from oracle import norm_loss_oracle as no
from paper_2406_06858_amd import ffn, loss

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24


def f64(t):
    return t.detach().cpu().double().numpy()


def assert_within(got, want, bound, what=""):
    g = f64(got)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    bad = ~(np.abs(g - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} out of bounds, first at {np.argwhere(bad)[0]}: {g[bad][0]} for {want[bad][0]}"


def padded(rows, cols, pitch, dtype, fill=7.0):
    buf = torch.full((rows * pitch + 8,), fill, dtype=dtype, device=DEV)
    return buf[:rows * pitch].view(rows, pitch)[:, :cols], buf


def untouched(view, buf):
    rows, cols = view.shape
    pitch = view.stride(0) if rows > 1 else cols
    assert (buf[rows * pitch:] == 7.0).all()
    assert (buf[:rows * pitch].view(rows, pitch)[:, cols:] == 7.0).all()


class Case:
    def __init__(self, M, V, K, seed, v0=0, vocab=0, pad=(0, 0), ignored=0.2, scale=1.0):
        gen = torch.Generator().manual_seed(seed)
        self.M, self.V, self.K, self.v0, self.vocab, self.pad = M, V, K, v0, vocab or v0 + V, pad
        self.X, _ = padded(M, K, K + pad[0], torch.bfloat16)
        self.W, _ = padded(V, K, K + pad[1], torch.bfloat16)
        self.X.copy_(torch.randn(M, K, generator=gen))
        self.W.copy_(torch.randn(V, K, generator=gen) * (scale * 2.0 / K ** 0.5))
        target = torch.randint(0, self.vocab, (M,), generator=gen)
        target[0], target[-1] = v0, v0 + V - 1                                    # the first and the last column
        skip = torch.rand(M, generator=gen) < ignored
        skip[0] = skip[-1] = False
        self.target = torch.where(skip, torch.tensor([-100, -1, self.vocab, self.vocab + 12345])[torch.arange(M) % 4], target)
        self.dloss = torch.randn(M, generator=gen)
        self.x, self.w, self.t = f64(self.X), f64(self.W), self.target.numpy()
        self.lse, self.logit, self.loss, self.z = no.loss(self.x, self.w, self.t, v0, self.vocab)
        self.z_off = np.abs(self.x) @ np.abs(self.w).T * (K / 16 + 16) * 2 * U

    def problem(self, **kw):
        return loss.loss_problem(self.M, self.V, self.K, v0=self.v0, vocab=self.vocab, ldx=self.K + self.pad[0], ldw=self.K + self.pad[1], **kw)

    def lse_off(self):
        below = self.z.max(axis=1, keepdims=True) - self.z
        p = np.exp(self.z - self.lse[:, None])
        return self.z_off.max(axis=1) + (p * (below + 2)).sum(axis=1) * 2 * U + (self.V / 256 + 64) * U + (np.abs(self.lse) + 8) * 4 * U

    def forward(self, target_dtype=torch.int64, **kw):
        p = self.problem(target_dtype=target_dtype, **kw)
        ws = workspace(loss.FLUX_LOSS_FORWARD, p)
        out = [torch.full((self.M + 1,), 7.0, device=DEV) for _ in range(3)]
        loss.flux_loss(p, self.X, self.W, self.target.to(target_dtype).to(DEV), *out, ws)
        torch.cuda.synchronize()
        assert all(t[self.M] == 7.0 for t in out)
        return [t[:self.M] for t in out]

    def check_forward(self, got):
        off = self.lse_off()
        assert_within(got[0], self.lse, off, "lse")
        here = (self.t >= self.v0) & (self.t < min(self.v0 + self.V, self.vocab))
        z_off = np.where(here, self.z_off[np.arange(self.M), np.where(here, self.t - self.v0, 0)], 0.0)
        assert_within(got[1], self.logit, z_off, "logit")
        counts = (self.t >= 0) & (self.t < self.vocab)
        assert_within(got[2], self.loss, np.where(counts, off + z_off + np.abs(self.loss) * U, 0.0), "loss")

    def backward(self, dloss, lse, target_dtype=torch.int64, want=("dX", "dW"), dW=None, **kw):
        p = self.problem(target_dtype=target_dtype, **kw)
        ws = workspace(loss.FLUX_LOSS_BACKWARD, p)
        dX, bx = padded(self.M, self.K, self.K + self.pad[0], (torch.bfloat16, torch.float32)[p.dx_dtype]) if "dX" in want else (None, None)
        bw = None
        if dW is None and "dW" in want:
            dW, bw = padded(self.V, self.K, self.K + self.pad[1], (torch.bfloat16, torch.float32)[p.dw_dtype])
        loss.flux_loss_backward(p, self.X, self.W, self.target.to(target_dtype).to(DEV), lse, dloss.to(DEV), dX, dW, ws)
        torch.cuda.synchronize()
        for view, buf in ((dX, bx), (dW, bw)):
            if buf is not None:
                untouched(view, buf)
        return dX, dW

    def gradients(self, lse, dloss):
        """Want and bound of dX and dW but for their last rounding, lse and dloss as they are handed over."""
        d = np.broadcast_to(f64(dloss), (self.M,))
        lse = f64(lse)
        dx, dw, dz = no.loss_backward(self.x, self.w, self.t, self.v0, self.vocab, lse, d)
        counts = (self.t >= 0) & (self.t < self.vocab)
        p = np.exp(self.z - lse[:, None]) * (np.abs(d) * counts)[:, None]
        # p: the logit's error, the difference's and exp's roundings; then the difference to 1, the product with dloss, and the rounding to bf16
        dz_off = p * (self.z_off + (np.abs(self.z - lse[:, None]) + np.abs(self.z) + 4) * 2 * U) + np.abs(dz) * (HALF["bf16"] + 4 * U)
        dx_off = dz_off @ np.abs(self.w) + np.abs(dz) @ np.abs(self.w) * (self.V / 16 + 16) * 2 * U
        dw_off = dz_off.T @ np.abs(self.x) + np.abs(dz).T @ np.abs(self.x) * (self.M / 16 + 16) * 2 * U
        return dx, dx_off, dw, dw_off

    def check_backward(self, got, lse, dloss, dx="bf16", dw="bf16"):
        dx64, dx_off, dw64, dw_off = self.gradients(lse, dloss)
        # (a denormal gradient has bf16's smallest step)
        assert_within(got[0], dx64, dx_off + (np.abs(dx64) + dx_off) * HALF[dx] + 2.0 ** -133, "dX")
        assert_within(got[1], dw64, dw_off + (np.abs(dw64) + dw_off) * HALF[dw] + 2.0 ** -133, "dW")


def workspace(op, p):
    """Ready for its first call, and full of NaN but for what has to be zero."""
    n = loss.flux_loss_workspace_bytes(op, p)
    ws = torch.full(((n + 3) // 4,), float("nan"), device=DEV)
    ffn.flux_ffn_init(ws)
    return ws


SHAPES = [(1, 1, 8), (1, 2, 8), (2, 1, 64), (1, 1000, 64), (3, 257, 72), (17, 50, 8), (64, 4000, 512), (65, 129, 200), (130, 1000, 256), (257, 513, 136), (300, 777, 1000),
          (512, 2048, 1024), (33, 5003, 320)]


@pytest.mark.parametrize("M,V,K", SHAPES)
def test_forward(M, V, K):
    for pad, dtype in (((0, 0), torch.int64), ((24, 8), torch.int32)):
        c = Case(M, V, K, M + V + K, pad=pad)
        c.check_forward(c.forward(dtype))


@pytest.mark.parametrize("M,V,K", SHAPES)
def test_backward(M, V, K):
    for pad, dtype, dx, dw in (((0, 0), torch.int64, "bf16", "bf16"), ((24, 8), torch.int32, "f32", "f32")):
        c = Case(M, V, K, 3 * M + V + K, pad=pad)
        lse = torch.from_numpy(c.lse).float().to(DEV)
        got = c.backward(c.dloss, lse, dtype, dx_dtype=dx, dw_dtype=dw)
        c.check_backward(got, lse, c.dloss, dx, dw)
        skipped = torch.from_numpy((c.t < 0) | (c.t >= c.vocab))
        assert not got[0].cpu()[skipped].any()
        for one in (("dX",), ("dW",)):
            alone = c.backward(c.dloss, lse, dtype, want=one, dx_dtype=dx, dw_dtype=dw)
            for a, b in zip(alone, got):
                assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("config", range(1, 7))
@pytest.mark.parametrize("split", [0, 1, 5])
def test_every_tile(config, split):
    """All tiles, whole and cut, over edges in every direction and over none."""
    for M, V, K in ((300, 777, 1000), (256, 512, 1536), (70, 130, 1000)):
        c = Case(M, V, K, config * 10 + split)
        c.check_forward(c.forward(tile_config=config, split_k=split))
        lse = torch.from_numpy(c.lse).float().to(DEV)
        c.check_backward(c.backward(c.dloss, lse, tile_config=config, split_k=split), lse, c.dloss)


@pytest.mark.parametrize("M", [1, 8, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("V,K", [(1, 8), (15, 256), (33, 264), (4096, 512), (4099, 520), (777, 1544), (300, 4096)])
def test_few_rows_on_their_own_kernel(M, V, K):
    """Short and long rows, with whole pieces and without, 16 and 32 columns a workgroup; and the tiles for the same."""
    c = Case(M, V, K, M * V + K, pad=(8, 16))
    lse = torch.from_numpy(c.lse).float().to(DEV)
    for config in (ffn.flux_ffn_tile_config_count(), 5):
        c.check_forward(c.forward(tile_config=config))
        c.check_backward(c.backward(c.dloss, lse, tile_config=config), lse, c.dloss)


@pytest.mark.parametrize("piece", [64, 128, 192, 512, 1 << 20])
@pytest.mark.parametrize("dx,dw", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_pieces_of_the_vocabulary(piece, dx, dw):
    for M, V, K, pad in ((130, 1000, 256, (8, 16)), (9, 449, 64, (0, 0)), (257, 512, 136, (0, 8))):
        c = Case(M, V, K, piece + M, pad=pad)
        lse = torch.from_numpy(c.lse).float().to(DEV)
        got = c.backward(c.dloss, lse, dx_dtype=dx, dw_dtype=dw, piece=piece)
        c.check_backward(got, lse, c.dloss, dx, dw)
        again = c.backward(c.dloss, lse, dx_dtype=dx, dw_dtype=dw, piece=piece)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("ranks", [1, 2, 3, 8, 16])
def test_shards_and_their_join(ranks):
    M, V, K = 70, 48, 128
    gen = torch.Generator().manual_seed(ranks)
    shards = [Case(M, V, K, 100 + r, v0=r * V, vocab=ranks * V) for r in range(ranks)]
    target = torch.randint(0, ranks * V, (M,), generator=gen)
    target[5], target[6] = -100, ranks * V
    X = shards[0].X
    for r, c in enumerate(shards):
        c.X, c.target, c.t, c.x = X, target, target.numpy(), f64(X)
        c.lse, c.logit, c.loss, c.z = no.loss(c.x, c.w, c.t, c.v0, c.vocab)
        c.z_off = np.abs(c.x) @ np.abs(c.w).T * (K / 16 + 16) * 2 * U
    parts = [c.forward() for c in shards]
    for c, part in zip(shards, parts):
        c.check_forward(part)
    lse, logit, value = (torch.empty(M, device=DEV) for _ in range(3))
    loss.flux_loss_join(shards[0].problem(), [p[0] for p in parts], [p[1] for p in parts], target.to(DEV), lse, logit, value)
    whole = no.loss(f64(X), np.concatenate([c.w for c in shards]), target.numpy(), 0, ranks * V)
    off = np.max([c.lse_off() for c in shards], axis=0) + (ranks + 40) * 4 * U
    z_off = np.max([c.z_off.max(axis=1) for c in shards], axis=0)
    assert_within(lse, whole[0], off, "lse")
    assert_within(logit, whole[1], z_off, "logit")
    assert_within(value, whole[2], np.where(whole[2] == 0, 0.0, off + z_off + np.abs(whole[2]) * U), "loss")
    # into an input's place; and the gradients of every shard under the whole vocabulary's lse
    again = parts[0][0].clone()
    loss.flux_loss_join(shards[0].problem(), [again] + [p[0] for p in parts[1:]], [p[1] for p in parts], target.to(DEV), again)
    assert torch.equal(again, lse)
    dloss = torch.randn(M, generator=gen)
    for c in shards:
        c.check_backward(c.backward(dloss, lse), lse, dloss)


@pytest.mark.parametrize("M", [65, 40, 9])
def test_one_number_for_every_row_and_gradients_added_up(M):
    c = Case(M, 300, 136, 8, pad=(0, 8))
    lse = torch.from_numpy(c.lse).float().to(DEV)
    one = torch.tensor([0.125])
    got = c.backward(one, lse, dloss_one=1)
    c.check_backward(got, lse, one)
    for dw in ("bf16", "f32"):
        held, _ = padded(c.V, c.K, c.K + 8, TORCH[dw])
        held.copy_(torch.randn(c.V, c.K, generator=torch.Generator().manual_seed(3)))
        before = f64(held)
        _, dw64, off = c.gradients(lse, one)[1:]
        _, dW = c.backward(one, lse, dloss_one=1, dw_accumulate=1, dw_dtype=dw, dW=held, piece=128)
        assert_within(dW, dw64 + before, off + (np.abs(dw64 + before) + off) * (HALF[dw] + U), dw)


@pytest.mark.parametrize("M", [6, 70, 300])
def test_dloss_of_every_size(M):
    """From 2^-60 to 2^60 side by side, zeros, all zeros, one infinity."""
    c = Case(M, 333, 64, 16)
    lse = torch.from_numpy(c.lse).float().to(DEV)
    c.dloss *= 2.0 ** torch.randint(-60, 61, (M,), generator=torch.Generator().manual_seed(M))
    c.dloss[1] = 0
    c.check_backward(c.backward(c.dloss, lse, dx_dtype="f32", dw_dtype="f32"), lse, c.dloss, "f32", "f32")
    for one in (0, 1):
        dX, dW = c.backward(torch.zeros(1 if one else M), lse, dloss_one=one)
        assert not dX.any() and not dW.any()
    c.dloss[0] = float("inf")
    dX, _ = c.backward(c.dloss, lse, dx_dtype="f32")
    assert not bool(dX[0].isfinite().any())
    # (the other rows have no factor then: their dZ is rounded with dloss in it, within the same bound)
    dx64, off, _, _ = c.gradients(lse, torch.where(c.dloss == float("inf"), 0.0, c.dloss))
    assert_within(dX[1:], dx64[1:], off[1:] + np.abs(dx64[1:]) * 2 * U, "other rows")


def test_rows_that_do_not_count_hide_what_they_hold():
    """A row without a target and with dloss or lse that are no numbers adds nothing; a row of NaN logits keeps to itself in the forward pass."""
    c = Case(70, 200, 64, 4)
    c.target[3], c.t[3] = -100, -100
    c.dloss[3] = float("nan")
    lse = torch.from_numpy(c.lse).float().to(DEV)
    lse[3] = float("inf")
    got = c.backward(c.dloss, lse)
    assert not got[0][3].any() and bool(got[0].isfinite().all()) and bool(got[1].isfinite().all())
    want = c.forward()
    c.X[7, 5] = float("nan")
    c.X[9, 5] = 1e38
    lse, logit, value = c.forward()
    rows = [r for r in range(70) if r not in (7, 9)]
    assert bool(lse[7].isnan())
    for a, b in zip(want, (lse, logit, value)):
        assert torch.equal(a[rows], b[rows])


@pytest.mark.parametrize("M,V,K", [(5, 77, 136), (70, 300, 264), (300, 520, 512), (31, 4100, 2056)])
@pytest.mark.parametrize("dloss", [float("inf"), float("nan")])
def test_a_mean_over_no_row_has_no_gradient(M, V, K, dloss):
    c = Case(M, V, K, 41)
    target = torch.full((M,), -100, device=DEV)
    for accumulate in (0, 1):
        p = c.problem(dloss_one=1, dw_dtype="f32", dw_accumulate=accumulate)
        dX, dW = torch.full_like(c.X, 5.0), torch.full((V, K), 3.0, device=DEV)
        loss.flux_loss_backward(p, c.X, c.W, target, torch.full((M,), float("nan"), device=DEV), torch.tensor([dloss], device=DEV), dX, dW,
                                workspace(loss.FLUX_LOSS_BACKWARD, p))
        assert (dX == 0).all() and (dW == 3.0 * accumulate).all()


@pytest.mark.parametrize("M", [5, 70])
def test_logits_beyond_all_measure(M):
    """Rows of equal logits of 2^100: what is left of the difference to the largest is nothing, not its rounding."""
    V, K = 300, 64
    X, W = torch.full((M, K), 2.0 ** 47, device=DEV).to(torch.bfloat16), torch.full((V, K), 2.0 ** 47, device=DEV).to(torch.bfloat16)
    W[:, 0] *= 1.5                                                     # (64.5 2^94: log2 e times that is no number of 24 bits)
    X[1] *= -1
    target, one = torch.arange(M, device=DEV), torch.ones(1, device=DEV)
    for config in (1, 5) + ((ffn.flux_ffn_tile_config_count(),) if M <= 64 else ()):
        p = loss.loss_problem(M, V, K, tile_config=config, dloss_one=1, dx_dtype="f32", dw_dtype="f32")
        lse, logit, value = (torch.empty(M, device=DEV) for _ in range(3))
        loss.flux_loss(p, X, W, target, lse, logit, value, workspace(loss.FLUX_LOSS_FORWARD, p))
        want = torch.full((M,), 64.5 * 2.0 ** 94, device=DEV)
        want[1] *= -1
        assert torch.equal(logit, want) and torch.equal(lse, want) and not value.any()
        dX, dW = torch.empty(M, K, device=DEV), torch.empty(V, K, device=DEV)
        loss.flux_loss_backward(p, X, W, target, lse, one, dX, dW, workspace(loss.FLUX_LOSS_BACKWARD, p))
        # (lse has no room for log 300: every exp is 1, dZ 1 but 0 at the target)
        dz = torch.ones(M, V, dtype=torch.float64, device=DEV) - torch.nn.functional.one_hot(target, V)
        assert torch.equal(dX.double(), dz @ W.double()) and torch.equal(dW.double(), dz.t() @ X.double())


@pytest.mark.parametrize("M", [5, 70])
def test_large_and_infinite_logits(M):
    """Logits of thousands: the sums neither overflow nor vanish.  One of infinity: lse is infinite, and a column of minus infinity counts for nothing."""
    c = Case(M, 300, 64, 6, scale=4000.0)
    c.check_forward(c.forward())
    lse = torch.from_numpy(c.lse).float().to(DEV)
    c.check_backward(c.backward(c.dloss, lse), lse, c.dloss)
    c.X.fill_(1.0)
    c.W.fill_(0.5)
    c.W[17, 0] = float("-inf")
    lse = c.forward()[0]
    assert_within(lse, np.full(M, 32 + np.log(299.0)), 1e-4)
    c.W[17, 0] = float("inf")
    assert bool((c.forward()[0] == float("inf")).all())
    c.W[:, 0] = float("-inf")
    assert bool((c.forward()[0] == float("-inf")).all())


def test_long_lists_of_columns():
    """More columns than the largest vocabularies have."""
    c = Case(3, 300001, 8, 12)
    c.check_forward(c.forward())
    lse = torch.from_numpy(c.lse).float().to(DEV)
    c.check_backward(c.backward(c.dloss, lse, piece=1 << 16), lse, c.dloss)


def test_rows_that_are_no_whole_lines():
    """X in rows that begin anywhere in a line is laid out anew where that pays: the bits are those of X in rows of whole lines."""
    M, V, K = 1000, 20001, 4104
    gen = torch.Generator(device=DEV).manual_seed(1)
    X = torch.randn(M, K, generator=gen, device=DEV).to(torch.bfloat16)
    W = (0.02 * torch.randn(V, K, generator=gen, device=DEV)).to(torch.bfloat16)
    target, dloss = torch.randint(0, V, (M,), generator=gen, device=DEV), torch.randn(M, generator=gen, device=DEV)
    got = []
    for pitch in (K, K + 8, (K + 63) // 64 * 64):
        x, _ = padded(M, K, pitch, torch.bfloat16)
        x.copy_(X)
        p = loss.loss_problem(M, V, K, ldx=pitch, piece=4096)
        out = [torch.empty(M, device=DEV) for _ in range(3)]
        loss.flux_loss(p, x, W, target, *out, workspace(loss.FLUX_LOSS_FORWARD, p))
        (dX, buf), dW = padded(M, K, pitch, torch.bfloat16), torch.empty_like(W)
        loss.flux_loss_backward(p, x, W, target, out[0], dloss, dX, dW, workspace(loss.FLUX_LOSS_BACKWARD, p))
        torch.cuda.synchronize()
        untouched(dX, buf)
        got.append((*out, dX, dW))
    sizes = [loss.flux_loss_workspace_bytes(op, loss.loss_problem(M, V, K, ldx=ld, piece=4096)) for op in (0, 1) for ld in (K, (K + 63) // 64 * 64)]
    assert sizes[0] > sizes[1] and sizes[2] > sizes[3]                # (the copy was made)
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("M,V,ldx,ldw", [(40, 8, 0, 150_000_000), (14, 96, 150_000_000, 0), (40, 31, 0, 71_000_000), (31, 30, 71_000_000, 71_000_000), (3, 3, 0, 1_000_000_000)])
def test_pitches_whose_offsets_take_all_32_bits(M, V, ldx, ldw):
    """The bits of rows side by side; what lies between the rows is no number."""
    K = 136
    gen = torch.Generator(device=DEV).manual_seed(3)
    X, W = (torch.randn(n, K, generator=gen, device=DEV).to(torch.bfloat16) for n in (M, V))
    target, dloss = torch.arange(M, device=DEV) % (V + 1), torch.randn(M, generator=gen, device=DEV)
    got = []
    for lx, lw in ((0, 0), (ldx, ldw)):
        views = []
        for t, ld in ((X, lx), (W, lw), (X, lx), (W, lw)):
            n = t.shape[0]
            buf = torch.full(((n - 1) * (ld or K) + K,), float("nan"), dtype=torch.bfloat16, device=DEV)
            views.append(buf.as_strided((n, K), (ld or K, 1)))
        x, w, dX, dW = views
        x.copy_(X)
        w.copy_(W)
        p = loss.loss_problem(M, V, K, ldx=lx, ldw=lw)
        out = [torch.empty(M, device=DEV) for _ in range(3)]
        loss.flux_loss(p, x, w, target, *out, workspace(loss.FLUX_LOSS_FORWARD, p))
        loss.flux_loss_backward(p, x, w, target, out[0], dloss, dX, dW, workspace(loss.FLUX_LOSS_BACKWARD, p))
        torch.cuda.synchronize()
        got.append([*out, dX.contiguous(), dW.contiguous()])
        del x, w, dX, dW, views, buf
        torch.cuda.empty_cache()
    assert torch.isfinite(got[0][4]).all()
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("M,config", [(1, 6), (40, 5), (64, 6), (65, 3), (100, 4)])
def test_weights_that_are_read_past_the_caches(M, config):
    """Large matrices in whole lines are, others are not: the same bits."""
    V, K = 25001, 4096
    gen = torch.Generator(device=DEV).manual_seed(M)
    X = torch.randn(M, K, generator=gen, device=DEV).to(torch.bfloat16)
    W = (0.02 * torch.randn(V, K, generator=gen, device=DEV)).to(torch.bfloat16)
    target, dloss = torch.randint(0, V, (M,), generator=gen, device=DEV), torch.randn(M, generator=gen, device=DEV)
    got = []
    for pitch in (K, K + 8):
        w, _ = padded(V, K, pitch, torch.bfloat16)
        w.copy_(W)
        p = loss.loss_problem(M, V, K, ldw=pitch, tile_config=config)
        out = [torch.empty(M, device=DEV) for _ in range(3)]
        loss.flux_loss(p, X, w, target, *out, workspace(loss.FLUX_LOSS_FORWARD, p))
        dX, (dW, buf) = torch.empty_like(X), padded(V, K, pitch, torch.bfloat16)
        loss.flux_loss_backward(p, X, w, target, out[0], dloss, dX, dW, workspace(loss.FLUX_LOSS_BACKWARD, p))
        torch.cuda.synchronize()
        untouched(dW, buf)
        got.append((*out, dX, dW))
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("M", [1, 31, 33, 64, 65, 128])
@pytest.mark.parametrize("dw,accumulate", [("bf16", 0), ("f32", 1)])
def test_large_weight_gradients_of_few_rows(M, dw, accumulate):
    """dW as an outer product: every count of terms, an odd number of rows, columns that end inside a strip, set and added to."""
    V, K = 4099, 2056
    gen = torch.Generator(device=DEV).manual_seed(M)
    X = torch.randn(M, K, generator=gen, device=DEV).to(torch.bfloat16)
    W = (0.02 * torch.randn(V, K, generator=gen, device=DEV)).to(torch.bfloat16)
    target, dloss = torch.randint(0, V, (M,), generator=gen, device=DEV), torch.randn(M, generator=gen, device=DEV)
    z = X.double() @ W.double().t()
    lse = torch.logsumexp(z, 1).float()
    p = loss.loss_problem(M, V, K, ldw=K + 8, dw_dtype=dw, dw_accumulate=accumulate)
    w, _ = padded(V, K, K + 8, torch.bfloat16)
    w.copy_(W)
    dW, buf = padded(V, K, K + 8, TORCH[dw])
    loss.flux_loss_backward(p, X, w, target, lse, dloss, None, dW, workspace(loss.FLUX_LOSS_BACKWARD, p))
    torch.cuda.synchronize()
    untouched(dW, buf)
    pr = torch.exp(z - lse.double()[:, None])
    dz = (pr - torch.nn.functional.one_hot(target, V)) * dloss.double()[:, None]
    want = dz.t() @ X.double() + 7.0 * accumulate
    # (bounds as in Case.gradients; what Z is off by from the sum of magnitudes)
    z_off = X.double().abs() @ W.double().abs().t() * (K / 16 + 16) * 2 * U
    dz_off = pr * dloss.double().abs()[:, None] * (z_off + (z.abs() + (z - lse.double()[:, None]).abs() + 4) * 2 * U) + dz.abs() * (HALF["bf16"] + 4 * U)
    off = dz_off.t() @ X.double().abs() + dz.abs().t() @ X.double().abs() * (M / 16 + 16) * 2 * U
    bad = ~((dW.double() - want).abs() <= off + (want.abs() + off) * (HALF[dw] + U))
    assert not bad.any(), int(bad.sum())


def test_captured_and_replayed():
    c = Case(200, 3000, 512, 14)
    target = c.target.to(DEV)
    pf = c.problem(piece=1024)
    ws = workspace(loss.FLUX_LOSS_BACKWARD, pf)
    n = loss.flux_loss_workspace_bytes(loss.FLUX_LOSS_FORWARD, pf)
    if ws.numel() * 4 < n:
        ws = workspace(loss.FLUX_LOSS_FORWARD, pf)
    lse, logit, value = (torch.empty(c.M, device=DEV) for _ in range(3))
    dX, dW, dloss = torch.empty_like(c.X), torch.empty_like(c.W), c.dloss.to(DEV)

    def step():
        loss.flux_loss(pf, c.X, c.W, target, lse, logit, value, ws)
        loss.flux_loss_backward(pf, c.X, c.W, target, lse, dloss, dX, dW, ws)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for i in range(4):
        c.X.copy_(torch.randn(c.M, c.K, generator=torch.Generator().manual_seed(50 + i)))
        step()
        outs = (lse, logit, value, dX, dW)
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            assert torch.equal(a, b), i


def test_streams_of_their_own():
    c = Case(130, 1000, 1000, 15)
    target = c.target.to(DEV)
    p = c.problem()
    want = c.forward()
    runs = []
    for _ in range(3):
        runs.append((torch.cuda.Stream(), workspace(loss.FLUX_LOSS_FORWARD, p), [torch.empty(c.M, device=DEV) for _ in range(3)]))
    torch.cuda.synchronize()
    for _ in range(5):
        for s, ws, out in runs:
            loss.flux_loss(p, c.X, c.W, target, *out, ws, stream=s)
    torch.cuda.synchronize()
    for _, _, out in runs:
        for a, b in zip(want, out):
            assert torch.equal(a, b)


def test_tensors_of_another_type_or_device_are_refused():
    c = Case(4, 64, 64, 1)
    p, f = c.problem(), torch.empty(4, device=DEV)
    t = c.target.to(DEV)
    ws = workspace(loss.FLUX_LOSS_FORWARD, p)
    for args in ((c.X.float(), c.W, t, f, f, f, ws), (c.X, c.W.cpu(), t, f, f, f, ws), (c.X, c.W, t.int(), f, f, f, ws), (c.X, c.W, t, f.double(), f, f, ws),
                 (c.X, c.W, t, f, f, f, ws.cpu()), (c.X, c.W, t.cpu(), f, f, f, ws)):
        with pytest.raises(ValueError):
            loss.flux_loss(p, *args)
    with pytest.raises(ValueError):
        loss.flux_loss_backward(p, c.X, c.W, t, f, f, c.X.float(), None, ws)
    with pytest.raises(ValueError):
        loss.flux_loss_join(p, [f], [f, f], t, f)
    with pytest.raises(ValueError):
        loss.flux_loss_join(p, [f.cpu()], [f], t, f)
