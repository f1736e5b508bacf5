"""Adapters beside the shared projections (mbq_lora_sort, mbq_lora_group, mbq_lora_backward_group) against the definition in
64 bits, at the sizes, ranks, assignments and alignments where they can go wrong.

Tolerances.  Products of bf16 values are exact in fp32 and every other operand is fp32, so an output is off by the roundings
of its sums.  A sum of n terms in fp32, in any order, is off by at most (n - 1) u sum |terms| (u = 2^-24) and, as the roundings
are independent, by about sqrt(n) u sum |terms| at most; a value passes within (4 sqrt(n) + 16) u sum |terms|, an array within
(sqrt(n) + 8) u of its norm, where sums of sums add up."""
import ctypes

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def factor(n):
    return (4.0 * n ** 0.5 + 16.0) * U


class Case:
    """Inputs on the GPU and what the definition makes of them (fp64, CPU)."""

    def __init__(self, T, K, Ns, n, r, seed=0, ragged=False, bare=0.2, assignment=None, poison=False, with_base=True):
        gen = torch.Generator().manual_seed(seed)
        self.T, self.K, self.Ns, self.n, self.r = T, K, list(Ns), n, r
        self.X = torch.randn((T, K), generator=gen).to(torch.bfloat16)
        if assignment is None:
            assignment = torch.randint(0, n, (T,), generator=gen)
            assignment = torch.where(torch.rand(T, generator=gen) < bare, -1, assignment)
        self.adapter = torch.as_tensor(assignment).to(torch.int32)
        self.scale = torch.rand(n, generator=gen) + 0.5
        self.ranks = torch.randint(0, r + 1, (n,), generator=gen).to(torch.int32) if ragged else None
        self.A = [(torch.randn((n, r, K), generator=gen) / K ** 0.5).to(torch.bfloat16) for _ in Ns]
        self.B = [torch.randn((n, r, N), generator=gen).to(torch.bfloat16) for N in Ns]
        self.base = [torch.randn((T, N), generator=gen) if with_base else None for N in Ns]
        self.dY = [torch.randn((T, N), generator=gen) for N in Ns]
        self.dx_base = torch.randn((T, K), generator=gen) if with_base else None
        self.own = [r if self.ranks is None else int(self.ranks[a]) for a in range(n)]
        self.tokens_of = [torch.nonzero(self.adapter == a)[:, 0] for a in range(n)]
        self.H = [torch.zeros((T, r)) for _ in Ns]
        for p in range(len(Ns)):
            for a in range(n):
                at, k = self.tokens_of[a], self.own[a]
                self.H[p][at, :k] = (self.X[at].double() @ self.A[p][a, :k].double().t()).float()
        if poison:  # what is not to be used: rows beyond a rank, tokens without an adapter
            for a in range(n):
                for p in range(len(Ns)):
                    self.A[p][a, self.own[a]:] = float("nan")
                    self.B[p][a, self.own[a]:] = float("inf")
            none = (self.adapter < 0) | (self.adapter >= n)
            self.X[none] = float("nan")
            for p in range(len(Ns)):
                self.dY[p][none] = float("nan")
                for a in range(n):
                    for t in self.tokens_of[a]:
                        self.H[p][t, self.own[a]:] = float("nan")
                self.H[p][none] = float("inf")

    def tokens(self, mbq):
        adapter = self.adapter.cuda()
        return (adapter, *mbq.mbq_lora_sort(adapter, self.n))

    def forward(self, mbq, **more):
        on = lambda v: None if v is None else [None if t is None else t.cuda() for t in v]  # noqa: E731
        Y = mbq.mbq_lora_group(self.X.cuda(), on(self.A), on(self.B), self.tokens(mbq), self.scale.cuda(),
                               ranks=None if self.ranks is None else self.ranks.cuda(), base=on(self.base), **more)
        torch.cuda.synchronize()
        return Y

    def backward(self, mbq, **more):
        on = lambda v: [t.cuda() for t in v]  # noqa: E731
        d = mbq.mbq_lora_backward_group(self.X.cuda(), on(self.A), on(self.B), self.tokens(mbq), self.scale.cuda(),
                                        on(self.dY), on(self.H), ranks=None if self.ranks is None else self.ranks.cuda(),
                                        base=None if self.dx_base is None else self.dx_base.cuda(), **more)
        torch.cuda.synchronize()
        return d

    def check_forward(self, Y, H=None):
        for p, N in enumerate(self.Ns):
            want = torch.zeros((self.T, N), dtype=torch.float64) if self.base[p] is None else self.base[p].double().clone()
            size = want.abs()
            want_h, size_h = torch.zeros((self.T, self.r), dtype=torch.float64), torch.zeros((self.T, self.r), dtype=torch.float64)
            for a in range(self.n):
                at, k, s = self.tokens_of[a], self.own[a], float(self.scale[a])
                x, A, B = self.X[at].double(), self.A[p][a, :k].double(), self.B[p][a, :k].double()
                want_h[at, :k], size_h[at, :k] = x @ A.t(), x.abs() @ A.abs().t()
                want[at] += s * (want_h[at, :k] @ B)
                size[at] += s * (size_h[at, :k] @ B.abs())
            close(Y[p], want, size, self.K + self.r, f"Y[{p}]")
            if H is not None:
                close(H[p], want_h, size_h, self.K, f"H[{p}]")
                assert torch.equal(H[p].cpu() == 0, want_h == 0)

    def check_backward(self, dX, dA, dB):
        want_x = torch.zeros((self.T, self.K), dtype=torch.float64) if self.dx_base is None else self.dx_base.double().clone()
        size_x = want_x.abs()
        for p, N in enumerate(self.Ns):
            want_a, size_a = torch.zeros((2, self.n, self.r, self.K), dtype=torch.float64)
            want_b, size_b = torch.zeros((2, self.n, self.r, N), dtype=torch.float64)
            for a in range(self.n):
                at, k, s = self.tokens_of[a], self.own[a], float(self.scale[a])
                if not len(at):
                    continue
                x, dy, h = self.X[at].double(), self.dY[p][at].double(), self.H[p][at, :k].double()
                A, B = self.A[p][a, :k].double(), self.B[p][a, :k].double()
                g, size_g = s * dy @ B.t(), s * dy.abs() @ B.abs().t()
                want_x[at] += g @ A
                size_x[at] += size_g @ A.abs()
                want_a[a, :k], size_a[a, :k] = g.t() @ x, size_g.t() @ x.abs()
                want_b[a, :k], size_b[a, :k] = s * h.t() @ dy, s * h.abs().t() @ dy.abs()
            close(dA[p], want_a, size_a, N + self.T, f"dA[{p}]")
            close(dB[p], want_b, size_b, self.T, f"dB[{p}]")
        close(dX, want_x, size_x, max(self.Ns) + len(self.Ns) * self.r, "dX")


def close(got, want, size, terms, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    off = (got - want).abs()
    limit = factor(terms) * size
    bad = ~(off <= limit)
    assert not bad.any(), (what, int(bad.sum()), float(off[bad].max()), float(limit[bad].max()))
    norm = float(want.norm())
    if norm:
        rel = float((got - want).norm()) / norm
        print(f"[lora] {what}: relative error {rel:.2e}", flush=True)
        assert rel <= (terms ** 0.5 + 8) * U, (what, rel)


@pytest.mark.parametrize("T,n", [(0, 3), (1, 1), (5, 1), (16, 16), (64, 3), (257, 40), (1000, 7), (4099, 300)])
def test_sort_groups_stably(mbq, T, n):
    gen = torch.Generator().manual_seed(T + n)
    adapter = torch.randint(-1, n, (T,), generator=gen).to(torch.int32)
    if T > 4:  # none, whatever the value
        adapter[1], adapter[2], adapter[T // 2] = n, 2 ** 31 - 1, -(2 ** 31)
    perm, offsets = mbq.mbq_lora_sort(adapter.cuda(), n)
    key = torch.where((adapter < 0) | (adapter >= n), n, adapter.long())
    assert torch.equal(perm.cpu().long(), torch.argsort(key, stable=True))
    want = torch.cat([torch.zeros(1, dtype=torch.long), torch.bincount(key, minlength=n + 1).cumsum(0)[:n]])
    assert torch.equal(offsets.cpu().long(), want)


SHAPES = [  # T, K, Ns, adapters, r
    (1, 128, (1,), 1, 1),
    (1, 2048, (2048,), 4, 16),
    (2, 256, (7, 16), 3, 3),
    (15, 384, (130,), 40, 8),
    (16, 1024, (256, 64, 64), 16, 16),
    (17, 128, (257,), 2, 20),
    (31, 640, (1000, 24, 8, 40), 5, 33),
    (64, 1024, (1024, 1024), 64, 32),
    (65, 1024, (520,), 3, 16),
    (100, 128, (16,), 1, 256),
    (129, 2176, (300, 101), 11, 20),
    (300, 512, (1024,), 2, 64),
    (333, 256, (77,), 29, 100),
    (777, 384, (512, 128, 128), 4, 12),
    (1030, 256, (264,), 1, 16),
    (2050, 128, (136,), 3, 8),
]


@pytest.mark.parametrize("T,K,Ns,n,r", SHAPES)
@pytest.mark.parametrize("ragged", [False, True])
def test_forward(mbq, T, K, Ns, n, r, ragged):
    case = Case(T, K, Ns, n, r, seed=T + K, ragged=ragged)
    H = [torch.full((T, r), float("nan"), device="cuda") for _ in Ns]
    case.check_forward(case.forward(mbq, H=H), H)


@pytest.mark.parametrize("T,K,Ns,n,r", SHAPES)
@pytest.mark.parametrize("ragged", [False, True])
def test_backward(mbq, T, K, Ns, n, r, ragged):
    case = Case(T, K, Ns, n, r, seed=T + r, ragged=ragged)
    case.check_backward(*case.backward(mbq))


@pytest.mark.parametrize("T", [9, 64, 150, 700])
def test_what_is_not_to_be_used_is_not(mbq, T):
    """NaN and infinity in pool rows beyond a rank, in activations and gradients of tokens without an adapter, in H there."""
    case = Case(T, 256, (72, 33), 5, 24, seed=T, ragged=True, bare=0.3, poison=True)
    case.ranks[1] = 0
    case.own[1] = 0
    for p in range(2):
        case.A[p][1], case.B[p][1] = float("nan"), float("nan")
    H = [torch.empty((T, 24), device="cuda") for _ in range(2)]
    Y = case.forward(mbq, H=H)
    dX, dA, dB = case.backward(mbq)
    case.X[(case.adapter < 0)] = 0  # for the reference
    case.check_forward(Y, H)
    case.check_backward(dX, dA, dB)
    for p, N in enumerate(case.Ns):  # what nobody uses is zero, not small
        for a in range(5):
            assert torch.count_nonzero(dA[p][a, case.own[a]:]) == 0 and torch.count_nonzero(dB[p][a, case.own[a]:]) == 0


@pytest.mark.parametrize("T", [1, 20, 64, 90, 200])
@pytest.mark.parametrize("ids", ["none", "last", "far", "first and last"])
def test_assignments(mbq, T, ids):
    n = 70
    assignment = {"none": [-1] * T, "last": [n - 1] * T, "far": [[n, -(2 ** 31), 2 ** 31 - 1][i % 3] for i in range(T)],
                  "first and last": [0 if i % 2 else n - 1 for i in range(T)]}[ids]
    case = Case(T, 256, (136,), n, 8, seed=T, assignment=assignment)
    Y = case.forward(mbq)
    case.check_forward(Y)
    if ids in ("none", "far"):
        assert torch.equal(Y[0].cpu(), case.base[0])
    dX, dA, dB = case.backward(mbq)
    case.check_backward(dX, dA, dB)
    if ids in ("none", "far"):
        assert torch.equal(dX.cpu(), case.dx_base) and not torch.count_nonzero(dA[0]) and not torch.count_nonzero(dB[0])


@pytest.mark.parametrize("T", [3, 70, 300])
def test_base_left_out_and_in_place(mbq, T):
    case = Case(T, 512, (200, 48), 4, 16, seed=T)
    Y = case.forward(mbq)
    tokens = case.tokens(mbq)
    on = lambda v: [t.cuda() for t in v]  # noqa: E731
    kept = on(case.base)
    got = mbq.mbq_lora_group(case.X.cuda(), on(case.A), on(case.B), tokens, case.scale.cuda(), base=kept, Y=kept)
    assert all(torch.equal(a, b) for a, b in zip(got, Y)) and got[0] is kept[0]
    dX, dA, dB = case.backward(mbq)
    grad = case.dx_base.cuda()
    got = mbq.mbq_lora_backward_group(case.X.cuda(), on(case.A), on(case.B), tokens, case.scale.cuda(), on(case.dY),
                                      on(case.H), base=grad, dX=grad)
    assert torch.equal(got[0], dX) and all(torch.equal(a, b) for a, b in zip(got[1] + got[2], dA + dB))
    one = mbq.mbq_lora_group(case.X.cuda(), on(case.A), on(case.B), tokens, case.scale.cuda(), base=[kept[0], None])
    bare = Case(T, 512, (200, 48), 4, 16, seed=T, with_base=False)
    bare.base[0] = kept[0].cpu()
    bare.check_forward(one)
    bare.base[0] = None
    bare.check_forward(bare.forward(mbq))
    bare.check_backward(*bare.backward(mbq))


@pytest.mark.parametrize("T", [6, 66, 270])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_alignment(mbq, T, shift):
    """Outputs, bases, gradients and B that begin anywhere, with columns that would allow wide accesses."""
    case = Case(T, 256, (136, 64), 3, 16, seed=shift)
    Y, (dX, dA, dB) = case.forward(mbq), case.backward(mbq)

    def moved(t):
        flat = torch.empty(t.numel() + 8, dtype=t.dtype, device="cuda")
        out = flat[shift: shift + t.numel()].view(t.shape)
        out.copy_(t)
        return out

    tokens, X, scale = case.tokens(mbq), case.X.cuda(), case.scale.cuda()
    A, B = [a.cuda() for a in case.A], [moved(b) for b in case.B]
    got = mbq.mbq_lora_group(X, A, B, tokens, scale, base=[moved(b) for b in case.base], Y=[moved(y) for y in Y])
    case.check_forward(got)
    got = mbq.mbq_lora_backward_group(X, A, B, tokens, scale, [moved(d) for d in case.dY], [moved(h) for h in case.H],
                                      base=moved(case.dx_base), dX=moved(dX), dA=[moved(d) for d in dA],
                                      dB=[moved(d) for d in dB])
    case.check_backward(*got)


@pytest.mark.parametrize("T", [7, 64, 65, 500])
def test_neighbours_are_left_alone_and_equal_calls_give_equal_bits(mbq, T):
    case = Case(T, 384, (70, 264), 4, 20, seed=T)
    n, r = case.n, case.r

    def guarded(*shape):
        flat = torch.full((int(np.prod(shape)) + 512,), 7.0, device="cuda")
        return flat, flat[256:-256].view(shape)

    found = []
    for _ in range(2):
        Y, H = [guarded(T, N) for N in case.Ns], [guarded(T, r) for _ in case.Ns]
        dX, dA, dB = guarded(T, case.K), [guarded(n, r, case.K) for _ in case.Ns], [guarded(n, r, N) for N in case.Ns]
        case.forward(mbq, Y=[y[1] for y in Y], H=[h[1] for h in H])
        case.backward(mbq, dX=dX[1], dA=[d[1] for d in dA], dB=[d[1] for d in dB])
        every = Y + H + [dX] + dA + dB
        for flat, _ in every:
            assert (flat[:256] == 7).all() and (flat[-256:] == 7).all()
        found.append([v.clone() for _, v in every])
    assert all(torch.equal(a, b) for a, b in zip(*found))


def test_workspace_contents_do_not_matter(mbq):
    for T in (5, 300):
        case = Case(T, 256, (200,), 3, 16, seed=T)
        want, want_d = case.forward(mbq), case.backward(mbq)
        for fill in (0, 255):
            ws = mbq.lora_workspace(T, 256, 1, 16, "cuda").fill_(fill)
            back = mbq.lora_backward_workspace(T, 256, [200], 3, 16, "cuda").fill_(fill)
            assert torch.equal(case.forward(mbq, ws=ws)[0], want[0])
            got = case.backward(mbq, ws=back)
            assert torch.equal(got[0], want_d[0]) and torch.equal(got[1][0], want_d[1][0]) and torch.equal(got[2][0], want_d[2][0])


@pytest.mark.parametrize("T,n,ids", [(65, 70, "any"), (100, 300, "any"), (130, 200, "one"), (300, 2000, "few"), (70, 4100, "none")])
def test_more_adapters_than_tokens(mbq, T, n, ids):
    """Beyond the sizes of a decode batch, with a pool that most of the call does not touch."""
    gen = torch.Generator().manual_seed(n)
    some = {"any": n, "one": 1, "few": 3, "none": 1}[ids]
    assignment = torch.randint(0, some, (T,), generator=gen) * (n // some) + (n // some - 1)
    if ids == "none":
        assignment[:] = -1
    elif ids != "one":
        assignment[torch.rand(T, generator=gen) < 0.2] = -1
    case = Case(T, 256, (136, 33), n, 20, seed=T, ragged=True, assignment=assignment)
    H = [torch.full((T, 20), float("nan"), device="cuda") for _ in range(2)]
    case.check_forward(case.forward(mbq, H=H), H)
    case.check_backward(*case.backward(mbq))


@pytest.mark.parametrize("T,K,Ns,n,r", [(3, 4224, (136, 33), 2, 4), (5, 8192, (2056,), 3, 8), (2, 16384, (24, 7), 2, 3),
                                        (9, 2176, (300, 101), 5, 40), (6, 1024, (512, 264), 4, 100), (1, 20608, (600,), 1, 70)])
def test_decode_batches_of_long_rows_and_large_ranks(mbq, T, K, Ns, n, r):
    """One launch whose rows take several passes, and the two launches that larger factors take."""
    for ragged in (False, True):
        case = Case(T, K, Ns, n, r, seed=K + r, ragged=ragged)
        H = [torch.full((T, r), float("nan"), device="cuda") for _ in Ns]
        case.check_forward(case.forward(mbq, H=H), H)


@pytest.mark.parametrize("T", [20, 300])
@pytest.mark.parametrize("wanted", ["dX", "dA", "dB", "dX dA", "dX dB", "dA dB", ""])
def test_gradients_that_are_not_wanted(mbq, T, wanted):
    """Each subset of the gradients through the C interface, the others and what only they read null, has the bits of the full
    call."""
    case = Case(T, 384, (136, 40), 3, 24, seed=T, ragged=True)
    dX, dA, dB = case.backward(mbq)
    lib, N = mbq.load(), (ctypes.c_int64 * 2)(*case.Ns)
    at = lambda ts: (ctypes.c_void_p * len(ts))(*(t.data_ptr() for t in ts))  # noqa: E731
    X, base, tokens, scale, ranks = case.X.cuda(), case.dx_base.cuda(), case.tokens(mbq), case.scale.cuda(), case.ranks.cuda()
    A, B, dY, H = ([t.cuda() for t in ts] for ts in (case.A, case.B, case.dY, case.H))
    ws = mbq.lora_backward_workspace(T, 384, case.Ns, 3, 24, "cuda")
    got = [torch.full_like(dX, 5.0), *(torch.full_like(d, 5.0) for d in dA + dB)]
    want = [d if name in wanted.split() else torch.full_like(d, 5.0)
            for d, name in zip([dX, *dA, *dB], ["dX", "dA", "dA", "dB", "dB"])]
    status = lib.mbq_lora_backward_group(
        X.data_ptr(), T, 384, 2, at(A), at(B), N, 3, 24, ranks.data_ptr(), scale.data_ptr(), *(t.data_ptr() for t in tokens), at(dY),
        at(H) if "dB" in wanted else None, base.data_ptr(), got[0].data_ptr() if "dX" in wanted else None,
        at(got[1:3]) if "dA" in wanted else None, at(got[3:]) if "dB" in wanted else None, ws.data_ptr(), ws.numel(),
        torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert status == 0 and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("T", [20, 300])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_what_is_not_finite_stays_with_its_token_and_adapter(mbq, T, value):
    """One token's activations and one other's gradient: their rows and their adapters' gradients, the rest to the bit."""
    case = Case(T, 256, (136, 33), 4, 20, seed=T)
    case.adapter[3], case.adapter[7] = 1, 2
    H = [torch.empty((T, 20), device="cuda") for _ in range(2)]
    Y, (dX, dA, dB) = case.forward(mbq, H=H), case.backward(mbq)
    case.X[3, 200] = value
    H2 = [torch.empty((T, 20), device="cuda") for _ in range(2)]
    Y2 = case.forward(mbq, H=H2)
    others = torch.arange(T) != 3
    for p in range(2):
        assert torch.equal(Y2[p][others], Y[p][others]) and torch.equal(H2[p][others], H[p][others])
        assert not torch.isfinite(Y2[p][3]).any() and not torch.isfinite(H2[p][3]).any()
    dX2, dA2, dB2 = case.backward(mbq)
    assert torch.equal(dX2, dX) and all(torch.equal(a, b) for a, b in zip(dB2, dB))
    for p in range(2):
        assert torch.equal(dA2[p][[0, 2, 3]], dA[p][[0, 2, 3]]) and not torch.isfinite(dA2[p][1, :, 200]).any()
        keep = torch.arange(256) != 200
        assert torch.equal(dA2[p][1][:, keep], dA[p][1][:, keep])
    case.X[3, 200] = 1.0
    _, dA, _ = case.backward(mbq)
    case.dY[0][7, 5] = value
    dX2, dA2, dB2 = case.backward(mbq)
    others = torch.arange(T) != 7
    assert torch.equal(dX2[others], dX[others]) and not torch.isfinite(dX2[7]).any()
    assert torch.equal(dA2[1], dA[1]) and torch.equal(dB2[1], dB[1])
    assert torch.equal(dA2[0][[0, 1, 3]], dA[0][[0, 1, 3]]) and torch.equal(dB2[0][[0, 1, 3]], dB[0][[0, 1, 3]])
    assert not torch.isfinite(dA2[0][2]).any() and not torch.isfinite(dB2[0][2, :, 5]).any()


def test_no_tokens(mbq):
    case = Case(0, 128, (24,), 2, 8)
    assert case.forward(mbq)[0].shape == (0, 24)
    dX, dA, dB = case.backward(mbq, dA=[torch.full((2, 8, 128), 3.0, device="cuda")], dB=[torch.full((2, 8, 24), 3.0, device="cuda")])
    assert dX.shape == (0, 128) and not torch.count_nonzero(dA[0]) and not torch.count_nonzero(dB[0])


def test_gradients_against_differences(mbq):
    """The gradients of L = sum_p <dY_p, Y_p> along random directions, by central differences of the call itself.  L is bilinear
    in (X, A), (A, B), .. so a central difference is exact but for rounding; steps keep bf16 inputs exact (multiples of 2^-6 in
    small numbers), outputs round to 2^-24 of their size, and the difference of two sums of T N values is good to 1e-4."""
    T, K, Ns, n, r = 70, 128, (40, 24), 3, 8
    gen = torch.Generator().manual_seed(5)
    whole = lambda *s: torch.randint(-8, 9, s, generator=gen).float()  # noqa: E731
    case = Case(T, K, Ns, n, r, seed=1, bare=0.1)
    X, A, B = whole(T, K) / 8, [whole(n, r, K) / 8 for _ in Ns], [whole(n, r, N) / 8 for N in Ns]
    dY = [whole(T, N) / 8 for N in Ns]
    tokens, scale = case.tokens(mbq), case.scale.cuda()
    bf = lambda t: t.to(torch.bfloat16).cuda()  # noqa: E731

    def loss(X, A, B, H=None):
        Y = mbq.mbq_lora_group(bf(X), [bf(a) for a in A], [bf(b) for b in B], tokens, scale, H=H)
        return sum(float((d.double() * y.double().cpu()).sum()) for d, y in zip(dY, Y))

    H = [torch.empty((T, r), device="cuda") for _ in Ns]
    loss(X, A, B, H)
    dX, dA, dB = mbq.mbq_lora_backward_group(bf(X), [bf(a) for a in A], [bf(b) for b in B], tokens, scale,
                                             [d.cuda() for d in dY], H)
    dX, dA, dB = dX.double().cpu(), [d.double().cpu() for d in dA], [d.double().cpu() for d in dB]
    e = 1.0 / 64  # X + e D has at most eight significant bits: |X| <= 1, |D| <= 1
    sign = lambda t: torch.randint(0, 2, t.shape, generator=gen).float() * 2 - 1  # noqa: E731
    D = sign(X)
    slope = (loss(X + e * D, A, B) - loss(X - e * D, A, B)) / (2 * e)
    assert abs(slope - float((dX * D).sum())) <= 1e-4 * float((dX * D).norm()) * 10
    for p in range(2):
        D = sign(A[p])
        up, down = [a.clone() for a in A], [a.clone() for a in A]
        up[p], down[p] = A[p] + e * D, A[p] - e * D
        slope = (loss(X, up, B) - loss(X, down, B)) / (2 * e)
        assert abs(slope - float((dA[p] * D).sum())) <= 1e-4 * float((dA[p] * D).norm()) * 10
        D = sign(B[p])
        up, down = [b.clone() for b in B], [b.clone() for b in B]
        up[p], down[p] = B[p] + e * D, B[p] - e * D
        slope = (loss(X, A, up) - loss(X, A, down)) / (2 * e)
        assert abs(slope - float((dB[p] * D).sum())) <= 1e-4 * float((dB[p] * D).norm()) * 10


@pytest.mark.parametrize("T", [8, 200])
def test_captured_calls_on_another_stream(mbq, T):
    """Forward and backward captured on a side stream and replayed, with eager work and new inputs between the replays."""
    case = Case(T, 512, (136, 72), 4, 16, seed=T)
    on = lambda v: [t.cuda() for t in v]  # noqa: E731
    X, A, B, tokens, scale = case.X.cuda(), on(case.A), on(case.B), case.tokens(mbq), case.scale.cuda()
    base, dY, H = on(case.base), on(case.dY), [torch.empty((T, 16), device="cuda") for _ in case.Ns]
    Y = [torch.empty_like(b) for b in base]
    ws, back = mbq.lora_workspace(T, 512, 2, 16, "cuda"), mbq.lora_backward_workspace(T, 512, case.Ns, 4, 16, "cuda")
    dX, dA, dB = torch.empty((T, 512), device="cuda"), [torch.empty_like(a, dtype=torch.float32) for a in A], [
        torch.empty_like(b, dtype=torch.float32) for b in B]

    def step():
        mbq.mbq_lora_group(X, A, B, tokens, scale, base=base, Y=Y, H=H, ws=ws)
        mbq.mbq_lora_backward_group(X, A, B, tokens, scale, dY, H, dX=dX, dA=dA, dB=dB, ws=back)
        return [*Y, *H, dX, *dA, *dB]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for turn in range(4):
        X.copy_(torch.randn((T, 512), device="cuda").to(torch.bfloat16))
        for d in dY:
            d.normal_()
        want = [v.clone() for v in step()]
        torch.cuda.synchronize()
        for v in out:
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), turn


def test_two_streams_at_once(mbq):
    """Two calls that do not share a workspace, in flight together."""
    cases = [Case(T, 512, (264,), 3, 16, seed=T) for T in (40, 400)]
    want = [c.forward(mbq)[0] for c in cases]
    args = [(c.X.cuda(), [c.A[0].cuda()], [c.B[0].cuda()], c.tokens(mbq), c.scale.cuda()) for c in cases]
    base = [[c.base[0].cuda()] for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for a, b, s in zip(args, base, streams):
            with torch.cuda.stream(s):
                got.append(mbq.mbq_lora_group(*a, base=b)[0])
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 2])


def test_offsets_beyond_32_bits(mbq):
    """An output of more than 2^31 values, and a pool of more than 2^31 values."""
    T, K, N, r = 70000, 128, 32768, 4
    gen = torch.Generator(device="cuda").manual_seed(3)
    X = torch.randn((T, K), generator=gen, device="cuda").to(torch.bfloat16)
    A = (torch.randn((2, r, K), generator=gen, device="cuda") / K ** 0.5).to(torch.bfloat16)
    B = torch.randn((2, r, N), generator=gen, device="cuda").to(torch.bfloat16)
    adapter = (torch.arange(T, device="cuda") % 2).to(torch.int32)
    scale = torch.ones(2, device="cuda")
    Y = mbq.mbq_lora_group(X, [A], [B], (adapter, *mbq.mbq_lora_sort(adapter, 2)), scale)[0]
    for t in (0, 1, 65535, 65536, 69998, 69999):
        h = A[t % 2].double() @ X[t].double()
        size = (A[t % 2].double().abs() @ X[t].double().abs()) @ B[t % 2].double().abs()
        assert ((Y[t].double() - h @ B[t % 2].double()).abs() <= factor(K + r) * size).all(), t
    del Y
    torch.cuda.empty_cache()
    n, r = 4100, 16
    B = torch.zeros((n, r, N), dtype=torch.bfloat16, device="cuda")
    A = torch.zeros((n, r, K), dtype=torch.bfloat16, device="cuda")
    scale = torch.ones(n, device="cuda")
    A[-1].normal_(generator=gen)
    B[-1].normal_(generator=gen)
    for T in (3, 100):
        adapter = torch.full((T,), n - 1, dtype=torch.int32, device="cuda")
        Y = mbq.mbq_lora_group(X[:T], [A], [B], (adapter, *mbq.mbq_lora_sort(adapter, n)), scale)[0]
        h, size = X[:T].double() @ A[-1].double().t(), X[:T].double().abs() @ A[-1].double().abs().t()
        assert ((Y.double() - h @ B[-1].double()).abs() <= factor(K + r) * (size @ B[-1].double().abs())).all()


def test_beside_the_shared_projections(mbq):
    """A stage of a decoder block as it is served: routed linears, then every request's adapter added in place."""
    T, K, Ns, n, r = 24, 512, [256, 128], 6, 16
    case = Case(T, K, Ns, n, r, seed=9, ragged=True)
    gen = torch.Generator().manual_seed(2)
    blobs = [mbq.mbq_encode(0.02 * torch.randn((N, K), generator=gen).cuda()) for N in Ns]
    Wr = [(torch.randn((4, K), generator=gen) / K ** 0.5).cuda() for _ in Ns]
    br = [torch.zeros(4, device="cuda") for _ in Ns]
    X = case.X.cuda()
    routing, Y = mbq.mbq_routed_linear_group(X, Wr, br, blobs, Ns)
    case.base = [y.cpu() for y in Y]
    mbq.mbq_lora_group(X, [a.cuda() for a in case.A], [b.cuda() for b in case.B], case.tokens(mbq), case.scale.cuda(),
                       ranks=case.ranks.cuda(), base=Y, Y=Y)
    case.check_forward(Y)


def test_many_stages_of_a_wavefront(mbq):
    """Enough tiles that a wavefront takes eight and more stages of a row through its part of LDS, the last one not whole."""
    case = Case(3200, 8192, (24,), 2, 16, seed=6)
    H = [torch.full((3200, 16), float("nan"), device="cuda")]
    case.check_forward(case.forward(mbq, H=H), H)
    case = Case(3200, 128, (8200,), 2, 40, seed=7)
    case.check_backward(*case.backward(mbq))


@pytest.mark.parametrize("T,r", [(20, 16), (300, 24), (700, 16), (700, 40), (1300, 64)])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_rows_beyond_a_rank_are_zero_whatever_the_values(mbq, T, r, value):
    """A token of every adapter with values that are not finite, in X and in dY: dA and dB are zero beyond the adapter's rank
    (in the first chunk of its tokens and in later ones), and the columns that such a value does not enter keep their bits."""
    own = [r // 2 - 3, r, 0, 1]
    case = Case(T, 256, (136, 33), 4, r, seed=T + r, assignment=[a % 5 if a % 5 < 4 else -1 for a in range(T)])
    case.ranks, case.own = torch.tensor(own, dtype=torch.int32), own
    _, dA, dB = case.backward(mbq)
    for a in range(4):
        at = case.tokens_of[a]
        case.X[at[0], 200], case.X[at[-1], 7] = value, -value
    keep = torch.ones(256, dtype=torch.bool)
    keep[[7, 200]] = False
    _, dA2, dB2 = case.backward(mbq)
    for p in range(2):
        assert torch.equal(dB2[p], dB[p]) and torch.equal(dA2[p][:, :, keep], dA[p][:, :, keep])
        for a in range(4):
            assert torch.count_nonzero(dA2[p][a, own[a]:]) == 0 and not torch.isfinite(dA2[p][a, :own[a]][:, ~keep]).any()
    case.X[~torch.isfinite(case.X)] = 1.0
    for a in range(4):
        at = case.tokens_of[a]
        for dY in case.dY:
            dY[at[0], 5], dY[at[-1], 30] = value, -value
    _, dA2, dB2 = case.backward(mbq)
    for p, N in enumerate(case.Ns):
        keep = torch.ones(N, dtype=torch.bool)
        keep[[5, 30]] = False
        assert torch.equal(dB2[p][:, :, keep], dB[p][:, :, keep])
        for a in range(4):
            assert torch.count_nonzero(dA2[p][a, own[a]:]) == 0 and torch.count_nonzero(dB2[p][a, own[a]:]) == 0
            assert not torch.isfinite(dB2[p][a, :own[a]][:, ~keep]).any() and not torch.isfinite(dA2[p][a, :own[a]]).any()


@pytest.mark.parametrize("r", [16, 40])
def test_factor_gradients_hold_products_of_all_their_bits(mbq, r):
    """Adapters of one token each, so that dB is one product h dy per value.  Operands are cut into pieces of eight bits, each
    the rest rounded to nearest: the second is at most 2^-8 of the power of two below the operand, the third 2^-17.  The products
    of second and third pieces are left out, 2 x 2^-25 of h dy.  Of the six sums the last is rounded at its full size, to a step
    2^-23 off if the matrix cores truncate, the others at 2^-7 of it and less, 5 x 2^-30: together under 4 x 2^-24."""
    T, N = 96, 264
    gen = torch.Generator().manual_seed(r)
    awkward = torch.tensor([1 + 2.0 ** -7 - 2.0 ** -23, 1 + 2.0 ** -8 - 2.0 ** -23, 1 + 2.0 ** -8 + 2.0 ** -16 - 2.0 ** -23,
                            1 + 2.0 ** -8 - 2.0 ** -16 + 2.0 ** -23, 2 - 2.0 ** -23, 1.0])

    def values(*shape):
        v = torch.where(torch.rand(shape, generator=gen) < 0.5, awkward[torch.randint(0, 6, shape, generator=gen)],
                        1 + torch.rand(shape, generator=gen))
        return v * 2.0 ** torch.randint(-30, 31, shape, generator=gen) * (torch.randint(0, 2, shape, generator=gen) * 2 - 1)

    case = Case(T, 128, (N,), T, r, seed=r, assignment=list(range(T)))
    case.scale[:] = 1.0
    case.H, case.dY = [values(T, r)], [values(T, N)]
    largest = torch.finfo(torch.float32).max  # nothing next to it becomes an infinity
    case.dY[0][:, :3] = torch.tensor([largest, -largest, 2.0 ** 127 * (2 - 2.0 ** -8)])
    case.H[0][::2] = case.H[0][::2].sign() * 2.0 ** -10 * (1 + torch.rand((T // 2, r), generator=gen))
    case.H[0][1::2] = case.H[0][1::2].clamp(-0.99, 0.99)
    _, _, (dB,) = case.backward(mbq)
    want = case.H[0].double()[:, :, None] * case.dY[0].double()[:, None, :]
    off = (dB.double().cpu() - want).abs() / want.abs()
    print(f"[lora] products: worst {float(off.max()) / U:.2f} x 2^-24", flush=True)
    assert (off <= 4 * U).all()


def test_one_workspace_for_calls_of_several_lengths(mbq):
    """Buffers for 2000 tokens serve shorter calls, which stay inside what they ask for themselves."""
    K, Ns, n, r = 2048, [520, 33], 3, 20
    large = (mbq.lora_workspace(2000, K, 2, r, "cuda"), mbq.lora_backward_workspace(2000, K, Ns, n, r, "cuda"))
    for T in (5, 64, 65, 760, 1504, 1505, 2000):
        case = Case(T, K, Ns, n, r, seed=T)
        Y, (dX, dA, dB) = case.forward(mbq, ws=large[0]), case.backward(mbq, ws=large[1])
        own = []
        for need in (mbq.lora_workspace(T, K, 2, r, "cuda").numel(), mbq.lora_backward_workspace(T, K, Ns, n, r, "cuda").numel()):
            own.append(torch.full((need + 512,), 7, dtype=torch.uint8, device="cuda"))
        Y2, (dX2, dA2, dB2) = case.forward(mbq, ws=own[0][:-512]), case.backward(mbq, ws=own[1][:-512])
        assert all((w[-512:] == 7).all() for w in own)
        assert torch.equal(dX, dX2) and all(torch.equal(a, b) for a, b in zip(Y + dA + dB, Y2 + dA2 + dB2))
