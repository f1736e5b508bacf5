"""The balance loss (mbq_balance_loss_group) and the routers' gradients (mbq_route_backward_group) against their definition in
64 bits.

Tolerances.  The loss is computed in fp64 throughout and rounded once: a value is off by half a step of fp32, 2^-24 of it, and
a hundred roundings of fp64.  The routers' gradients are fp32 sums; a sum of n terms passes within
(4 sqrt(n) + 16) 2^-24 sum |terms|, its array within (sqrt(n) + 8) 2^-24 of its norm."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def balance_reference(S, coef, mask, target):
    T, P = S.shape
    kept = range(T) if mask is None else [t for t in range(T) if mask[t]]
    counts, sums, rows = [0] * P, [0.0] * P, {}
    for t in kept:
        row = S[t].tolist()
        best = max(range(P), key=lambda e: (row[e], -e))
        counts[best] += 1
        m = max(row)
        w = [math.exp(v - m) for v in row]
        rows[t] = [v / math.fsum(w) for v in w]
        for e in range(P):
            sums[e] += rows[t][e]
    n = len(rows)
    grad = torch.zeros((T, P), dtype=torch.float64)
    if n == 0:
        return counts, 0.0, grad
    u = [counts[e] / n / (1.0 / P if target is None else target[e]) for e in range(P)]
    loss = coef * sum(u[e] * sums[e] / n for e in range(P))
    for t, p in rows.items():
        mean = math.fsum(u[e] * p[e] for e in range(P))
        for e in range(P):
            grad[t, e] = coef / n * p[e] * (u[e] - mean)
    return counts, loss, grad


def check_balance(got, S, coef, mask, target):
    counts, loss, grad = got
    want_counts, want_loss, want_grad = balance_reference(S, coef, mask, target)
    assert counts.tolist() == want_counts
    assert abs(float(loss) - want_loss) <= (U + 1e-13) * abs(want_loss)
    n = max(1, sum(want_counts))
    P = S.shape[1]
    largest = max(want_counts) / n * (P if target is None else 1 / min(target))  # u - mean is exact to 2^-50 of the largest u
    assert ((grad.double().cpu() - want_grad).abs() <= U * want_grad.abs() + abs(coef) / n * largest * 1e-14 + 2 ** -149).all()


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 255, 257, 1000, 4097, 20011])
@pytest.mark.parametrize("P,routers", [(4, 1), (3, 4), (2, 2), (1, 1), (4, 4)])
def test_balance_loss(mbq, T, P, routers):
    gen = torch.Generator().manual_seed(T + P)
    logits = [3.0 * torch.randn((T, P), generator=gen, dtype=torch.float64) for _ in range(routers)]
    mask = None if T % 2 else torch.rand(T, generator=gen) < 0.7
    target = None if routers % 2 else [(e + 1.0) / 7 for e in range(P)]
    got = mbq.mbq_balance_loss_group([S.cuda() for S in logits], 0.02, mask=None if mask is None else mask.cuda(), target=target)
    again = mbq.mbq_balance_loss_group([S.cuda() for S in logits], 0.02, mask=None if mask is None else mask.to(torch.uint8).cuda(),
                                       target=target)
    plain = mbq.mbq_balance_loss_group([S.cuda() for S in logits], 0.02, mask=None if mask is None else mask.cuda(),
                                       target=target, want_grad=False)
    for S, a, b, c in zip(logits, got, again, plain):
        check_balance(a, S, 0.02, mask, target)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1]) and c[2] is None


@pytest.mark.parametrize("T", [70, 9000])
def test_balance_loss_at_the_borders(mbq, T):
    gen = torch.Generator().manual_seed(T)
    S = torch.randint(-2, 3, (T, 4), generator=gen).double()  # many ties
    S[::7, 1] = -math.inf                                      # a precision that is off
    S[3] = torch.tensor([1e300, -1e300, 1e300, 0.0], dtype=torch.float64)  # far apart
    S[5] = torch.finfo(torch.float64).min                      # masks of the lowest value: all equal
    mask = torch.ones(T, dtype=torch.bool)
    mask[[8, 20]] = False
    S[8], S[20] = math.nan, -math.inf                          # masked: not used
    got = mbq.mbq_balance_loss_group([S.cuda()], 1.0, mask=mask.cuda())[0]
    check_balance(got, S, 1.0, mask, None)
    assert torch.count_nonzero(got[2][[8, 20]]) == 0
    assert torch.count_nonzero(got[2][::7, 1]) == 0
    for row in (math.nan, -math.inf, math.inf):                # the same among the tokens kept
        bad = S.clone()
        bad[20] = 0.0
        bad[8] = row
        mask[:] = True
        counts, loss, grad = mbq.mbq_balance_loss_group([bad.cuda()], 1.0, mask=mask.cuda())[0]
        assert math.isnan(float(loss)) and grad[8].isnan().all() and int(counts.sum()) == T
        assert not grad[torch.arange(T) != 8].isnan().any()
    none = mbq.mbq_balance_loss_group([S.cuda()], 1.0, mask=torch.zeros(T, dtype=torch.bool, device="cuda"))[0]
    assert none[0].tolist() == [0] * 4 and float(none[1]) == 0.0 and not torch.count_nonzero(none[2])


def test_balance_loss_without_tokens(mbq):
    counts, loss, grad = mbq.mbq_balance_loss_group([torch.zeros((0, 4), dtype=torch.float64, device="cuda")])[0]
    assert counts.tolist() == [0] * 4 and float(loss) == 0.0 and grad.shape == (0, 4)


def test_balance_gradient_against_differences(mbq):
    """Central differences of the loss with the counts held (the steps move no choice): the loss is rounded to 2^-24 of about 1
    and the step is 1e-2, so a difference is good to 2^-24 / 1e-2 = 6e-6 beside its own 1e-4 / 6 curvature."""
    gen = torch.Generator().manual_seed(11)
    S = torch.randn((6, 4), generator=gen, dtype=torch.float64)
    S[torch.arange(6), torch.argmax(S, 1)] += 0.5
    _, _, grad = mbq.mbq_balance_loss_group([S.cuda()], 1.0, target=[0.4, 0.3, 0.2, 0.1])[0]
    for t in range(6):
        for e in range(4):
            up, down = S.clone(), S.clone()
            up[t, e] += 1e-2
            down[t, e] -= 1e-2
            a, b = [float(mbq.mbq_balance_loss_group([v.cuda()], 1.0, target=[0.4, 0.3, 0.2, 0.1])[0][1]) for v in (up, down)]
            assert abs((a - b) / 2e-2 - float(grad[t, e])) <= 2.5e-5


def close(got, want, size, terms, what):
    got = got.double().cpu()
    off, limit = (got - want).abs(), (4.0 * terms ** 0.5 + 16.0) * U * size
    bad = ~(off <= limit)
    assert not bad.any(), (what, int(bad.sum()), float(off[bad].max()), float(limit[bad].max()))
    if float(want.norm()):
        assert float((got - want).norm()) <= (terms ** 0.5 + 8) * U * float(want.norm()), what


def check_route_backward(got, X, Wr, d, mask, base):
    dX, dWr, dbr = got
    keep = torch.ones(len(X), dtype=torch.bool) if mask is None else mask.bool()
    x = torch.where(keep[:, None], X.double(), 0.0)
    want = torch.zeros_like(x) if base is None else base.double()
    size = want.abs()
    for p in range(len(Wr)):
        g = torch.where(keep[:, None], d[p].double(), 0.0)
        want, size = want + g @ Wr[p].double(), size + g.abs() @ Wr[p].double().abs()
        close(dWr[p], g.t() @ x, g.abs().t() @ x.abs(), len(X), f"dWr[{p}]")
        close(dbr[p], g.sum(0), g.abs().sum(0), len(X), f"dbr[{p}]")
    close(dX, want, size, 4 * len(Wr), "dX")


def router_case(T, K, P, n, seed, masked=True, with_base=True):
    gen = torch.Generator().manual_seed(seed)
    X = torch.randn((T, K), generator=gen).to(torch.bfloat16)
    Wr = [torch.randn((P, K), generator=gen) / K ** 0.5 for _ in range(n)]
    d = [torch.randn((T, P), generator=gen) for _ in range(n)]
    mask = torch.rand(T, generator=gen) < 0.7 if masked else None
    base = torch.randn((T, K), generator=gen) if with_base else None
    return X, Wr, d, mask, base


def call(mbq, X, Wr, d, mask, base, **more):
    on = lambda t: None if t is None else t.cuda()  # noqa: E731
    got = mbq.mbq_route_backward_group(X.cuda(), [w.cuda() for w in Wr], [v.cuda() for v in d], mask=on(mask), base=on(base), **more)
    torch.cuda.synchronize()
    return got


@pytest.mark.parametrize("T,K,P,n", [(1, 128, 4, 1), (2, 256, 3, 4), (17, 128, 1, 1), (64, 1024, 4, 4), (65, 2176, 2, 3),
                                     (333, 2176, 4, 1), (700, 384, 4, 2), (1025, 640, 4, 3), (4100, 256, 3, 2)])
@pytest.mark.parametrize("masked,with_base", [(False, False), (True, True)])
def test_route_backward(mbq, T, K, P, n, masked, with_base):
    case = router_case(T, K, P, n, T + K, masked, with_base)
    got = call(mbq, *case)
    check_route_backward(got, *case)
    again = call(mbq, *case)
    assert torch.equal(got[0], again[0]) and all(torch.equal(a, b) for a, b in zip(got[1] + got[2], again[1] + again[2]))


@pytest.mark.parametrize("T", [40, 600])
def test_masked_tokens_are_not_used(mbq, T):
    X, Wr, d, mask, base = router_case(T, 256, 4, 3, T)
    X[~mask] = float("nan")
    for v in d:
        v[~mask] = float("inf")
    got = call(mbq, X, Wr, d, mask, base)
    check_route_backward(got, X, Wr, d, mask, base)
    assert torch.equal(got[0].cpu()[~mask], base[~mask])
    nothing = call(mbq, X, Wr, d, torch.zeros(T, dtype=torch.bool), None)
    assert not torch.count_nonzero(nothing[0]) and not any(torch.count_nonzero(v) for v in nothing[1] + nothing[2])


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_alignment_in_place_and_neighbours(mbq, shift):
    T, K, P, n = 130, 384, 4, 2
    X, Wr, d, mask, base = router_case(T, K, P, n, shift)

    def moved(t):
        flat = torch.full((t.numel() + 520,), 7.0, dtype=t.dtype, device="cuda")
        out = flat[256 + shift: 256 + shift + t.numel()].view(t.shape)
        out.copy_(t)
        return flat, out

    grad, d_moved = moved(base), [moved(v) for v in d]
    dWr, dbr = [moved(w) for w in Wr], [moved(w[:, 0].contiguous()) for w in Wr]
    got = mbq.mbq_route_backward_group(X.cuda(), [w.cuda() for w in Wr], [v[1] for v in d_moved], mask=mask.cuda(), base=grad[1],
                                       dX=grad[1], dWr=[v[1] for v in dWr], dbr=[v[1] for v in dbr])
    torch.cuda.synchronize()
    check_route_backward(got, X, Wr, d, mask, base)
    for flat, view in [grad, *dWr, *dbr]:
        assert (flat[:256 + shift] == 7).all() and (flat[256 + shift + view.numel():] == 7).all()


def test_route_backward_without_tokens(mbq):
    X, Wr, d, _, _ = router_case(0, 128, 4, 2, 0, False, False)
    dX, dWr, dbr = call(mbq, X, Wr, d, None, None, dWr=[torch.ones((4, 128), device="cuda") for _ in range(2)],
                        dbr=[torch.ones(4, device="cuda") for _ in range(2)])
    assert dX.shape == (0, 128) and not any(torch.count_nonzero(v) for v in dWr + dbr)


def test_route_backward_offsets_beyond_32_bits(mbq):
    T, K = 70000, 32768
    X = torch.ones((T, K), dtype=torch.bfloat16, device="cuda")
    X[T - 1] = 3.0
    Wr = torch.randn((1, K), device="cuda")
    d = torch.zeros((T, 1), device="cuda")
    d[T - 1], d[0] = 0.5, 0.25
    dX, dWr, dbr = mbq.mbq_route_backward_group(X, [Wr], [d])
    assert torch.equal(dX[T - 1], 0.5 * Wr[0]) and torch.equal(dX[0], 0.25 * Wr[0])
    assert not torch.count_nonzero(dX[1000]) and not torch.count_nonzero(dX[T - 2])
    assert torch.equal(dWr[0], torch.full_like(Wr, 1.75)) and float(dbr[0]) == 0.75


def test_a_training_step_of_the_routers(mbq):
    """Route, loss, gradients, the activations' gradient joined with the adapters': as a program runs them; captured and
    replayed with new activations, each replay against the eager step."""
    T, K, n, r, N = 300, 512, 2, 8, 136
    gen = torch.Generator().manual_seed(4)
    X = torch.randn((T, K), generator=gen).to(torch.bfloat16).cuda()
    Wr, br = (torch.randn((4, K), generator=gen) / K ** 0.5).cuda(), torch.zeros(4, device="cuda")
    A = (torch.randn((n, r, K), generator=gen) / K ** 0.5).to(torch.bfloat16).cuda()
    B = torch.randn((n, r, N), generator=gen).to(torch.bfloat16).cuda()
    adapter = (torch.arange(T) // 130 - 1).to(torch.int32).cuda()  # none, 0, 1
    tokens, scale = (adapter, *mbq.mbq_lora_sort(adapter, n)), torch.ones(n, device="cuda")
    mask = (torch.arange(T) % 50 < 40).cuda()
    dY = [torch.randn((T, N), generator=gen).cuda()]
    ws = [mbq.route_workspace(T, K, "cuda"), mbq.lora_workspace(T, K, 1, r, "cuda"),
          mbq.lora_backward_workspace(T, K, [N], n, r, "cuda"), mbq.balance_loss_workspace(T, 1, "cuda"),
          mbq.route_backward_workspace(T, K, 1, 4, "cuda")]

    def step():
        prec, perm, offsets, logits = mbq.mbq_route(X, Wr, br, want_logits=True, ws=ws[0])
        H = [torch.empty((T, r), device="cuda")]
        Y = mbq.mbq_lora_group(X, [A], [B], tokens, scale, H=H, ws=ws[1])
        counts, loss, d = mbq.mbq_balance_loss_group([logits], 0.1, mask=mask, target=[0.4, 0.3, 0.2, 0.1], ws=ws[3])[0]
        dX, dA, dB = mbq.mbq_lora_backward_group(X, [A], [B], tokens, scale, dY, H, ws=ws[2])
        adapters = dX.clone()
        dX, dWr, dbr = mbq.mbq_route_backward_group(X, [Wr], [d], mask=mask, base=dX, dX=dX, ws=ws[4])
        return [prec, logits, counts, loss, d, Y[0], adapters, dX, dA[0], dB[0], dWr[0], dbr[0]]

    prec, logits, counts, loss, d, Y, adapters, dX, dA, dB, dWr, dbr = step()
    assert counts.tolist() == torch.bincount(prec[mask].cpu().long(), minlength=4).tolist()
    check_balance((counts, loss, d), logits.cpu(), 0.1, mask.cpu(), [0.4, 0.3, 0.2, 0.1])
    check_route_backward((dX, [dWr], [dbr]), X.cpu(), [Wr.cpu()], [d.cpu()], mask.cpu(), adapters.cpu())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for turn in range(4):
        X.copy_(torch.randn((T, K), device="cuda").to(torch.bfloat16))
        want = [v.clone() for v in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), turn
