"""What the calls beside a frozen blob (adapters, balance loss, routers' gradients) refuse: decided on the host, before any
launch, without a GPU."""
import ctypes
import os

import pytest
import torch

import paper_2602_20191_amd as pkg

OK, INVALID, SHAPE, WORKSPACE = 0, 1, 2, 3
F = 0x10000  # an address that is never dereferenced: the calls are refused first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pkg.LIB_PATH):
        import paper_2602_20191_amd.build as b

        b.build()
    return pkg.load()


def pointers(*p):
    return (ctypes.c_void_p * len(p))(*p)


def widths(*n):
    return (ctypes.c_int64 * len(n))(*n)


def test_lora_sort(lib):
    assert lib.mbq_lora_sort(F, -1, 4, F, F, None) == SHAPE
    assert lib.mbq_lora_sort(F, 4, 0, F, F, None) == SHAPE
    assert lib.mbq_lora_sort(F, 4, 65537, F, F, None) == SHAPE
    assert lib.mbq_lora_sort(None, 4, 4, F, F, None) == INVALID
    assert lib.mbq_lora_sort(F, 4, 4, None, F, None) == INVALID
    assert lib.mbq_lora_sort(F, 4, 4, F, None, None) == INVALID
    assert lib.mbq_lora_sort(F + 2, 4, 4, F, F, None) == INVALID


def lora(lib, **change):
    v = dict(X=F, T=4, K=128, n=1, A=pointers(F), B=pointers(F), N=widths(16), adapters=2, r=8, ranks=None, scale=F, adapter=F,
             perm=F, offsets=F, base=None, Y=pointers(F), H=None, ws=F, ws_bytes=0)
    v.update(change)
    return lib.mbq_lora_group(*v.values(), None)


def test_lora_forward(lib):
    assert lora(lib, n=0) == INVALID and lora(lib, n=5) == INVALID
    assert lora(lib, K=100) == SHAPE and lora(lib, K=0) == SHAPE and lora(lib, T=-1) == SHAPE and lora(lib, T=1 << 25) == SHAPE
    assert lora(lib, r=0) == SHAPE and lora(lib, r=257) == SHAPE and lora(lib, adapters=0) == SHAPE
    assert lora(lib, adapters=65537) == SHAPE and lora(lib, N=widths(0)) == SHAPE
    for name in ("X", "A", "B", "N", "scale", "adapter", "perm", "offsets", "Y"):
        assert lora(lib, **{name: None}) == INVALID, name
    for name in ("A", "B", "Y"):
        assert lora(lib, **{name: pointers(None)}) == INVALID, name
    assert lora(lib, H=pointers(None)) == INVALID
    assert lora(lib, X=F + 8) == INVALID and lora(lib, A=pointers(F + 2)) == INVALID and lora(lib, B=pointers(F + 1)) == INVALID
    assert lora(lib, Y=pointers(F + 2)) == INVALID and lora(lib, base=pointers(F + 2)) == INVALID
    need = lib.mbq_lora_workspace_bytes(4, 128, 1, 8)
    assert need > 0
    assert lora(lib, ws_bytes=need - 1) == WORKSPACE and lora(lib, ws=None, ws_bytes=need) == WORKSPACE
    assert lora(lib, ws=F + 16, ws_bytes=need) == WORKSPACE
    assert b"workspace" in lib.mbq_last_error()
    assert lora(lib, T=0, X=None, scale=None, Y=None, ws=None) == OK  # no tokens: nothing to do
    for T, K, n, r in [(-1, 128, 1, 8), (4, 100, 1, 8), (4, 128, 0, 8), (4, 128, 5, 8), (4, 128, 1, 0), (4, 128, 1, 257)]:
        assert lib.mbq_lora_workspace_bytes(T, K, n, r) == 0


def lora_backward(lib, **change):
    v = dict(X=F, T=4, K=128, n=1, A=pointers(F), B=pointers(F), N=widths(16), adapters=2, r=8, ranks=None, scale=F, adapter=F,
             perm=F, offsets=F, dY=pointers(F), H=pointers(F), base=None, dX=F, dA=pointers(F), dB=pointers(F), ws=F, ws_bytes=0)
    v.update(change)
    return lib.mbq_lora_backward_group(*v.values(), None)


def test_lora_backward(lib):
    assert lora_backward(lib, n=5) == INVALID and lora_backward(lib, K=64) == SHAPE and lora_backward(lib, r=300) == SHAPE
    for name in ("X", "A", "B", "N", "scale", "adapter", "perm", "offsets", "dY", "H"):
        assert lora_backward(lib, **{name: None}) == INVALID, name
    for name in ("A", "B", "dY", "H", "dA", "dB"):
        assert lora_backward(lib, **{name: pointers(None)}) == INVALID, name
    assert lora_backward(lib, dX=F + 2) == INVALID and lora_backward(lib, base=F + 1) == INVALID
    assert lora_backward(lib, dA=pointers(F + 2)) == INVALID
    need = lib.mbq_lora_backward_workspace_bytes(4, 128, 1, widths(16), 2, 8)
    assert need > 0
    assert lora_backward(lib, ws_bytes=need - 1) == WORKSPACE
    assert lib.mbq_lora_backward_workspace_bytes(4, 128, 1, widths(0), 2, 8) == 0
    assert lib.mbq_lora_backward_workspace_bytes(4, 128, 1, None, 2, 8) == 0


def test_launches_that_no_grid_holds(lib):
    wide = widths(1 << 24)
    assert lora(lib, T=1 << 20, adapters=65536, N=wide) == SHAPE
    assert lora(lib, T=1 << 20, adapters=65536, N=widths(4096)) == WORKSPACE  # (the widths decide)
    assert lora(lib, T=65, adapters=65536, N=wide) == WORKSPACE  # a tile per token at most
    assert lora_backward(lib, T=64, K=1 << 20, adapters=65536, r=256) == SHAPE
    assert lora_backward(lib, T=64, adapters=65536, N=wide) == SHAPE
    assert lib.mbq_lora_backward_workspace_bytes(64, 128, 1, wide, 65536, 8) == 0
    assert lib.mbq_lora_backward_workspace_bytes(64, 128, 1, widths(4096), 65536, 8) > 0


def balance(lib, **change):
    v = dict(n=1, logits=pointers(F), T=4, P=4, mask=None, target=None, coef=1.0, counts=pointers(F), loss=pointers(F),
             dlogits=pointers(F), ws=F, ws_bytes=0)
    v.update(change)
    return lib.mbq_balance_loss_group(*v.values(), None)


def test_balance_loss(lib):
    assert balance(lib, n=0) == INVALID and balance(lib, n=5) == INVALID
    assert balance(lib, P=0) == SHAPE and balance(lib, P=5) == SHAPE and balance(lib, T=-1) == SHAPE
    for name in ("logits", "counts", "loss"):
        assert balance(lib, **{name: None}) == INVALID and balance(lib, **{name: pointers(None)}) == INVALID, name
    assert balance(lib, dlogits=pointers(None)) == INVALID
    assert balance(lib, logits=pointers(F + 8)) == INVALID and balance(lib, logits=pointers(F + 4), P=3) == INVALID
    for q in (0.0, -0.1, float("nan"), float("inf")):
        assert balance(lib, target=(ctypes.c_double * 4)(0.5, 0.3, q, 0.1)) == INVALID, q
    assert balance(lib, coef=float("nan")) == INVALID and balance(lib, coef=float("inf")) == INVALID
    need = lib.mbq_balance_loss_workspace_bytes(4, 1)
    assert balance(lib, ws_bytes=need - 1) == WORKSPACE and balance(lib, ws=F + 128, ws_bytes=need) == WORKSPACE
    assert lib.mbq_balance_loss_workspace_bytes(4, 5) == 0 and lib.mbq_balance_loss_workspace_bytes(-1, 1) == 0


def route_backward(lib, **change):
    v = dict(X=F, T=4, K=128, n=1, Wr=pointers(F), P=4, dlogits=pointers(F), mask=None, base=None, dX=F, dWr=pointers(F),
             dbr=pointers(F), ws=F, ws_bytes=0)
    v.update(change)
    return lib.mbq_route_backward_group(*v.values(), None)


def test_route_backward(lib):
    assert route_backward(lib, n=0) == INVALID and route_backward(lib, P=5) == SHAPE and route_backward(lib, K=96) == SHAPE
    for name in ("X", "Wr", "dlogits"):
        assert route_backward(lib, **{name: None}) == INVALID, name
    for name in ("Wr", "dlogits", "dWr", "dbr"):
        assert route_backward(lib, **{name: pointers(None)}) == INVALID, name
    assert route_backward(lib, X=F + 2) == INVALID and route_backward(lib, Wr=pointers(F + 4)) == INVALID
    assert route_backward(lib, dX=F + 2) == INVALID
    need = lib.mbq_route_backward_workspace_bytes(4, 128, 1, 4)
    assert route_backward(lib, ws_bytes=need - 1) == WORKSPACE
    assert lib.mbq_route_backward_workspace_bytes(4, 128, 1, 5) == 0


def test_binding_refuses_host_memory_and_wrong_types():
    X = torch.zeros((4, 128), dtype=torch.bfloat16)
    ids = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(pkg.MbqError):
        pkg.mbq_lora_sort(ids, 2)
    with pytest.raises(pkg.MbqError):
        pkg.mbq_lora_group(X, [X[None]], [X[None]], (ids, ids, ids), torch.zeros(1))
    with pytest.raises(pkg.MbqError):
        pkg.mbq_balance_loss_group([torch.zeros((4, 4), dtype=torch.float64)])
    with pytest.raises(pkg.MbqError):
        pkg.mbq_route_backward_group(X, [torch.zeros((4, 128))], [torch.zeros((4, 4))])


@pytest.mark.gpu
def test_binding_refuses_on_the_gpu(mbq):
    X = torch.zeros((4, 128), dtype=torch.bfloat16, device="cuda")
    A = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device="cuda")
    B = torch.zeros((2, 8, 24), dtype=torch.bfloat16, device="cuda")
    ids, offsets = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    tokens, scale = (ids, ids, offsets), torch.ones(2, device="cuda")
    for change in (dict(X=X.float()), dict(A=[A.float()]), dict(B=[B[:, :4]]), dict(tokens=(ids.long(), ids, offsets)),
                   dict(tokens=(ids, ids[:3], offsets)), dict(scale=scale[:1]), dict(A=[A, A]), dict(ranks=scale),
                   dict(base=[torch.zeros((4, 23), device="cuda")]), dict(Y=[torch.zeros((3, 24), device="cuda")]),
                   dict(H=[torch.zeros((4, 7), device="cuda")])):
        v = dict(X=X, A=[A], B=[B], tokens=tokens, scale=scale)
        v.update(change)
        with pytest.raises(AssertionError):
            mbq.mbq_lora_group(**v)
    for change in (dict(base=[torch.zeros((24, 4), device="cuda").t()]), dict(base=[torch.zeros((4, 24))]), dict(scale=scale.cpu()),
                   dict(X=torch.zeros((128, 4), dtype=torch.bfloat16, device="cuda").t())):
        v = dict(X=X, A=[A], B=[B], tokens=tokens, scale=scale)
        v.update(change)
        with pytest.raises(mbq.MbqError):
            mbq.mbq_lora_group(**v)
    S = torch.zeros((4, 4), dtype=torch.float64, device="cuda")
    for bad in (dict(logits=[S.float()]), dict(logits=[S], mask=ids), dict(logits=[S], target=[0.5, 0.5]), dict(logits=[])):
        with pytest.raises(AssertionError):
            mbq.mbq_balance_loss_group(**bad)
    with pytest.raises(mbq.MbqError):
        mbq.mbq_balance_loss_group([S], target=[0.5, 0.5, 0.0, 0.1])
    with pytest.raises(AssertionError):
        mbq.mbq_route_backward_group(X, [torch.zeros((4, 128), device="cuda")], [torch.zeros((4, 3), device="cuda")])


LENGTHS = sorted({*range(0, 700), *range(700, 13000, 16), *range(1, 13000, 31), *(1 << i for i in range(10, 25)), 12256, 12288, 12289})


@pytest.mark.parametrize("K,n,r", [(128, 1, 1), (2048, 1, 16), (4096, 3, 16), (4096, 2, 64), (8192, 3, 16), (2176, 2, 20), (28672, 4, 256)])
def test_a_workspace_serves_shorter_calls(lib, K, n, r):
    """A buffer that is large enough for T tokens is large enough for fewer."""
    N = widths(*[K, 1000, K // 4, 3 * K][:n])
    for of in (lambda T: lib.mbq_lora_workspace_bytes(T, K, n, r),
               lambda T: lib.mbq_lora_backward_workspace_bytes(T, K, n, N, 4, r),
               lambda T: lib.mbq_route_backward_workspace_bytes(T, K, n, 1 + r % 4),
               lambda T: lib.mbq_balance_loss_workspace_bytes(T, n)):
        sizes = [of(T) for T in LENGTHS]
        while not sizes[-1]:  # more than a launch holds
            sizes.pop()
        assert len(sizes) > 900 and all(sizes) and sizes == sorted(sizes)
