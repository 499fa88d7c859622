"""Infinite and NaN values of rows that a token sees, wherever they lie and however small their weight (no softmax weight
of a finite score is zero): the column is infinite, NaN with both signs or a NaN, and every other column and every token
that does not see the row keep their bits."""
import pytest
import torch

from gpu_cases import note
from rows_cases import call, make, shape

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def places(T_prefix, T, N):
    """(store, row) of values to spoil: first, inside a full block, the last that every token sees, the last."""
    rows = {("p", 0), ("p", T_prefix // 2), ("p", T_prefix - 1)} if T_prefix else set()
    if T:
        rows |= {("", 0), ("", T // 2), ("", max(T - N, 0)), ("", T - 1)}
    return sorted(rows)


def spoil(x, at, bad, column):
    store, row = at
    x[store + "v"][..., row, column] = bad


def seen_by(at, T, N):
    """Tokens that see the row."""
    return [i for i in range(N) if at[0] == "p" or at[1] <= T - N + i]


def check(got, clean, tokens, column, bad, what):
    N, hd = got.shape[1], got.shape[-1]
    rest = [c for c in range(hd) if c != column]
    assert torch.equal(got[..., rest], clean[..., rest]), f"{what}: other columns"
    for i in range(N):
        g = got[:, i, :, column]
        if i not in tokens:
            assert torch.equal(g, clean[:, i, :, column]), f"{what}: token {i} does not see it"
        elif bad != bad:
            assert torch.isnan(g).all(), f"{what}: token {i}"
        else:
            assert (g == bad).all(), f"{what}: token {i} has {g.flatten()[:4].tolist()}"


# query heads, KV heads, new tokens: 1, 2, 16, 12 and 16 rows to a key range, then tiles
ROWS = [(2, 2, 1), (4, 2, 1), (32, 2, 1), (6, 2, 4), (8, 2, 4), (6, 2, 40)]
# one slot; joint; two full blocks; several slots of the prefix, the own rows, both
LENGTHS = [(0, 37), (37, 5), (16, 0), (0, 160), (64, 96), (700, 600), (0, 2000), (1500, 0), (0, 16384)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("n_q,n_kv,N", ROWS)
@pytest.mark.parametrize("T_prefix,T", LENGTHS)
def test_seen_values_that_are_not_finite(dtype, hd, n_q, n_kv, N, T_prefix, T):
    if T and T < N:
        T = N
    s = shape(dtype, n_q, n_kv, hd)
    x = make(dtype, n_q, n_kv, hd, 2, N, T_prefix, T, 41)
    clean = call(s, x, T_prefix, T)
    assert torch.isfinite(clean).all()
    for n, at in enumerate(places(T_prefix, T, N)):
        bad, column = (INF, -INF, NAN)[n % 3], (7 * n) % hd
        y = dict(x, v=x["v"].clone(), pv=x["pv"].clone())
        spoil(y, at, bad, column)
        check(call(s, y, T_prefix, T), clean, seen_by(at, T, N), column, bad, f"{at} {bad}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,N", ROWS)
def test_both_signs(dtype, n_q, n_kv, N):
    for T_prefix, T in ((0, 160), (64, 96), (700, 600)):
        s = shape(dtype, n_q, n_kv, 128)
        x = make(dtype, n_q, n_kv, 128, 2, N, T_prefix, T, 43)
        clean = call(s, x, T_prefix, T)
        a, b = places(T_prefix, T - N + 1, 1)[0], places(T_prefix, T - N + 1, 1)[-1]
        spoil(x, a, INF, 5)
        spoil(x, b, -INF, 5)
        check(call(s, x, T_prefix, T), clean, range(N), 5, NAN, "both")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 256])
@pytest.mark.parametrize("n_q,n_kv,N", ROWS)
@pytest.mark.parametrize("T_prefix,T", LENGTHS)
def test_weights_below_the_smallest_number(dtype, hd, n_q, n_kv, N, T_prefix, T):
    # the row's weight is e^(-40 sqrt(hd)) of the others': 0 in 32 bits, yet not zero
    if T and T < N:
        T = N
    s = shape(dtype, n_q, n_kv, hd)
    x = make(dtype, n_q, n_kv, hd, 2, N, T_prefix, T, 45)
    x["q"].fill_(1.0)
    for n, at in enumerate(places(T_prefix, T, N)):
        if at == ("", 0) and not T_prefix and T == N:
            continue  # token 0 sees that row alone: its weight is one
        y = {m: t.clone() for m, t in x.items()}
        y[at[0] + "k"][..., at[1], :] = -40.0
        clean = call(s, y, T_prefix, T)
        assert torch.isfinite(clean).all()
        bad, column = (INF, -INF, NAN)[n % 3], (5 * n + 1) % hd
        spoil(y, at, bad, column)
        check(call(s, y, T_prefix, T), clean, seen_by(at, T, N), column, bad, f"{at} {bad}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("n_q,n_kv,N", ROWS)
@pytest.mark.parametrize("T_prefix,T", LENGTHS)
def test_ranges_below_the_smallest_number(dtype, hd, n_q, n_kv, N, T_prefix, T):
    # so are the weights of every other row up to it: whole waves' and whole slots' states merge with a factor of 0
    T = max(T, N) if T else 0
    s = shape(dtype, n_q, n_kv, hd)
    x = make(dtype, n_q, n_kv, hd, 2, N, T_prefix, T, 49)
    x["q"].fill_(1.0)
    low = T_prefix if T_prefix and T else (T_prefix or T - N + 1) // 2
    if low == 0:
        return  # token 0 sees one row
    at = "p" if T_prefix else ""
    x[at + "k"][..., :low, :] = -40.0
    clean = call(s, x, T_prefix, T)
    assert torch.isfinite(clean).all()
    for n, row in enumerate(sorted({0, low // 2, low - 1})):
        bad, column = (INF, -INF, NAN)[n], (5 * n + 1) % hd
        y = dict(x, v=x["v"].clone(), pv=x["pv"].clone())
        spoil(y, (at, row), bad, column)
        check(call(s, y, T_prefix, T), clean, range(N), column, bad, f"{row} of {low} {bad}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,N", ROWS)
def test_weights_of_such_calls(dtype, n_q, n_kv, N):
    # the weights that rows receive come from q and K alone
    for T_prefix, T in ((0, 160), (64, 96), (700, 600)):
        s = shape(dtype, n_q, n_kv, 64)
        x = make(dtype, n_q, n_kv, 64, 2, N, T_prefix, T, 47)
        w, w2 = x["weight"].clone(), x["weight"].clone()
        call(s, x, T_prefix, T, None, None, w, 0.5)
        for at in places(T_prefix, T, N):
            spoil(x, at, NAN, 3)
        call(s, x, T_prefix, T, None, None, w2, 0.5)
        assert torch.equal(w, w2)
