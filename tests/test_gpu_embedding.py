"""Embedding lookup with scaling and its gradient by sorted tokens, against
float64.

Tolerances.  u = 2^-24 is float32's unit roundoff, u_t that of the output's
type.  The lookup rounds one product to float32 and once more to the output's
type.  A sum of k float32 terms in any order is off by at most (k - 1) u times
the sum of magnitudes (to first order), the scaling adds one rounding, the
addition to what was there one more, and the store u_t of the result; half the
smallest subnormal of the type bounds what underflows."""
import numpy as np
import pytest
import torch

import paper_2205_11048_amd as gba

pytestmark = pytest.mark.gpu
DEV = "cuda"
U32 = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _matrix(rng, n, D, dtype, pad, sigma=1.0):
    """[n, D] values on the GPU inside a wider tensor whose other columns are NaN, and the same in float64."""
    x = torch.from_numpy(rng.normal(0.0, sigma, (n, D))).to(dtype)
    wide = torch.full((n, D + pad), float("nan"), dtype=dtype)
    wide[:, :D] = x
    return wide.to(DEV)[:, :D], x.double().numpy()


def _out(n, D, dtype, pad):
    wide = torch.full((n, D + pad), float("nan"), dtype=dtype, device=DEV)
    return wide, wide[:, :D]


def _workspace(n, D, R):
    return torch.full((gba.gba_embedding_grad_workspace_size(n, D, R),), 255, dtype=torch.uint8, device=DEV)


def _err():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def _close(got, ref, bound, name):
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (name, int(bad.sum()), got[bad][:3], ref[bad][:3], bound[bad][:3])


# ------------------------------------------------------------------- lookup
@pytest.mark.parametrize("n,D,table_type,out_type,pad", [
    (1, 1, F32, F32, 0), (1, 2048, BF16, BF16, 0), (3, 7, F16, F16, 0), (17, 8, BF16, F32, 0), (64, 32, F32, BF16, 0),
    (65, 33, BF16, BF16, 0), (255, 100, F32, F32, 3), (1000, 257, F16, BF16, 5), (300, 1001, BF16, F16, 7),
    (129, 4096, F32, F16, 0), (37, 8200, BF16, BF16, 0), (5000, 16, F32, F32, 0), (513, 64, BF16, BF16, 1)])
def test_lookup(n, D, table_type, out_type, pad):
    rng = np.random.default_rng(n * 7 + D)
    R = 501
    table, t64 = _matrix(rng, R, D, table_type, pad)
    ids = rng.integers(0, R, n)
    ids[0], ids[-1] = R - 1, 0
    wide, out = _out(n, D, out_type, pad)
    scale = np.float32(np.sqrt(D) * 0.7)
    err = _err()
    gba.gba_embedding_lookup(torch.from_numpy(ids).to(DEV), table, out, scale=float(scale), err=err)
    ref = t64[ids] * float(scale)
    _close(out, ref, (1.01 * U32 + ROUND[out_type]) * np.abs(ref) * 1.01 + TINY[out_type], "lookup")
    assert int(err.item()) == 0
    again = torch.empty_like(out)   # the same from 32-bit IDs
    gba.gba_embedding_lookup(torch.from_numpy(ids.astype(np.int32)).to(DEV), table, again, scale=float(scale), err=err)
    assert torch.equal(again, out) and int(err.item()) == 0
    if pad:
        assert torch.isnan(wide[:, D:]).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_lookup_without_scaling_keeps_the_bits(dtype):
    rng = np.random.default_rng(3)
    table, _ = _matrix(rng, 40, 65, dtype, 0)
    table[3, 5], table[4, 6] = float("inf"), -0.0
    ids = torch.tensor([3, 39, 0, 4, 3], device=DEV)
    _, out = _out(5, 65, dtype, 0)
    gba.gba_embedding_lookup(ids, table, out)
    assert torch.equal(out.view(torch.uint8), table[ids].contiguous().view(torch.uint8))


def test_lookup_of_more_rows_than_a_launch_has_blocks():
    """Just over 2^24 rows of more than a block's columns: 34 GB of output."""
    n, D, R = (1 << 24) + 5, 1032, 11
    table = torch.arange(R, device=DEV, dtype=BF16)[:, None].expand(R, D).contiguous()
    ids = torch.arange(n, device=DEV, dtype=torch.int32) % R
    out = torch.full((n, D), float("nan"), device=DEV, dtype=BF16)
    gba.gba_embedding_lookup(ids, table, out)
    for at in range(0, n, 1 << 20):
        assert bool((out[at:at + (1 << 20)] == ids[at:at + (1 << 20), None]).all()), at


def test_lookup_of_no_tokens_and_bad_ids():
    table = torch.ones((10, 12), device=DEV)
    out = torch.full((4, 12), 5.0, device=DEV)
    err = _err()
    gba.gba_embedding_lookup(torch.zeros(0, dtype=torch.int64, device=DEV), table, out, err=err)
    assert (out == 5.0).all() and int(err.item()) == 0
    ids = torch.tensor([2, -1, 10, 2 ** 40], device=DEV)
    gba.gba_embedding_lookup(ids, table, out, err=err)
    assert int(err.item()) == gba.DERR_ID_RANGE
    assert (out[0] == 1.0).all() and (out[1:] == 0.0).all()


def test_offsets_past_31_bits():
    """A table of more than 2^31 elements: its last rows are looked up, and get a gradient."""
    R, D = 270_000, 8_200
    table = torch.zeros((R, D), dtype=BF16, device=DEV)
    table[-3:] = torch.arange(3, device=DEV, dtype=F32)[:, None] + 1.0
    ids = torch.tensor([R - 1, 5, R - 3, R - 1], device=DEV)
    out = torch.empty((4, D), dtype=BF16, device=DEV)
    gba.gba_embedding_lookup(ids, table, out, scale=2.0)
    assert out.float().mean(1).tolist() == [6.0, 0.0, 2.0, 6.0]
    g = torch.full((4, D), 1.5, dtype=BF16, device=DEV)
    gba.gba_embedding_grad_dense(ids, g, table, _workspace(4, D, R))
    assert (table[-1] == 3.0).all() and (table[-3] == 1.5).all() and (table[5] == 1.5).all()
    assert (table[-2] == 0.0).all() and float(table.float().sum(1).count_nonzero()) == 3.0


# ----------------------------------------------------------------- gradient
def _ids(rng, pattern, n, R, padding):
    if pattern == "same":
        ids = np.full(n, R // 2)
    elif pattern == "distinct":
        ids = rng.permutation(R)[:n]
    elif pattern == "runs":   # IDs that occur 1, 2, 4, ... times
        ids = np.repeat(np.arange(n) * 3, np.minimum(2 ** np.minimum(np.arange(n), 20), n))[:n] % R
        ids = rng.permutation(ids)
    elif pattern == "padding":
        ids = np.full(n, padding)
    else:
        ids = (rng.zipf(1.2, n) * 7919) % R
    ids = ids.astype(np.int64)
    if padding >= 0 and pattern not in ("padding", "same") and padding < R:
        ids[rng.random(n) < 0.15] = padding
    return ids


def _reference(ids, g64, R, padding, scale):
    """G, sum of magnitudes and number of terms per row, in float64."""
    keep = ids != padding
    G, mag = np.zeros((R, g64.shape[1])), np.zeros((R, g64.shape[1]))
    np.add.at(G, ids[keep], g64[keep])
    np.add.at(mag, ids[keep], np.abs(g64[keep]))
    return G * scale, mag * scale, np.bincount(ids[keep], minlength=R)


GRADS = [
    # n, R, D, type, out type, pattern, padding, pad
    (1, 1, 1, F32, F32, "zipf", -1, 0),
    (1, 100, 64, BF16, F32, "zipf", -1, 0),
    (2, 50, 4, F32, F32, "same", -1, 0),
    (63, 64, 3, F16, F16, "zipf", 5, 0),
    (128, 300, 512, BF16, F32, "distinct", -1, 0),
    (129, 129, 520, BF16, BF16, "distinct", 0, 4),
    (1000, 97, 32, F32, F32, "zipf", 96, 0),
    (1024, 4000, 16, BF16, F32, "runs", -1, 0),
    (1025, 4000, 8, BF16, BF16, "runs", 3, 0),
    (3000, 20, 1, F32, F32, "zipf", 7, 2),
    (2999, 5000, 7, BF16, F32, "zipf", 4999, 0),
    (5000, 9, 100, F16, F32, "zipf", -1, 3),
    (5000, 100_000, 257, F32, F32, "zipf", 0, 0),
    (4097, 3, 33, BF16, F32, "same", -1, 0),
    (20_000, 2, 64, F32, F32, "same", -1, 0),
    (40_003, 1_000_000, 20, F32, F32, "runs", 12, 0),
    (700, 700, 1001, F16, BF16, "padding", 3, 7),
    (900, 64, 2048, F32, BF16, "zipf", 1, 0),
    (1500, 30, 4100, BF16, F32, "runs", -1, 0),
    (4095, 2000, 24, F16, F32, "zipf", 0, 1),
    (4096, 70, 40, F32, F32, "runs", -1, 0),
    (4097, 1 << 20, 12, BF16, F32, "distinct", 17, 0),
    (9001, 50, 130, F32, F16, "zipf", 2, 0),
]


def _bound(G, mag, count, out_type, prior=None):
    k = count[:, None].astype(np.float64)
    b = 1.01 * (k + 1.0) * U32 * mag + 1.01 * ROUND[out_type] * np.abs(G) + TINY[out_type]
    if prior is not None:
        b += 1.01 * U32 * np.abs(G)
    return b


@pytest.mark.parametrize("n,R,D,dtype,out_type,pattern,padding,pad", GRADS)
def test_gradient(n, R, D, dtype, out_type, pattern, padding, pad):
    rng = np.random.default_rng(n * 31 + D)
    ids = _ids(rng, pattern, n, R, padding)
    grad, g64 = _matrix(rng, n, D, dtype, pad)
    if padding >= 0:   # what a padding token holds does not matter
        grad[torch.from_numpy(ids == padding).to(DEV)] = float("nan")
    scale = float(np.float32(1.7))
    G, mag, count = _reference(ids, g64, R, padding, scale)
    ids_d, err = torch.from_numpy(ids).to(DEV), _err()

    # one row per distinct ID
    wide, rows = _out(n, D, F32, pad)
    unique = torch.full((n,), -7, dtype=torch.int64, device=DEV)
    num = torch.full((1,), -7, dtype=torch.int64, device=DEV)
    gba.gba_embedding_grad_rows(ids_d, grad, R, unique, rows, num, _workspace(n, D, R), scale=scale,
                                padding_id=padding, err=err)
    want = np.flatnonzero(count)
    U = int(num.item())
    assert U == len(want) and np.array_equal(unique[:U].cpu().numpy(), want)
    _close(rows[:U], G[want], _bound(G[want], mag[want], count[want], F32), "rows")
    assert torch.isnan(rows[U:]).all() and (unique[U:] == -7).all()
    if pad:
        assert torch.isnan(wide[:, D:]).all()

    # the whole table, twice: the same bits
    ws = _workspace(n, D, R)
    tables = []
    for _ in range(2):
        wide, table = _out(R, D, out_type, pad)
        gba.gba_embedding_grad_dense(ids_d, grad, table, ws, scale=scale, padding_id=padding, err=err)
        tables.append(table)
        if pad:
            assert torch.isnan(wide[:, D:]).all()
    _close(tables[0], G, _bound(G, mag, count, out_type), "table")
    assert (tables[0][torch.from_numpy(count == 0).to(DEV)] == 0.0).all()
    assert torch.equal(tables[0], tables[1])

    # added to what is there
    prior, p64 = _matrix(rng, R, D, out_type, pad)
    before = prior.clone()
    gba.gba_embedding_grad_dense(ids_d, grad, prior, ws, scale=scale, padding_id=padding, accumulate=True, err=err)
    ref = G + p64
    _close(prior, ref, _bound(ref, mag, count, out_type, prior=p64), "accumulated")
    idle = torch.from_numpy(count == 0).to(DEV)
    assert torch.equal(prior[idle], before[idle])
    assert int(err.item()) == 0


@pytest.mark.parametrize("n,R,D,dtype,out_type,pattern,padding,pad", [
    (5, 9, 8192, BF16, F32, "zipf", -1, 0), (63, 7, 1800, BF16, F32, "zipf", 3, 2), (64, 64, 600, F16, F32, "distinct", 0, 0),
    (64, 3000, 4096, F32, F32, "zipf", 1, 0), (32, 700, 2048, BF16, F32, "zipf", 1, 0), (33, 70, 1500, BF16, F32, "runs", 6, 0), (17, 30, 4096, F32, BF16, "zipf", 2, 1),
    (64, 50, 200, BF16, F32, "zipf", 2, 0), (40, 50, 250, F16, F16, "same", 3, 3), (31, 400, 8200, BF16, F32, "runs", -1, 0), (65, 40, 2048, BF16, BF16, "zipf", 39, 0), (127, 3, 256, BF16, F32, "same", 1, 0),
    (128, 500, 250, BF16, F32, "runs", 2, 1), (129, 500, 256, F16, F16, "zipf", -1, 0), (255, 11, 12, F32, F32, "zipf", 10, 0),
    (256, 300, 100, BF16, F32, "distinct", -1, 0), (256, 256, 1, F32, F32, "zipf", 0, 0), (257, 60, 31, F32, F32, "zipf", 4, 3), (191, 1 << 16, 64, BF16, F32, "distinct", -1, 0), (254, 5, 8, F16, F32, "zipf", 2, 0),
    (130, 130, 30, F32, F32, "distinct", 129, 0),
    (200, 90, 64, BF16, F32, "padding", 8, 0)])
def test_gradient_of_few_tokens(n, R, D, dtype, out_type, pattern, padding, pad):
    """Sizes at and around those that one launch sorts and adds up."""
    test_gradient(n, R, D, dtype, out_type, pattern, padding, pad)


@pytest.mark.parametrize("n,R,D,dtype,out_type,pattern,padding,pad", [
    (6144, 1 << 18, 9, F32, F32, "zipf", 3, 0), (6145, 1 << 18, 9, F32, F32, "runs", 3, 0),
    (8192, (1 << 18) + 1, 20, BF16, F32, "zipf", 0, 0), (8193, (1 << 18) + 1, 20, BF16, F32, "distinct", 0, 0),
    (8191, 300_000, 33, F16, F16, "runs", -1, 1), (7000, 400, 64, BF16, F32, "same", 2, 0)])
def test_gradient_around_the_counting_sort(n, R, D, dtype, out_type, pattern, padding, pad):
    """Sizes at the limits of the sort in one launch, with run heads counted by a launch of their own."""
    test_gradient(n, R, D, dtype, out_type, pattern, padding, pad)


def test_few_tokens_of_the_largest_ids():
    """Rows up to 2^32 - 1, whose number fills 32 bits."""
    R = 1 << 32
    ids = torch.tensor([R - 1, 5, R - 1, R - 2, 0, R - 1, 5], device=DEV).repeat(27)[:187]
    g = torch.ones((187, 8), device=DEV)
    unique, rows = torch.full((187,), -7, dtype=torch.int64, device=DEV), torch.empty((187, 8), device=DEV)
    num, err = torch.zeros(1, dtype=torch.int64, device=DEV), _err()
    gba.gba_embedding_grad_rows(ids, g, R, unique, rows, num, _workspace(187, 8, R), err=err)
    want, count = torch.unique(ids, return_counts=True)
    assert int(err.item()) == 0 and int(num.item()) == 4
    assert torch.equal(unique[:4], want) and torch.equal(rows[:4], count[:, None].float().expand(4, 8))


def test_few_tokens_outside_the_table_are_reported():
    ids = torch.tensor([1, 50, -2, 1], device=DEV)
    g = torch.ones((4, 8), device=DEV)
    rows, unique = torch.full((6, 8), 5.0, device=DEV), torch.full((6,), -7, dtype=torch.int64, device=DEV)
    num, err = torch.zeros(1, dtype=torch.int64, device=DEV), _err()
    gba.gba_embedding_grad_rows(ids, g, 50, unique, rows, num, _workspace(4, 8, 50), err=err)
    assert int(err.item()) == gba.DERR_ID_RANGE
    assert (rows[4:] == 5.0).all() and (unique[4:] == -7).all()
    table, err = torch.full((50, 8), 2.0, device=DEV), _err()
    gba.gba_embedding_grad_dense(ids, g, table, _workspace(4, 8, 50), accumulate=True, err=err)
    assert int(err.item()) == gba.DERR_ID_RANGE


@pytest.mark.parametrize("n,R,D,out_type,pad", [
    (4100, 376_000, 33, F32, 0), (4097, 640_000, 33, F32, 0), (5003, 1_600_000, 33, F32, 0), (16_384, 2_100_000, 33, F32, 3),
    (16_384, 400_000, 1003, BF16, 0), (16_385, 400_000, 1003, BF16, 0), (3, 5000, 40, F32, 1), (777, 20_000, 250, BF16, 0),
    (64, 1_100_000, 130, F16, 2)])
def test_gradient_of_a_large_table(n, R, D, out_type, pad):
    """The sorts that share their launch with the clear, by the bytes to clear per token; tables around 256 MB."""
    rng = np.random.default_rng(n + R)
    ids = (rng.zipf(1.1, n).astype(np.uint64) * 40_503 % R).astype(np.int64)
    ids[::9] = 4
    ids[1::50] = R - 1
    grad, g64 = _matrix(rng, n, D, BF16, pad)
    unique, place, count = np.unique(ids, return_inverse=True, return_counts=True)
    G, mag, _ = _reference(place, g64, len(unique), -1, 1.0)
    wide, table = _out(R, D, out_type, pad)
    err = _err()
    gba.gba_embedding_grad_dense(torch.from_numpy(ids).to(DEV), grad, table, _workspace(n, D, R), err=err)
    at = torch.from_numpy(unique).to(DEV)
    _close(table[at], G, _bound(G, mag, count, out_type), "touched rows")
    if pad:
        assert torch.isnan(wide[:, D:]).all()
    table[at] = 0.0
    assert int(table.count_nonzero()) == 0 and int(err.item()) == 0


def test_gradient_of_no_tokens():
    ids = torch.zeros(0, dtype=torch.int64, device=DEV)
    g = torch.zeros((0, 12), device=DEV)
    num = torch.full((1,), 9, dtype=torch.int64, device=DEV)
    rows = torch.zeros((0, 12), device=DEV)
    gba.gba_embedding_grad_rows(ids, g, 50, ids, rows, num, _workspace(0, 12, 50))
    assert int(num.item()) == 0
    table = torch.full((50, 12), 3.0, device=DEV)
    gba.gba_embedding_grad_dense(ids, g, table, _workspace(0, 12, 50), accumulate=True)
    assert (table == 3.0).all()
    gba.gba_embedding_grad_dense(ids, g, table, _workspace(0, 12, 50))
    assert (table == 0.0).all()


def test_a_token_outside_the_table_is_reported():
    ids = torch.tensor([1, 50, 2], device=DEV)
    g = torch.ones((3, 8), device=DEV)
    table, err = torch.empty((50, 8), device=DEV), _err()
    gba.gba_embedding_grad_dense(ids, g, table, _workspace(3, 8, 50), err=err)
    assert int(err.item()) == gba.DERR_ID_RANGE


def test_infinite_and_missing_values_stay_in_their_row():
    ids = torch.tensor([4, 1, 4, 2, 0, 4], device=DEV)
    g = torch.ones((6, 40), dtype=BF16, device=DEV)
    g[1], g[3, 7] = float("inf"), float("nan")
    table = torch.empty((6, 40), device=DEV)
    gba.gba_embedding_grad_dense(ids, g, table, _workspace(6, 40, 6))
    assert torch.isinf(table[1]).all() and torch.isnan(table[2, 7]) and int(torch.isnan(table).sum()) == 1
    assert (table[4] == 3.0).all() and (table[0] == 1.0).all() and (table[3] == 0.0).all()


def test_the_gradient_is_the_lookups():
    """Differences of sum(c * lookup) in the table's elements (the sum is linear: a step of 1 is exact to rounding)."""
    rng = np.random.default_rng(11)
    R, D, n, scale = 30, 24, 90, 4.0
    ids = torch.from_numpy(rng.integers(0, R, n)).to(DEV)
    table, _ = _matrix(rng, R, D, F32, 0)
    c = torch.from_numpy(rng.normal(0, 1, (n, D)).astype(np.float32)).to(DEV)
    G = torch.empty((R, D), device=DEV)
    gba.gba_embedding_grad_dense(ids, c, G, _workspace(n, D, R), scale=scale)
    out, moved = torch.empty((n, D), device=DEV), torch.empty((n, D), device=DEV)
    gba.gba_embedding_lookup(ids, table, out, scale=scale)
    for r, k in [(0, 0), (3, 23), (29, 11), (17, 5)]:
        t = table.clone()
        t[r, k] += 1.0
        gba.gba_embedding_lookup(ids, t, moved, scale=scale)
        diff = float(((moved.double() - out.double()) * c.double()).sum())
        terms = float((c.double().abs() * (ids == r)[:, None])[:, k].sum())
        assert abs(diff - float(G[r, k])) <= 100 * U32 * scale * terms + 1e-30


def test_another_stream():
    rng = np.random.default_rng(5)
    ids = torch.from_numpy(rng.integers(0, 60, 700)).to(DEV)
    g = torch.from_numpy(rng.normal(0, 1, (700, 48)).astype(np.float32)).to(DEV)
    a, b = torch.empty((60, 48), device=DEV), torch.empty((60, 48), device=DEV)
    ws = _workspace(700, 48, 60)
    gba.gba_embedding_grad_dense(ids, g, a, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    gba.gba_embedding_grad_dense(ids, g, b, ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, b)


def test_refusals():
    ids = torch.zeros(8, dtype=torch.int64, device=DEV)
    g = torch.zeros((8, 16), device=DEV)
    table = torch.zeros((20, 16), device=DEV)
    ws = _workspace(8, 16, 20)
    num, unique = torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(8, dtype=torch.int64, device=DEV)
    for bad in [lambda: gba.gba_embedding_lookup(ids.short(), table, g), lambda: gba.gba_embedding_lookup(ids, table, g[:7]),
                lambda: gba.gba_embedding_lookup(ids, table, g[:, :8]), lambda: gba.gba_embedding_lookup(ids, table.double(), g),
                lambda: gba.gba_embedding_lookup(ids, table.T, g), lambda: gba.gba_embedding_lookup(ids, table[:0], g),
                lambda: gba.gba_embedding_lookup(ids, table.cpu(), g),
                lambda: gba.gba_embedding_lookup(ids, table[:1].expand(20, 16), g),
                lambda: gba.gba_embedding_grad_dense(ids, g, table, ws[:-1]),
                lambda: gba.gba_embedding_grad_dense(ids, g[:, :15], table, ws),
                lambda: gba.gba_embedding_grad_dense(ids[1:], g[1:], table, ws),   # not 16-byte aligned
                lambda: gba.gba_embedding_grad_rows(ids, g, 20, unique, g.half(), num, ws),
                lambda: gba.gba_embedding_grad_rows(ids, g, 20, unique[:7], g, num, ws),
                lambda: gba.gba_embedding_grad_rows(ids, g, 0, unique, g, num, ws),
                lambda: gba.gba_embedding_grad_workspace_size(-1, 16, 20),
                lambda: gba.gba_embedding_grad_workspace_size(8, 0, 20),
                lambda: gba.gba_embedding_grad_workspace_size(8, 16, (1 << 32) + 1)]:
        with pytest.raises(gba.GBAError):
            bad()
