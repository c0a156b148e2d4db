"""GPU parity of the serving operators against the 64-bit reference (oracle/sol_cache_oracle.py).

Tolerances count roundings.  A bf16 value is off by at most 2^-8 of itself, an f32 value by 2^-24.  The other terms are
stated at each check.
"""
import math

import numpy as np
import pytest
import torch

from oracle import sol_cache_oracle as ora
from paper_2607_24027_amd import binding as sb
from paper_2607_24027_amd import cache as sc

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    sc.lib()
    return torch.device("cuda:0")


def i32(x, dev):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=dev)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def placed(x, how, dev):
    """x [..., d] on the GPU as a view of that kind: 'plain', 'tokens' (the last two leading dimensions exchanged in memory),
    'odd' (rows that start anywhere)."""
    x = x.to(dev)
    if how == "tokens":
        return x.transpose(-3, -2).contiguous().transpose(-3, -2)
    if how == "odd":
        big = torch.zeros(*x.shape[:-1], x.shape[-1] + 3, dtype=x.dtype, device=dev)
        big[..., 1:-2] = x
        return big[..., 1:-2]
    return x.contiguous()


# ------------------------------------------------------------------------------------------------ norm and rotation
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,pairs,how,B,N,Hq,Hk", [
    (128, 128, False, "plain", 1, 1, 1, 1), (128, 128, True, "tokens", 2, 37, 5, 3), (128, 0, False, "tokens", 1, 16, 2, 2),
    (128, 64, False, "odd", 1, 19, 3, 1), (128, 24, True, "plain", 1, 33, 2, 7), (128, 8, False, "tokens", 3, 5, 4, 0),
    (64, 64, False, "tokens", 1, 70, 9, 2), (64, 64, True, "odd", 1, 8, 2, 2), (64, 32, False, "plain", 2, 129, 1, 4),
    (64, 40, True, "tokens", 1, 65, 0, 3), (128, 128, False, "tokens", 1, 700, 40, 8),
])
def test_qk_norm_rope(dev, dtype, d, rot, pairs, how, B, N, Hq, Hk):
    g = torch.Generator().manual_seed(d + rot + N)
    P = 50
    xs = [torch.randn(B, H, N, d, generator=g).mul(torch.exp2(torch.randint(-6, 7, (B, H, N, 1), generator=g))).to(DT[dtype])
          if H else None for H in (Hq, Hk)]
    for x in xs:
        if x is not None:
            x[0, 0, 0] = 0.0                                     # a row without a length
    ws = [torch.randn(d, generator=g).to(DT[dtype]) if x is not None else None for x in xs]
    if how == "plain":
        ws[1] = None
    cos = sin = None
    if rot:
        angle = torch.rand(P, rot // 2, generator=g, dtype=torch.float64) * 7
        cos, sin = angle.cos().float(), angle.sin().float()
    positions = torch.randint(0, P, (B, N), generator=g, dtype=torch.int32)
    positions[torch.rand(B, N, generator=g) < 0.2] = -1
    positions[-1, -1] = P if rot else -5                         # not a row of the tables
    gpu = [None if x is None else placed(x, how, dev) for x in xs]
    outs = [None if x is None else placed(torch.full(x.shape, 7.0, dtype=x.dtype), how, dev) for x in xs]
    got = sc.qk_norm_rope(gpu[0], gpu[1], *(None if w is None else w.to(dev) for w in ws), None if cos is None else cos.to(dev),
                          None if sin is None else sin.to(dev), positions.to(dev), eps=1e-5, interleaved=pairs, q_out=outs[0],
                          k_out=outs[1])
    for x, w, y in zip(xs, ws, got):
        if x is None:
            assert y is None
            continue
        ref, written = ora.norm_rope(f64(x), None if w is None else f64(w), None if cos is None else cos.numpy(),
                                     None if sin is None else sin.numpy(), positions.numpy(), 1e-5, pairs)
        y = f64(y)
        mask = np.broadcast_to(written[:, None, :, None], y.shape)
        assert (y[~mask] == 7.0).all()
        # f32: the sum of squares is off by at most 8 + 6 roundings, half of that in its root, then root, quotient, two factors
        # (2 + 3 + 2) and two products and a sum of the pair: below 24 roundings of the pair's length.
        length = np.abs(ref)
        half = rot // 2
        if half:
            ia = np.arange(half) * 2 if pairs else np.arange(half)
            ib = ia + 1 if pairs else ia + half
            length[..., ia] = length[..., ib] = np.hypot(ref[..., ia], ref[..., ib])
        tol = HALF_STEP[dtype] * np.abs(ref) * (1 + 2.0 ** -7) + 24 * 2.0 ** -24 * length
        assert (np.abs(y - ref)[mask] <= tol[mask]).all()


def test_qk_norm_rope_far_strides_and_defaults(dev):
    # offsets past 2^31 elements in a strided view; default outputs and positions
    big = torch.zeros(1, 3, 1 << 23, 128, dtype=torch.bfloat16, device=dev)      # 6.4 GB
    g = torch.Generator().manual_seed(3)
    part = torch.randn(1, 3, 5, 128, generator=g).bfloat16()
    q = big[:, :, -5:]
    q.copy_(part.to(dev))
    angle = torch.rand(5, 64, generator=g, dtype=torch.float64)
    y, none = sc.qk_norm_rope(q, None, cos=angle.cos().float().to(dev), sin=angle.sin().float().to(dev))
    assert none is None and y.is_contiguous()
    ref, _ = ora.norm_rope(f64(part), None, angle.cos().float().numpy(), angle.sin().float().numpy(), np.arange(5)[None], 1e-6, False)
    assert (np.abs(f64(y) - ref) <= 2.0 ** -8 * np.abs(ref) * 1.01 + 2.0 ** -18).all()


# ------------------------------------------------------------------------------------------------------ page tables
def run_tables(dev, lens, add, table, ring, state, rows):
    t, r = i32(table, dev), i32(ring, dev)
    new = sc.tables(i32(lens, dev), i32(add, dev), t, r, i32(state, dev), rows)
    return [x.cpu().numpy() for x in (new.row_start, new.slots, new.positions, new.lens, new.state, t, r)]


@pytest.mark.parametrize("seed", range(24))
def test_tables_random_steps(dev, seed):
    rng = np.random.default_rng(seed)
    S = int(rng.choice([1, 2, 63, 64, 65, 300, 1025, 4096]) if seed < 16 else rng.integers(1, 40))
    MP = int(rng.integers(1, 30))
    lens = rng.integers(0, MP * 64 + 1, S)
    if seed % 3 == 0:
        lens[rng.random(S) < 0.5] //= 64
        lens[rng.random(S) < 0.3] = 0
    held = -(-lens // 64)
    P = int(held.sum() + rng.integers(1, 2 * S + 5))
    pages = rng.permutation(P)
    table = np.full((S, MP), -1)
    table[np.arange(MP)[None] < held[:, None]] = pages[:held.sum()]
    head = int(rng.integers(0, P))
    ring = np.full(P, -1)
    free = P - held.sum()
    ring[(head + np.arange(free)) % P] = pages[held.sum():]
    state = np.array([head, free])
    table[rng.random(table.shape) < 0.02] = -1                   # pages that were dropped
    for step in range(3):
        add = rng.integers(-100, 150, S)
        add[rng.random(S) < 0.2] = 0
        add[rng.random(S) < 0.1] = -(1 << 30)
        add[rng.random(S) < 0.02] = 1 << 30 if step == 2 else 64 * 31
        rows = min(int(np.maximum(add, 0).astype(np.int64).sum()), 300000) + int(rng.integers(0, 50))
        got = run_tables(dev, lens, add, table, ring, state, rows)
        if np.maximum(add, 0).sum() > 300000:                    # the plain form goes row by row
            add = np.minimum(add, 64 * 31)
            got = run_tables(dev, lens, add, table, ring, state, rows)
        want = ora.tables(lens, add, table, ring, state, rows)
        for name, x, y in zip(("row_start", "slots", "positions", "lens", "state", "table", "ring"), got, want):
            assert np.array_equal(x, y), (name, step)
        lens, state, table, ring = want[3], want[4], want[5], want[6]


def test_tables_more_rows_than_an_int_counts(dev):
    # refused requests keep their rows: the sums stop at the largest int
    add = [1 << 30] * 5 + [3]
    got = run_tables(dev, [0] * 6, add, np.full((6, 2), -1), np.arange(4), [0, 4], 10)
    assert got[0].tolist() == [0, 1 << 30] + [(1 << 31) - 1] * 5
    assert (got[1] == -1).all() and got[3].tolist() == [0] * 5 + [3] and got[5][5, 0] == 0


def test_tables_bad_values_stay_in_bounds(dev):
    got = run_tables(dev, [-5, 1 << 30, 100], [70, -3, 5], [[9, 99], [7, -7], [1 << 30, 2]], [3, 1 << 30, -9, 2], [-3, 1 << 30], 80)
    want = ora.tables([-5, 1 << 30, 100], [70, -3, 5], np.array([[9, 99], [7, -7], [1 << 30, 2]]), np.array([3, 1 << 30, -9, 2]),
                      [-3, 1 << 30], 80)
    for x, y in zip(got, want):
        assert np.array_equal(x, y)


def test_tables_give_the_same_step_again(dev):
    lens, add = i32([100, 64, 0], dev), i32([40, -64, 10], dev)
    table, ring, state = i32([[0, 1, -1], [2, -1, -1], [-1, -1, -1]], dev), i32([3, 4, 5, -1, -1, -1], dev), i32([0, 3], dev)
    a = sc.tables(lens, add, table, ring, state, 50)
    keep = [x.clone() for x in (*a, table, ring)]
    b = sc.tables(lens, add, table, ring, state, 50, out=a)
    assert b is a and all(torch.equal(x, y) for x, y in zip((*b, table, ring), keep))
    last = sc.tables(lens, -lens, table, ring, state, 0)         # no rows at all
    assert last.slots.numel() == 0 and last.lens.tolist() == [0, 0, 0]


# -------------------------------------------------------------------------------------------------- append and read
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,T,how", [(128, 1, 1, "plain"), (128, 3, 200, "tokens"), (128, 8, 48, "odd"), (64, 1, 1, "odd"), (64, 5, 131, "tokens"),
                                       (64, 2, 64, "plain")])
def test_append_and_read(dev, dtype, d, H, T, how):
    rng = np.random.default_rng(d + T)
    P = -(-T // 64) + 2
    k = rng.standard_normal((H, T, d)) * np.exp2(rng.integers(-12, 12, (H, T, 1)))
    v = rng.standard_normal((H, T, d)) * np.exp2(rng.integers(-12, 12, (H, T, 1)))
    k[0, 0, :32] = 0.0
    v[-1, -1, :32] = np.resize([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -5], 32)        # ties
    k[0, -1, -32:] = 7.0
    k, v = (torch.tensor(x).to(DT[dtype]) for x in (k, v))
    if T > 8:
        k[0, 3, :32], v[0, 3, :32] = 3e38, 1e5                   # past what a value's scale may be
        k[0, 4, :32], v[0, 4, :32] = 1e-38, 1e-38
        k[0, 5, 1], v[0, 6, 2] = 2e-20, 2.0 ** -25
    slots = rng.permutation(P * 64)[:T].astype(np.int32)
    if how == "tokens":
        slots = (np.arange(T) + 37).astype(np.int32)
    skip = rng.random(T) < 0.1
    skip[0] = False
    slots[skip] = rng.choice([-1, -(1 << 31), P * 64, (1 << 31) - 1], skip.sum())
    before = torch.randint(0, 256, (P, H, 68 * d), dtype=torch.uint8, generator=torch.Generator().manual_seed(1))
    store = before.to(dev)
    sc.append(placed(k, how, dev), placed(v, how, dev), store, i32(slots, dev))
    want = before.numpy().copy()
    (kc, ke), (vc, ve) = ora.quantise(f64(k), ora.K_SCALES), ora.quantise(f64(v), ora.V_SCALES)
    for t in range(T):
        if not skip[t]:
            for h in range(H):
                ora.write_page_token(want[slots[t] // 64, h], int(slots[t] % 64), d, (kc[h, t], ke[h, t]), (vc[h, t], ve[h, t]))
    assert np.array_equal(store.cpu().numpy(), want)             # every byte, those of other tokens too
    rk, rv = ora.values(kc, ke), ora.values(vc, ve)
    rk[:, skip] = rv[:, skip] = 0.0
    for dt in ("bf16", "f32"):
        gk, gv = sc.read(store, i32(slots, dev), dtype=DT[dt])
        assert np.array_equal(f64(gk), rk) and np.array_equal(f64(gv), rv)
    out = placed(torch.full((H, T, d), 5.0), how, dev)
    nothing, only = sc.read(store, i32(slots, dev), v_out=out)
    assert nothing is None and only is out and np.array_equal(f64(out), rv)


@pytest.mark.parametrize("d", [64, 128])
def test_tokens_that_are_not_finite(dev, d):
    k, v = torch.randn(2, 6, d), torch.randn(2, 6, d)
    k[0, 1, 5], v[1, 2, d - 1], k[1, 3, 0], v[0, 4, 40] = math.nan, math.inf, -math.inf, math.nan
    store = sc.empty(1, 2, d, dev)
    slots = i32([9, 63, 0, 17, 40, 41], dev)
    sc.append(k.to(dev), v.to(dev), store, slots)
    gk, gv = (f64(x) for x in sc.read(store, slots, dtype=torch.float32))
    bad = np.zeros((2, 6), bool)
    bad[0, 1] = bad[1, 2] = bad[1, 3] = bad[0, 4] = True
    assert np.isnan(gk[bad]).all() and np.isnan(gv[bad]).all()
    assert np.isfinite(gk[~bad]).all() and np.isfinite(gv[~bad]).all()


# ----------------------------------------------------------------------------------------------------- attention
def make_store(rng, P, H, d, dev, fill=None):
    """A store whose tokens were appended, and its values [H, P * 64, d]."""
    k = torch.tensor(rng.standard_normal((H, P * 64, d)) * np.exp(0.4 * rng.standard_normal((H, 1, d))), dtype=torch.float32)
    v = torch.tensor(rng.standard_normal((H, P * 64, d)) + 0.5 * rng.standard_normal((H, 1, d)), dtype=torch.float32)
    store = sc.empty(P, H, d, dev)
    if fill is not None:
        store.fill_(fill)
    slots = torch.arange(P * 64, dtype=torch.int32, device=dev)
    sc.append(k.to(dev), v.to(dev), store, slots)
    return store, ora.values(*ora.quantise(k.numpy().astype(np.float64), ora.K_SCALES)), \
        ora.values(*ora.quantise(v.numpy().astype(np.float64), ora.V_SCALES))


def tolerance(dtype, q, k, v, out, spread, reach):
    """Bound of the error of one row of outputs.  With ds the error of a logit, a probability is off by 2 ds of itself at most
    (ds is small), and an output by that times sum p |v - out|: weights that all change alike leave it as it is.

    ds: q log2(e) / sqrt(d) is split into 6-bit floats.  With 32 channels scaled so that the largest magnitude lies in (3.75, 7.5],
    what a term leaves is at most half its step of 1/4 for magnitudes up to 4, and the next term is taken of 16 times that: three
    terms (bf16) leave 2^-3 / 16^2, six (f32) 2^-3 / 16^5, and the factor two roundings.  Sums of d products in f32, 2^-24 a
    term, on sum |q k|; the accumulator starts at a number below |s| + 16, four roundings of that.  Probabilities are rounded to
    f16, half a step of 2^-11, or in two terms 2^-22 (f32), and their sum is taken before: an error on sum p |v|.  They are held as
    2^7 p / p_max at least, and f16 has no steps below 2^-24: none is exact to more than 2^-32, half of that step, of the row's
    sum, an error on sum |v|.  Sums of probabilities times values: f32, at most one rounding for 16 keys and 64
    more for shares and their join, on sum p |v|.  The result: one rounding of its type, and a quotient."""
    d, L = q.shape[0], k.shape[0]
    top = np.repeat(np.abs(q).reshape(-1, 32).max(1), 32)
    lost = top * (2.0 ** -11 if dtype == "bf16" else 2.0 ** -23) / 3.75 + 2 * 2.0 ** -24 * np.abs(q)
    s = np.abs(k) @ np.abs(q) / math.sqrt(d)
    ds = (np.abs(k) @ lost) / math.sqrt(d) + d * 2.0 ** -24 * s + 4 * 2.0 ** -24 * (s + 16)
    cut = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
    return (HALF_STEP[dtype] * 1.01 + 2.0 ** -23) * np.abs(out) + 2 * ds.max() * spread + cut * reach + 2.0 ** -32 * np.abs(v).sum(0) \
        + (L / 16 + 64) * 2.0 ** -24 * reach


def check_forward(dev, dtype, d, Hq, Hk, lens, rows, granule, how="tokens", seed=0, positions=None, drop=(), max_rows=None, extra=0,
                  fill=255, wide=0):
    """One call against the reference; lens: with the new rows."""
    rng = np.random.default_rng(seed)
    S = len(lens)
    held = [-(-n // 64) for n in lens]
    P = sum(held) + 2
    store, k, v = make_store(rng, P, Hk, d, dev)
    pages = rng.permutation(P)
    MP = max(held + [1]) + 1 + wide
    table = rng.integers(-1, 2 * P, (S, MP))                     # what lies behind a request's pages is never read
    at = 0
    raw = store.cpu().numpy()
    for s in range(S):
        table[s, :held[s]] = pages[at:at + held[s]]
        at += held[s]
    keep = np.zeros((P, 64), bool)
    for s in range(S):
        for t in range(lens[s]):
            keep[table[s, t // 64], t % 64] = True
    # bytes of tokens that are in no request are the worst there are
    for p in range(P):
        if not keep[p].any():
            raw[p] = fill
        elif not keep[p].all():
            n = int(keep[p].sum())
            for h in range(Hk):
                for t in range(n, 64):
                    w = d // 64
                    raw[p, h, t * (d // 2):(t + 1) * (d // 2)] = fill
                    t2 = (t & 0b10011) | (((t >> 2) & 1) << 3) | (((t >> 3) & 1) << 2)
                    for g in range(d // 32):
                        raw[p, h, 32 * d + (((g % 2) * 32 + t2 % 32) * w + g // 2) * 2 + t // 32] = fill
                        raw[p, h, 66 * d + ((t // 8) * (d // 32) + g) * 8 + t % 8] = fill
    store = torch.tensor(raw, device=dev)
    for s, p, bad in drop:
        table[s, p] = bad
    T = sum(rows) + extra
    q = torch.tensor(rng.standard_normal((Hq, T, d)), dtype=torch.float32).to(DT[dtype])
    if positions is None:
        positions = np.concatenate([np.arange(n - r, n) for n, r in zip(lens, rows)] + [np.full(extra, 3)]) if T else np.zeros(0)
    row_start = np.concatenate([[0], np.cumsum(rows)])
    out = placed(torch.full((Hq, T, d), 9.0, dtype=DT[dtype]), how, dev)
    args = (placed(q, how, dev), store, i32(table, dev), i32(lens, dev), i32(row_start, dev), i32(positions, dev))
    got = sc.forward(*args, causal_granule=granule, max_rows=max_rows, out=out)
    assert got is out
    y, qn = f64(out), f64(q)
    assert (y[:, sum(rows):] == 9.0).all()
    G = Hq // Hk
    worst = 0.0
    for s in range(S):
        n = lens[s]
        ok = np.array([0 <= table[s, t // 64] < P for t in range(n)], bool)
        slots = np.array([table[s, t // 64] * 64 + t % 64 if ok[t] else 0 for t in range(n)], int)
        r0, r1 = row_start[s], row_start[s + 1]
        if max_rows is not None:
            r1 = min(r1, r0 + max_rows)
        if r1 == r0:
            continue
        pos = positions[r0:r1]
        limit = np.where(pos < 0, 0, np.minimum((pos // granule + 1) * granule, n))
        sees = (np.arange(n)[None] < limit[:, None]) & ok[None]
        for h in range(Hq):
            kk, vv = k[h // G][slots], v[h // G][slots]
            ref, spread, reach = ora.attend(qn[h, r0:r1], kk, vv, sees)
            for r in range(r1 - r0):
                tol = tolerance(dtype, qn[h, r0 + r], kk if n else np.zeros((1, d)), vv, ref[r], spread[r], reach[r])
                err = np.abs(y[h, r0 + r] - ref[r])
                assert (err <= tol).all(), (s, h, r, float((err / np.maximum(tol, 1e-300)).max()))
                worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
    # the same call again gives the same bits
    again = sc.forward(*args, causal_granule=granule, max_rows=max_rows, out=torch.full_like(out, 9.0))
    assert torch.equal(again, out)
    return worst


FORWARD = [
    # d, Hq, Hk, lens, rows, granule, layout
    (128, 1, 1, [1], [1], 1, "plain"),
    (128, 8, 2, [64], [1], 1, "tokens"),
    (64, 6, 2, [65, 1, 300], [1, 1, 1], 1, "odd"),
    (128, 4, 1, [1000], [1], 1, "tokens"),
    (64, 3, 3, [700, 63, 128], [5, 63, 1], 1, "tokens"),
    (128, 10, 2, [200, 77], [40, 77], 1, "plain"),
    (128, 2, 2, [333], [150], 37, "odd"),
    (64, 4, 4, [500], [260], 100, "tokens"),
    (128, 3, 1, [400, 90], [200, 30], 1 << 30, "tokens"),
    (64, 8, 1, [2000], [9], 1, "plain"),
    (128, 33, 1, [130], [2], 1, "tokens"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,Hq,Hk,lens,rows,granule,how", FORWARD)
def test_forward(dev, dtype, d, Hq, Hk, lens, rows, granule, how):
    check_forward(dev, dtype, d, Hq, Hk, lens, rows, granule, how, seed=d + sum(lens))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("wide", [0, 4000])
def test_forward_few_and_many_rows(dev, dtype, d, wide):
    # requests of both kernels in one call; a table with room for long sequences gives each kernel its own launch
    check_forward(dev, dtype, d, 8, 2, [700, 64, 333, 1500, 65, 200], [1, 2, 150, 90, 12, 1], 1, "tokens", seed=d, wide=wide)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("wide", [0, 6, 60])
def test_forward_short_prefills(dev, dtype, wide):
    # many rows, not cut: by few rows' kernel, by the table's width, by the tiles; 2,049 rows of 8 heads are too many for the first
    rows = [256, 255, 256, 1, 256, 256, 256, 256, 257] if wide == 6 else [100, 300, 1, 200]
    check_forward(dev, dtype, 64, 8 if wide == 6 else 4, 2, [n + 20 for n in rows], rows, 1, "tokens", seed=wide, wide=wide)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("S", [40, 200])
@pytest.mark.parametrize("wide", [0, 100])
def test_forward_short_requests(dev, dtype, d, S, wide):
    # tiles that are not cut: a workgroup's (40 requests) or a wave's (200), by the table's width or by the lengths
    rng = np.random.default_rng(S + d)
    lens = [int(n) for n in rng.integers(0, 400, S)]
    rows = [int(min(n, r)) for n, r in zip(lens, rng.integers(0, 3, S))]
    check_forward(dev, dtype, d, 8, 8, lens, rows, 1, "tokens", seed=S, wide=wide, max_rows=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fill", [0, 127, 254, 255])
def test_forward_empty_requests_and_rows(dev, dtype, fill):
    # no tokens, no rows, rows that see nothing, rows behind the last request, whatever lies behind the lengths
    positions = np.array([-1, 0, 5, 89, -1, 2, 3, 3])
    check_forward(dev, dtype, 128, 4, 2, [90, 0, 70, 0, 4], [4, 2, 0, 0, 1], 1, positions=positions, extra=1, fill=fill, seed=fill)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 150])
def test_forward_dropped_pages(dev, dtype, rows):
    drop = [(0, 0, -1), (0, 3, 1 << 30), (0, 4, -(1 << 31)), (1, 0, -1), (1, 1, -1), (1, 2, -1)]
    check_forward(dev, dtype, 64, 4, 2, [600, 160], [rows, 1], 1, drop=drop, seed=rows)


@pytest.mark.parametrize("rows", [[3, 200], [1, 40]])
def test_forward_max_rows_leaves_the_rest(dev, rows):
    rng = np.random.default_rng(5)
    store, _, _ = make_store(rng, 8, 1, 128, dev)
    q = torch.randn(2, sum(rows), 128, device=dev)
    table = np.pad([[0, 1, 2, 3], [4, 5, 6, 7]], ((0, 0), (0, 60)), constant_values=-1)      # wide enough to need a workspace
    args = (store, i32(table, dev), i32([250, 256], dev), i32(np.cumsum([0] + rows), dev),
            i32(list(range(rows[0])) + list(range(rows[1])), dev))
    full = sc.forward(q, *args)
    part = sc.forward(q, *args, max_rows=max(rows))
    assert torch.equal(full, part)
    workspace = torch.empty(sc.workspace_bytes(2, sum(rows), max(rows), 2, 1, 128, 64), dtype=torch.uint8, device=dev)
    assert torch.equal(sc.forward(q, *args, max_rows=max(rows), workspace=workspace), full)
    with pytest.raises(sb.SolAttnError):
        sc.forward(q, *args, max_rows=max(rows), workspace=workspace[:16])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forward_not_finite(dev, dtype):
    """A token held as NaN, and queries that are not finite: their rows are NaN, every other row is as without them."""
    rng = np.random.default_rng(8)
    d, T = 128, 130
    k, v = (torch.tensor(rng.standard_normal((1, 200, d)), dtype=torch.float32, device=dev) for _ in range(2))
    q = torch.tensor(rng.standard_normal((2, T, d)), dtype=torch.float32, device=dev).to(DT[dtype])
    table, lens, row_start = i32([[2, 0, 3, 1]], dev), i32([200], dev), i32([0, T], dev)
    slots = i32([[2, 0, 3, 1][t // 64] * 64 + t % 64 for t in range(200)], dev)
    positions = i32(np.arange(70, 200), dev)

    def run(bad_k=None, bad_v=None, bad_q=None):
        kk, vv, qq = k.clone(), v.clone(), q.clone()
        if bad_k is not None:
            kk[0, bad_k, 77] = math.nan
        if bad_v is not None:
            vv[0, bad_v, 3] = math.inf
        if bad_q is not None:
            qq[1, bad_q, 100] = math.inf
        store = sc.empty(4, 1, d, dev)
        store.fill_(255)
        sc.append(kk, vv, store, slots)
        return sc.forward(qq, store, table, lens, row_start, positions)
    clean = run()
    assert bool(torch.isfinite(clean).all())
    for kw in (dict(bad_k=110), dict(bad_v=131), dict(bad_k=199)):
        at = next(iter(kw.values()))
        y = run(**kw)
        sees = (positions >= at)[None, :, None].expand_as(y)
        assert bool(torch.isnan(y[sees]).all()) and torch.equal(y[~sees], clean[~sees])
    y = run(bad_q=17)
    assert bool(torch.isnan(y[1, 17]).all())
    y[1, 17] = clean[1, 17]
    assert torch.equal(y, clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("peak", [0, 3000, 69999])
def test_forward_long_and_peaked(dev, dtype, peak):
    """70,000 tokens, of which one has nearly all the weight; a maximum that comes late."""
    d, L = 128, 70000
    P = -(-L // 64)
    g = torch.Generator(device=dev).manual_seed(peak)
    k, v = (torch.randn(1, P * 64, d, generator=g, device=dev) for _ in range(2))
    q = torch.randn(1, 1, d, generator=g, device=dev).to(DT[dtype])
    k[0, peak] = q.float()[0, 0] * 3
    store = sc.empty(P, 1, d, dev)
    order = torch.randperm(P, generator=g, device=dev)
    slots = (order[:, None] * 64 + torch.arange(64, device=dev)).flatten().int()
    sc.append(k, v, store, slots)
    out = sc.forward(q, store, order[None].int(), i32([L], dev), i32([0, 1], dev), i32([L - 1], dev))
    kk, vv = (f64(x)[0, :L] for x in sc.read(store, slots, dtype=torch.float32))
    ref, spread, reach = ora.attend(f64(q)[0], kk, vv, np.ones((1, L), bool))
    tol = tolerance(dtype, f64(q)[0, 0], kk, vv, ref[0], spread[0], reach[0])
    assert (np.abs(f64(out)[0, 0] - ref[0]) <= tol).all()


def test_forward_many_requests(dev):
    """More requests than lanes: 300 of them, some with several rows, some with none."""
    rng = np.random.default_rng(11)
    lens = [int(x) for x in rng.integers(0, 200, 300)]
    rows = [min(n, int(r)) for n, r in zip(lens, rng.choice([0, 1, 1, 1, 2, 40], 300))]
    check_forward(dev, "bf16", 64, 2, 1, lens, rows, 1, seed=12)


@pytest.mark.parametrize("seed", range(24))
def test_forward_random(dev, seed):
    """Shapes, lengths, masks and layouts at random; positions that are no run; dropped pages."""
    rng = np.random.default_rng(1000 + seed)
    d = int(rng.choice([64, 128]))
    Hk, G = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 4, 7, 16]))
    S = int(rng.integers(1, 8))
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(900), S))]
    rows = [int(rng.integers(0, max(2, min(n, 2000 // (S * Hk * G))) + 1)) for n in lens]
    rows[0] = max(1, rows[0])
    positions = np.concatenate([rng.integers(-1, n + 3, r) for n, r in zip(lens, rows)])
    drop = [(s, int(rng.integers(0, -(-n // 64))), int(rng.choice([-1, 1 << 28]))) for s, n in enumerate(lens) if rng.random() < 0.3 and n]
    granule = int(rng.choice([1, 1, 17, 64, 300, 1 << 30]))
    check_forward(dev, str(rng.choice(["bf16", "f32"])), d, Hk * G, Hk, lens, rows, granule, str(rng.choice(["plain", "tokens", "odd"])),
                  seed=seed, positions=positions, drop=drop, extra=0)


# The same edges where requests are cut into pieces and rows go to both kernels: tables with room for long sequences.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,Hq,Hk,lens,rows,granule,how", FORWARD)
def test_forward_wide_tables(dev, dtype, d, Hq, Hk, lens, rows, granule, how):
    check_forward(dev, dtype, d, Hq, Hk, lens, rows, granule, how, seed=d + sum(lens), wide=40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fill", [0, 127, 254, 255])
@pytest.mark.parametrize("rows", [3, 70])
def test_forward_cut_rows_that_see_nothing(dev, dtype, fill, rows):
    positions = np.concatenate([np.resize([-1, 0, 2100, 89, -1, 2199], rows), [2, 3, 3]])
    check_forward(dev, dtype, 64, 4, 2, [2200, 0, 70, 0, 4], [rows, 0, 2, 0, 1], 1, positions=positions, fill=fill, seed=fill, wide=40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 150])
def test_forward_cut_dropped_pages(dev, dtype, rows):
    drop = [(0, p, -1) for p in (0, 3, 4, 5, 6, 7, 8, 30)] + [(0, 20, 1 << 30), (0, 39, -(1 << 31))] + [(1, p, -1) for p in range(40)]
    check_forward(dev, dtype, 128, 4, 2, [2560, 2500], [rows, rows], 1, drop=drop, seed=rows, wide=40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [3, 130])
def test_forward_cut_not_finite(dev, dtype, d, T):
    # as test_forward_not_finite, of pieces that are joined
    rng = np.random.default_rng(T)
    L = 3000
    P = -(-L // 64)
    k, v = (torch.tensor(rng.standard_normal((1, P * 64, d)), dtype=torch.float32, device=dev) for _ in range(2))
    q = torch.tensor(rng.standard_normal((2, T, d)), dtype=torch.float32, device=dev).to(DT[dtype])
    order = torch.tensor(rng.permutation(P), device=dev)
    slots = (order[:, None] * 64 + torch.arange(64, device=dev)).flatten().int()
    table = torch.nn.functional.pad(order[None].int(), (0, 40), value=-1)
    positions = i32(np.linspace(L - 1, 700, T), dev)

    def run(bad_k=None, bad_v=None, bad_q=None):
        kk, vv, qq = k.clone(), v.clone(), q.clone()
        if bad_k is not None:
            kk[0, bad_k, 7] = math.nan
        if bad_v is not None:
            vv[0, bad_v, 3] = -math.inf
        if bad_q is not None:
            qq[1, bad_q, 10] = math.nan
        store = sc.empty(P, 1, d, dev)
        sc.append(kk, vv, store, slots)
        return sc.forward(qq, store, table, i32([L], dev), i32([0, T], dev), positions)
    clean = run()
    assert bool(torch.isfinite(clean).all())
    for kw in (dict(bad_k=0), dict(bad_k=1500), dict(bad_v=2900), dict(bad_k=2999)):
        at = next(iter(kw.values()))
        y = run(**kw)
        sees = (positions >= at)[None, :, None].expand_as(y)
        assert bool(torch.isnan(y[sees]).all()) and torch.equal(y[~sees], clean[~sees])
    y = run(bad_q=1)
    assert bool(torch.isnan(y[1, 1]).all())
    y[1, 1] = clean[1, 1]
    assert torch.equal(y, clean)


@pytest.mark.parametrize("seed", range(12))
def test_forward_random_wide(dev, seed):
    rng = np.random.default_rng(3000 + seed)
    d = int(rng.choice([64, 128]))
    Hk, G = int(rng.integers(1, 4)), int(rng.choice([1, 2, 4, 7]))
    S = int(rng.integers(1, 12))
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(2500), S))]
    rows = [int(rng.integers(0, max(2, min(n, 2000 // (S * Hk * G))) + 1)) for n in lens]
    rows[0] = max(1, rows[0])
    positions = np.concatenate([rng.integers(-1, n + 3, r) for n, r in zip(lens, rows)])
    drop = [(s, int(rng.integers(0, -(-n // 64))), int(rng.choice([-1, 1 << 28]))) for s, n in enumerate(lens) if rng.random() < 0.3 and n]
    check_forward(dev, str(rng.choice(["bf16", "f32"])), d, Hk * G, Hk, lens, rows, int(rng.choice([1, 17, 300, 1 << 30])),
                  str(rng.choice(["plain", "tokens", "odd"])), seed=seed, positions=positions, drop=drop, wide=int(rng.choice([40, 5000])))


@pytest.mark.parametrize("dtype,d,Hq,Hk,S,rows,lens,granule", [
    ("bf16", 128, 32, 16, 1, 700, 5000, 1),            # one request, tiles of 128 rows past half of what the GPU holds, cut
    ("bf16", 64, 64, 16, 3, 300, 2500, 1 << 30),       # few requests, all fillings looked at at once
    ("f32", 128, 16, 16, 12, 200, 900, 50),            # more than eight requests, one filling after the other
    ("bf16", 128, 4, 4, 90, 60, 500, 1),               # more requests than lanes, each of many rows
    ("f32", 64, 12, 12, 70, 3, 700, 1),                # more requests than lanes, each of few rows
    ("bf16", 64, 8, 8, 90, 2, 3000, 1),                # few rows, lengths alike: not cut
    ("bf16", 128, 4, 4, 30, 2, 4000, 1),               # few rows, cut
    ("bf16", 128, 8, 1, 1, 2, 200000, 1),              # one long request
])
def test_forward_cut_into_pieces(dev, dtype, d, Hq, Hk, S, rows, lens, granule):
    """Work of a size that is cut, against attention in 64 bits on the GPU, on the values that read() gives."""
    g = torch.Generator(device=dev).manual_seed(S + rows)
    rng = np.random.default_rng(S)
    length = [int(lens * f) for f in rng.uniform(0.4, 1.0, S)]
    rows = [min(n, max(1, int(rows * f))) for n, f in zip(length, rng.uniform(0.5, 1.0, S))]
    held = [-(-n // 64) for n in length]
    P, T = sum(held) + 1, sum(rows)
    k, v = (torch.randn(Hk, P * 64, d, generator=g, device=dev) for _ in range(2))
    store = sc.empty(P, Hk, d, dev)
    slots = torch.arange(P * 64, dtype=torch.int32, device=dev)
    sc.append(k, v, store, slots)
    k, v = (x.double() for x in sc.read(store, slots, dtype=torch.float32))
    order = torch.randperm(P, generator=g, device=dev).int()
    table = torch.full((S, max(held) + 3), -1, dtype=torch.int32, device=dev)
    at = 0
    for s in range(S):
        table[s, :held[s]] = order[at:at + held[s]]
        at += held[s]
    q = torch.randn(T, Hq, d, generator=g, device=dev).to(DT[dtype]).transpose(0, 1)
    row_start = np.concatenate([[0], np.cumsum(rows)])
    positions = torch.cat([torch.arange(n - r, n, dtype=torch.int32, device=dev) for n, r in zip(length, rows)])
    out = sc.forward(q, store, table, i32(length, dev), i32(row_start, dev), positions, causal_granule=granule)
    off = norm = 0.0
    for s in range(S):
        slot = (order[sum(held[:s]):sum(held[:s + 1]), None].long() * 64 + torch.arange(64, device=dev)).flatten()[:length[s]]
        r0, r1 = row_start[s], row_start[s + 1]
        limit = (positions[r0:r1].long() // granule + 1) * granule
        hidden = torch.arange(length[s], device=dev)[None] >= limit[:, None]
        for h in range(Hq):
            kk, vv = k[h // (Hq // Hk), slot], v[h // (Hq // Hk), slot]
            logits = (q[h, r0:r1].double() @ kk.T.contiguous()) / math.sqrt(d)
            ref = torch.softmax(logits.masked_fill(hidden, -math.inf), -1) @ vv
            err = out[h, r0:r1].double() - ref
            # as in tolerance(), with the largest |v| for sum p |v| and half of sum p |v - out|, and the largest |q| for that of a block
            top, sum_k = q[h, r0:r1].double().abs().amax(), kk.abs().sum(-1).amax()
            s_abs = top * sum_k / math.sqrt(d)
            ds = s_abs * ((2.0 ** -11 if dtype == "bf16" else 2.0 ** -23) / 3.75 + (d + 6) * 2.0 ** -24) + 64 * 2.0 ** -24
            cut = (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) + (length[s] / 16 + 64) * 2.0 ** -24 + length[s] * 2.0 ** -32
            bound = (HALF_STEP[dtype] * 1.01 + 2.0 ** -23) * ref.abs() + (4 * ds + cut) * vv.abs().amax()
            assert bool((err.abs() <= bound).all()), (s, h, float((err.abs() / bound).max()))
            off, norm = off + float(err.square().sum()), norm + float(ref.square().sum())
    # Over all values errors add up by their squares: a rounding to bf16 is at most 2^-8 / sqrt(3) of the values, to f16 an eighth
    # of that; a logit's, 2^-11 / sqrt(3) of a block's largest channel over 3.75 for each of d channels, comes to less than
    # that of f16, and a row's sum is over weights whose squares add up alike.  f32: as many terms of 2^-22 and less.
    assert math.sqrt(off / norm) <= (2.0 ** -8 / math.sqrt(3) * 1.25 if dtype == "bf16" else 2.0 ** -20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("how", ["tokens", "odd"])
@pytest.mark.parametrize("rows", [[3, 20, 1], [150], [3, 150, 1]])      # few rows, many, both in one call
def test_forward_every_term_of_the_queries(dev, dtype, d, how, rows):
    """The error over all values: a term of a query that is lost or wrong is 16 times what the terms leave.

    Errors of independent values add up by their squares.  With keys and values that are independent and have the mean 0, a logit
    that is off by e changes an output by e times what that key gives to it.  A channel of q, with the scaled top of its block in
    (3.75, 7.5], is left with an error of at most 2^-11 top / 3.75 (bf16; f32: 2^-23), evenly spread: over sqrt(3).  d channels of keys
    with squares k2 on average: sqrt(k2) times that, the 1 / sqrt(d) of the logits included.  Probabilities: half a step of 2^-11
    over sqrt(3) (f32: 2^-22).  Results: half a step over sqrt(3); f32: 16 roundings of 2^-24 for sums."""
    rng = np.random.default_rng(d + len(rows))
    lens = [400, 350, 600][:len(rows)]
    held = [-(-n // 64) for n in lens]
    store, k, v = make_store(rng, sum(held), 2, d, dev)
    pages = np.concatenate([[0], np.cumsum(held)])
    table = np.full((len(rows), max(held) + 30), -1)
    for s, n in enumerate(held):
        table[s, :n] = np.arange(pages[s], pages[s] + n)
    T = sum(rows)
    q = torch.tensor(4.0 * rng.standard_normal((4, T, d)), dtype=torch.float32).to(DT[dtype])
    row_start = np.concatenate([[0], np.cumsum(rows)])
    positions = np.concatenate([np.full(r, n - 1) for n, r in zip(lens, rows)])
    out = placed(torch.zeros(4, T, d, dtype=DT[dtype]), how, dev)
    sc.forward(placed(q, how, dev), store, i32(table, dev), i32(lens, dev), i32(row_start, dev), i32(positions, dev), out=out)
    y, qn = f64(out), f64(q)
    off = norm = 0.0
    for s, n in enumerate(lens):
        at = slice(pages[s] * 64, pages[s] * 64 + n)
        for h in range(4):
            ref = ora.attend(qn[h, row_start[s]:row_start[s + 1]], k[h // 2, at], v[h // 2, at], np.ones((rows[s], n), bool))[0]
            off, norm = off + np.square(y[h, row_start[s]:row_start[s + 1]] - ref).sum(), norm + np.square(ref).sum()
    left = (2.0 ** -11 if dtype == "bf16" else 2.0 ** -23) / 3.75 * np.abs(qn).max() * math.sqrt(np.square(k).mean())
    parts = [left, 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22, HALF_STEP[dtype] if dtype == "bf16" else 16 * 2.0 ** -24]
    assert math.sqrt(off / norm) <= math.sqrt(sum(x * x for x in parts) / 3), math.sqrt(off / norm)


def test_pages_past_four_gigabytes(dev):
    """Pages whose bytes lie past 2^32 in the store, and pages that two requests share."""
    P, H, d = 260000, 2, 128
    assert P * H * 68 * d > 2 ** 32
    store = torch.empty((P, H, 68 * d), dtype=torch.uint8, device=dev)
    pages = [P - 1, 5, P - 2, 3, P // 2]
    g = torch.Generator().manual_seed(9)
    k, v = (torch.randn(H, 300, d, generator=g) for _ in range(2))
    slots = np.array([pages[t // 64] * 64 + t % 64 for t in range(300)])
    sc.append(k.to(dev), v.to(dev), store, i32(slots, dev))
    kk, vv = (f64(x) for x in sc.read(store, i32(slots, dev), dtype=torch.float32))
    assert np.array_equal(kk, ora.values(*ora.quantise(f64(k), ora.K_SCALES)))
    assert np.array_equal(vv, ora.values(*ora.quantise(f64(v), ora.V_SCALES)))
    rows = [1, 90]                       # the second request has the first three pages only, the first all
    q = torch.randn(4, sum(rows), d, generator=g)
    table = np.array([pages, pages[:3] + [-1, -1]])
    out = f64(sc.forward(q.to(dev), store, i32(table, dev), i32([300, 190], dev), i32([0, 1, 91], dev),
                         i32([299] + list(range(100, 190)), dev)))
    for s, (r0, r1, n) in enumerate(((0, 1, 300), (1, 91, 190))):
        pos = np.array([299]) if s == 0 else np.arange(100, 190)
        for h in range(4):
            ref, spread, reach = ora.attend(f64(q)[h, r0:r1], kk[h // 2, :n], vv[h // 2, :n], np.arange(n)[None] <= pos[:, None])
            for r in range(r1 - r0):
                tol = tolerance("f32", f64(q)[h, r0 + r], kk[h // 2, :n], vv[h // 2, :n], ref[r], spread[r], reach[r])
                assert (np.abs(out[h, r0 + r] - ref[r]) <= tol).all()


def test_empty_calls(dev):
    """No rows at all, and a granule past an int."""
    rng = np.random.default_rng(3)
    store, _, _ = make_store(rng, 2, 2, 64, dev)
    none = torch.empty(0, dtype=torch.int32, device=dev)
    q = torch.empty(4, 0, 64, device=dev)
    assert sc.forward(q, store, i32([[0, 1]], dev), i32([100], dev), i32([0, 0], dev), none).shape == (4, 0, 64)
    before = store.clone()
    sc.append(q[:2], q[:2], store, none)
    assert torch.equal(store, before)
    k, v = sc.read(store, none)
    assert k.shape == v.shape == (2, 0, 64)
    y, _ = sc.qk_norm_rope(q[None], None)
    assert y.shape == (1, 4, 0, 64)
    q = torch.randn(4, 3, 64, device=dev)
    args = (store, i32([[0, 1]], dev), i32([100], dev), i32([0, 3], dev), i32([5, 6, 7], dev))
    assert torch.equal(sc.forward(q, *args, causal_granule=10 ** 15), sc.forward(q, *args, causal_granule=100))


# ------------------------------------------------------------------------------------------------------ as one step
class Server:
    """Requests that grow step by step through the four operators; the reference keeps plain lists."""

    def __init__(self, dev, dtype, d, Hq, Hk, S, MP, P, seed, interleaved):
        self.dev, self.dtype, self.d, self.Hq, self.Hk, self.S = dev, dtype, d, Hq, Hk, S
        self.rng = np.random.default_rng(seed)
        self.lens, self.state = i32([0] * S, dev), i32([0, P], dev)
        self.table, self.ring = i32(np.full((S, MP), -1), dev), i32(self.rng.permutation(P), dev)
        self.store = sc.empty(P, Hk, d, dev)
        self.store.fill_(255)
        angle = np.arange(MP * 64)[:, None] * 100.0 ** (-np.arange(d // 2) / (d // 2))
        self.cos, self.sin = (torch.tensor(f(angle), dtype=torch.float32, device=dev) for f in (np.cos, np.sin))
        self.w = [torch.tensor(1 + 0.1 * self.rng.standard_normal(d), dtype=torch.float32, device=dev) for _ in range(2)]
        self.inter = interleaved
        self.held = [[np.zeros((Hk, 0, d))] * 2 for _ in range(S)]

    def qkv(self, rows):
        x = self.rng.standard_normal((rows, self.Hq + 2 * self.Hk, self.d))
        return torch.tensor(x, dtype=torch.float32, device=self.dev).to(DT[self.dtype])

    def split(self, qkv):
        x = qkv.transpose(0, 1)
        return x[:self.Hq], x[self.Hq:self.Hq + self.Hk], x[self.Hq + self.Hk:]

    def step(self, qkv, add, granule=1):
        """The calls of one step on tensors `qkv` [rows, heads, d] and add [S]."""
        q, k, v = self.split(qkv)
        new = sc.tables(self.lens, add, self.table, self.ring, self.state, qkv.shape[0])
        q, k = sc.qk_norm_rope(q[None], k[None], *self.w, self.cos, self.sin, new.positions[None], interleaved=self.inter)
        sc.append(k[0], v, self.store, new.slots)
        out = sc.forward(q[0], self.store, self.table, new.lens, new.row_start, new.positions, causal_granule=granule)
        return new, q[0], k[0], out

    def check(self, qkv, add, new, q, k, out, granule=1):
        _, _, v = self.split(qkv)
        kq = ora.values(*ora.quantise(f64(k), ora.K_SCALES))
        vq = ora.values(*ora.quantise(f64(v), ora.V_SCALES))
        at = 0
        for s, a in enumerate(add):
            ks, vs = self.held[s]
            if a <= 0:
                n = max(0, ks.shape[1] + a)
                self.held[s] = [ks[:, :n], vs[:, :n]]
                continue
            self.held[s] = ks, vs = [np.concatenate([x, y[:, at:at + a]], 1) for x, y in zip((ks, vs), (kq, vq))]
            n = ks.shape[1]
            assert int(new.lens[s]) == n
            sees = np.arange(n)[None] < np.minimum((np.arange(n - a, n) // granule + 1) * granule, n)[:, None]
            for h in range(self.Hq):
                kk, vv = ks[h // (self.Hq // self.Hk)], vs[h // (self.Hq // self.Hk)]
                ref, spread, reach = ora.attend(f64(q[h, at:at + a]), kk, vv, sees)
                for r in range(a):
                    tol = tolerance(self.dtype, f64(q[h, at + r]), kk, vv, ref[r], spread[r], reach[r])
                    assert (np.abs(f64(out[h, at + r]) - ref[r]) <= tol).all(), (s, h, r)
            at += a


STEPS = [[70, 3, 0, 130], [1, 1, 1, 1], [1, -1, 5, -130], [40, 1, 1, 64], [-1000, 2, 1, 1], [65, 1, -2, 1]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,Hq,Hk,interleaved", [(128, 4, 2, False), (64, 3, 1, True)])
def test_serving_steps(dev, dtype, d, Hq, Hk, interleaved):
    server = Server(dev, dtype, d, Hq, Hk, 4, 6, 12, d, interleaved)
    for add in STEPS:
        qkv = server.qkv(max(1, sum(max(a, 0) for a in add)))
        got = server.step(qkv, i32(add, dev))
        server.check(qkv, add, *got)
        server.lens, server.state = got[0].lens, got[0].state


def test_frames_match_the_dense_forward(dev):
    """Frame by frame through the cache against the framework's own frame-causal forward on the values that the cache holds."""
    d, H, frame, frames = 128, 3, 90, 4
    N = frame * frames
    server = Server(dev, "bf16", d, H, H, 1, 8, 8, 4, True)
    outs, qs, ks, vs = [], [], [], []
    for f in range(frames):
        qkv = server.qkv(frame)
        new, q, k, out = server.step(qkv, i32([frame], dev), granule=frame)
        server.lens, server.state = new.lens, new.state
        hk, hv = sc.read(server.store, new.slots)
        outs.append(out), qs.append(q), ks.append(hk), vs.append(hv)
    q, k, v = (torch.cat(x, 1)[None].contiguous() for x in (qs, ks, vs))
    dense = sb.forward(q, k, v, 128, 64, 0.0, "dense", causal_granule=frame)
    a, b = f64(torch.cat(outs, 1)), f64(dense[0])
    # two bf16 results of the same products: each is within 2^-8 of its value and 2^-9 of the values' reach
    assert np.abs(a - b).max() <= 2 * (2.0 ** -8 * np.abs(b).max() + 2.0 ** -9 * np.abs(f64(v)).max())
    assert np.linalg.norm(a - b) <= 2 * 2.0 ** -8 * np.linalg.norm(b)


def test_captured_steps(dev):
    """Two steps captured into two graphs that share a store: each replay against an eager step on the same inputs."""
    S, Hq, Hk, d = 3, 4, 2, 128

    def server():
        s = Server(dev, "bf16", d, Hq, Hk, S, 6, 20, 3, False)
        first = torch.randn(150, Hq + 2 * Hk, d, generator=torch.Generator().manual_seed(1)).bfloat16().to(dev)
        new, *_ = s.step(first, i32([100, 30, 20], dev))
        s.lens, s.state = new.lens.clone(), new.state.clone()
        return s
    a, b = server(), server()
    stream = torch.cuda.Stream()
    graphs = []
    for rows, add in ((3, [1, 1, 1]), (12, [4, 0, 7])):
        qkv, adds = torch.zeros(rows, Hq + 2 * Hk, d, dtype=torch.bfloat16, device=dev), i32(add, dev)
        with torch.cuda.stream(stream):
            a.step(qkv, adds * 0)                                # a step that adds nothing, before the capture
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            new, q, k, out = a.step(qkv, adds)
            a.lens.copy_(new.lens)
            a.state.copy_(new.state)
        graphs.append((graph, qkv, adds, out, new))
    for turn in range(6):
        graph, qkv, adds, out, new = graphs[turn % 2]
        rows = qkv.shape[0]
        x = torch.randn(qkv.shape, generator=torch.Generator().manual_seed(10 + turn)).bfloat16().to(dev)
        if turn == 4:
            adds.copy_(i32([1, -60, 1], dev))                    # a step of fewer rows than were captured
        live = int(adds.clamp(min=0).sum())
        qkv.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        want, _, _, eager = b.step(x, adds.clone())
        b.lens, b.state = want.lens.clone(), want.state.clone()
        torch.cuda.synchronize()
        assert torch.equal(out[:, :live], eager[:, :live]), turn
        assert torch.equal(new.slots, want.slots) and torch.equal(a.lens, b.lens) and torch.equal(a.state, b.state)
        assert live <= rows


def test_streams_of_their_own(dev):
    """Calls on two other streams at once, each with its own workspace."""
    rng = np.random.default_rng(2)
    store, _, _ = make_store(rng, 40, 2, 128, dev)
    torch.cuda.synchronize()
    table, lens, row_start, positions = i32([list(range(40))], dev), i32([2500], dev), i32([0, 2], dev), i32([2498, 2499], dev)
    qs = [torch.randn(4, 2, 128, generator=torch.Generator().manual_seed(i)).to(dev) for i in range(2)]
    want = [sc.forward(q, store, table, lens, row_start, positions) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(sc.forward(qs[i], store, table, lens, row_start, positions))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


# ------------------------------------------------------------------------------------------------ the plan of pieces
FEW_TILE, MANY_TILE, HEADER, SENTINEL = 16, 128, 256, 0x5A5A5A5A


def pages_of_pieces(ws, d, need, both):
    """Pages of a piece as the parts of a call planned them: the words in front of the parts' results.  A workspace that held the
    sentinel before has that word, 63 untouched ones and the results; the second part starts behind a whole number of results of
    16 rows of the first and ends with a whole number of 128 results of 128 rows."""
    w = ws.view(torch.int32).cpu().numpy()

    def header(at):
        return w[at // 4] != SENTINEL and (w[at // 4 + 1:at // 4 + HEADER // 4] == SENTINEL).all()
    assert header(0)
    if not both:
        return [int(w[0])]
    few, many = FEW_TILE * (d + 2) * 4, 128 * MANY_TILE * (d + 2) * 4
    at = [a for a in range(HEADER, need - many, few) if (need - a - HEADER) % many == 0 and header(a)]
    assert len(at) == 1, at
    return [int(w[0]), int(w[at[0] // 4])]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("Hq,Hk,S,rows,lens,parts", [
    # parts: for the few and the many rows, least and most pages of a piece; None: the part is not there
    (32, 8, 4, [300], [4500, 1800], [None, (2, 60)]),             # few requests, all fillings at once
    (16, 8, 12, [200], [5000, 900], [None, (2, 60)]),             # one filling after the other
    (4, 4, 70, [60], [6000, 300], [None, (2, 60)]),               # more requests than lanes
    (4, 4, 150, [60, 1, 2], [6000, 300], [(2, 60), (2, 60)]),     # the same, of both kinds (rows of the long ones: 60 and 1)
    (3, 3, 90, [2, 1], [5000, 200], [(2, 60), None]),             # the same, of few rows
    (70, 70, 8, [40], [3000, 400], [(2, 40), None]),              # few rows: all fillings at once
    (34, 34, 60, [1], [4000, 300], [(2, 50), None]),              # few rows: one filling after the other
])
def test_forward_every_way_of_cutting(dev, dtype, d, Hq, Hk, S, rows, lens, parts):
    """Every way in which the pages of a piece are chosen, each shown by what the plan left in the workspace: less than the longest
    request has.  One request of each part in the middle is long (lens[0] tokens), the others have half of lens[1] to lens[1]."""
    rng = np.random.default_rng(S)
    length = [int(lens[1] * f) for f in rng.uniform(0.5, 1.0, S)]
    few_too = parts[1] is not None and parts[0] is not None
    length[S // 2:S // 2 + 1 + few_too] = [lens[0]] * (1 + few_too)
    rows = [rows[s % len(rows)] for s in range(S)]
    held = [-(-n // 64) for n in length]
    start, P, T = np.cumsum([0] + held), sum(held), sum(rows)
    g = torch.Generator(device=dev).manual_seed(S)
    k, v = (torch.randn(Hk, P * 64, d, generator=g, device=dev) for _ in range(2))
    store = sc.empty(P, Hk, d, dev)
    order = torch.randperm(P, generator=g, device=dev)
    slots = (order[:, None] * 64 + torch.arange(64, device=dev)).flatten().int()
    sc.append(k, v, store, slots)
    k, v = (x.double() for x in sc.read(store, slots, dtype=torch.float32))
    table = torch.full((S, max(held) + 3), -1, dtype=torch.int32, device=dev)
    for s in range(S):
        table[s, :held[s]] = order[start[s]:start[s + 1]].int()
    q = torch.randn(T, Hq, d, generator=g, device=dev).to(DT[dtype]).transpose(0, 1)
    row_start = np.cumsum([0] + rows)
    positions = torch.cat([torch.arange(n - r, n, dtype=torch.int32, device=dev) for n, r in zip(length, rows)])
    need = sc.workspace_bytes(S, T, max(rows), Hq, Hk, d, table.shape[1])
    ws = torch.full((need,), 0x5A, dtype=torch.uint8, device=dev)
    out = sc.forward(q, store, table, i32(length, dev), i32(row_start, dev), positions, max_rows=max(rows), workspace=ws)
    # with the many rows' kernel and several requests, the few rows' part is there too, even if no request is for it
    per = pages_of_pieces(ws, d, need, both=parts[1] is not None)
    for part, got in zip(parts, per):
        if part is not None:
            assert part[0] <= got <= part[1], per
    off = norm = 0.0
    for s in range(S):
        r0, r1, k0 = row_start[s], row_start[s + 1], start[s] * 64
        hidden = torch.arange(length[s], device=dev)[None] > positions[r0:r1, None]
        for h in range(Hk):
            kk, vv = (x[h, k0:k0 + length[s]] for x in (k, v))
            qq = q[h * (Hq // Hk):(h + 1) * (Hq // Hk), r0:r1].double()
            logits = (qq.reshape(-1, d) @ kk.T.contiguous()).view(Hq // Hk, r1 - r0, -1) / math.sqrt(d)
            p = torch.softmax(logits.masked_fill(hidden, -math.inf), -1).flatten(0, 1)
            ref, reach = p @ vv, p @ vv.abs()
            err = out[h * (Hq // Hk):(h + 1) * (Hq // Hk), r0:r1].double().reshape(-1, d) - ref
            # as in tolerance(), with the largest |q| for that of a block, and 2 sum p |v| for sum p |v - out|; a third term of the
            # queries leaves half a step of 2^-3 (its values reach 2), so three leave 2^-4 / 16^2, six 2^-4 / 16^5
            s_abs = qq.abs().amax() * kk.abs().sum(-1).amax() / math.sqrt(d)
            ds = s_abs * ((2.0 ** -12 if dtype == "bf16" else 2.0 ** -24) / 3.75 + (d + 6) * 2.0 ** -24) + 64 * 2.0 ** -24
            cut = (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) + (length[s] / 16 + 64) * 2.0 ** -24
            bound = (HALF_STEP[dtype] * 1.01 + 2.0 ** -23) * ref.abs() + (4 * ds + cut) * reach + 2.0 ** -32 * vv.abs().sum(0)
            assert bool((err.abs() <= bound).all()), (s, h, float((err.abs() / bound).max()))
            off, norm = off + float(err.square().sum()), norm + float(ref.square().sum())
    # over all values: as in test_forward_cut_into_pieces
    assert math.sqrt(off / norm) <= (2.0 ** -8 / math.sqrt(3) * 1.25 if dtype == "bf16" else 2.0 ** -20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [1, 60])                   # both kernels
@pytest.mark.parametrize("L,wide", [(700, 0), (3000, 0), (20000, 100)])
@pytest.mark.parametrize("gap", [17, 22, 45])
def test_forward_beside_a_token_of_nearly_all_the_weight(dev, dtype, d, rows, L, wide, gap):
    """A token whose value is 0 stands `gap` nats above all others: what the others give is all that there is to see.

    f32: as in tolerance(), with the error of each key's own logit, but no probability is too small to be exact: an exponential is off
    by an ulp, which the 2^-22 of tolerance() holds.  bf16: as there, each is off by up to 2^-32 of the largest, an error on sum |v|."""
    P = -(-L // 64)
    g = torch.Generator(device=dev).manual_seed(L + gap)
    k = 0.1 * torch.randn(1, P * 64, d, generator=g, device=dev)
    v = torch.randn(1, P * 64, d, generator=g, device=dev) + 1.0
    k[..., :32] = 0.0
    k[0, L // 3], v[0, L // 3] = 0.0, 0.0
    q = 0.25 * torch.randn(1, rows, d, generator=g, device=dev)
    q[..., :32] = 0.0
    k[0, L // 3, 0] = 3.0 * 2.0 ** round(math.log2(gap * math.sqrt(d) / 8.0 / 3.0))
    q[..., 0] = gap * math.sqrt(d) / float(k[0, L // 3, 0])
    q = q.to(DT[dtype])
    store = sc.empty(P, 1, d, dev)
    slots = torch.arange(P * 64, dtype=torch.int32, device=dev)
    sc.append(k, v, store, slots)
    table = torch.nn.functional.pad(torch.arange(P, dtype=torch.int32, device=dev)[None], (0, wide), value=-1)
    out = sc.forward(q, store, table, i32([L], dev), i32([0, rows], dev), i32([L - 1] * rows, dev))
    k, v = (x.double()[0, :L] for x in sc.read(store, slots, dtype=torch.float32))
    q = q.double()[0]
    s = (q @ k.T.contiguous()) / math.sqrt(d)
    p = torch.softmax(s, -1)
    assert bool((s[:, L // 3, None] - s >= gap - 2)[:, torch.arange(L, device=dev) != L // 3].all())
    ref = p @ v
    top = q.abs().unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, -1)
    lost = top * (2.0 ** -12 if dtype == "bf16" else 2.0 ** -24) / 3.75 + 2 * 2.0 ** -24 * q.abs()
    size = (q.abs() @ k.abs().T.contiguous()) / math.sqrt(d)
    ds = (lost @ k.abs().T.contiguous()) / math.sqrt(d) + d * 2.0 ** -24 * size + 4 * 2.0 ** -24 * (size.amax(-1, keepdim=True) + 16)
    spread = ((p * ds)[..., None] * (v[None] - ref[:, None]).abs()).sum(1) if rows == 1 else ds.amax(-1, keepdim=True) * 2 * (p @ v.abs())
    reach = p @ v.abs()
    bound = (HALF_STEP[dtype] * 1.01 + 2.0 ** -23) * ref.abs() + 2 * spread + (L / 16 + 64) * 2.0 ** -24 * reach
    bound += (2.0 ** -11 * reach + 2.0 ** -32 * v.abs().sum(0)) if dtype == "bf16" else 2.0 ** -22 * reach
    err = (out[0].double() - ref).abs()
    assert bool((err <= bound).all()), (float((err / bound).max()), float(err.norm() / ref.norm()))


@pytest.mark.parametrize("Hq,Hk,S,rows,lens,most", [
    (64, 8, 1, 7500, [7600], 2),             # 3,752 tiles of 128 rows, more than seven fillings of 512 workgroups
    (70, 70, 100, 1, [3000, 100], 70),       # 7,000 tiles of 16 rows, more than two fillings of the GPU
    (8, 2, 150, 30, [3000, 200, 250], 2),    # both parts, cut
])
def test_forward_keeps_to_its_workspace(dev, Hq, Hk, S, rows, lens, most):
    """A workspace of the very size, with other memory behind it; every request by itself gives the same to rounding."""
    d = 64
    g = torch.Generator(device=dev).manual_seed(S)
    length = [lens[0]] + [lens[1 + s % (len(lens) - 1)] for s in range(S - 1)]
    rows = [rows + 20 * (s % 3 == 0) * (S == 150) for s in range(S)]
    held = [-(-n // 64) for n in length]
    start, P, T = np.cumsum([0] + held), sum(held), sum(rows)
    k, v = (torch.randn(Hk, P * 64, d, generator=g, device=dev) for _ in range(2))
    store = sc.empty(P, Hk, d, dev)
    sc.append(k, v, store, torch.arange(P * 64, dtype=torch.int32, device=dev))
    table = torch.full((S, max(held) + 500), -1, dtype=torch.int32, device=dev)
    for s in range(S):
        table[s, :held[s]] = torch.arange(start[s], start[s + 1], dtype=torch.int32, device=dev)
    q = torch.randn(T, Hq, d, generator=g, device=dev).transpose(0, 1)
    row_start = np.cumsum([0] + rows)
    positions = torch.cat([torch.arange(n - r, n, dtype=torch.int32, device=dev) for n, r in zip(length, rows)])
    need = sc.workspace_bytes(S, T, max(rows), Hq, Hk, d, table.shape[1])
    block = torch.full((need + (1 << 20),), 0x5A, dtype=torch.uint8, device=dev)
    out = sc.forward(q, store, table, i32(length, dev), i32(row_start, dev), positions, max_rows=max(rows), workspace=block[:need])
    assert bool((block[need:] == 0x5A).all())
    for s in [0, 1, S // 2, S - 1] if S > 1 else [0]:
        at = slice(row_start[s], row_start[s + 1])
        for h in range(0, Hk, most):
            part = slice(h, h + most)
            one = sc.forward(q[part.start * (Hq // Hk):part.stop * (Hq // Hk), at], store[:, part].contiguous(), table[s:s + 1],
                             i32([length[s]], dev), i32([0, rows[s]], dev), positions[at].contiguous())
            # f32: sums in another order, a rounding for 16 keys and 64 more on sum p |v| below the largest |v|
            bound = 2 * (length[s] / 16 + 64 + 8) * 2.0 ** -24 * v.abs().amax()
            assert bool(((one - out[part.start * (Hq // Hk):part.stop * (Hq // Hk), at]).abs() <= bound).all()), (s, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("how", ["plain", "tokens", "odd"])
@pytest.mark.parametrize("d,rot,B,N,Hq,Hk", [
    (128, 128, 1, 3000, 37, 6),      # three heads to a workgroup: one has the last query head and two key heads, the last one has one
    (128, 64, 2, 1000, 50, 25),      # four
    (64, 32, 1, 9001, 21, 10),       # four, one with a query head and three key heads, the last one three
    (64, 64, 3, 4000, 0, 33),        # keys only: six, the last one three
    (128, 0, 1, 20000, 40, 3),       # sixteen, at most
])
def test_qk_norm_rope_several_heads_to_a_workgroup(dev, dtype, pairs, how, d, rot, B, N, Hq, Hk):
    """Large calls: a workgroup goes through several heads, across the border of queries and keys."""
    blocks = -(-B * N // (2048 // d))
    assert min(blocks * (Hq + Hk) // 2048, Hq + Hk, 16) > 1
    g = torch.Generator(device=dev).manual_seed(N)
    P = N + 7
    xs = [torch.randn(B, H, N, d, generator=g, device=dev).to(DT[dtype]) if H else None for H in (Hq, Hk)]
    ws = [(1 + 0.3 * torch.randn(d, generator=g, device=dev)).to(DT[dtype]) if H else None for H in (Hq, Hk)]
    angle = 7 * torch.rand(P, rot // 2, generator=g, device=dev, dtype=torch.float64)
    cos, sin = (angle.cos().float(), angle.sin().float()) if rot else (None, None)
    positions = torch.randint(0, P, (B, N), generator=g, device=dev, dtype=torch.int32)
    positions[:, ::97] = -1
    gpu = [None if x is None else placed(x, how, dev) for x in xs]
    outs = [None if x is None else placed(torch.full_like(x, 7.0), how, dev) for x in xs]
    got = sc.qk_norm_rope(*gpu, *ws, cos, sin, positions, interleaved=pairs, q_out=outs[0], k_out=outs[1])
    there = (positions >= 0)[:, None, :, None]
    for x, w, y in zip(xs, ws, got):
        if x is None:
            continue
        ref = x.double()
        ref = ref / (ref.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
        length = ref.abs()
        if rot:
            at = positions.clamp(min=0).long()
            c, s = cos.double()[at][:, None], sin.double()[at][:, None]
            half = rot // 2
            ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, half), slice(half, rot))
            a, b = ref[..., ia].clone(), ref[..., ib].clone()
            ref[..., ia], ref[..., ib] = a * c - b * s, b * c + a * s
            length[..., ia] = length[..., ib] = torch.hypot(a, b)
        # as in test_qk_norm_rope
        tol = HALF_STEP[dtype] * ref.abs() * (1 + 2.0 ** -7) + 24 * 2.0 ** -24 * length
        assert bool(torch.where(there, (y.double() - ref).abs() <= tol, y == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [3, 150])
def test_forward_channels_beside_a_large_one(dev, dtype, d, rows):
    """What the terms of a query leave of the other channels of a block whose largest one is 500 times as large (and meets keys of 0).

    Of a top in (3.75, 7.5] the first term leaves up to 1/4, which is 4 to the second (steps of 1/4 from 2 on), that one up to
    1/8, which is 2 to the third (steps of 1/8), and that one up to 1/16: three terms 2^-4 / 16^2, six 2^-4 / 16^5, of 3.75 at least.  Over all
    values as in test_forward_every_term_of_the_queries: evenly spread, a logit's over sqrt(3) times the keys' root mean square."""
    L = 4000
    P = -(-L // 64)
    g = torch.Generator(device=dev).manual_seed(d + rows)
    k, v = (torch.randn(1, P * 64, d, generator=g, device=dev) for _ in range(2))
    k[..., ::32] = 0.0
    store = sc.empty(P, 1, d, dev)
    slots = torch.arange(P * 64, dtype=torch.int32, device=dev)
    sc.append(k, v, store, slots)
    k, v = (x.double()[0, :L] for x in sc.read(store, slots, dtype=torch.float32))
    q = torch.randn(2, rows, d, generator=g, device=dev)
    q[..., ::32] = 500.0 + 24 * torch.rand(2, rows, d // 32, generator=g, device=dev)
    q = q.to(DT[dtype])
    table = torch.arange(P, dtype=torch.int32, device=dev)[None]
    out = sc.forward(q, store, table, i32([L], dev), i32([0, rows], dev), i32([L - 1] * rows, dev)).double()
    ref = torch.softmax((q.double().flatten(0, 1) @ k.T.contiguous()) / math.sqrt(d), -1) @ v
    left = (2.0 ** -12 if dtype == "bf16" else 2.0 ** -24) / 3.75 * 524 * float(k.square().mean().sqrt())
    parts = [left, 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22, HALF_STEP[dtype] if dtype == "bf16" else 16 * 2.0 ** -24]
    off = float((out.flatten(0, 1) - ref).norm() / ref.norm())
    assert off <= math.sqrt(sum(x * x for x in parts) / 3), (off, left)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outputs_in_one_buffer(dev, dtype):
    """Outputs that are parts of the rows of one buffer hold what outputs of their own hold, and nothing between them is written."""
    d, N, Hq, Hk = 128, 70, 6, 2
    g = torch.Generator(device=dev).manual_seed(1)
    q, k = (torch.randn(1, H, N, d, generator=g, device=dev).to(DT[dtype]) for H in (Hq, Hk))
    buffer = torch.full((1, N, Hq + 2 * Hk, d), 3.0, dtype=DT[dtype], device=dev)
    parts = [buffer[:, :, a:b].transpose(1, 2) for a, b in ((0, Hq), (Hq, Hq + Hk), (Hq + Hk, Hq + 2 * Hk))]
    want = sc.qk_norm_rope(q, k)
    sc.qk_norm_rope(q, k, q_out=parts[0], k_out=parts[1])
    assert torch.equal(parts[0], want[0]) and torch.equal(parts[1], want[1]) and bool((parts[2] == 3.0).all())
    store = sc.empty(2, Hk, d, dev)
    slots = torch.arange(N, dtype=torch.int32, device=dev)
    sc.append(want[1][0], k[0], store, slots)
    held = sc.read(store, slots, dtype=DT[dtype])
    sc.read(store, slots, k_out=parts[1][0], v_out=parts[2][0])
    assert torch.equal(parts[1][0], held[0]) and torch.equal(parts[2][0], held[1]) and torch.equal(parts[0], want[0])
    args = (store, i32([[0, 1]], dev), i32([N], dev), i32([0, N], dev), slots)
    attn = sc.forward(want[0][0], *args)
    sc.forward(want[0][0], *args, out=parts[0][0])
    assert torch.equal(parts[0][0], attn) and torch.equal(parts[1][0], held[0]) and torch.equal(parts[2][0], held[1])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("rows", [3, 90])
@pytest.mark.parametrize("wide", [0, 60])
def test_forward_takes_values_as_clamped(dev, dtype, d, rows, wide):
    """Lengths and rows that say too much are taken as clamped; positions past the length see all there is."""
    rng = np.random.default_rng(rows)
    store, _, _ = make_store(rng, 12, 2, d, dev)
    table = np.pad(rng.permutation(12).reshape(3, 4), ((0, 0), (0, wide)), constant_values=-1)
    T, room = 2 * rows + 4, 64 * (4 + wide)
    q = torch.randn(6, T, d, generator=torch.Generator().manual_seed(rows)).to(DT[dtype]).to(dev)
    positions = np.concatenate([np.arange(rows), np.arange(rows) + 150, [0, (1 << 31) - 1, -(1 << 31), 999]])
    bad = sc.forward(q, store, i32(table, dev), i32([-(1 << 31), (1 << 31) - 1, 1 << 20], dev), i32([-9, rows, 2 * rows, (1 << 31) - 1], dev),
                     i32(positions, dev), causal_granule=7)
    good = sc.forward(q, store, i32(table, dev), i32([0, room, room], dev), i32([0, rows, 2 * rows, T], dev),
                      i32(np.clip(positions, -1, room), dev), causal_granule=7)
    assert torch.equal(bad, good) and bool(torch.isfinite(good).all())
    assert bool((good[:, :rows] == 0).all()) and bool((good[:, T - 2] == 0).all()) and bool((good[:, T - 3] != 0).any())
    # rows that end before they start are none, and leave what is there
    out = torch.full_like(q, 5.0)
    sc.forward(q, store, i32(table, dev), i32([200] * 3, dev), i32([T, 2, 1, 0], dev), i32(np.clip(positions, 0, 199), dev), out=out)
    assert bool((out == 5.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [2, 100])
def test_forward_pages_twice_and_queries_without_strides(dev, dtype, rows):
    """A page that a request's table names twice is there twice; one query for all heads, one for all tokens."""
    d = 128
    rng = np.random.default_rng(rows)
    store, _, _ = make_store(rng, 3, 2, d, dev)
    copied = torch.cat([store, store[1:2], store[1:2]])
    g = torch.Generator().manual_seed(rows)
    lens, row_start, positions = i32([300], dev), i32([0, rows], dev), i32([299] * rows, dev)
    heads = torch.randn(1, rows, d, generator=g).to(DT[dtype]).to(dev).expand(8, rows, d)
    tokens = torch.randn(8, 1, d, generator=g).to(DT[dtype]).to(dev).expand(8, rows, d)
    for q in (heads, tokens):
        twice = sc.forward(q, store, i32([[1, 0, 1, 2, 1]], dev), lens, row_start, positions)
        apart = sc.forward(q.contiguous(), copied, i32([[1, 0, 3, 2, 4]], dev), lens, row_start, positions)
        assert torch.equal(twice, apart)
