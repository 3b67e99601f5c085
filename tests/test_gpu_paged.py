"""The paged operators on the GPU against their plain definitions in 64 bits (tests/paged_ref.py): each alone at the sizes, masks and
layouts where it can go wrong, then together, captured into a graph, and on what a Locret prefill retains."""
import math

import numpy as np
import pytest
import torch

from paper_2410_01805_amd import binding as B
from paper_2410_01805_amd import synth
from tests import paged_ref as R
from tests.gpu_util import DEV, dev, host, make_layer

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device=DEV)


def tt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def config(dtype="bf16", h=8, h_kv=2, d=64, page=16, n_pages=64, max_reqs=8, max_pages=16, window=0, sink=0, scale=0.0):
    return B.locret_paged_config(h, h_kv, d, B.LOCRET_BF16 if dtype == "bf16" else B.LOCRET_F32, page, n_pages, max_reqs, max_pages, window, sink, scale)


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), **I32)


def numbers(rng, dtype, *shape):
    """Device tensor of storable normal numbers and the same in 64 bits."""
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(tt(dtype))
    return t.to(DEV), t.double().numpy()


# ---- bookkeeping -----------------------------------------------------------------------------------------------------
def plan_state(rng, n_req, page, max_pages, spare, longest=None):
    lens = rng.integers(0, (longest or max_pages * page) + 1, n_req)
    held = -(-lens // page)
    n_pages = int(held.sum()) + spare
    order = rng.permutation(max(1, n_pages))
    table = np.full((n_req, max_pages), -7, dtype=np.int32)
    at = 0
    for r in range(n_req):
        table[r, : held[r]] = order[at: at + held[r]]
        at += held[r]
    free = np.concatenate([order[at:], order[:at]])
    return lens, table, free, n_pages - at if n_pages else 0, max(1, n_pages)


def check_plan(lens, new, table, free, n_free, n_pages, page, max_tokens, in_place):
    n_req, max_pages = table.shape
    want = R.plan(list(lens), list(new), table.tolist(), free.tolist(), n_free, page, max_pages, max_tokens)
    cfg = config(page=page, n_pages=n_pages, max_reqs=max(1, n_req), max_pages=max_pages)
    L, N, Tb, F, nf = ints(lens), ints(new), ints(table), ints(free), ints([n_free])
    L2, nf2 = (L, nf) if in_place else (torch.full_like(L, -5), torch.full_like(nf, -5))
    cu, slots, pos = torch.full((n_req + 1,), -9, **I32), torch.full((max_tokens + 3,), -9, **I32), torch.full((max_tokens + 3,), -9, **I32)
    B.locret_paged_plan(cfg, n_req, L, N, L2, Tb, F, nf, nf2, max_tokens, cu, slots, pos)
    got = dict(lens=L2, table=Tb, free=F, n_free=nf2[0], cu=cu, slots=slots[:max_tokens], positions=pos[:max_tokens])
    for k, v in got.items():
        np.testing.assert_array_equal(v.cpu().numpy(), np.asarray(want[k], dtype=np.int32).reshape(v.shape), err_msg=k)
    assert (slots[max_tokens:] == -9).all() and (pos[max_tokens:] == -9).all()
    return want


@pytest.mark.parametrize("n_req,page,max_pages,spare,new_hi,max_tokens", [
    (1, 16, 4, 4, 1, 1), (3, 16, 5, 40, 40, 200), (48, 64, 30, 200, 1, 48), (200, 32, 9, 500, 100, 9000), (255, 16, 7, 20, 3, 600),
    (257, 128, 3, 60, 200, 30000), (1023, 16, 6, 900, 30, 16000), (4096, 16, 3, 3000, 10, 30000), (4096, 256, 2, 9000, 2, 4096),
    (7, 16, 600, 3000, 5000, 20000), (5, 16, 4, 0, 20, 100), (64, 16, 8, 5000, 30, 333),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan_follows_its_definition(n_req, page, max_pages, spare, new_hi, max_tokens, in_place):
    rng = np.random.default_rng(n_req * 7 + page + max_tokens)
    lens, table, free, n_free, n_pages = plan_state(rng, n_req, page, max_pages, spare)
    new = rng.integers(0, new_hi + 1, n_req)
    new[rng.random(n_req) < 0.15] = -1
    check_plan(lens, new, table, free, n_free, n_pages, page, max_tokens, in_place)


def test_plan_serves_a_prefix_and_skips_rows_that_are_too_short():
    rng = np.random.default_rng(3)
    lens, table, free, n_free, n_pages = plan_state(rng, 6, 16, 4, 3, longest=20)
    # request 1's row cannot hold its tokens, request 3's pages are not there, 4 would need none and still takes nothing
    lens[:] = [5, 20, 0, 16, 17, 3]
    lens, table, free, n_free, n_pages = _state_of(lens, 16, 4, 3)
    out = check_plan(lens, np.array([3, 60, 20, 33, 2, 1]), table, free, n_free, n_pages, 16, 100, False)
    assert out["cu"] == [0, 3, 3, 23, 23, 23, 23]
    # and by tokens
    out = check_plan(lens, np.array([3, 1, 8, 1, 1, 1]), table, free, n_free, n_pages, 16, 11, False)
    assert out["cu"] == [0, 3, 4, 4, 4, 4, 4]
    # pages that are given back are there for the others
    out = check_plan(lens, np.array([-1, -1, 33, 33, -2, 0]), table, free, n_free, n_pages, 16, 100, True)
    assert out["cu"] == [0, 0, 0, 33, 66, 66, 66]


def _state_of(lens, page, max_pages, spare):
    lens = np.asarray(lens)
    held = -(-lens // page)
    n_pages = int(held.sum()) + spare
    order = np.random.default_rng(1).permutation(n_pages)
    table, at = np.full((len(lens), max_pages), -7, dtype=np.int32), 0
    for r in range(len(lens)):
        table[r, : held[r]] = order[at: at + held[r]]
        at += held[r]
    return lens, table, np.concatenate([order[at:], order[:at]]), n_pages - at, n_pages


def test_plan_bounds_its_device_data():
    """Lengths outside 0 .. max_pages * page_size, a free count above the pool, tokens beyond every row, ids that are not the pool's."""
    cfg = config(n_pages=6, max_pages=3, max_reqs=4)
    lens, new = ints([-4, 1000, 5, 0]), ints([2, 1, 2 ** 31 - 1, 0])
    table, free, nf = ints(np.zeros((4, 3))), ints([99, -3, 5, 2, 1, 0]), ints([77])
    out, cu, slots, pos, nf2 = torch.empty(4, **I32), torch.empty(5, **I32), torch.empty(8, **I32), torch.empty(8, **I32), torch.empty(1, **I32)
    B.locret_paged_plan(cfg, 4, lens, new, out, table, free, nf, nf2, 8, cu, slots, pos)
    assert out.tolist() == [2, 48, 5, 0] and cu.tolist() == [0, 2, 2, 2, 2] and nf2.item() == 5
    assert slots.tolist() == [0, 1] + [-1] * 6 and pos.tolist() == [0, 1] + [0] * 6
    free[5] = 99                                            # not a page of the pool: its tokens have no slot
    B.locret_paged_plan(cfg, 4, lens, new, out, table, free, nf, nf2, 8, cu, slots, pos)
    assert slots.tolist() == [-1] * 8 and pos.tolist() == [0, 1] + [0] * 6


def test_plan_without_requests():
    cfg = config(n_pages=6)
    nf, nf2, cu, slots, pos = ints([4]), ints([0]), ints([9]), torch.full((5000,), 3, **I32), torch.full((5000,), 3, **I32)
    B.locret_paged_plan(cfg, 0, None, None, None, None, ints(range(6)), nf, nf2, 5000, cu, slots, pos)
    assert nf2.item() == 4 and cu.item() == 0 and (slots == -1).all() and (pos == 0).all()
    B.locret_paged_plan(cfg, 0, None, None, None, None, ints(range(6)), nf, nf, 0, cu, None, None)
    assert nf.item() == 4


def test_plan_with_the_largest_number_of_tokens():
    most = 2 ** 31 - 1
    cfg = config(n_pages=6, max_pages=3, max_reqs=2)
    slots, pos = torch.full((most,), 3, **I32), torch.full((most,), 3, **I32)
    cu, nf2, out = ints([9] * 3), ints([0]), ints([0, 0])
    B.locret_paged_plan(cfg, 2, ints([0, 17]), ints([20, 3]), out, ints([[-1, -1, -1], [4, 5, -1]]), ints([0, 1, 2, 3, 9, 9]), ints([4]), nf2, most, cu, slots, pos)
    assert nf2.item() == 2 and cu.tolist() == [0, 20, 23] and out.tolist() == [20, 20]
    assert slots[:23].tolist() == [48 + i for i in range(16)] + [32 + i for i in range(4)] + [80 + i for i in range(1, 4)]
    assert pos[:23].tolist() == list(range(20)) + [17, 18, 19]
    assert slots[23:].max().item() == slots[23:].min().item() == -1 and pos[23:].max().item() == pos[23:].min().item() == 0
    del slots, pos
    torch.cuda.empty_cache()


# ---- append ----------------------------------------------------------------------------------------------------------
APPEND = [
    # dtype, h, h_kv, d, T, rot, interleaved, norm, page, strided
    ("bf16", 8, 2, 128, 1, 128, False, False, 16, False), ("bf16", 8, 2, 128, 37, 128, False, True, 64, True),
    ("bf16", 6, 6, 96, 23, 96, False, True, 16, True), ("bf16", 6, 2, 96, 23, 48, False, False, 32, False),
    ("bf16", 4, 1, 64, 50, 64, True, True, 16, True), ("bf16", 12, 2, 32, 9, 32, False, False, 256, False),
    ("bf16", 12, 2, 32, 9, 16, True, True, 16, True), ("bf16", 4, 4, 64, 11, 0, False, True, 16, False),
    ("bf16", 2, 1, 128, 2051, 64, False, True, 128, True), ("f32", 8, 2, 64, 19, 64, False, True, 16, True),
    ("f32", 3, 3, 96, 40, 48, True, True, 32, False), ("f32", 5, 1, 128, 2049, 112, False, False, 16, True),
    ("f32", 2, 2, 32, 1, 16, False, False, 16, False), ("f32", 2, 1, 128, 7, 128, True, False, 16, False),
]


@pytest.mark.parametrize("dtype,h,h_kv,d,T,rot,il,norm,page,strided", APPEND)
def test_append_follows_its_definition(dtype, h, h_kv, d, T, rot, il, norm, page, strided):
    rng = np.random.default_rng(T * 131 + d + rot)
    n_pages = 2 * T // page + 2
    cfg = config(dtype, h, h_kv, d, page, n_pages)
    R_all = h + 2 * h_kv
    x, x64 = numbers(rng, dtype, T, R_all, d)
    if strided:                                            # as one product leaves them, heads side by side
        q, k, v = x[:, :h], x[:, h: h + h_kv], x[:, h + h_kv:]
    else:
        q, k, v = (y.contiguous() for y in (x[:, :h], x[:, h: h + h_kv], x[:, h + h_kv:]))
    positions = rng.integers(0, 1 << 20, T)
    positions[0] = 0
    slots = rng.permutation(n_pages * page)[:T]
    slots[rng.random(T) < 0.2] = -1
    slots[T // 2] = n_pages * page + 5                     # outside the pool
    freq, _ = B.locret_rope_frequencies(rot, 10000.0) if rot else ([], 1.0)
    wq, wk = (1 + 0.3 * rng.standard_normal((2, d)).astype(np.float32)) if norm else (None, None)
    K, K64 = numbers(rng, dtype, n_pages, h_kv, page, d)
    V, V64 = numbers(rng, dtype, n_pages, h_kv, page, d)
    out = torch.full((T + 1, h, d), 7.0, dtype=tt(dtype), device=DEV)
    f32 = lambda w: None if w is None else torch.from_numpy(np.ascontiguousarray(w)).to(DEV)
    B.locret_paged_append(cfg, T, q, k, v, ints(positions), ints(slots), torch.tensor(freq + [0.0], dtype=torch.float64, device=DEV), rot, il, 1.25,
                          f32(wq), f32(wk), 1e-5, out, K, V)
    # sums of d squares, a root and two products before the rotation's two: 2^-19 covers them at d = 128 (a sum of d terms of
    # one sign is off by at most 16 rounded steps in lanes and tree), angles by 2^-24 turns are 2^-21 radians
    rel = 2.0 ** -19
    yq, sq = R.rows(x64[:, :h], wq, 1e-5, positions, freq, rot, il, 1.25)
    yk, sk = R.rows(x64[:, h: h + h_kv], wk, 1e-5, positions, freq, rot, il, 1.25)
    assert (np.abs(host(out[:T]).astype(np.float64) - yq) <= R.STEP[dtype] * np.abs(yq) + rel * sq).all()
    assert (out[T] == 7.0).all()
    tolK = np.zeros_like(K64)
    for t in range(T):
        if 0 <= slots[t] < n_pages * page:
            p, i = divmod(slots[t], page)
            K64[p, :, i], V64[p, :, i] = yk[t], x64[t, h + h_kv:]
            tolK[p, :, i] = R.STEP[dtype] * np.abs(yk[t]) + rel * sk[t]
    assert (np.abs(host(K).astype(np.float64) - K64) <= tolK).all()
    np.testing.assert_array_equal(host(V).astype(np.float64), V64)


def test_append_of_queries_alone_keys_alone_and_in_place():
    rng = np.random.default_rng(5)
    cfg = config("bf16", 4, 2, 64, 16, 4)
    x, _ = numbers(rng, "bf16", 9, 8, 64)
    q, k, v = (y.contiguous() for y in (x[:, :4], x[:, 4:6], x[:, 6:]))
    pos, slots = ints(range(100, 109)), ints(range(9))
    freq = torch.tensor(B.locret_rope_frequencies(64, 10000.0)[0], dtype=torch.float64, device=DEV)
    w = torch.linspace(0.5, 1.5, 64, device=DEV)
    K, V, K2, V2 = (torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device=DEV) for _ in range(4))
    both, alone = torch.empty_like(q), torch.empty_like(q)
    B.locret_paged_append(cfg, 9, q, k, v, pos, slots, freq, 64, False, 1.0, w, w, 1e-6, both, K, V)
    B.locret_paged_append(cfg, 9, q, None, None, pos, None, freq, 64, False, 1.0, w, None, 1e-6, alone, None, None)
    B.locret_paged_append(cfg, 9, None, k, v, pos, slots, freq, 64, False, 1.0, None, w, 1e-6, None, K2, V2)
    assert torch.equal(both, alone) and torch.equal(K, K2) and torch.equal(V, V2)
    B.locret_paged_append(cfg, 9, q, None, None, pos, None, freq, 64, False, 1.0, w, None, 1e-6, q, None, None)
    assert torch.equal(both, q)
    B.locret_paged_append(cfg, 0, q, k, v, pos, slots, freq, 64, False, 1.0, w, w, 1e-6, q, K, V)
    assert torch.equal(both, q)


def test_append_of_more_tokens_than_a_grid_dimension_has_workgroups():
    T = (1 << 24) + 5
    cfg = config("bf16", 1, 1, 32, 16, 2)
    q = torch.randn(T, 1, 32, device=DEV).bfloat16()
    out = torch.zeros_like(q)
    B.locret_paged_append(cfg, T, q, None, None, None, None, None, 0, False, 1.0, None, None, 0.0, out, None, None)
    assert torch.equal(q, out)


# ---- attention -------------------------------------------------------------------------------------------------------
def paged_case(rng, dtype, h, h_kv, d, page, lens, window=0, sink=0, scale=0.0, spread=1.0):
    """Pages in a random order with other numbers everywhere behind the lengths."""
    held = [-(-n // page) for n in lens]
    n_pages, max_pages = sum(held) + 2, max(held + [1]) + 1
    order = rng.permutation(n_pages)
    table, at = rng.integers(-3, n_pages + 3, (len(lens), max_pages)).astype(np.int32), 0
    for r, n in enumerate(held):
        table[r, :n] = order[at: at + n]
        at += n
    K, K64 = numbers(rng, dtype, n_pages, h_kv, page, d)
    V, V64 = numbers(rng, dtype, n_pages, h_kv, page, d)
    cfg = config(dtype, h, h_kv, d, page, n_pages, len(lens), max_pages, window, sink, scale)
    return dict(cfg=cfg, K=K, V=V, K64=K64, V64=V64, table=table, lens=list(lens), dtype=dtype, h=h, h_kv=h_kv, d=d, page=page, window=window,
                sink=sink, scale=scale or 1 / math.sqrt(d))


def units(c, X, r, m):
    """[unit][d] of request r; rows of pages outside the pool are NaN and not seen (second result)."""
    n = c["lens"][r]
    ids = c["table"][r, : -(-n // c["page"])]
    ok = (ids >= 0) & (ids < X.shape[0])
    x = X[np.where(ok, ids, 0), m].reshape(-1, c["d"])[:n]
    return x, np.repeat(ok, c["page"])[:n]


# the decode step's probabilities are two bf16 factors, the second of what the first one leaves
DECODE_FACTOR = 2.0 ** -16


def reference(c, q64, new, factor=None):
    """Outputs, lse and their tolerances for the last new[r] tokens of every request."""
    T, h, d, g = q64.shape[0], c["h"], c["d"], c["h"] // c["h_kv"]
    out, lse, tol, ltol = np.zeros((T, h, d)), np.full((T, h), -np.inf), np.zeros((T, h, d)), np.zeros((T, h))
    t = 0
    for r, k in enumerate(new):
        for m in range(c["h_kv"]):
            K, ok = units(c, c["K64"], r, m)
            V, _ = units(c, c["V64"], r, m)
            for i in range(k):
                see = R.visible(c["lens"][r] - k + i, c["lens"][r], c["window"], c["sink"]) & ok
                for j in range(m * g, (m + 1) * g):
                    out[t + i, j], lse[t + i, j], tol[t + i, j], ltol[t + i, j] = R.attend(q64[t + i, j], K, V, see, c["scale"], c["dtype"],
                                                                                                       factor)
        t += k
    return out, lse, tol, ltol


def close(got, want, tol, what):
    got = got.astype(np.float64)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(all="ignore"):
        bad = ~(same | (np.abs(got - want) <= tol))
    if np.isfinite(want).any():
        with np.errstate(all="ignore"):
            ratio = np.where(same | ~np.isfinite(want), 0, np.abs(got - want) / np.maximum(tol, 1e-300))
        print(f"[paged] {what}: worst {np.nanmax(ratio):.3f} of the bound", flush=True)
    assert not bad.any(), (what, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


def workspace(cfg):
    return torch.empty(B.locret_paged_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)


def run_decode(c, q):
    out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device=DEV)
    B.locret_paged_decode(c["cfg"], len(c["lens"]), q, c["K"], c["V"], ints(c["table"]), ints(c["lens"]), out, lse, workspace(c["cfg"]))
    return host(out), host(lse)


def run_prefill(c, q, cu, rows=None):
    T = q.shape[0]
    out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device=DEV)
    B.locret_paged_prefill(c["cfg"], len(c["lens"]), T, q, c["K"], c["V"], ints(c["table"]), ints(c["lens"]), ints(cu), out, lse, workspace(c["cfg"]))
    return host(out), host(lse)


LENS = [0, 1, 15, 16, 17, 33, 63, 64, 65, 127, 128, 129, 200, 257, 511, 640]
DECODE = [
    # dtype, h, h_kv, d, page, lens, window, sink
    ("bf16", 8, 2, 128, 16, LENS, 0, 0), ("bf16", 32, 8, 128, 64, [3000, 0, 77], 0, 0), ("bf16", 8, 8, 96, 32, LENS, 0, 0),
    ("bf16", 16, 1, 64, 128, LENS, 0, 0), ("bf16", 6, 2, 32, 16, LENS, 0, 0), ("bf16", 40, 2, 128, 16, [300, 5], 0, 0),
    ("bf16", 33, 1, 64, 16, [129, 40, 700], 0, 0), ("bf16", 128, 1, 32, 256, [600], 0, 0),
    ("bf16", 8, 2, 128, 16, LENS, 50, 0), ("bf16", 8, 2, 64, 32, LENS, 100, 4), ("bf16", 12, 4, 96, 16, LENS, 1, 0),
    ("bf16", 8, 2, 128, 64, LENS, 33, 70), ("bf16", 4, 1, 128, 256, [5000, 2500], 129, 300), ("bf16", 4, 2, 32, 16, LENS, 7, 1000),
    ("bf16", 4, 2, 128, 16, [1] * 200, 0, 0), ("bf16", 4, 1, 128, 16, [9000], 0, 0), ("bf16", 2, 1, 64, 16, [20000, 3], 0, 0),
    ("f32", 8, 2, 64, 16, LENS, 0, 0), ("f32", 4, 4, 128, 32, LENS, 40, 3), ("f32", 5, 1, 96, 64, [2000, 1, 0], 0, 0),
    ("f32", 24, 1, 32, 16, LENS, 0, 0), ("f32", 2, 1, 128, 16, [7000, 12], 0, 0),
]


@pytest.mark.parametrize("dtype,h,h_kv,d,page,lens,window,sink", DECODE)
def test_decode_follows_its_definition(dtype, h, h_kv, d, page, lens, window, sink):
    rng = np.random.default_rng(h * 1000 + d + page + len(lens) + window)
    c = paged_case(rng, dtype, h, h_kv, d, page, lens, window, sink)
    q, q64 = numbers(rng, dtype, len(lens), h, d)
    q, q64 = q * 2, q64 * 2
    out, lse = run_decode(c, q)
    want, wl, tol, ltol = reference_with_empty(c, q64)
    close(out, want, tol, "out")
    close(lse, wl, ltol, "lse")


@pytest.mark.parametrize("n", [63, 64, 65, 128])
@pytest.mark.parametrize("ends", [0, 300])
def test_decode_of_about_a_wavefront_of_requests(n, ends):
    rng = np.random.default_rng(n + ends)
    lens = rng.integers(0, 200, n).tolist()
    lens[0] = lens[1] = lens[-2] = lens[-1] = ends
    lens[20] = lens[21] = 0
    lens[40] = 3000
    c = paged_case(rng, "bf16", 8, 2, 64, 16, lens, window=900, sink=3)
    q, q64 = numbers(rng, "bf16", n, 8, 64)
    out, lse = run_decode(c, q)
    want, wl, tol, ltol = reference_with_empty(c, q64)
    close(out, want, tol, "out")
    close(lse, wl, ltol, "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_as_many_requests_as_a_call_takes(dtype):
    rng = np.random.default_rng(90)
    n = B.LOCRET_PAGED_MAX_REQS
    lens = rng.integers(0, 4, n).tolist()
    lens[7] = 700
    c = paged_case(rng, dtype, 16, 1, 128, 16, lens)
    q, q64 = numbers(rng, dtype, n, 16, 128)
    out, lse = run_decode(c, q)
    want, wl, tol, ltol = reference_with_empty(c, q64)
    close(out, want, tol, "decode")
    close(lse, wl, ltol, "decode lse")
    c = paged_case(rng, dtype, 2, 1, 32, 16, lens)
    new = [int(rng.integers(0, x + 1)) for x in lens]
    q, q64 = numbers(rng, dtype, sum(new), 2, 32)
    out, lse = run_prefill(c, q, np.cumsum([0] + new))
    want, wl, tol, ltol = reference(c, q64, new)
    close(out, want, tol, "prefill")
    close(lse, wl, ltol, "prefill lse")


def reference_with_empty(c, q64):
    T, h, d = q64.shape
    some = [r for r, n in enumerate(c["lens"]) if n]
    got = reference(c, q64[some], [1 if n else 0 for n in c["lens"]], DECODE_FACTOR)
    full = np.zeros((T, h, d)), np.full((T, h), -np.inf), np.zeros((T, h, d)), np.zeros((T, h))
    for a, b in zip(full, got):
        a[some] = b
    return full


PREFILL = [
    # dtype, h, h_kv, d, page, lens, new, window, sink
    ("bf16", 8, 2, 128, 16, [100, 1, 65, 0, 300], [100, 1, 30, 0, 7], 0, 0), ("bf16", 8, 8, 96, 32, [70, 200], [70, 64], 0, 0),
    ("bf16", 4, 1, 64, 64, [257, 31], [129, 31], 0, 0), ("bf16", 6, 2, 32, 16, [150, 40, 90], [90, 40, 1], 0, 0),
    ("bf16", 10, 2, 128, 128, [400], [333], 0, 0), ("bf16", 33, 1, 64, 16, [90, 20], [50, 20], 0, 0), ("bf16", 7, 7, 128, 256, [300], [270], 0, 0),
    ("bf16", 8, 2, 128, 16, [300, 64], [260, 10], 50, 0), ("bf16", 8, 2, 64, 32, [500, 130], [90, 130], 64, 4), ("bf16", 4, 2, 96, 16, [200], [150], 1, 3),
    ("bf16", 4, 1, 128, 64, [700, 350], [40, 350], 65, 130), ("bf16", 4, 4, 32, 16, [333], [333], 20, 1000), ("bf16", 8, 2, 128, 64, [3000], [5], 0, 0),
    ("bf16", 8, 1, 128, 16, [2500, 60], [64, 3], 0, 0), ("bf16", 4, 2, 64, 16, [5000], [33], 2000, 70), ("bf16", 128, 1, 64, 16, [40], [9], 0, 0),
    ("f32", 8, 2, 64, 16, [100, 1, 65, 0], [100, 1, 30, 0], 0, 0), ("f32", 3, 1, 128, 32, [200, 77], [60, 77], 50, 3),
    ("f32", 4, 4, 96, 64, [130], [130], 0, 0), ("f32", 12, 2, 32, 16, [150, 33], [150, 1], 7, 1), ("f32", 2, 1, 128, 16, [2100], [20], 0, 0),
]


@pytest.mark.parametrize("dtype,h,h_kv,d,page,lens,new,window,sink", PREFILL)
def test_prefill_follows_its_definition(dtype, h, h_kv, d, page, lens, new, window, sink):
    rng = np.random.default_rng(h * 1000 + d + page + sum(new) + window)
    c = paged_case(rng, dtype, h, h_kv, d, page, lens, window, sink)
    first, T = 3, sum(new)                                 # rows in front of the first request and behind the last one belong to nobody
    q, q64 = numbers(rng, dtype, T + 8, h, d)
    q, q64 = q * 2, q64 * 2
    cu = first + np.cumsum([0] + new)
    out, lse = run_prefill(c, q, cu)
    want, wl, tol, ltol = reference(c, q64[first: first + T], new)
    close(out[first: first + T], want, tol, "out")
    close(lse[first: first + T], wl, ltol, "lse")
    for x in (out, lse):
        assert (x[:first] == 9).all() and (x[first + T:] == 9).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 96), ("bf16", 64), ("bf16", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("window,sink", [(0, 0), (40, 5)])
@pytest.mark.parametrize("what", ["nan", "inf", "lowest"])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_what_is_masked_does_not_reach_the_result(dtype, d, window, sink, what, page):
    """Not-a-number, infinite and lowest values behind the lengths, in later tokens and in front of the window; the tokens that do see such a
    value row get what the definition gives them."""
    rng = np.random.default_rng(d + window)
    lens, new = [150, 37, 64], [100, 37, 3]
    c = paged_case(rng, dtype, 4, 2, d, page, lens, window, sink)
    bad = {"nan": float("nan"), "inf": float("inf"), "lowest": torch.finfo(tt(dtype)).min}[what]
    at = [(0, 120), (0, 60), (1, 20), (2, 63), (2, 9), (0, 149)]
    for r, u in at:
        p, i = c["table"][r, u // page], u % page
        # (values that are seen are at most 2^64 in size)
        seen = bad if what != "lowest" else -2.0 ** 64
        c["V"][p, 1, i, :: 3] = seen
        c["V64"][p, 1, i, :: 3] = seen
    for r, n in enumerate(lens):                           # behind the lengths, keys too
        p, i = c["table"][r, (n - 1) // page], (n - 1) % page + 1
        c["V"][p, :, i:], c["K"][p, :, i:] = bad, bad
        c["V64"][p, :, i:], c["K64"][p, :, i:] = bad, bad
    spare = [p for p in range(c["K"].shape[0]) if p not in {c["table"][r, k] for r, n in enumerate(lens) for k in range(-(-n // page))}]
    for p in spare:
        c["K"][p], c["V"][p] = bad, bad
    q, q64 = numbers(rng, dtype, sum(new), 4, d)
    cu = np.cumsum([0] + new)
    out, lse = run_prefill(c, q, cu)
    want, wl, tol, ltol = reference(c, q64, new)
    close(out, want, tol, "prefill")
    close(lse, wl, ltol, "prefill lse")
    last = cu[1:] - 1
    out, lse = run_decode(c, q[torch.from_numpy(last).to(DEV)].contiguous())
    want, wl, tol, ltol = reference(c, q64[last], [1, 1, 1])
    close(out, want, tol, "decode")
    close(lse, wl, ltol, "decode lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_pages_outside_the_pool_are_not_seen(dtype, page):
    rng = np.random.default_rng(11)
    c = paged_case(rng, dtype, 4, 2, 64, page, [150 * page // 16, 40, 20])
    c["table"][0, [2, 5]] = [-1, 1 << 27]
    c["table"][1, : -(-40 // page)] = c["K"].shape[0]      # nothing is left of this request
    new = [9, 40, 2]
    q, q64 = numbers(rng, dtype, sum(new), 4, 64)
    out, lse = run_prefill(c, q, np.cumsum([0] + new))
    want, wl, tol, ltol = reference(c, q64, new)
    assert (out[9:49] == 0).all() and np.isneginf(lse[9:49]).all()
    close(out, want, tol, "prefill")
    close(lse, wl, ltol, "prefill lse")
    last = torch.tensor([8, 48, 50], device=DEV)
    out, lse = run_decode(c, q[last].contiguous())
    want, wl, tol, ltol = reference(c, q64[[8, 48, 50]], [1, 1, 1])
    close(out, want, tol, "decode")
    close(lse, wl, ltol, "decode lse")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 96)])
def test_logits_of_any_size(dtype, d):
    """Large logits late and early, rows whose visible logits are all far below the hidden ones, and a scale of its own."""
    rng = np.random.default_rng(d)
    c = paged_case(rng, dtype, 4, 2, d, 16, [400, 200], 60, 3, scale=0.5)
    for r, u in [(0, 5), (0, 130), (0, 399), (1, 180)]:
        p, i = c["table"][r, u // 16], u % 16
        c["K"][p, :, i] *= 24
        c["K64"][p, :, i] = host(c["K"][p, :, i])           # as stored: 24 times a bf16 number is rounded
    new = [300, 60]
    q, q64 = numbers(rng, dtype, sum(new), 4, d)
    out, lse = run_prefill(c, q, np.cumsum([0] + new))
    want, wl, tol, ltol = reference(c, q64, new)
    close(out, want, tol, "prefill")
    close(lse, wl, ltol, "prefill lse")
    last = torch.tensor([299, 359], device=DEV)
    out, lse = run_decode(c, q[last].contiguous())
    want, wl, tol, ltol = reference(c, q64[[299, 359]], [1, 1])
    close(out, want, tol, "decode")
    close(lse, wl, ltol, "decode lse")


def test_cu_new_is_taken_within_the_tokens_and_more_new_tokens_than_units_see_nothing():
    rng = np.random.default_rng(2)
    c = paged_case(rng, "bf16", 4, 2, 64, 16, [5, 30, 30])
    q, q64 = numbers(rng, "bf16", 20, 4, 64)
    out, lse = run_prefill(c, q, [-3, 8, 14, 900])        # requests of 8, 6 and 6 tokens
    assert (out[:3] == 0).all() and np.isneginf(lse[:3]).all()
    c2 = dict(c, lens=[5, 30, 30])
    want, wl, tol, ltol = reference(c2, q64[3:], [5, 6, 6])
    close(out[3:], want, tol, "out")
    close(lse[3:], wl, ltol, "lse")


def test_lengths_are_taken_within_the_row():
    rng = np.random.default_rng(4)
    c = paged_case(rng, "bf16", 4, 2, 64, 16, [64, 20])
    full = int(c["cfg"].max_pages) * 16
    order = rng.integers(0, c["K"].shape[0], c["table"].shape)
    c["table"][:] = order
    q, q64 = numbers(rng, "bf16", 2, 4, 64)
    c["lens"] = [full + 999, -5]
    out, lse = run_decode(c, q)
    c["lens"] = [full, 0]
    want, wl, tol, ltol = reference_with_empty(c, q64)
    close(out, want, tol, "out")
    close(lse, wl, ltol, "lse")


def test_a_chunk_of_many_rows_on_a_long_cache_of_small_pages():
    """More page numbers than a workgroup keeps at hand (4096), and no parts; sampled rows."""
    rng = np.random.default_rng(77)
    n, new = 70001, 4400
    c = paged_case(rng, "bf16", 8, 8, 32, 16, [n])
    q, q64 = numbers(rng, "bf16", new, 8, 32)
    out, lse = run_prefill(c, q, [0, new])
    rows = [0, 1, 63, 255, 256, 2047, 4350, 4399]
    KV = [[units(c, c[x], 0, m)[0] for m in range(8)] for x in ("K64", "V64")]
    for t in rows:
        see = R.visible(n - new + t, n, 0, 0)
        for j in range(8):
            want, wl, tol, ltol = R.attend(q64[t, j], KV[0][j], KV[1][j], see, c["scale"], "bf16")
            close(out[t, j], want, tol, f"row {t} head {j}")
            assert abs(lse[t, j] - wl) <= ltol


def test_units_behind_four_gigabytes_of_the_pool():
    """Pages whose offset passes 32 bits."""
    page, h_kv, d = 256, 8, 128
    n_pages = (1 << 32) // (page * h_kv * d * 2) + 40      # 512 KB a page: 4 GB and some
    cfg = config("bf16", 16, h_kv, d, page, n_pages, 2, 4)
    K = torch.zeros(n_pages, h_kv, page, d, dtype=torch.bfloat16, device=DEV)
    V = torch.zeros_like(K)
    rng = np.random.default_rng(8)
    lens, new = [700, 300], [10, 300]
    table = np.array([[n_pages - 1, 3, n_pages - 20, 0], [n_pages - 2, n_pages - 7, 1, 0]], dtype=np.int32)
    k, k64 = numbers(rng, "bf16", sum(lens), h_kv, d)
    v, v64 = numbers(rng, "bf16", sum(lens), h_kv, d)
    slots = np.concatenate([table[r, np.arange(n) // page] * page + np.arange(n) % page for r, n in enumerate(lens)])
    B.locret_paged_append(cfg, sum(lens), None, k, v, None, ints(slots), None, 0, False, 1.0, None, None, 0.0, None, K, V)
    q, q64 = numbers(rng, "bf16", sum(new), 16, d)
    small = sorted(set(table.flatten().tolist()))
    at = {p: i for i, p in enumerate(small)}
    idx = torch.tensor(small, device=DEV)
    c = dict(cfg=cfg, K=K, V=V, K64=host(K[idx]).astype(np.float64), V64=host(V[idx]).astype(np.float64), dtype="bf16", h=16, h_kv=h_kv, d=d, page=page,
             window=0, sink=0, scale=1 / math.sqrt(d), lens=lens, table=table)
    out, lse = run_prefill(c, q, np.cumsum([0] + new))
    last = torch.tensor([9, 309], device=DEV)
    dec, dlse = run_decode(c, q[last].contiguous())
    c["table"] = np.vectorize(at.get)(table)
    want, wl, tol, ltol = reference(c, q64, new)
    close(out, want, tol, "prefill")
    close(lse, wl, ltol, "prefill lse")
    close(dec, want[[9, 309]], tol[[9, 309]], "decode")
    close(dlse, wl[[9, 309]], ltol[[9, 309]], "decode lse")


# ---- together --------------------------------------------------------------------------------------------------------
def dense_reference(tokens, freq, rot, weights, new, window, sink, dtype, g):
    """Attention outputs of the last `new` tokens of one request, from its raw q, k, v in 64 bits.  Stored keys and queries are rounded to the
    type, which the reference does too, so that the tolerance is that of the attention alone."""
    q, k, v = tokens
    n, d = q.shape[0], q.shape[2]
    pos = np.arange(n)
    store = lambda x: torch.from_numpy(x).to(tt(dtype)).double().numpy()
    qr, kr = store(R.rows(q, weights[0], 1e-6, pos, freq, rot, False, 1.0)[0]), store(R.rows(k, weights[1], 1e-6, pos, freq, rot, False, 1.0)[0])
    out, tol = np.zeros((new, q.shape[1], d)), np.zeros((new, q.shape[1], d))
    for i in range(new):
        see = R.visible(n - new + i, n, window, sink)
        for j in range(q.shape[1]):
            out[i, j], _, tol[i, j], _ = R.attend(qr[n - new + i, j], kr[:, j // g], v[:, j // g], see, 1 / math.sqrt(d), dtype)
    return out, tol


@pytest.mark.parametrize("dtype,window,sink", [("bf16", 0, 0), ("bf16", 48, 4), ("f32", 0, 0)])
def test_a_run_of_all_of_them(dtype, window, sink):
    """Prompts arrive, are continued in chunks and generated, finish and give their pages to others."""
    h, h_kv, d, page = 8, 2, 64, 16
    rng = np.random.default_rng(21)
    cfg = config(dtype, h, h_kv, d, page, n_pages=40, max_reqs=3, max_pages=16, window=window, sink=sink)
    cache = B.PagedCache(cfg, DEV, rope=dict(rotary_dim=64, theta=10000.0))
    freq = B.locret_rope_frequencies(64, 10000.0)[0]
    w = 1 + 0.2 * rng.standard_normal((2, d)).astype(np.float32)
    wq, wk = (torch.from_numpy(x).to(DEV) for x in w)
    streams = [[np.zeros((0, h, d)), np.zeros((0, h_kv, d)), np.zeros((0, h_kv, d))] for _ in range(3)]
    steps = [[70, 33, 0], [50, 1, 90], [1, 1, 1], [1, 1, 1], [1, -1, 1], [1, 40, -1], [1, 1, 17], [1, 1, 1]]
    for new in steps:
        T = sum(max(n, 0) for n in new)
        x, x64 = numbers(rng, dtype, T, h + 2 * h_kv, d)
        cu, slots, pos = cache.plan(ints(new), T + 2)
        slots, pos = slots[:T], pos[:T]
        q = cache.append(x[:, :h], x[:, h: h + h_kv], x[:, h + h_kv:], pos, slots, wq, wk)
        one = all(n == 1 for n in new)
        out = host(cache.decode(q) if one else cache.prefill(q, cu))
        t = 0
        for r, n in enumerate(new):
            if n < 0:
                streams[r] = [y[:0] for y in streams[r]]
            n = max(n, 0)
            for i, (lo, hi) in enumerate(((0, h), (h, h + h_kv), (h + h_kv, h + 2 * h_kv))):
                streams[r][i] = np.concatenate([streams[r][i], x64[t: t + n, lo: hi]])
            if n:
                want, tol = dense_reference(streams[r], freq, 64, w, n, window, sink, dtype, h // h_kv)
                # keys and queries that lie within a rounding of two neighbours may be stored a step apart: 2^-8 (2^-24) of a logit's summands
                # in few of them, an eighth of the sum of sizes covers it (bf16 logits of these normed rows are at most 8)
                close(out[t: t + n], want, tol + (0.02 if dtype == "bf16" else 1e-5), f"request {r} of {new}")
            t += n
        assert cache.lens.tolist() == [s[0].shape[0] for s in streams]
        assert cache.n_free.item() == 40 - sum(-(-s[0].shape[0] // page) for s in streams)


def test_a_captured_decode_step_is_replayed_as_the_cache_grows():
    """plan, append and decode as one graph: lengths, tables and slots move on the device from replay to replay; eager work in between."""
    h, h_kv, d, page = 8, 2, 128, 16
    rng = np.random.default_rng(31)
    mk = lambda: B.PagedCache(config("bf16", h, h_kv, d, page, 64, 4, 16), DEV, rope=dict(rotary_dim=128, theta=500000.0))
    a, b = mk(), mk()
    prompt = [40, 15, 1, 96]
    x, _ = numbers(rng, "bf16", sum(prompt), h + 2 * h_kv, d)
    for c in (a, b):
        cu, slots, pos = c.plan(ints(prompt), sum(prompt))
        q = c.append(x[:, :h], x[:, h: h + h_kv], x[:, h + h_kv:], pos, slots)
        c.prefill(q, cu)
    one = ints([1, 1, 1, 1])
    x = torch.zeros(4, h + 2 * h_kv, d, dtype=torch.bfloat16, device=DEV)

    def step(c):
        _, slots, pos = c.plan(one, 4)
        return c.decode(c.append(x[:, :h], x[:, h: h + h_kv], x[:, h + h_kv:], pos, slots), want_lse=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm = mk()
        step(warm)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(a)
    for i in range(9):
        x.copy_(numbers(rng, "bf16", 4, h + 2 * h_kv, d)[0])
        graph.replay()
        torch.cuda.synchronize()
        want = step(b)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), i
        assert torch.equal(a.lens, b.lens) and torch.equal(a.n_free, b.n_free)


def test_a_captured_prefill_is_replayed():
    rng = np.random.default_rng(32)
    c = paged_case(rng, "bf16", 8, 2, 64, 16, [200, 90])
    q, _ = numbers(rng, "bf16", 100, 8, 64)
    table, lens, cu, out, lse, ws = ints(c["table"]), ints(c["lens"]), ints([0, 60, 100]), torch.zeros_like(q), torch.zeros(100, 8, device=DEV), workspace(c["cfg"])
    call = lambda o, l: B.locret_paged_prefill(c["cfg"], 2, 100, q, c["K"], c["V"], table, lens, cu, o, l, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse)
    for i in range(4):
        q.copy_(numbers(rng, "bf16", 100, 8, 64)[0])
        cu.copy_(ints([[0, 60, 100], [5, 5, 95], [0, 100, 100], [0, 99, 100]][i]))
        out.fill_(3.0)
        lse.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        o, l = torch.full_like(q, 3.0), torch.full_like(lse, 3.0)
        call(o, l)
        assert torch.equal(out, o) and torch.equal(lse, l), i


@pytest.mark.parametrize("dtype,d,h,h_kv,rope", [("bf16", 128, 8, 2, True), ("bf16", 96, 6, 6, True), ("bf16", 64, 4, 1, False), ("f32", 64, 8, 2, True)])
def test_what_a_prefill_retains_is_generated_from_pages(dtype, d, h, h_kv, rope):
    """Two streams of their own contexts, evicted to their budgets, adopted into one pool and generated together: each token's output is
    that of locret_decode_step, up to what bf16 factors differ by."""
    theta = 10000.0
    ws = [synth.tiny(name=f"adopt{i}", dtype=dtype, h=h, h_kv=h_kv, d=d, N=300 + 40 * i, B=100, b=180 + 40 * i, n_s=20, d_R=128, rope=rope, theta=theta)
          for i in range(2)]
    cfg = config(dtype, h, h_kv, d, 16, n_pages=64, max_reqs=2, max_pages=24)
    cache = B.PagedCache(cfg, DEV, rope=dict(rotary_dim=d, theta=theta) if rope else None)
    layers = []
    for r, w in enumerate(ws):
        layer, _, _ = make_layer(w)
        lo = 0
        while lo < w.N:
            hi = min(w.N, lo + w.B)
            layer.prefill_chunk(*(dev(x, w) for x in synth.tokens(w, lo, hi)), w.n_s)
            lo = hi
        cache.adopt(layer, r)
        layers.append(layer)
    assert cache.lens.tolist() == [w.b for w in ws]
    rng = np.random.default_rng(6)
    for step in range(20):
        x, _ = numbers(rng, dtype, 2, h + 2 * h_kv, d)
        want = torch.cat([layer.decode_step(*(y[r: r + 1].contiguous() for y in (x[:, :h], x[:, h: h + h_kv], x[:, h + h_kv:])))[0]
                          for r, layer in enumerate(layers)])
        _, slots, pos = cache.plan(ints([1, 1]), 2)
        got = cache.decode(cache.append(x[:, :h], x[:, h: h + h_kv], x[:, h + h_kv:], pos, slots))
        got, want = host(got).astype(np.float64), host(want).astype(np.float64)
        # locret_decode_step rounds a query after scaling it: every product of a logit is off by at most 2^-8, at random, the logit by
        # 2^-8 / sqrt(3) in standard deviation (they are normal numbers of size 1), an output by as much of its row's size, since it is a sum
        # over units of independent errors; five of those are 0.012.  Probabilities as 16-bit factors add as much here, the two outputs'
        # rounding 2^-7: 0.03, taken twice.  In float32 the same with 2^-24 and sums of up to 128 terms: 2^-17, taken twice.
        size = np.sqrt((want ** 2).mean(-1, keepdims=True))
        tol = (0.06 if dtype == "bf16" else 2.0 ** -16) * (size + np.abs(want))
        close(got, want, tol, f"token {step}")


def test_calls_on_another_stream():
    rng = np.random.default_rng(41)
    c = paged_case(rng, "bf16", 8, 2, 64, 16, [200, 90])
    q, _ = numbers(rng, "bf16", 2, 8, 64)
    want = run_decode(c, q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run_decode(c, q)
    side.synchronize()
    np.testing.assert_array_equal(got[0], want[0])
    out, ws = torch.empty_like(q), workspace(c["cfg"])
    table, lens = ints(c["table"]), ints(c["lens"])
    torch.cuda.synchronize()
    B.locret_paged_decode(c["cfg"], 2, q, c["K"], c["V"], table, lens, out, None, ws, stream=side)
    side.synchronize()
    np.testing.assert_array_equal(host(out), want[0])


def test_calls_at_once_with_a_workspace_each():
    """Decode and prefill on two streams together, many times, against the same calls one after the other."""
    rng = np.random.default_rng(43)
    c = paged_case(rng, "bf16", 8, 2, 128, 16, [3000, 900, 40])
    q, _ = numbers(rng, "bf16", 90, 8, 128)
    table, lens, cu = ints(c["table"]), ints(c["lens"]), ints([0, 40, 75, 90])
    ws = [workspace(c["cfg"]) for _ in range(2)]
    outs = [[torch.zeros_like(q) for _ in range(2)] for _ in range(2)]

    def call(i, o):
        if i == 0:
            B.locret_paged_decode(c["cfg"], 3, q[:3], c["K"], c["V"], table, lens, o[:3], None, ws[0])
        else:
            B.locret_paged_prefill(c["cfg"], 3, 90, q, c["K"], c["V"], table, lens, cu, o, None, ws[1])

    for i in range(2):
        call(i, outs[0][i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                call(i, outs[1][i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[0][i], outs[1][i])


def test_the_same_request_twice_in_a_batch():
    """Two rows of the block table with the same pages (a shared prompt)."""
    rng = np.random.default_rng(44)
    c = paged_case(rng, "bf16", 8, 2, 64, 32, [500, 500, 100], 200, 4)
    c["table"][1] = c["table"][0]
    q, q64 = numbers(rng, "bf16", 60, 8, 64)
    new = [25, 25, 10]
    out, lse = run_prefill(c, q, np.cumsum([0] + new))
    want, wl, tol, ltol = reference(c, q64, new)
    close(out, want, tol, "prefill")
    close(lse, wl, ltol, "prefill lse")


def test_results_do_not_depend_on_what_the_workspace_held():
    rng = np.random.default_rng(42)
    c = paged_case(rng, "bf16", 4, 1, 128, 16, [9000, 500])
    q, _ = numbers(rng, "bf16", 64, 4, 128)
    table, lens, cu = ints(c["table"]), ints(c["lens"]), ints([0, 40, 64])
    for n, call in ((2, lambda o, ws: B.locret_paged_decode(c["cfg"], 2, q[:2], c["K"], c["V"], table, lens, o, None, ws)),
                    (64, lambda o, ws: B.locret_paged_prefill(c["cfg"], 2, 64, q, c["K"], c["V"], table, lens, cu, o, None, ws))):
        outs = []
        for fill in (0, 255):
            ws = torch.full((B.locret_paged_workspace_bytes(c["cfg"]),), fill, dtype=torch.uint8, device=DEV)
            o = torch.empty_like(q[:n])
            call(o, ws)
            call(o, ws)
            outs.append(o)
        assert torch.equal(*outs)


# ---- the ends of what a call takes -----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 64), ("bf16", 96, 16), ("bf16", 64, 128), ("bf16", 32, 16), ("f32", 64, 16)])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 120, 2 ** 30, "row", "row - 1"])
@pytest.mark.parametrize("sink", [0, 5, 2 ** 31 - 1])
def test_windows_longer_than_the_requests(dtype, d, page, window, sink):
    """Windows up to the largest number, as long as a row of the block table and one less: all units up to a token's own are seen."""
    rng = np.random.default_rng(d + page)
    lens, new = [200, 3, 90, 1], [200, 3, 20, 1]
    c = paged_case(rng, dtype, 8, 2, d, page, lens)
    row = c["cfg"].max_pages * page
    c["cfg"].window = {"row": row, "row - 1": row - 1}.get(window, window)
    c["cfg"].n_sink = sink
    q, q64 = numbers(rng, dtype, sum(new), 8, d)
    cu = np.cumsum([0] + new)
    out, lse = run_prefill(c, q, cu)
    want, wl, tol, ltol = reference(c, q64, new)
    close(out, want, tol, "prefill")
    close(lse, wl, ltol, "prefill lse")
    last = cu[1:] - 1
    out, lse = run_decode(c, q[torch.from_numpy(last).to(DEV)].contiguous())
    want, wl, tol, ltol = reference(c, q64[last], [1] * 4, DECODE_FACTOR)
    close(out, want, tol, "decode")
    close(lse, wl, ltol, "decode lse")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("window", [0, 1, 20, 2 ** 31 - 1])
@pytest.mark.parametrize("sink", [0, 3, 2 ** 31 - 1])
def test_chunks_longer_than_their_requests(dtype, d, window, sink):
    """Tokens in front of a request's first unit see nothing, with windows and sinks of any size; the others see what they do elsewhere."""
    rng = np.random.default_rng(d + 1)
    lens, new = [5, 70, 0, 33], [40, 70, 6, 300]
    c = paged_case(rng, dtype, 8, 2, d, 16, lens, window, sink)
    q, q64 = numbers(rng, dtype, sum(new), 8, d)
    cu = np.cumsum([0] + new)
    out, lse = run_prefill(c, q, cu)
    some = [min(k, n) for k, n in zip(new, lens)]          # the last ones of each
    there = np.concatenate([np.arange(cu[r + 1] - k, cu[r + 1]) for r, k in enumerate(some)])
    want, wl, tol, ltol = reference(c, q64[there], some)
    close(out[there], want, tol, "out")
    close(lse[there], wl, ltol, "lse")
    rest = np.setdiff1d(np.arange(sum(new)), there)
    assert (out[rest] == 0).all() and np.isneginf(lse[rest]).all()


# ---- adopting what a context retained --------------------------------------------------------------------------------
def retained(n=150, budget=90):
    """A context that has evicted to its budget."""
    w = synth.tiny(name="adopted", dtype="bf16", h=8, h_kv=2, d=64, N=n, B=50, b=budget, n_s=10, d_R=128, rope=True, theta=10000.0)
    layer, _, _ = make_layer(w)
    for lo in range(0, w.N, w.B):
        layer.prefill_chunk(*(dev(x, w) for x in synth.tokens(w, lo, min(w.N, lo + w.B))), w.n_s)
    return layer


@pytest.mark.parametrize("n_pages,max_pages,taken,code", [
    (5, 16, 0, B.LOCRET_ENOMEM),      # 90 units are 6 pages of 16
    (8, 16, 37, B.LOCRET_ENOMEM),     # 3 pages belong to another request
    (20, 5, 0, B.LOCRET_ESHAPE),      # a row holds 80 units
    (3, 5, 0, B.LOCRET_ESHAPE),       # both
])
def test_adopt_refuses_what_the_pool_cannot_hold(n_pages, max_pages, taken, code):
    """An error, a pool that stays as it was, and one that goes on to be used."""
    layer = retained()
    assert layer.cache_len == 90
    cache = B.PagedCache(config("bf16", 8, 2, 64, 16, n_pages, 3, max_pages), DEV, rope=dict(rotary_dim=64, theta=10000.0))
    cache.K.fill_(3.0)
    cache.V.fill_(4.0)
    if taken:
        cache.plan(ints([taken]), taken)
    state = lambda: [x.clone() for x in (cache.K, cache.V, cache.block_table, cache.lens, cache.free_pages, cache.n_free)]
    before = state()
    with pytest.raises(B.LocretError) as e:
        cache.adopt(layer, 1)
    assert e.value.code == code
    assert all(torch.equal(a, b) for a, b in zip(before, state()))
    cu, slots, _ = cache.plan(ints([0, 20]), 20)
    assert cu.tolist() == [0, 0, 20] and (slots >= 0).all()


def test_adopt_behind_units_that_fill_the_row_to_its_end():
    layer = retained()
    cache = B.PagedCache(config("bf16", 8, 2, 64, 16, 40, 2, 7), DEV, rope=dict(rotary_dim=64, theta=10000.0))
    cache.plan(ints([0, 22]), 22)                          # 22 + 90 units: the row's 112
    cache.adopt(layer, 1)
    assert cache.lens.tolist() == [0, 112] and cache.n_free.item() == 33
    with pytest.raises(B.LocretError) as e:
        cache.adopt(layer, 1)
    assert e.value.code == B.LOCRET_ESHAPE and cache.lens.tolist() == [0, 112] and cache.n_free.item() == 33
    cache.adopt(layer, 0)
    assert cache.lens.tolist() == [90, 112]


def test_adopt_of_a_context_on_a_device_without_a_number():
    """"cuda" is the current device, for the pool and for the context."""
    layer = retained()
    cache = B.PagedCache(config("bf16", 8, 2, 64, 16, 20, 2, 16), "cuda", rope=dict(rotary_dim=64, theta=10000.0))
    cache.adopt(layer, 0)
    other = B.LocretLayer(layer.cfg, "cuda")
    other.set_weights(*(torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in ((12 * 64, 128), (128, 2))))
    x = torch.randn(10, 12, 64, device=DEV).bfloat16()
    other.prefill_chunk(x[:, :8].contiguous(), x[:, 8:10].contiguous(), x[:, 10:].contiguous(), 1)
    cache.adopt(other, 1)
    assert cache.lens.tolist() == [90, 10]


# ---- strides that lead nowhere ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_one_token_of_a_fused_product(dtype):
    """In place on one token's slice, which is dense whatever its token stride, and with a token stride that no vector load could take."""
    rng = np.random.default_rng(61)
    h, h_kv, d = 8, 2, 64
    cfg = config(dtype, h, h_kv, d, 16, 4)
    pos, slots = ints([77]), ints([21])
    freq = torch.tensor(B.locret_rope_frequencies(d, 10000.0)[0], dtype=torch.float64, device=DEV)
    x, _ = numbers(rng, dtype, 1, h + 2 * h_kv, d)
    want, K, V, K2, V2 = (torch.zeros(s, dtype=tt(dtype), device=DEV) for s in ((1, h, d), *((4, h_kv, 16, d),) * 4))
    parts = lambda y: (y[:, :h], y[:, h: h + h_kv], y[:, h + h_kv:])
    B.locret_paged_append(cfg, 1, *(y.contiguous() for y in parts(x)), pos, slots, freq, d, False, 1.0, None, None, 0.0, want, K, V)
    for stride in (12 * d, 7, 0):
        y = x.clone()
        q, k, v = (z.as_strided((1, z.shape[1], d), (stride, d, 1)) for z in parts(y))
        B.locret_paged_append(cfg, 1, q, k, v, pos, slots, freq, d, False, 1.0, None, None, 0.0, q, K2, V2)
        assert torch.equal(q, want) and torch.equal(K, K2) and torch.equal(V, V2), stride
        assert torch.equal(y[:, h:], x[:, h:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_one_head(dtype):
    rng = np.random.default_rng(62)
    T, d = 9, 32
    cfg = config(dtype, 1, 1, d, 16, 4)
    pos, slots = ints(range(T)), ints(range(5, 5 + T))
    freq = torch.tensor(B.locret_rope_frequencies(d, 10000.0)[0], dtype=torch.float64, device=DEV)
    x, _ = numbers(rng, dtype, T, 3, d)
    want, got, K, V, K2, V2 = (torch.zeros(s, dtype=tt(dtype), device=DEV) for s in (*((T, 1, d),) * 2, *((4, 1, 16, d),) * 4))
    q, k, v = (x[:, i: i + 1] for i in range(3))
    B.locret_paged_append(cfg, T, q.contiguous(), k.contiguous(), v.contiguous(), pos, slots, freq, d, False, 1.0, None, None, 0.0, want, K, V)
    q, k, v = (y.as_strided((T, 1, d), (3 * d, 1, 1)) for y in (q, k, v))
    B.locret_paged_append(cfg, T, q, k, v, pos, slots, freq, d, False, 1.0, None, None, 0.0, got, K2, V2)
    assert torch.equal(got, want) and torch.equal(K, K2) and torch.equal(V, V2)
    q = q.contiguous()                                     # in place, where the head stride is no more looked at
    B.locret_paged_append(cfg, T, q.data_ptr(), None, None, pos.data_ptr(), None, freq.data_ptr(), d, False, 1.0, None, None, 0.0, q.data_ptr(), None, None,
                          strides=[d, 5, 0, 0, 0, 0])
    assert torch.equal(q, want)
    with pytest.raises(B.LocretError) as e:                # the token stride is
        B.locret_paged_append(cfg, T, q.data_ptr(), None, None, pos.data_ptr(), None, freq.data_ptr(), d, False, 1.0, None, None, 0.0, q.data_ptr(), None, None,
                              strides=[2 * d, d, 0, 0, 0, 0])
    assert e.value.code == B.LOCRET_EINVAL


def test_addresses_and_tensors_in_one_call():
    """Any argument may be an address beside tensors; results are those of tensors alone."""
    rng = np.random.default_rng(63)
    c = paged_case(rng, "bf16", 8, 2, 64, 16, [70, 33])
    q, _ = numbers(rng, "bf16", 20, 8, 64)
    table, lens, cu, ws = ints(c["table"]), ints(c["lens"]), ints([0, 12, 20]), workspace(c["cfg"])
    calls = {
        "decode": lambda o, l, f: B.locret_paged_decode(c["cfg"], 2, *(f(i, x) for i, x in enumerate((q, c["K"], c["V"], table, lens, o, l, ws))),
                                                        workspace_bytes=ws.nbytes),
        "prefill": lambda o, l, f: B.locret_paged_prefill(c["cfg"], 2, 20, *(f(i, x) for i, x in enumerate((q, c["K"], c["V"], table, lens, cu, o, l, ws))),
                                                          workspace_bytes=ws.nbytes),
    }
    for what, call in calls.items():
        n = 2 if what == "decode" else 20
        mk = lambda: (torch.zeros(n, 8, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(n, 8, device=DEV))
        want, got = mk(), mk()
        call(*want, lambda i, x: x)
        for keep in range(8):                              # one tensor left
            for x in got:
                x.zero_()
            call(*got, lambda i, x: x if i == keep else x.data_ptr())
            assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]), (what, keep)
    x, _ = numbers(rng, "bf16", 5, 12, 64)
    k, v, pos, slots = x[:, 8:10].contiguous(), x[:, 10:].contiguous(), ints(range(5)), ints(range(3, 8))
    want, got = torch.empty_like(q[:5]), torch.empty_like(q[:5])
    freq = torch.tensor(B.locret_rope_frequencies(64, 10000.0)[0], dtype=torch.float64, device=DEV)
    pools = [torch.zeros_like(c["K"]) for _ in range(4)]
    args = lambda o, K, V: (q[:5], k, v, pos, slots, freq, o, K, V)
    call = lambda a: B.locret_paged_append(c["cfg"], 5, *a[:6], 64, False, 1.0, None, None, 0.0, *a[6:])
    call(args(want, *pools[:2]))
    for keep in range(9):
        got.zero_(), pools[2].zero_(), pools[3].zero_()
        call([x if i == keep else x.data_ptr() for i, x in enumerate(args(got, *pools[2:]))])
        assert torch.equal(want, got) and torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3]), keep
    state = lambda: [ints([5, 17]), ints([20, 3]), ints([0, 0]), ints([[4, -1, -1], [2, 3, -1]]), ints([0, 1, 5, 6, 9, 9, 9]), ints([4]), ints([0]), ints([9] * 3),
                     torch.zeros(30, **I32), torch.zeros(30, **I32)]
    cfg = config(n_pages=7, max_pages=3, max_reqs=2)
    call = lambda a: B.locret_paged_plan(cfg, 2, *a[:7], 30, *a[7:])
    want = state()
    call(want)
    for keep in range(10):
        got = state()
        call([x if i == keep else x.data_ptr() for i, x in enumerate(got)])
        assert all(torch.equal(a, b) for a, b in zip(want, got)), keep


@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 64), ("bf16", 64, 16), ("f32", 64, 16), ("f32", 96, 32)])
@pytest.mark.parametrize("window,sink", [(0, 0), (50, 4)])
@pytest.mark.parametrize("value", [None, float("inf"), float("nan")])
def test_rows_whose_logits_are_all_minus_infinity(dtype, d, page, window, sink, value):
    """Keys of -inf weigh nothing: rows that see only such are zeros and -inf, whatever their values hold, the others are what is left of theirs."""
    rng = np.random.default_rng(d + page + window)
    lens, new = [700, 200, 90], [30, 200, 90]
    c = paged_case(rng, dtype, 4, 2, d, page, lens, window, sink)
    gone = [np.zeros(n, dtype=bool) for n in lens]
    gone[0][:] = True                                      # all of them
    gone[1][:120] = True                                   # rows up to 119, and later ones whose window starts with them
    for r, g in enumerate(gone):
        for u in np.flatnonzero(g):
            p, i = c["table"][r, u // page], u % page
            c["K"][p, :, i, 0] = -math.inf
            if value is not None and r == 0 and u % 3 == 0:
                c["V"][p, :, i, :: 5] = value
    q, q64 = numbers(rng, dtype, sum(new), 4, d)
    q[..., 0] = 1.0
    q64[..., 0] = 1.0
    cu = np.cumsum([0] + new)

    def check(rows, out, lse, what):
        want, wl, tol, ltol = (np.zeros((len(rows),) + s) for s in ((4, d), (4,), (4, d), (4,)))
        for t, (r, i) in enumerate(rows):
            for j in range(4):
                see = R.visible(lens[r] - new[r] + i, lens[r], window, sink) & ~gone[r]
                K, V = (units(c, c[x], r, j // 2)[0] for x in ("K64", "V64"))
                want[t, j], wl[t, j], tol[t, j], ltol[t, j] = R.attend(q64[cu[r] + i, j], K, V, see, c["scale"], dtype)
        close(out, want, tol, what)
        close(lse, wl, ltol, what + " lse")

    out, lse = run_prefill(c, q, cu)
    check([(r, i) for r in range(3) for i in range(new[r])], out, lse, "prefill")
    assert (out[:30] == 0).all() and (out[30: 150] == 0).all() and np.isneginf(lse[:150]).all()
    out, lse = run_decode(c, q[torch.from_numpy(cu[1:] - 1).to(DEV)].contiguous())
    check([(r, new[r] - 1) for r in range(3)], out, lse, "decode")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_in_which_requests_wait_finish_or_are_not_served(dtype):
    """One token each for the others: packed rows through prefill, rows by request through decode, against the definition."""
    h, h_kv, d, page = 8, 2, 64, 16
    rng = np.random.default_rng(71)
    cache = B.PagedCache(config(dtype, h, h_kv, d, page, n_pages=20, max_reqs=6, max_pages=5), DEV)
    streams = [[np.zeros((0, n, d)) for n in (h, h_kv, h_kv)] for _ in range(6)]
    # request 1 waits, 3 is finished; in the last step the row of 4 is too short and there is no page left for 5
    for new in ([33, 50, 0, 20, 64, 48], [1, 0, 1, -1, 1, 1], [10, 0, 40, 5, 30, 20]):
        T = sum(max(n, 0) for n in new)
        x, x64 = numbers(rng, dtype, T, h + 2 * h_kv, d)
        cu, slots, pos = cache.plan(ints(new), T)
        q = cache.append(x[:, :h], x[:, h: h + h_kv], x[:, h + h_kv:], pos, slots)
        at = cu.tolist()
        for r, n in enumerate(new):
            if n < 0:
                streams[r] = [y[:0] for y in streams[r]]
            for i, (lo, hi) in enumerate(((0, h), (h, h + h_kv), (h + h_kv, h + 2 * h_kv))):
                streams[r][i] = np.concatenate([streams[r][i], x64[at[r]: at[r + 1], lo: hi]])
        assert cache.lens.tolist() == [s[0].shape[0] for s in streams]
        out = host(cache.prefill(q, cu))
        rows = torch.zeros(6, h, d, dtype=q.dtype, device=DEV)
        last = [at[r + 1] - 1 for r in range(6)]
        has = [r for r in range(6) if at[r + 1] > at[r]]
        rows[has] = q[[last[r] for r in has]]
        dec = host(cache.decode(rows))
        for r in has:
            n = at[r + 1] - at[r]
            want, tol = dense_reference(streams[r], [], 0, (None, None), n, 0, 0, dtype, h // h_kv)
            close(out[at[r]: at[r + 1]], want, tol, f"prefill of request {r} of {new}")
            close(dec[r: r + 1], want[-1:], tol[-1:], f"decode of request {r} of {new}")
        assert (dec[[r for r in range(6) if not streams[r][0].shape[0]]] == 0).all()
    assert at == [0, 10, 10, 50, 55, 55, 55]


@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 64), ("bf16", 64, 16), ("f32", 64, 16)])
@pytest.mark.parametrize("window,sink", [(0, 0), (50, 4)])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_rows_with_a_logit_of_infinity_or_nan_are_nan(dtype, d, page, window, sink, value):
    """Rows that see such a key, and no others."""
    rng = np.random.default_rng(d + page + window)
    lens, new = [700, 200, 90], [30, 200, 90]
    c = paged_case(rng, dtype, 4, 2, d, page, lens, window, sink)
    at = [(0, 690), (0, 100), (1, 60), (2, 0)]
    for r, u in at:
        c["K"][c["table"][r, u // page], :, u % page, 0] = value
    q, q64 = numbers(rng, dtype, sum(new), 4, d)
    q[..., 0] = 1.0
    q64[..., 0] = 1.0
    cu = np.cumsum([0] + new)
    rows = [(r, i) for r in range(3) for i in range(new[r])]

    def check(rows, out, lse, what):
        for t, (r, i) in enumerate(rows):
            see = R.visible(lens[r] - new[r] + i, lens[r], window, sink)
            if any(see[u] for s, u in at if s == r):
                assert np.isnan(out[t]).all() and np.isnan(lse[t]).all(), (what, r, i)
                continue
            for j in range(4):
                K, V = (units(c, c[x], r, j // 2)[0] for x in ("K64", "V64"))
                want, wl, tol, ltol = R.attend(q64[cu[r] + i, j], K, V, see, c["scale"], dtype)
                assert (np.abs(out[t, j] - want) <= tol).all() and abs(lse[t, j] - wl) <= ltol, (what, r, i, j)

    out, lse = run_prefill(c, q, cu)
    check(rows, out, lse, "prefill")
    last = cu[1:] - 1
    out, lse = run_decode(c, q[torch.from_numpy(last).to(DEV)].contiguous())
    check([(r, new[r] - 1) for r in range(3)], out, lse, "decode")
