"""Paged entry points without a GPU: refusals that are found on the host, and the rotary frequencies."""
import ctypes as C
import math

import pytest
import torch

from paper_2410_01805_amd import binding as B

GOOD = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, dtype=B.LOCRET_BF16, page_size=16, n_pages=100, max_reqs=4, max_pages=10, window=0, n_sink=0,
            softmax_scale=0.0)
OK, EINVAL, ESHAPE, EALIGN, ENOMEM = B.LOCRET_OK, B.LOCRET_EINVAL, B.LOCRET_ESHAPE, B.LOCRET_EALIGN, B.LOCRET_ENOMEM
P = 0x10000           # an address that no refused call may touch


def cfg(**kw):
    return B.locret_paged_config(**{**GOOD, **kw})


BAD = [
    (dict(n_q_heads=0), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(n_kv_heads=3), ESHAPE), (dict(n_q_heads=2048), ESHAPE),
    (dict(n_q_heads=256, n_kv_heads=1), ESHAPE), (dict(head_dim=16), ESHAPE), (dict(head_dim=80), ESHAPE), (dict(head_dim=256), ESHAPE),
    (dict(dtype=2), EINVAL), (dict(page_size=0), ESHAPE), (dict(page_size=8), ESHAPE), (dict(page_size=48), ESHAPE), (dict(page_size=512), ESHAPE),
    (dict(n_pages=0), EINVAL), (dict(n_pages=1 << 27), ESHAPE), (dict(max_pages=0), EINVAL), (dict(max_pages=1 << 27), ESHAPE), (dict(max_pages=(1 << 26) + 1), ESHAPE), (dict(max_pages=1 << 26, max_reqs=129), ESHAPE),
    (dict(max_reqs=0), EINVAL), (dict(max_reqs=4097), ESHAPE), (dict(window=-1), EINVAL), (dict(n_sink=-1), EINVAL),
    (dict(softmax_scale=-1.0), EINVAL), (dict(softmax_scale=float("nan")), EINVAL), (dict(softmax_scale=float("inf")), EINVAL),
]


@pytest.mark.parametrize("kw,code", BAD)
def test_bad_configurations_are_refused(kw, code):
    c = cfg(**kw)
    assert B.locret_paged_workspace_bytes(c) == 0
    assert plan(c) == append(c) == decode(c) == prefill(c) == code


def test_no_configuration():
    assert B.lib.locret_paged_workspace_bytes(None) == 0
    assert B.lib.locret_paged_decode(None, 1, P, P, P, P, P, P, P, P, 1 << 40, None) == EINVAL


def plan(c, n_req=2, ptrs=None, max_tokens=5, **kw):
    names = ["lens", "n_new", "lens_out", "table", "free", "n_free", "n_free_out", "cu", "slots", "positions"]
    p = [kw.get(n, P) for n in names]
    return B.lib.locret_paged_plan(C.byref(c), n_req, *p[:7], max_tokens, *p[7:], None)


def append(c, T=3, rot=32, il=0, amp=1.0, eps=1e-6, strides=None, **kw):
    g = lambda n: kw.get(n, P)
    st = None if strides is None else (C.c_int64 * 6)(*strides)
    return B.lib.locret_paged_append(C.byref(c), T, g("q"), g("k"), g("v"), st, g("positions"), g("slots"), g("freq"), rot, il, amp, g("wq"), g("wk"), eps,
                                     kw.get("q_out", 0x20000), g("K"), g("V"), None)


def decode(c, n_req=2, bytes_=1 << 40, **kw):
    p = [kw.get(n, P) for n in ("q", "K", "V", "table", "lens", "out", "lse", "ws")]
    return B.lib.locret_paged_decode(C.byref(c), n_req, *p, bytes_, None)


def prefill(c, n_req=2, T=7, bytes_=1 << 40, **kw):
    p = [kw.get(n, P) for n in ("q", "K", "V", "table", "lens", "cu", "out", "lse", "ws")]
    return B.lib.locret_paged_prefill(C.byref(c), n_req, T, *p, bytes_, None)


@pytest.mark.parametrize("kw,code", [
    (dict(n_req=-1), EINVAL), (dict(n_req=5), ESHAPE), (dict(max_tokens=-1), EINVAL), *((dict([(n, None)]), EINVAL) for n in (
        "lens", "n_new", "lens_out", "table", "free", "n_free", "n_free_out", "cu", "slots", "positions")),
    *((dict([(n, P + 2)]), EALIGN) for n in ("lens", "table", "free", "cu", "slots")),
])
def test_plan_refuses(kw, code):
    assert plan(cfg(), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), EINVAL), (dict(il=2), EINVAL), (dict(amp=float("nan")), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("inf")), EINVAL),
    (dict(rot=8), ESHAPE), (dict(rot=80), ESHAPE), (dict(rot=-16), ESHAPE), (dict(q=None, k=None, v=None), EINVAL), (dict(q_out=None), EINVAL),
    (dict(v=None), EINVAL), (dict(k=None), EINVAL), (dict(K=None), EINVAL), (dict(V=None), EINVAL), (dict(slots=None), EINVAL), (dict(freq=None), EINVAL),
    (dict(positions=None), EINVAL), (dict(q=P + 8), EALIGN), (dict(K=P + 8), EALIGN), (dict(wq=P + 4), EALIGN), (dict(freq=P + 4), EALIGN),
    (dict(slots=P + 2), EALIGN), (dict(strides=[512, 64, 128, 64, 128, 60]), EALIGN), (dict(strides=[512, 64, 128, -64, 128, 64]), EINVAL),
    (dict(strides=[1024, 64, 128, 64, 128, 64], q=P, q_out=P), EINVAL),
])
def test_append_refuses(kw, code):
    assert append(cfg(), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n_req=-1), EINVAL), (dict(n_req=5), ESHAPE), *((dict([(n, None)]), EINVAL) for n in ("q", "K", "V", "table", "lens", "out", "ws")),
    *((dict([(n, P + 8)]), EALIGN) for n in ("q", "K", "V", "out", "ws")), (dict(table=P + 2), EALIGN), (dict(lens=P + 1), EALIGN), (dict(lse=P + 2), EALIGN),
    (dict(ws=P + 16), EALIGN), (dict(bytes_=0), ENOMEM), (dict(bytes_=255), ENOMEM),
])
def test_attention_refuses(kw, code):
    assert decode(cfg(), **kw) == code
    assert prefill(cfg(), **kw) == code


def test_prefill_refuses():
    assert prefill(cfg(n_q_heads=16), T=(1 << 31) - 1, n_req=1) == ESHAPE
    assert prefill(cfg(), T=-1) == EINVAL and prefill(cfg(), cu=None) == EINVAL and prefill(cfg(), cu=P + 2) == EALIGN


def test_empty_calls_need_nothing():
    assert decode(cfg(), n_req=0, q=None, ws=None) == OK
    assert prefill(cfg(), T=0, q=None) == OK and prefill(cfg(), n_req=0) == OK
    assert append(cfg(), T=0, q=None, k=None) == OK


def test_the_workspace_grows_with_the_layout_only():
    small, large = B.locret_paged_workspace_bytes(cfg()), B.locret_paged_workspace_bytes(cfg(n_q_heads=32, n_kv_heads=8, head_dim=128))
    assert 0 < small <= large < 1 << 28
    assert B.locret_paged_workspace_bytes(cfg(n_pages=1 << 20, max_reqs=4096, max_pages=1 << 16)) < 1 << 28


def test_the_binding_checks_tensors():
    """Host tensors, wrong types and sizes never reach the library."""
    c, i32 = cfg(), torch.zeros(400, dtype=torch.int32)
    x = torch.zeros(4, 8, 64, dtype=torch.bfloat16)
    K = torch.zeros(100, 2, 16, 64, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 10, dtype=torch.uint8)
    for f in (lambda: B.locret_paged_plan(c, 2, i32, i32, i32, i32, i32, i32, i32, 2, i32, i32, i32),
              lambda: B.locret_paged_append(c, 4, x, x[:, :2], x[:, :2], i32, i32, None, 0, False, 1.0, None, None, 0.0, x, K, K),
              lambda: B.locret_paged_decode(c, 4, x, K, K, i32, i32, x, None, ws),
              lambda: B.locret_paged_prefill(c, 2, 4, x, K, K, i32, i32, i32, x, None, ws)):
        with pytest.raises(B.LocretError) as e:
            f()
        assert e.value.code == EINVAL


# ---- rotary frequencies ----------------------------------------------------------------------------------------------
def test_plain_frequencies():
    f, a = B.locret_rope_frequencies(64, 10000.0)
    assert a == 1.0 and f[0] == 1.0
    for i in range(32):
        assert math.isclose(f[i], 10000.0 ** (-i / 32), rel_tol=1e-14)


def test_linear_frequencies():
    f, a = B.locret_rope_frequencies(128, 500000.0, B.LOCRET_ROPE_LINEAR, factor=4.0)
    g, _ = B.locret_rope_frequencies(128, 500000.0)
    assert a == 1.0 and all(math.isclose(4 * x, y, rel_tol=1e-14) for x, y in zip(f, g))


def test_frequencies_by_bands():
    f, a = B.locret_rope_frequencies(128, 500000.0, B.LOCRET_ROPE_BANDS, factor=8.0, original=8192, low=1.0, high=4.0)
    g, _ = B.locret_rope_frequencies(128, 500000.0)
    kinds = set()
    for x, y in zip(f, g):
        wave = 2 * math.pi / y
        if wave < 8192 / 4:
            want, kind = y, "kept"
        elif wave > 8192 / 1:
            want, kind = y / 8, "stretched"
        else:
            s = (8192 / wave - 1) / 3
            want, kind = s * y + (1 - s) * y / 8, "mixed"
        kinds.add(kind)
        assert math.isclose(x, want, rel_tol=1e-12)
    assert a == 1.0 and kinds == {"kept", "stretched", "mixed"}


def test_frequencies_by_a_ramp():
    f, a = B.locret_rope_frequencies(64, 10000.0, B.LOCRET_ROPE_RAMP, factor=16.0, original=4096, low=1.0, high=32.0)
    g, _ = B.locret_rope_frequencies(64, 10000.0)
    assert math.isclose(a, 0.1 * math.log(16) + 1, rel_tol=1e-6)
    # pairs that turn more than 32 times over the first context are kept, those that turn less than once are stretched
    first = max(i for i in range(32) if 4096 * g[i] / (2 * math.pi) >= 32)
    last = min(i for i in range(32) if 4096 * g[i] / (2 * math.pi) <= 1)
    for i in range(32):
        w = min(1.0, max(0.0, (i - first) / (last - first)))
        assert math.isclose(f[i], w * g[i] / 16 + (1 - w) * g[i], rel_tol=1e-12), i


def test_frequencies_by_factors():
    factors = [1.0 + 0.25 * i for i in range(48)]
    f, a = B.locret_rope_frequencies(96, 10000.0, B.LOCRET_ROPE_FACTORS, factor=32.0, original=4096, factors=factors)
    g, _ = B.locret_rope_frequencies(96, 10000.0)
    assert math.isclose(a, math.sqrt(1 + math.log(32) / math.log(4096)), rel_tol=1e-6)
    assert all(math.isclose(x, y / z, rel_tol=1e-14) for x, y, z in zip(f, g, factors))
    assert B.locret_rope_frequencies(96, 10000.0, B.LOCRET_ROPE_FACTORS, factor=0.5, original=4096, factors=factors)[1] == 1.0


@pytest.mark.parametrize("kw,code", [
    (dict(rotary_dim=0), ESHAPE), (dict(rotary_dim=33), ESHAPE), (dict(rotary_dim=8192), ESHAPE), (dict(theta=1.0), EINVAL), (dict(theta=float("nan")), EINVAL),
    (dict(scaling=5), EINVAL), (dict(scaling=-1), EINVAL), (dict(scaling=1, factor=0.0), EINVAL), (dict(scaling=2, factor=8.0), EINVAL),
    (dict(scaling=2, factor=8.0, original=8192.0, low=4.0, high=1.0), EINVAL), (dict(scaling=3, factor=8.0, original=8192.0, low=0.0, high=1.0), EINVAL),
    (dict(scaling=4, factor=8.0, original=8192.0), EINVAL), (dict(scaling=4, factor=8.0, original=8192.0, factors=[1.0] * 31 + [0.0]), EINVAL),
])
def test_frequencies_refuse(kw, code):
    with pytest.raises(B.LocretError) as e:
        B.locret_rope_frequencies(**{**dict(rotary_dim=64, theta=10000.0), **kw})
    assert e.value.code == code


@pytest.mark.parametrize("dtype,most", [(B.LOCRET_F32, 1 << 31), (B.LOCRET_BF16, 1 << 34)])
@pytest.mark.parametrize("h", [16, 1024])
def test_prefill_takes_rows_up_to_its_limit(dtype, most, h):
    c = cfg(n_q_heads=h, n_kv_heads=h // 16, dtype=dtype)
    assert prefill(c, T=most // h, bytes_=0) == ENOMEM     # (the workspace is looked at behind the sizes)
    assert prefill(c, T=most // h + 1) == ESHAPE


def test_layouts_of_up_to_1024_heads():
    assert B.locret_paged_workspace_bytes(cfg(n_q_heads=1024, n_kv_heads=8)) > 0
    assert B.locret_paged_workspace_bytes(cfg(n_q_heads=1032, n_kv_heads=129)) == 0


def test_a_ramp_that_does_not_extend_keeps_its_amplitude():
    kw = dict(original=4096, low=1.0, high=32.0)
    assert B.locret_rope_frequencies(64, 10000.0, B.LOCRET_ROPE_RAMP, factor=0.5, **kw)[1] == 1.0
    f, a = B.locret_rope_frequencies(64, 10000.0, B.LOCRET_ROPE_RAMP, factor=1.0, **kw)
    # the mixture k f + (1 - k) f of a pair: four roundings of numbers that add up to f, each off by at most 2^-53 of its own
    assert a == 1.0 and all(math.isclose(x, y, rel_tol=2.0 ** -51) for x, y in zip(f, B.locret_rope_frequencies(64, 10000.0)[0]))
