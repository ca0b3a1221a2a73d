"""What the calls on the paged 8-bit cache and the adapters refuse, without a GPU: through the binding (ValueError) and through the C ABI (codes, nothing
launched)."""
import ctypes

import pytest
import torch

import paper_2502_15779_amd as rcp

D, P, H, N_PAGES = 64, 16, 2, 3
KC, KS = rcp.kv8_new_cache(N_PAGES, H, "cpu", page=P, head_dim=D)
LEN, TABLE = torch.ones(2, dtype=torch.int32), torch.zeros((2, 4), dtype=torch.int32)
X = torch.zeros((2, H, D), dtype=torch.float16)
CACHE = (KC, KS, KC, KS)


@pytest.mark.parametrize("call, message", [
    (lambda: rcp.kv8_append(X, X, LEN, TABLE, *CACHE), "must be a"),
    (lambda: rcp.kv8_append(X, X, LEN, TABLE, KC.view(torch.uint8), KS, KC, KS), "codes must be float8_e4m3fn"),
    (lambda: rcp.kv8_append(X, X, LEN, TABLE, KC, KS.double(), KC, KS), "codes must be float8_e4m3fn"),
    (lambda: rcp.kv8_append(X, X, LEN, TABLE, KC, KS, KC[:2], KS[:2]), "codes must be float8_e4m3fn"),
    (lambda: rcp.kv8_append(X, X, LEN, TABLE, KC.transpose(1, 2), KS, KC, KS), "codes must be float8_e4m3fn"),
    (lambda: rcp.kv8_append("k", X, LEN, TABLE, *CACHE), "k must be"),
    (lambda: rcp.kv8_append(X[:, :1], X, LEN, TABLE, *CACHE), "must be a"),
    (lambda: rcp.kv8_attn(X, LEN, TABLE, *CACHE, 1.0), "must be a contiguous CUDA tensor"),
    (lambda: rcp.kv8_attn(X[..., :32], LEN, TABLE, *CACHE, 1.0), "must be a contiguous CUDA tensor"),
    (lambda: rcp.lowrank_add(X[0].float(), X, X, LEN, LEN, X[0]), "x must be float16 or bfloat16"),
    (lambda: rcp.lowrank_add(X[0], X[:, :, :32], X, LEN, LEN, X[0]), "A must be"),
    (lambda: rcp.lowrank_add(X[0], torch.zeros(1, 8, D).half(), torch.zeros(1, 32, 8).half(), LEN, torch.zeros(1), X[0]), "base and out must be"),
    (lambda: rcp.lowrank_add(X[0], torch.zeros(1, 8, D).half(), torch.zeros(1, D, 8).half(), LEN, torch.zeros(2), X[0]), "scaling must be"),
    (lambda: rcp.lowrank_add(X[0], torch.zeros(1, 8, D).half(), torch.zeros(1, D, 8).half(), LEN, torch.zeros(1), X[0]), "CUDA tensor"),
])
def test_arguments_that_do_not_fit_are_value_errors(call, message):
    with pytest.raises(ValueError, match=message):
        call()


FAKE, ODD = 0x1000, 0x1008   # never dereferenced: every call below fails its validation first


def _cache(**change):
    return rcp._Kv8Cache(**{**dict(k_codes=FAKE, k_scales=FAKE, v_codes=FAKE, v_scales=FAKE, n_pages=8, H=2, page=16, D=64), **change})


def _batch(**change):
    return rcp._Kv8Batch(**{**dict(starts=FAKE, lengths=FAKE, table=FAKE, rows=5, sequences=2, width=4), **change})


@pytest.mark.parametrize("cache, batch, code", [
    (dict(k_codes=None), {}, -1), (dict(v_scales=None), {}, -1), ({}, dict(lengths=None), -1), ({}, dict(table=None), -1),
    (dict(D=96), {}, -4), (dict(D=0), {}, -4), (dict(page=24), {}, -4), (dict(page=256), {}, -4), (dict(page=0), {}, -4),
    (dict(n_pages=0), {}, -2), (dict(H=0), {}, -2), (dict(H=4097), {}, -2),
    ({}, dict(sequences=0), -2), ({}, dict(sequences=1025), -2), ({}, dict(rows=-1), -2), ({}, dict(rows=(1 << 20) + 1), -2),
    ({}, dict(starts=None), -2), ({}, dict(width=0), -2), ({}, dict(width=1 << 21), -2), (dict(page=128), dict(width=1 << 17, sequences=512), -2),
    (dict(k_codes=ODD), {}, -3), ({}, dict(lengths=ODD), -3), ({}, dict(table=ODD), -3), ({}, dict(starts=ODD), -3),
])
def test_caches_and_batches_are_checked_before_the_device_is_touched(cache, batch, code):
    L, c, b = rcp.lib(), _cache(**cache), _batch(**batch)
    assert L.rcp_kv8_append(c, b, FAKE, 128, FAKE, 128, 0, None, 0, None, 0, 0, None, None) == code
    assert L.rcp_kv8_attn(c, b, FAKE, 0, 4, 1.0, FAKE, 0, FAKE, 1 << 30, None) == code


def test_append_refusals():
    L, c, b = rcp.lib(), _cache(), _batch()
    f = lambda k=FAKE, ks=128, v=FAKE, vs=128, dt=0, rope=None, q=None, qs=0, H_q=0, qo=None, b=b: L.rcp_kv8_append(
        c, b, k, ks, v, vs, dt, rope, 0, q, qs, H_q, qo, None)
    assert f(k=None) == -1 and f(v=None) == -1 and f(q=FAKE, qs=256, H_q=4) == -1
    assert f(dt=3) == -4 and f(dt=-1) == -4
    assert f(ks=127) == -2 and f(ks=120) == -2 and f(vs=0) == -2 and f(vs=-128) == -2 and f(q=FAKE, qs=248, H_q=4, qo=FAKE) == -2
    assert f(q=FAKE, qs=256, H_q=0, qo=FAKE) == -2 and f(q=FAKE, qs=1 << 20, H_q=4097, qo=FAKE) == -2
    assert f(k=ODD) == -3 and f(v=ODD) == -3 and f(rope=ODD) == -3 and f(q=ODD, qs=256, H_q=4, qo=FAKE) == -3 and f(q=FAKE, qs=256, H_q=4, qo=ODD) == -3
    assert f(q=FAKE, qs=4096 * 64, H_q=4096, qo=FAKE, b=_batch(rows=1 << 20)) == -2 and b"too many" in L.rcp_last_error()
    assert f(k=None, v=None, b=_batch(rows=0)) == 0     # no new tokens: nothing to do


def test_attention_refusals():
    L, c = rcp.lib(), _cache()
    f = lambda q=FAKE, qd=0, H_q=4, out=FAKE, od=0, ws=FAKE, wb=1 << 30, b=_batch(): L.rcp_kv8_attn(c, b, q, qd, H_q, 1.0, out, od, ws, wb, None)
    assert f(H_q=3) == -2 and f(H_q=0) == -2 and f(H_q=4098) == -2
    assert f(qd=3) == -4 and f(od=7) == -4 and f(q=None) == -1 and f(out=None) == -1
    assert f(q=ODD) == -3 and f(out=ODD) == -3 and f(ws=ODD) == -3
    need = L.rcp_kv8_workspace_bytes(5, 2, 4, 2, 64, 0)
    assert need > 0 and f(ws=None) == -5 and f(wb=need - 1) == -5 and b"workspace" in L.rcp_last_error()
    one = _batch(starts=None, rows=2)
    assert f(wb=L.rcp_kv8_workspace_bytes(2, 2, 4, 2, 64, 1) - 1, b=one) == -5
    assert f(q=None, out=None, ws=None, wb=0, b=_batch(rows=0)) == 0
    for scale in (-0.1, float("inf"), float("nan")):
        assert L.rcp_kv8_attn(c, _batch(), FAKE, 0, 4, scale, FAKE, 0, FAKE, 1 << 30, None) == -4 and b"softmax_scale" in L.rcp_last_error()
    w = L.rcp_kv8_workspace_bytes
    assert w(5, 0, 4, 2, 64, 0) == 0 and w(5, 2, 3, 2, 64, 0) == 0 and w(5, 2, 4, 2, 80, 0) == 0 and w(-1, 2, 4, 2, 64, 0) == 0


def test_adapter_refusals():
    L = rcp.lib()

    def f(x=FAKE, dt=0, M=3, N=16, K=64, r=8, n=2, A=FAKE, B=FAKE, which=FAKE, scaling=FAKE, base=FAKE, out=FAKE, od=0, ws=FAKE, wb=1 << 30):
        return L.rcp_lowrank_add(x, dt, M, N, K, r, n, A, B, which, scaling, base, out, od, ws, wb, None)
    for name in ("x", "A", "B", "which", "scaling", "base", "out"):
        assert f(**{name: None}) == -1, name
        assert f(**{name: ODD}) == -3, name
    assert f(ws=ODD) == -3
    assert f(dt=1) == -4 and f(dt=5) == -4 and f(od=5) == -4
    assert f(M=-1) == -2 and f(M=(1 << 19) + 1) == -2 and f(N=0) == -2 and f(N=18) == -2 and f(K=48) == -2 and f(K=0) == -2
    assert f(r=0) == -2 and f(r=12) == -2 and f(r=136) == -2 and f(n=0) == -2
    need = L.rcp_lowrank_workspace_bytes(3, 16, 64, 8)
    assert need > 0 and f(wb=need - 1) == -5 and f(ws=None) == -5
    assert f(M=0, x=None, out=None, ws=None) == 0 and L.rcp_lowrank_workspace_bytes(3, 16, 64, 12) == 0
