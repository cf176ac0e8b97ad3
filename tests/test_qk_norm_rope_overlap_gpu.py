"""Results of the norm and rotation that overlap what a call still reads, or each other, are refused; neighbours in one allocation are not."""
import pytest
import torch

from test_qk_norm_rope_gpu import case, lib  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu

B, S, H, Hkv, D = 2, 16, 6, 2, 64
HALF = torch.float16


def buffer(n):
    return torch.zeros(n, device="cuda", dtype=HALF)


def taken(memory, first, *shape):
    n = 1
    for x in shape:
        n *= x
    return memory[first:first + n].view(shape)


def test_results(lib):  # noqa: F811
    q, k, _, qw, kw, pos, f, _ = case(B, S, H, Hkv, D, HALF, packed=True)
    packed = q.as_strided((B * S * (H + 2 * Hkv) * D,), (1,), q.storage_offset())
    nq, nk = B * S * H * D, B * S * Hkv * D
    m = buffer(2 * (nq + nk))
    good = taken(m, 0, B, H, S, D), taken(m, nq, B, Hkv, S, D)
    want = lib.qk_norm_rope(q, k, qw, kw, pos, f)
    got = lib.qk_norm_rope(q, k, qw, kw, pos, f, out=good)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    before = m.clone()
    for out in ((good[0], taken(m, nq - 8, B, Hkv, S, D)), (good[0], taken(m, 0, B, Hkv, S, D)), (taken(packed, 0, B, H, S, D), good[1]),
                (good[0], taken(packed, packed.numel() - nk, B, Hkv, S, D)), (good[0], taken(packed, D * H, B, Hkv, S, D))):
        with pytest.raises(ValueError, match="overlap"):
            lib.qk_norm_rope(q, k, qw, kw, pos, f, out=out)
    with pytest.raises(ValueError, match="overlap"):
        lib.qk_norm_rope(q, k, good[0].view(-1)[:D], kw, pos, f, out=good)
    assert torch.equal(m, before)


def test_caches(lib):  # noqa: F811
    q, k, v, qw, kw, pos, f, _ = case(B, S, H, Hkv, D, HALF, packed=True)
    packed = q.as_strided((B * S * (H + 2 * Hkv) * D,), (1,), q.storage_offset())
    slots = torch.arange(B * S, dtype=torch.int32, device="cuda").view(B, S)
    n, nq = Hkv * S * D, B * S * H * D              # a page; the result
    m = buffer(2 * B * n + nq + n)
    kc, vc, out = taken(m, 0, B, Hkv, S, D), taken(m, B * n, B, Hkv, S, D), taken(m, 2 * B * n, B, H, S, D)
    call = lambda kc, vc, out=None: lib.qk_norm_rope_cache(q, k, v, qw, kw, pos, f, kc, vc, slots, out=out)
    want = lib.qk_norm_rope(q, k, qw, kw, pos, f)
    assert torch.equal(call(kc, vc, out), want[0]) and torch.equal(kc, want[1]) and torch.equal(vc, v.transpose(1, 2))
    before, of_packed = m.clone(), packed.clone()
    for bad in ((kc, kc), (kc, taken(m, n, B, Hkv, S, D)), (kc, vc, taken(m, B * n + 8, B, H, S, D)), (taken(packed, 0, B, Hkv, S, D), vc),
                (kc, taken(packed, 8 * D, B, Hkv, S, D)), (kc, vc, taken(packed, 8, B, H, S, D))):
        with pytest.raises(ValueError, match="overlap"):
            call(*bad)
    assert torch.equal(m, before) and torch.equal(packed, of_packed)


def test_gradients(lib):  # noqa: F811
    q, k, _, qw, kw, pos, f, _ = case(B, S, H, Hkv, D, HALF, packed=True)
    dy = [torch.randn(B, n, S, D, device="cuda").to(HALF) for n in (H, Hkv)]
    m = buffer(B * S * (H + 2 * Hkv + 1) * D)
    rows = m.view(B, S, H + 2 * Hkv + 1, D)
    call = lambda dq, dk, w=(qw, kw): lib.qk_norm_rope_backward(*dy, q, k, *w, pos, f, grads=(dq, dk))
    want = lib.qk_norm_rope_backward(*dy, q, k, qw, kw, pos, f)
    # neighbouring heads of one tensor, and heads taken in turns
    for dq, dk in ((rows[:, :, :H], rows[:, :, H:H + Hkv]), (rows[:, :, 1:1 + H], rows[:, :, H + 2:H + 2 + Hkv]), (rows[:, :, 0:11:2], rows[:, :, 1:4:2])):
        got = call(dq, dk)
        assert torch.equal(dq, want[0]) and torch.equal(dk, want[1]) and torch.equal(got[2], want[2])
    before, of_q = m.clone(), q.clone()
    for dq, dk in ((rows[:, :, :H], rows[:, :, H - 1:H - 1 + Hkv]), (rows[:, :, 0:11:2], rows[:, :, 2:5:2]), (q, rows[:, :, :Hkv]), (rows[:, :, :H], k),
                   (rows[:, :, :H], q[:, :, H - Hkv:]), (dy[0].view(B, S, H, D), rows[:, :, :Hkv]), (rows[:, :, :H], dy[1].view(B, S, Hkv, D))):
        with pytest.raises(ValueError, match="overlap"):
            call(dq, dk)
    assert torch.equal(m, before) and torch.equal(q, of_q)
    # without weights q and k are not looked at
    want = lib.qk_norm_rope_backward(*dy, q, k, None, None, pos, f)
    got = call(q, k, (None, None))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
