"""Norm and rotation where only part of a head is rotated, or none of it: a column that is not rotated has to do with the others of its row by
the norm alone.  Values against the definition in 64 bits with the tolerances of test_qk_norm_rope_gpu.py, infinities and NaN exactly where the
definition has them."""
import math

import pytest
import torch

import reference64 as ref
from test_qk_norm_rope_gpu import case, check, lib  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu


def check_kinds(got, want, size, rel):
    """Infinities and NaN where the definition has them and nowhere else; the rest as check has it."""
    want, size = want.cpu(), size.cpu()
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(got.cpu()), kind(want)), f"{kind.__name__}: {int(kind(got).sum())} values, of the definition {int(kind(want).sum())}"
    there = torch.isfinite(want)
    check(torch.where(there.to(got.device), got, 0), torch.where(there, want, 0), torch.where(torch.isfinite(size), size, 0), rel)


def plant(x, rot, what, row0):
    """Values that are not finite into columns from rot on of [B, S, heads, D]: near the first of them and near the last."""
    D = x.shape[3]
    for i, value in enumerate(what):
        x[i % 2, row0 + i, i % 3, rot + 3 + i] = value
        x[i % 2, row0 + 3 + i, i % 3, D - 1 - 5 * i] = value


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 96, 128, 160])
@pytest.mark.parametrize("weights", [None, "own", "f32"])
def test_columns_that_are_not_rotated(lib, weights, D, dtype):  # noqa: F811
    """Infinities of both signs and NaN in such columns, and (FP32) a weight that is infinite: forward, cache form and backward, both pairings."""
    B, S, H, Hkv = 2, 12, 5, 3
    slots = torch.randperm(64, device="cuda", generator=torch.Generator("cuda").manual_seed(D))[:B * S].to(torch.int32).view(B, S)
    for rot in (0, 16, D // 2 // 16 * 16, D - 16):
        for interleaved in (False, True):
            q, k, v, qw, kw, pos, f, _ = case(B, S, H, Hkv, D, dtype, rot, 0, weights, seed=rot, packed=False)
            dy = [torch.randn(B, n, S, D, device="cuda", generator=torch.Generator("cuda").manual_seed(rot + n)).to(dtype) for n in (H, Hkv)]
            # (under a norm a row of x with a NaN makes all of the weights' gradients NaN: not with the weights of the rows' type)
            for x in (q, k):
                plant(x, rot, (math.inf, -math.inf, math.nan) if weights != "own" else (math.inf, -math.inf), 0)
            for x in dy:
                plant(x.transpose(1, 2), rot, (math.inf, -math.inf, math.nan), 6)
            phi = ref.angles(pos, f, None, B, S)
            if weights == "f32":
                qw[D - 9] = math.inf
            got = lib.qk_norm_rope(q, k, qw, kw, pos, f, interleaved=interleaved)
            kc, vc = (torch.zeros(1, Hkv, 64, D, device="cuda", dtype=dtype) for _ in range(2))
            q_out = lib.qk_norm_rope_cache(q, k, v, qw, kw, pos, f, kc, vc, slots, interleaved=interleaved)
            stored = kc[0][:, slots.long()].transpose(0, 1).contiguous()
            for y, x, w in ((got[0], q, qw), (got[1], k, kw), (q_out, q, qw), (stored, k, kw)):
                still = ref.norm_rope(x, w, phi[..., :0], 1e-6, False)
                size = torch.where(torch.isfinite(still), still.abs(), 0).amax(-1, keepdim=True) * math.sqrt(2)
                check_kinds(y, ref.norm_rope(x, w, phi, 1e-6, interleaved), size, 2.0 ** -19)
            if weights == "f32":
                qw[D - 9] = 1.0
            back = lib.qk_norm_rope_backward(*dy, q, k, qw, kw, pos, f, interleaved=interleaved)
            for which, (g, x, w) in enumerate(((dy[0], q, qw), (dy[1], k, kw))):
                dx, dw, size, _ = ref.norm_rope_backward(g, x, w, phi, 1e-6, interleaved)
                if w is None:
                    # (the error of a pair is one of its own two terms: of the row's finite values the greatest bounds it, and a value of a
                    # column that is not rotated is no term of another's.  The row's greatest of all is infinite here and bounds nothing.)
                    size = torch.where(torch.isfinite(g), g.abs(), 0).double().transpose(1, 2).amax(-1, keepdim=True)
                check_kinds(back[which], dx, size * math.sqrt(2), 2.0 ** -17)
                if w is not None:
                    # (sizes of the columns' terms without those that are not finite; a column with one of these is not finite itself)
                    fair = [torch.where(torch.isfinite(t), t, 0) for t in (g, x)]
                    dw_size = ref.norm_rope_backward(*fair, w, phi, 1e-6, interleaved)[3]
                    check_kinds(back[2 + which], dw, dw_size, (B * S * x.shape[2] + 64) * 2.0 ** -24 + 2.0 ** -18)


def test_a_call_that_only_turns_the_layout_copies_every_bit_pattern(lib):  # noqa: F811
    """No rotation, no weights: each of the 2^16 values of a type, beside every kind of neighbour, comes out as it went in."""
    for dtype in (torch.float16, torch.bfloat16):
        x = torch.randperm(1 << 16, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(torch.int32).to(torch.int16).view(dtype)
        q = x.view(2, 16, 32, 64)
        f, pos = torch.empty(0, device="cuda"), torch.arange(16, dtype=torch.int32, device="cuda")
        for interleaved in (False, True):
            got = lib.qk_norm_rope(q, q[:, :, :5], None, None, pos, f, interleaved=interleaved)
            back = lib.qk_norm_rope_backward(*got, q, q[:, :, :5], None, None, pos, f, interleaved=interleaved)
            for y, n in ((got[0].transpose(1, 2), 32), (got[1].transpose(1, 2), 5), (back[0], 32), (back[1], 5)):
                want = q[:, :, :n]
                assert torch.equal(torch.isnan(y), torch.isnan(want))
                assert torch.equal(torch.where(torch.isnan(y), 0, y), torch.where(torch.isnan(want), 0, want))
