"""Rotary positions against their definition in 64 bits."""
import numpy as np
import pytest

from _kv_util import bf16, bf16_cuda, host

pytestmark = pytest.mark.gpu


def reference(x, positions, inv_freq, interleaved, inverse, scale):
    """(y, tolerance): 2^-8 of y for its rounding to bf16; sine and cosine off by 2^-21 (the angle as a part of a turn in fp32,
    2 pi 2^-25, and a few half steps), the products and their sum by three half steps of fp32."""
    x = np.asarray(x, dtype=np.float64)
    R = 2 * len(inv_freq)
    a = np.asarray(positions, dtype=np.float64)[..., None] * inv_freq                 # [B, S, R/2] or [S, R/2]
    a = a[:, None] if a.ndim == 3 else a
    c, s = scale * np.cos(a), scale * np.sin(a) * (-1 if inverse else 1)
    first, second = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    y, tol = x.copy(), np.zeros_like(x)
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., first] * s + x[..., second] * c
    size = (np.abs(x[..., first]) + np.abs(x[..., second])) * abs(scale)
    for part in (first, second):
        tol[..., part] = 2.0 ** -8 * np.abs(y[..., part]) + 2.0 ** -20 * size
    return y, tol


def check(got, want):
    y, tol = want
    assert np.all(np.abs(host(got) - y) <= tol), float((np.abs(host(got) - y) - tol).max())


SHAPES = [
    # B, S, Hq, Hk, D, R
    (1, 1, 1, 0, 64, 64),
    (1, 1, 1, 1, 8, 2),
    (3, 5, 4, 2, 128, 128),
    (2, 33, 3, 1, 128, 64),
    (2, 7, 5, 5, 64, 20),
    (1, 100, 2, 2, 64, 24),
    (2, 9, 2, 1, 80, 40),
    (5, 1, 32, 8, 128, 128),
    (1, 300, 8, 1, 256, 6),
    (2, 3, 130, 2, 64, 32),
]


@pytest.mark.parametrize("B,S,Hq,Hk,D,R", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_against_the_definition(B, S, Hq, Hk, D, R, interleaved, inverse):
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(B + S + D + R)
    q, k = (bf16(rng.standard_normal((B, H, S, D))) for H in (Hq, max(Hk, 1)))
    positions = rng.integers(-10, 200000, (B, S)).astype(np.int32)
    inv = binding.rope_frequencies(R)
    got = binding.rope_bf16(bf16_cuda(q), torch.from_numpy(positions).cuda(), inv, k=bf16_cuda(k) if Hk else None,
                            interleaved=interleaved, inverse=inverse, scale=1.25)
    torch.cuda.synchronize()
    for g, x in zip(got if Hk else (got,), (q, k)):
        check(g, reference(x, positions, inv.cpu().numpy(), interleaved, inverse, 1.25))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [64, 36])
def test_in_place_on_strided_views_with_shared_positions(interleaved, R):
    """q and k are views of one buffer [B, S, heads, D], as a layer's projection leaves them, and turn where they lie."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(R)
    x = bf16(rng.standard_normal((2, 11, 10, 64)))
    buf = bf16_cuda(x)
    q, k, v = (t.transpose(1, 2) for t in buf.split((6, 2, 2), 2))
    inv = binding.rope_frequencies(R, base=500.0)
    got = binding.rope_bf16(q, torch.arange(11, dtype=torch.int32, device="cuda") + 5, inv, k=k, q_out=q, k_out=k, interleaved=interleaved)
    torch.cuda.synchronize()
    assert got[0].data_ptr() == q.data_ptr()
    xt = x.transpose(0, 2, 1, 3)
    for g, ref in ((q, xt[:, :6]), (k, xt[:, 6:8])):
        check(g, reference(ref, 5 + np.arange(11), inv.cpu().numpy(), interleaved, False, 1.0))
    assert np.array_equal(host(v), xt[:, 8:])


def test_far_positions():
    """Where fp32 angles would be off by many turns."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(1)
    x = bf16(rng.standard_normal((1, 2, 6, 64)))
    positions = np.array([2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7, 2 ** 24 + 1, 0, 131071], dtype=np.int32)
    inv = binding.rope_frequencies(64)
    got = binding.rope_bf16(bf16_cuda(x), torch.from_numpy(positions).cuda(), inv)
    torch.cuda.synchronize()
    check(got, reference(x, positions, inv.cpu().numpy(), False, False, 1.0))


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(interleaved):
    """The inverse rotation of an output's gradient is the gradient: against the formula's (its transpose, in 64 bits) and
    against differences of the operation itself, which is linear: <y(x + h d) - y(x), g> / h = <d, gradient>."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(2)
    x, g = (bf16(rng.standard_normal((2, 3, 4, 64))) for _ in range(2))
    positions = rng.integers(0, 5000, (2, 4)).astype(np.int32)
    inv, pos = binding.rope_frequencies(48), torch.from_numpy(positions).cuda()
    grad = host(binding.rope_bf16(bf16_cuda(g), pos, inv, interleaved=interleaved, inverse=True, scale=1.5))
    want, tol = reference(g, positions, inv.cpu().numpy(), interleaved, True, 1.5)
    assert np.all(np.abs(grad - want) <= tol)
    d = np.where(rng.random(x.shape) < 0.1, 1.0, 0.0)
    y0, t0 = reference(x, positions, inv.cpu().numpy(), interleaved, False, 1.5)
    y1, t1 = reference(x + d, positions, inv.cpu().numpy(), interleaved, False, 1.5)
    xs = [host(binding.rope_bf16(bf16_cuda(z), pos, inv, interleaved=interleaved, scale=1.5)) for z in (x, bf16(x + d))]
    moved = bf16(x + d) - (x + d)                                     # the step that bf16 makes of the sum
    slack = (np.abs(g) * (t0 + t1)).sum() + (tol * d).sum() + 1.5 * 2 * np.abs(moved).sum() * np.abs(g).max()
    assert abs(((xs[1] - xs[0]) * g).sum() - (d * grad).sum()) <= slack


def test_long_context_frequencies():
    from paper_2604_18616_amd import binding
    R, base, factor, length = 128, 10000.0, 8.0, 4096
    inv = base ** (-np.arange(0, R, 2) / R)
    keep = np.clip((length * inv / (2 * np.pi) - 1.0) / 31.0, 0, 1)
    got = binding.rope_frequencies(R, base, factor, length).cpu().numpy()
    assert np.allclose(got, inv * (keep + (1 - keep) / factor), rtol=1e-14, atol=0)
    assert got[0] == 1.0 and np.isclose(got[-1], inv[-1] / factor, rtol=1e-14)
    assert np.allclose(binding.rope_frequencies(R, base, factor).cpu().numpy(), inv / factor, rtol=1e-14, atol=0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_many_tokens(interleaved):
    """Enough of them for a thread to walk several heads, numbers of heads that do not divide."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(3)
    B, S, Hq, Hk, D, R = 1, 4500, 33, 7, 128, 96
    q, k = (bf16(rng.standard_normal((B, H, S, D), dtype=np.float32)) for H in (Hq, Hk))
    positions = rng.integers(0, 100000, (B, S)).astype(np.int32)
    inv = binding.rope_frequencies(R)
    got = binding.rope_bf16(bf16_cuda(q), torch.from_numpy(positions).cuda(), inv, k=bf16_cuda(k), interleaved=interleaved)
    torch.cuda.synchronize()
    for g, x in zip(got, (q, k)):
        check(g, reference(x, positions, inv.cpu().numpy(), interleaved, False, 1.0))


def test_outputs_given_and_not_dense():
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(4)
    q, k = bf16(rng.standard_normal((2, 3, 5, 64))), bf16(rng.standard_normal((1, 2, 5, 64)))
    room = torch.full((2, 7, 6, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    qo, ko = room[:, 1:6, :3, :64].transpose(1, 2), room[:, 1:6, 3:5, :64].transpose(1, 2)
    kd = bf16_cuda(k).expand(2, 2, 5, 64)                    # one sequence's keys for both
    positions, inv = np.array([[3, 1, 4, 1, 5], [9, 2, 6, 5, 3]], dtype=np.int32), binding.rope_frequencies(48)
    got = binding.rope_bf16(bf16_cuda(q), torch.from_numpy(positions).cuda(), inv, k=kd, q_out=qo, k_out=ko)
    own = binding.rope_bf16(bf16_cuda(q), torch.from_numpy(positions).cuda(), inv, k=kd)
    torch.cuda.synchronize()
    assert got[0] is qo and got[1] is ko
    for pair in (got, own):
        check(pair[0], reference(q, positions, inv.cpu().numpy(), False, False, 1.0))
        check(pair[1], reference(np.broadcast_to(k, (2, 2, 5, 64)), positions, inv.cpu().numpy(), False, False, 1.0))
    qo.fill_(7.0), ko.fill_(7.0)
    assert (room == 7.0).all()


@pytest.mark.parametrize("interleaved,layout", [(False, "bshd"), (True, "bhsd")])
def test_a_large_call_is_its_parts(interleaved, layout):
    """200 MB in one call against the same tokens in small calls: the same bits."""
    import torch
    from paper_2604_18616_amd import binding
    B, S, Hq, Hk, D = 2, 5001, 30, 5, 160
    shape = lambda H: (B, H, S, D) if layout == "bhsd" else (B, S, H, D)
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.randn(shape(H), generator=gen, device="cuda").to(torch.bfloat16) for H in (Hq, Hk))
    if layout == "bshd":
        q, k = q.transpose(1, 2), k.transpose(1, 2)
    positions = torch.arange(B * S, dtype=torch.int32, device="cuda").reshape(B, S)
    inv = binding.rope_frequencies(128)
    whole = binding.rope_bf16(q, positions, inv, k=k, interleaved=interleaved)
    for at in range(0, S, 500):
        part = binding.rope_bf16(q[:, :, at:at + 500], positions[:, at:at + 500], inv, k=k[:, :, at:at + 500], interleaved=interleaved)
        for w, x in zip(whole, part):
            assert torch.equal(w[:, :, at:at + 500], x)
