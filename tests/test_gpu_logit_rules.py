"""Rules on logits on the GPU against their definition in 64 bits.

Bound: a logit takes part in at most four operations of half a step each (division or product, penalty, its subtraction,
bias), on values no larger than |z| * repetition + |penalty| + |bias|: that * 4 * 2^-24; a bf16 output adds 2^-8 of its value.
Counts and minus infinities are exact."""
import math

import numpy as np
import pytest

from oracle import decoding_loop as D

pytestmark = pytest.mark.gpu


def random_tree(rng, R):
    return np.array([-1] + [int(rng.integers(0, r)) for r in range(1, R)], np.int32)


def case(seed, S, R, T, V, n_new=0):
    rng = np.random.default_rng(seed)
    words = (V + 31) // 32
    c = dict(S=S, R=R, T=T, V=V, z=(rng.standard_normal((S * R, V)) * 3).astype(np.float32), parent=np.concatenate([random_tree(rng, R) for _ in range(S)]),
             tokens=rng.integers(0, max(1, min(V, 9)), (S, T)).astype(np.int32),
             counts=(rng.integers(0, 4, (S, V)) * (rng.random((S, V)) < 0.3)).astype(np.int32), new=rng.integers(0, max(1, min(V, 7)), (S, n_new)).astype(np.int32),
             repetition=(1 + rng.random(S)).astype(np.float32), frequency=rng.random(S).astype(np.float32), presence=rng.random(S).astype(np.float32),
             bias=(rng.standard_normal((2, V)) * (rng.random((2, V)) < 0.2)).astype(np.float32), bias_row=rng.integers(-1, 2, S).astype(np.int32),
             masks=rng.integers(0, 1 << 32, (3, words), dtype=np.uint32), mask_row=rng.integers(-1, 3, S * R).astype(np.int32))
    return c


NAMES = ("counts", "repetition", "frequency", "presence", "bias", "bias_row", "masks", "mask_row")


def run(gpu, c, bf16, without=(), in_place=False, shift=0):
    lib, _, torch = gpu
    dev = lambda a: torch.from_numpy(a.view(np.int32) if a.dtype == np.uint32 else a).cuda()   # noqa: E731
    given = {n: None if n in without else dev(c[n]) for n in NAMES}
    S, R, T, V = (c[n] for n in "SRTV")
    dtype = torch.bfloat16 if bf16 else torch.float32
    flat = torch.zeros(S * R * V + shift, dtype=dtype, device="cuda")
    z = flat[shift:].view(S * R, V)
    z.copy_(dev(c["z"]))
    exact_z = z.double().cpu().numpy()
    out = z if in_place else torch.full_like(z, 5.0)
    rules = lib.LogitRules(S, R, T, V, lib.Y_BF16 if bf16 else lib.Y_FP32, dev(c["parent"]), **given)
    new = dev(c["new"]) if c["new"].size and given["counts"] is not None else None
    rules.run(z, dev(c["tokens"]), out, new_tokens=new)
    torch.cuda.synchronize()
    kw = {n: None if n in without else c[n] for n in NAMES}
    want, counts = D.logit_rules(exact_z, S, R, T, c["parent"], c["tokens"].tolist(), c["new"].tolist() if new is not None else None, **kw)
    got = out.double().cpu().numpy()
    if counts is not None:
        assert np.array_equal(given["counts"].cpu().numpy(), counts)
    most = 0 if counts is None else counts
    rep = np.ones(S) if "repetition" in without else c["repetition"]
    penalty = (0 if "frequency" in without else c["frequency"][:, None]) * (most + T) + (0 if "presence" in without else c["presence"][:, None])
    size = np.abs(exact_z) * np.repeat(rep, R)[:, None] + np.repeat(np.broadcast_to(penalty, (S, V)), R, 0) + (0 if "bias" in without else np.abs(c["bias"]).max(0)[None])
    with np.errstate(invalid="ignore"):
        bound = size * 4 * 2.0 ** -24 + (np.abs(want) * 2.0 ** -8 if bf16 else 0)
        same = (got == want) | (np.isnan(got) & np.isnan(want)) | (np.abs(got - want) <= bound)
    assert np.all(same), (int((~same).sum()), np.argwhere(~same)[:3].tolist())
    return got, want


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("S,R,T,V,n_new", [(1, 1, 1, 1, 0), (2, 1, 1, 7, 1), (3, 4, 2, 8, 3), (2, 30, 10, 9, 2), (1, 64, 64, 300, 9), (8, 3, 3, 2049, 3), (2, 5, 5, 5003, 40)])
def test_against_the_definition(gpu, S, R, T, V, n_new, bf16):
    run(gpu, case(S + R + V, S, R, T, V, n_new), bf16)


def test_blocks_of_four_waves(gpu):
    """Many streams of a vocabulary above 2048: the larger blocks."""
    run(gpu, case(5, 600, 1, 1, 2100, 1), True)
    run(gpu, case(6, 512, 2, 2, 2500, 1), False)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("without", [("counts",), ("repetition",), ("frequency", "presence"), ("bias", "bias_row"), ("masks", "mask_row"), NAMES])
def test_parts_that_are_not_wanted(gpu, without, bf16):
    run(gpu, case(11, 2, 6, 4, 77, 2), bf16, without=without)


@pytest.mark.parametrize("bf16", [True, False])
def test_in_place_and_at_any_alignment(gpu, bf16):
    for shift in (0, 1, 3):
        run(gpu, case(12 + shift, 3, 5, 5, 515, 2), bf16, in_place=True, shift=shift)
        run(gpu, case(22 + shift, 3, 5, 5, 515, 2), bf16, shift=shift)


def test_values_at_the_edge(gpu):
    for bf16 in (True, False):
        c = case(30, 2, 4, 3, 40, 2)
        c["z"][:, :8] = np.array([math.nan, math.inf, -math.inf, 0.0, -0.0, 3e38, -3e38, 1e-38], np.float32)
        c["repetition"][:] = 1.0
        c["masks"][0, :] = 0                                             # nothing is allowed: NaN and infinities too
        c["mask_row"][:4] = [0, -1, 1, 2]
        got, want = run(gpu, c, bf16)
        assert np.all(got[0] == -math.inf) and math.isnan(got[1, 0])


def test_what_the_device_arrays_may_hold(gpu):
    """Parents that are no earlier row, tokens and new tokens outside the vocabulary, rows of no table."""
    c = case(31, 3, 6, 6, 50, 4)
    c["parent"][:6] = [0, 5, 1, -7, 1 << 30, 4]
    c["tokens"][0] = [3, -1, 50, 1 << 30, 3, 3]
    c["new"][0] = [-1, 50, -(1 << 31), 2]
    c["new"][1] = [2, 2, 2, 2]
    c["bias_row"][:] = [2, -5, 1]
    c["mask_row"][:] = np.array([3, -9, 1 << 30] * 6)
    for bf16 in (True, False):
        run(gpu, c, bf16)


def test_repeated_calls_give_the_same_bits(gpu):
    c = case(32, 4, 10, 10, 3001, 0)
    a, _ = run(gpu, c, False)
    b, _ = run(gpu, c, False)
    assert np.array_equal(a, b)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("S,R,V", [(4, 3, 1400003), (3, 30, 187000), (3, 30, 187001)])
def test_results_that_outgrow_the_caches(gpu, S, R, V, bf16):
    """More than 32 MiB of results in a buffer of their own: the same bits as in place, which the definition checks; and the
    definition on the first and last tokens, which take part in no sum over others."""
    lib, _, torch = gpu
    assert S * R * V * 2 > 32 << 20
    c = case(40, S, R, min(R, 9), V, 2)
    dev = lambda a: torch.from_numpy(a.view(np.int32) if a.dtype == np.uint32 else a).cuda()   # noqa: E731
    z = dev(c["z"]).to(torch.bfloat16 if bf16 else torch.float32)
    results, counted = [], []
    for in_place in (False, True):
        given = {n: dev(c[n]) for n in NAMES}
        rules = lib.LogitRules(S, R, c["T"], V, lib.Y_BF16 if bf16 else lib.Y_FP32, dev(c["parent"]), **given)
        x = z.clone()
        out = x if in_place else torch.full_like(x, 5.0)
        rules.run(x, dev(c["tokens"]), out, new_tokens=dev(c["new"]))
        torch.cuda.synchronize()
        results.append(out)
        counted.append(given["counts"])
    bits = torch.int16 if bf16 else torch.int32
    assert torch.equal(results[0].view(bits), results[1].view(bits)) and torch.equal(counted[0], counted[1])
    for part in (slice(0, 64), slice((V - 40) // 32 * 32, V)):
        kw = {n: c[n] for n in NAMES}
        kw["counts"], kw["bias"] = c["counts"][:, part], c["bias"][:, part]
        kw["masks"] = c["masks"][:, part.start // 32:part.stop // 32 + 1]
        tokens = [[t - part.start for t in row] for row in c["tokens"].tolist()]
        new = [[t - part.start for t in row] for row in c["new"].tolist()]
        want, _ = D.logit_rules(z[:, part].double().cpu().numpy(), S, R, c["T"], c["parent"], tokens, new, **kw)
        got = results[0][:, part].double().cpu().numpy()
        size = np.abs(z[:, part].double().cpu().numpy()) * 2 + (4 + 2 + R) * 1.0 + 1 + np.abs(c["bias"][:, part]).max()
        with np.errstate(invalid="ignore"):
            same = (got == want) | (np.abs(got - want) <= size * 4 * 2.0 ** -24 + (np.abs(want) * 2.0 ** -8 if bf16 else 0))
        assert np.all(same), np.argwhere(~same)[:3].tolist()
