"""Rotary positions on the GPU against their definition in 64 bits.

Bounds: an angle's cosine and sine are off by at most 4 steps of 2^-24 (the reduced angle's rounding and the sums of their
series) and by the rounding of the frequency, position * 2^-52.  A turned feature is the sum of two products of them, each with
a rounding, and one more: (|a| + |b|) * (6 * 2^-24 + position * 2^-52); a bf16 output adds half a step, 2^-8 of its value."""
import numpy as np
import pytest

from oracle import decoding_loop as D

pytestmark = pytest.mark.gpu

SCALINGS = {"plain": {}, "linear": dict(factor=4.0), "base": dict(factor=8.0), "turns": dict(factor=8.0, low=1.0, high=4.0, context=8192.0)}


def make_rope(gpu, dim, rot, interleaved, scaling, theta=500000.0):
    lib = gpu[0]
    kinds = {"plain": lib.ROPE_PLAIN, "linear": lib.ROPE_LINEAR, "base": lib.ROPE_BASE, "turns": lib.ROPE_TURNS}
    return lib.Rope(dim, rot, lib.ROPE_INTERLEAVED if interleaved else lib.ROPE_HALF, kinds[scaling], theta, **SCALINGS[scaling])


def positions(rng, streams, rows, far):
    base = rng.integers(0, far, streams).astype(np.int32)
    offset = np.sort(rng.integers(0, 9, rows)).astype(np.int32)
    return base, offset, (base.astype(np.int64)[:, None] + offset[None, :]).reshape(-1)


@pytest.mark.parametrize("scaling", list(SCALINGS))
@pytest.mark.parametrize("streams,rows,rot,far", [(1, 1, 64, 16), (3, 5, 10, 1 << 17), (8, 30, 64, 1 << 20), (2, 257, 126, (1 << 31) - 10)])
def test_tables(gpu, scaling, streams, rows, rot, far):
    lib, _, torch = gpu
    base, offset, pos = positions(np.random.default_rng(rot + rows), streams, rows, far)
    M = streams * rows
    out = [torch.full((M, rot // 2), 7.0, device="cuda") for _ in range(2)]
    lib.RopeTables(make_rope(gpu, 128, rot, False, scaling), out[0], out[1], M, rows, torch.from_numpy(base).cuda(), torch.from_numpy(offset).cuda()).run()
    angles = D.rope_angles(pos, rot, scaling, 500000.0, **SCALINGS[scaling])
    bound = 4 * 2.0 ** -24 + pos[:, None] * 2.0 ** -52
    for got, want in zip(out, (np.cos(angles), np.sin(angles))):
        assert np.all(np.abs(got.cpu().numpy().astype(np.float64) - want) <= bound)


def check(gpu, streams, rows, heads, dim, rot, interleaved, scaling, bf16, inverse=False, far=1 << 17, in_place=False, pad=0, shift=0, seed=0):
    """Tensors with `pad` elements between heads, and `shift` elements behind an aligned address."""
    lib, _, torch = gpu
    rng = np.random.default_rng(seed)
    base, offset, pos = positions(rng, streams, rows, far)
    M, dtype = streams * rows, torch.bfloat16 if bf16 else torch.float32
    angles = D.rope_angles(pos, rot, scaling, 500000.0, **SCALINGS[scaling])

    def room(h, fill):
        flat = torch.full((M * h * (dim + pad) + shift + 3,), fill, dtype=dtype, device="cuda")
        return flat, flat[shift:shift + M * h * (dim + pad)].view(M, h, dim + pad)[..., :dim]

    moves, sources, outs, flats = [], [], [], []
    for i, h in enumerate(heads):
        flat_x, x = room(h, 0.0)
        x.copy_(torch.from_numpy(rng.standard_normal((M, h, dim))).to("cuda"))
        flat_y, y = (flat_x, x) if in_place else room(h, 11.0)
        sources.append(x.double().cpu().numpy())
        moves.append(lib.RopeTensor(x, y, rotate=i < 2))
        outs.append(y)
        flats.append((flat_y, flat_y.clone(), y))
    plan = lib.RopePlan(make_rope(gpu, dim, rot, interleaved, scaling), moves, M, lib.Y_BF16 if bf16 else lib.Y_FP32, inverse=inverse, rows_per_stream=rows,
                        base=torch.from_numpy(base).cuda(), offset=torch.from_numpy(offset).cuda())
    plan.run()
    torch.cuda.synchronize()
    for i, (x, y) in enumerate(zip(sources, outs)):
        got = y.double().cpu().numpy()
        if i >= 2:
            assert np.array_equal(got, x)
            continue
        want = D.rope(x, angles, rot, interleaved, inverse)
        assert np.array_equal(got[..., rot:], x[..., rot:])
        size = D.rope(np.abs(x), np.zeros_like(angles), rot, interleaved)
        for j in range(rot // 2):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
            size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
        bound = size * (6 * 2.0 ** -24 + pos[:, None, None] * 2.0 ** -52) + (np.abs(want) * 2.0 ** -8 if bf16 else 0)
        assert np.all(np.abs(got - want)[..., :rot] <= bound[..., :rot] * (1 + 2.0 ** -8)), i
    for flat, before, y in flats:                        # nothing between the heads or behind the tensor was touched
        inside = torch.zeros(flat.shape, dtype=torch.bool, device="cuda")
        torch.as_strided(inside, y.shape, y.stride(), y.storage_offset()).fill_(True)
        assert torch.equal(flat[~inside], before[~inside])


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(64, 64), (128, 128), (128, 32), (80, 80), (96, 46), (32, 4), (64, 22), (6, 2), (130, 118)])
def test_layouts_and_parts_of_the_head(gpu, dim, rot, interleaved, bf16):
    check(gpu, 3, 7, (6, 2, 2), dim, rot, interleaved, "turns", bf16)


@pytest.mark.parametrize("streams,rows,heads", [(1, 1, (1,)), (16, 1, (32, 8)), (1, 1030, (4, 1, 1)), (2, 800, (12, 3, 3)), (5, 33, (1, 1, 1, 1))])
def test_row_counts_and_several_tensors(gpu, streams, rows, heads):
    check(gpu, streams, rows, heads, 64, 64, False, "plain", True)
    check(gpu, streams, rows, heads, 128, 40, True, "base", False)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("interleaved", [False, True])
def test_any_stride_and_alignment_and_in_place(gpu, interleaved, bf16):
    for pad, shift, rot in [(3, 1, 64), (0, 1, 22), (5, 0, 46), (1, 3, 128)]:
        check(gpu, 2, 9, (5, 2, 2), 128, rot, interleaved, "linear", bf16, pad=pad, shift=shift)
        check(gpu, 2, 9, (5, 2, 2), 128, rot, interleaved, "linear", bf16, pad=pad, shift=shift, in_place=True)
    check(gpu, 1, 9, (5, 2), 128, 128, interleaved, "plain", bf16, far=(1 << 31) - 10)


def test_rows_without_base_and_offset(gpu):
    lib, _, torch = gpu
    x = torch.randn(12, 2, 64, device="cuda")
    one, two = torch.empty_like(x), torch.empty_like(x)
    rope = make_rope(gpu, 64, 64, False, "plain")
    lib.RopePlan(rope, [lib.RopeTensor(x, one)], 12, lib.Y_FP32, rows_per_stream=4).run()
    at = torch.arange(4, dtype=torch.int32, device="cuda")
    lib.RopePlan(rope, [lib.RopeTensor(x, two)], 12, lib.Y_FP32, rows_per_stream=4, base=torch.zeros(3, dtype=torch.int32, device="cuda"), offset=at).run()
    assert torch.equal(one, two) and torch.equal(one[0], x[0])


def test_a_transposed_destination(gpu):
    """Keys of [rows][heads] into a cache segment of [heads][rows], values beside them."""
    lib, _, torch = gpu
    k, v = (torch.randn(70, 3, 64, device="cuda").bfloat16() for _ in range(2))
    kc, vc, flat = torch.empty(3, 70, 64, device="cuda").bfloat16(), torch.empty(3, 70, 64, device="cuda").bfloat16(), torch.empty_like(k)
    rope = make_rope(gpu, 64, 64, False, "plain")
    lib.RopePlan(rope, [lib.RopeTensor(k, kc.permute(1, 0, 2)), lib.RopeTensor(v, vc.permute(1, 0, 2), rotate=False)], 70, lib.Y_BF16).run()
    lib.RopePlan(rope, [lib.RopeTensor(k, flat)], 70, lib.Y_BF16).run()
    assert torch.equal(kc, flat.permute(1, 0, 2)) and torch.equal(vc, v.permute(1, 0, 2))


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_inverse_is_the_gradient(gpu, interleaved):
    check(gpu, 2, 9, (5, 2), 96, 46, interleaved, "turns", False, inverse=True)
    check(gpu, 2, 9, (5, 2), 128, 128, interleaved, "plain", True, inverse=True)
    # <y(x + d) - y(x), g> = <d, inverse(g)>: a difference of a linear map, in fp32: 64 * 24 products of size 1 and their roundings
    lib, _, torch = gpu
    rope = make_rope(gpu, 64, 64, interleaved, "plain")
    x, d, g = (torch.randn(24, 1, 64, device="cuda") for _ in range(3))

    def run(t, inverse):
        y = torch.empty_like(t)
        lib.RopePlan(rope, [lib.RopeTensor(t, y)], 24, lib.Y_FP32, inverse=inverse).run()
        return y.double()

    moved = x + d
    left = ((run(moved, False) - run(x, False)) * g.double()).sum()
    right = ((moved.double() - x.double()) * run(g, True)).sum()
    assert abs(float(left - right)) <= 64 * 24 * 16 * 2.0 ** -24
