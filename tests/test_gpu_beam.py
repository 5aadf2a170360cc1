"""Selection over beams and vocabulary on the GPU: sources, tokens, lengths and ends match the definition exactly, scores to their roundings.

A log-sum's exponentials are fp32: each is off by 2^-23 and what its rounded argument makes of it (2 * 2^-24 of up to 32, where it counts at
all), 64 of them are added in fp32 (63 * 2^-24 at most): 2^-17 in all.  Ranks of different beams that are nearer than 2^-15 to each other are kept out of
the inputs, but for equals."""
import math

import numpy as np
import pytest

from oracle import beams as O
from workloads.generate import bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu


def clear(ranks, W):
    """Whether no choice turns on less than the bound."""
    for group in ranks:
        for (x, a), (y, b) in zip(group[:W], group[1:W + 1]):
            if a != b and x != y and abs(x - y) < 2.0 ** -15:
                return False
    return True


def run(gpu, z, score, length, done, W, dtype, eos=-1, pad=0, power=0.0, in_place=False, offset=0):
    lib, _, torch = gpu
    rows, V = z.shape
    op = lib.BeamSelect(rows // W, W, V, lib.Y_FP32 if dtype == "fp32" else lib.Y_BF16, eos, pad, power)
    flat = torch.empty(rows * V + offset, dtype=torch.float32 if dtype == "fp32" else torch.bfloat16).cuda()
    flat[offset:].copy_(torch.from_numpy(z.astype(np.float32)).view(-1))
    i32 = lambda a: torch.from_numpy(np.array(a, np.int32)).cuda()   # noqa: E731
    ins = [torch.from_numpy(np.array(score, np.float32)).cuda(), i32(length), i32(done)]
    outs = ins if in_place else [torch.empty_like(t) for t in ins]
    source, token = i32(np.full(rows, -9)), i32(np.full(rows, -9))
    ws = torch.full((op.workspace_bytes(),), 0xFF, dtype=torch.uint8).cuda()
    op.run(flat[offset:], *ins, source, token, *outs, ws)
    torch.cuda.synchronize()
    return {"source": source, "token": token, "score": outs[0], "length": outs[1], "finished": outs[2]}


def check(gpu, z, score, length, done, W, dtype="fp32", eos=-1, pad=0, power=0.0, **kw):
    want, ranks = O.beam_select(z, score, length, done, W, eos, pad, float(np.float32(power)))
    assert clear(ranks, W)
    got = {n: t.cpu().numpy() for n, t in run(gpu, z, score, length, done, W, dtype, eos, pad, power, **kw).items()}
    for n in ("source", "token", "length", "finished"):
        assert np.array_equal(got[n], want[n]), n
    with np.errstate(invalid="ignore"):
        assert np.all((got["score"] == want["score"]) | (np.abs(got["score"] - want["score"]) <= 2.0 ** -17 + np.abs(want["score"]) * 2.0 ** -24))


def inputs(seed, G, W, V, dtype, done=0.0, sigma=3.0, power=0.0, **kw):
    """The first seed from this one on whose choices are clear."""
    while True:
        rng = np.random.default_rng(seed)
        z = (rng.standard_normal((G * W, V)) * sigma).astype(np.float32)
        if dtype == "bf16":
            z = bf16_bits_to_f32(f32_to_bf16_bits(z))
        z = z.astype(np.float64)
        score = np.float32(-20 - 5 * rng.random(G * W))
        ended = (rng.random(G * W) < done).astype(np.int32)
        length = np.where(ended, rng.integers(1, 20, G * W), 20).astype(np.int32)
        if clear(O.beam_select(z, score, length, ended, W, power=float(np.float32(power)))[1], W):
            return z, score, length, ended, W
        seed += 1000


@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1003, 4095, 4096, 4097, 32003])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_vocabularies(gpu, V, dtype):
    check(gpu, *inputs(V, 2, 3, V, dtype), dtype=dtype)


@pytest.mark.parametrize("W", [1, 2, 5, 16, 31, 32])
@pytest.mark.parametrize("power,done", [(0.0, 0.0), (0.8, 0.3)])
def test_beams(gpu, W, power, done):
    check(gpu, *inputs(W, 3, W, 5000, "fp32", done=done, power=power), power=power, eos=2, pad=7)


@pytest.mark.parametrize("V", [450, 1000, 2047, 4000, 4500, 8192, 8200, 16380, 16385])
@pytest.mark.parametrize("W,done", [(3, 0.3), (8, 0.0), (12, 0.0), (17, 0.4), (24, 0.0), (32, 0.0)])
def test_few_tokens_for_many_beams(gpu, V, W, done):
    check(gpu, *inputs(V + W, 2, W, V, "fp32", done=done))


def test_a_large_vocabulary(gpu):
    check(gpu, *inputs(5, 2, 8, 128256, "bf16", done=0.2, power=1.0), dtype="bf16", power=1.0, eos=5)


def test_a_vocabulary_of_a_million(gpu):
    check(gpu, *inputs(16, 1, 3, 1000003, "bf16"), dtype="bf16")


@pytest.mark.parametrize("power", [50.0, 300.0, 1e30])
def test_scores_that_the_length_makes_nothing_of(gpu, power):
    """20^-50 leaves little of a score, 20^-300 and less nothing at all: then all candidates are equal, and the lower beam's best come first."""
    z, score, length, done, W = inputs(17, 2, 4, 3000, "fp32")
    done[2] = 1
    if power == 50.0:
        want, _ = O.beam_select(z, score, length, done, W, power=power)
    else:
        want = {"source": np.repeat([0, 4], 4), "token": np.concatenate([np.argsort(-z[0], kind="stable")[:4], np.argsort(-z[4], kind="stable")[:4]])}
    got = run(gpu, z, score, length, done, W, "fp32", power=power)
    assert np.array_equal(got["source"].cpu().numpy(), want["source"]) and np.array_equal(got["token"].cpu().numpy(), want["token"])


def test_more_groups_than_the_card_has_units(gpu):
    check(gpu, *inputs(6, 400, 2, 300, "fp32"))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("offset", [1, 2, 3])
def test_rows_that_are_not_aligned(gpu, dtype, offset):
    check(gpu, *inputs(7, 1, 4, 4103, dtype), dtype=dtype, offset=offset)


def test_in_place(gpu):
    check(gpu, *inputs(8, 3, 5, 700, "fp32", done=0.3), eos=3, in_place=True)


def test_the_first_step(gpu):
    """One beam with score 0, the others have none."""
    z, _, _, _, W = inputs(9, 3, 4, 2000, "fp32")
    check(gpu, z, np.tile([0.0] + [-math.inf] * 3, 3).astype(np.float32), np.zeros(12, np.int32), np.zeros(12, np.int32), W)


def test_a_token_that_ends(gpu):
    z, score, length, done, W = inputs(10, 1, 4, 500, "fp32")
    best = int(np.argmax(z[np.argmax(score)]))
    check(gpu, z, score, length, done, W, eos=best)
    z[1, best] = 60.0
    check(gpu, z, score, length, done, W, eos=best)


def test_masks_that_leave_few(gpu):
    """Fewer candidates than beams, none, one per beam."""
    rng = np.random.default_rng(11)
    for left in (0, 1, 2):
        z = np.full((4, 9000), -math.inf)
        for b in range(4):
            z[b, rng.permutation(9000)[:left]] = rng.standard_normal(left)
        check(gpu, z, np.float32([-1, -3.5, -2.25, -7]), np.full(4, 3), np.zeros(4, np.int32), 4, pad=6)
    z = np.full((4, 9000), -math.inf)
    z[2, 8999] = 1.5
    check(gpu, z, np.float32([-1, -3.5, -2.25, -7]), np.full(4, 3), np.zeros(4, np.int32), 4, pad=6)


@pytest.mark.parametrize("odd", [math.nan, math.inf])
def test_rows_that_are_no_distributions(gpu, odd):
    z, score, length, done, W = inputs(12, 2, 3, 4500, "fp32")
    z[1, 4400] = odd
    z[3], z[4], z[5, 17] = odd, odd, odd
    check(gpu, z, score, length, done, W)
    score[:] = [math.nan, -1, -math.inf, math.inf, -2, -3]
    z[1, 4400] = 0.0
    check(gpu, z, score, length, done, W)


def test_odd_logits(gpu):
    """The largest and smallest numbers, both zeros, an infinity below."""
    rng = np.random.default_rng(13)
    z = rng.choice(np.float32([0.0, -0.0, 1e-42, -1e-42, 3.4e38, -3.4e38, -1.0, 1.0]), (4, 700)).astype(np.float64)
    z[:, 5] = -math.inf
    check(gpu, z, np.float32([-1, -9, -17, -25]), np.full(4, 3), np.zeros(4, np.int32), 4)
    z = np.where(z > 1e30, 1.0, z)
    check(gpu, z, np.float32([-1, -9, -17, -25]), np.full(4, 3), np.zeros(4, np.int32), 4)


@pytest.mark.parametrize("W", [1, 4, 32])
@pytest.mark.parametrize("V", [100, 9000])
def test_equals(gpu, W, V):
    """All logits alike, all beams alike: the lower beam, then the lower token."""
    check(gpu, np.full((2 * W, V), 0.25), np.full(2 * W, -1.5, np.float32), np.full(2 * W, 3), np.zeros(2 * W, np.int32), W)
    rng = np.random.default_rng(14)
    z = np.tile(rng.integers(0, 3, V) * 0.5, (2 * W, 1))
    check(gpu, z, np.full(2 * W, -1.5, np.float32), np.full(2 * W, 3), np.zeros(2 * W, np.int32), W)


def test_more_equals_than_are_ranked_at_once(gpu):
    """Every chunk of 32 beams has the same best candidate; then all but one."""
    z = np.zeros((32, 40000))
    check(gpu, z, np.full(32, -1.5, np.float32), np.full(32, 3), np.zeros(32, np.int32), 32)
    z[:, 39999] = 1.0
    check(gpu, z, np.full(32, -1.5, np.float32), np.full(32, 3), np.zeros(32, np.int32), 32)
    done = np.zeros(32, np.int32)
    done[3:] = 1
    check(gpu, z, np.full(32, -1.5, np.float32), np.full(32, 3), done, 32, pad=4)


def test_equal_candidates_one_by_one_are_the_best_of_each_beam(gpu):
    """Beams whose only candidates stand in one chunk, and many candidates in one chunk of one beam."""
    rng = np.random.default_rng(15)
    z = rng.standard_normal((8, 6000)) - 40.0
    z[2, 640:704] = np.linspace(0.0, 3.0, 64)
    z = z.astype(np.float32).astype(np.float64)
    check(gpu, z, np.float32([-30, -31, -1, -32, -33, -34, -35, -36]), np.full(8, 3), np.zeros(8, np.int32), 8)


def test_replays(gpu):
    """Captured, replayed on other logits, with eager work in between."""
    lib, _, torch = gpu
    W, V = 4, 5000
    op = lib.BeamSelect(2, W, V, lib.Y_FP32, eos=2)
    z = torch.zeros((8, V)).cuda()
    state = [torch.zeros(8).cuda(), torch.zeros(8, dtype=torch.int32).cuda(), torch.zeros(8, dtype=torch.int32).cuda()]
    source, token = (torch.zeros(8, dtype=torch.int32).cuda() for _ in range(2))
    ws = torch.empty(op.workspace_bytes(), dtype=torch.uint8).cuda()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        op.run(z, *state, source, token, *state, ws)
    for seed in range(4):
        x, score, length, done, _ = inputs(20 + seed, 2, W, V, "fp32", done=0.2)
        z.copy_(torch.from_numpy(x))
        for t, a in zip(state, (score, length, done)):
            t.copy_(torch.from_numpy(a))
        ws.fill_(seed)
        graph.replay()
        torch.cuda.synchronize()
        want, _ = O.beam_select(x, score, length, done, W, 2)
        assert np.array_equal(source.cpu().numpy(), want["source"]) and np.array_equal(token.cpu().numpy(), want["token"])
        assert np.array_equal(state[1].cpu().numpy(), want["length"]) and np.array_equal(state[2].cpu().numpy(), want["finished"])


@pytest.mark.parametrize("W,V,dtype", [(4, 128256, "bf16"), (16, 32000, "bf16"), (32, 32000, "fp32")])
@pytest.mark.parametrize("left", ["nothing", "a token", "a finished beam", "a beam"])
def test_many_infinite_logits(gpu, W, V, dtype, left):
    """Groups of beams whose logits are +infinity all over (more groups of chunks than are looked at one by one), but for one beam: they have no
    candidates, and nothing of the next group, or of what lies behind the last, becomes one."""
    z, score, length, done, _ = inputs(18, 1, W, V, dtype)
    one, rest = W // 2, np.full((W, V), math.inf)
    if left == "a token":
        rest[one] = -math.inf
        rest[one, V - 3] = 0.5
    elif left == "a beam":
        rest[one] = z[one]
    ended = done.copy()
    ended[one] = left == "a finished beam"
    check(gpu, np.concatenate([rest, z, rest]), np.tile(score, 3), np.tile(length, 3), np.concatenate([ended, done, ended]), W, dtype=dtype, pad=9)
    check(gpu, rest, score, length, ended, W, dtype=dtype, pad=9)
