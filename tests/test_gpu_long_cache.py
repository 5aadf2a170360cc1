"""Stream caches at the largest number of slots: two heads of 2^24 slots with 128 features, so offsets of elements pass 2^32 within one
tensor and those of bytes within one head.  Keys and values are zeros but for a few rows at the far ends, and what is
expected follows by hand: n zero keys and one with score x share a soft-max as 1 : ... : 1 : e^x."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

H, CAP, DIM = 2, 1 << 24, 128
BF16_ONE = 0x3F80


@pytest.fixture(scope="module")
def long_cache(gpu):
    lib, _, torch = gpu
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB of device memory")
    k, v = (torch.zeros((1, 1, H, CAP, DIM), dtype=torch.int16, device="cuda") for _ in range(2))
    t = dict(k=k, v=v, mass=torch.ones((1, 1, H, CAP), device="cuda"), slot_pos=torch.zeros((1, 1, H, CAP), dtype=torch.int32, device="cuda"),
             len=torch.tensor([CAP], dtype=torch.int32, device="cuda"), next_pos=torch.tensor([CAP], dtype=torch.int32, device="cuda"))
    yield t, lib.StreamCache(*t.values())
    del t, k, v
    torch.cuda.empty_cache()


def test_append_at_the_far_end(gpu, long_cache):
    _, _, torch = gpu
    t, cache = long_cache
    give_way = [CAP - 3, CAP - 70000]                            # of the two heads
    for h, slot in enumerate(give_way):
        t["mass"][0, 0, h, slot] = 0.25
    new = torch.arange(2 * H * DIM, dtype=torch.int16, device="cuda").view(2, 1, 1, H, DIM) + 1
    cache.append(new[0].contiguous(), new[1].contiguous(), 1, None, CAP)
    torch.cuda.synchronize()
    for h, slot in enumerate(give_way):
        for name, rows in (("k", new[0]), ("v", new[1])):
            assert torch.equal(t[name][0, 0, h, slot], rows[0, 0, h])
            assert int(t[name][0, 0, h, slot - 1].abs().max()) == 0 and int(t[name][0, 0, h, slot + 1].abs().max()) == 0
            t[name][0, 0, h, slot] = 0
        assert float(t["mass"][0, 0, h, slot]) == 0 and int(t["slot_pos"][0, 0, h, slot]) == CAP
        t["mass"][0, 0, h, slot] = 1
        t["slot_pos"][0, 0, h, slot] = 0
    assert int(t["len"][0]) == CAP and int(t["next_pos"][0]) == CAP + 1
    assert int(t["slot_pos"].max()) == 0 and float(t["mass"].min()) == 1
    t["next_pos"][0] = CAP


@pytest.mark.parametrize("budget", [100, 700])                   # copied by the block that finds the slots, and by others
def test_compress_from_the_far_end(gpu, long_cache, budget):
    lib, _, torch = gpu
    t, cache = long_cache
    t["mass"][..., CAP - budget:] = 2
    for name in ("k", "v"):
        t[name][0, 0, :, CAP - budget:, 0] = torch.arange(budget, dtype=torch.int16, device="cuda") + (7 if name == "v" else 1)
    small = [torch.zeros((1, 1, H, budget, DIM), dtype=torch.int16, device="cuda") for _ in range(2)]
    to = lib.StreamCache(*small, torch.zeros((1, 1, H, budget), device="cuda"), torch.zeros((1, 1, H, budget), dtype=torch.int32, device="cuda"),
                         *(torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2)))
    kept = torch.empty((1, 1, H, budget), dtype=torch.int32, device="cuda")
    cache.compress(to, kept, budget)
    torch.cuda.synchronize()
    assert torch.equal(kept, (torch.arange(budget, dtype=torch.int32, device="cuda") + CAP - budget).expand(1, 1, H, budget))
    assert torch.equal(small[0], t["k"][:, :, :, CAP - budget:]) and torch.equal(small[1], t["v"][:, :, :, CAP - budget:])
    t["mass"][..., CAP - budget:] = 1
    for name in ("k", "v"):
        t[name][0, 0, :, CAP - budget:] = 0


@pytest.mark.parametrize("rows", [1, 64])                        # few query vectors, and the wide products
@pytest.mark.parametrize("shared", [False, True])
def test_masses_at_the_far_end(gpu, long_cache, rows, shared):
    """Head h's key CAP - 2 - h has score x with every query vector.  The sum of CAP weights 1 is off by at most CAP^(1/2) + 16 steps of
    2^-23, as the masses of the definition's test; x is exact."""
    lib, _, torch = gpu
    t, long = long_cache
    G, x = 4, 20.0
    far = [CAP - 2, CAP - 3]
    for h in range(H):
        t["k"][0, 0, h, far[h], 0] = BF16_ONE
    q = torch.zeros((1, rows, H * G, DIM), dtype=torch.int16, device="cuda")
    q[..., 0] = 0x41A0                                           # 20 in bf16
    if shared:
        empty = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device="cuda")   # noqa: E731
        cache = lib.StreamCache(empty(1, 1, H, 8, DIM, dtype=torch.int16), empty(1, 1, H, 8, DIM, dtype=torch.int16),
                                empty(1, 1, H, 8, dtype=torch.float32), empty(1, 1, H, 8), empty(1), empty(1))
        mass = torch.ones((1, H, CAP), device="cuda")
        op = lib.AttentionMass(cache, H * G, rows, 1.0, k_prefill=t["k"][0], mass_prefill=mass)
    else:
        mass = t["mass"]
        op = lib.AttentionMass(long, H * G, rows, 1.0)
    ws = torch.empty(max(256, op.workspace_bytes(0)), dtype=torch.uint8, device="cuda")
    op.run(q, None, ws)
    torch.cuda.synchronize()
    got = mass.view(H, CAP).cpu().numpy().astype(np.float64) - 1
    total = CAP - 1 + math.exp(x)
    want = np.full((H, CAP), rows * G / total)
    for h in range(H):
        want[h, far[h]] *= math.exp(x)
        t["k"][0, 0, h, far[h]] = 0
    t["mass"][:] = 1
    bound = want * ((CAP ** 0.5 + 16) * 2.0 ** -23) + (1 + want) * 2.0 ** -23
    assert np.all(np.abs(got - want) <= bound)
