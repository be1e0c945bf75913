"""Which kernel runs a product of the linear, on the host: what each kernel
needs holds for every plan, and each kernel is reached."""

import random

import pytest

from tests import _linear_rules as R

KINDS = [R.FORWARD, R.INPUT, R.WEIGHT]


def sizes(n, seed=1):
    rng = random.Random(seed)
    for _ in range(n):
        yield tuple(round(2 ** rng.uniform(0, 14)) for _ in range(3))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_plans_hold_what_the_kernels_need(kind, dtype):
    for M, N, K in list(sizes(1500)) + [(1, 1, 1), (1, 1, 1 << 20), (1 << 20, 8, 8), (64, 64, 193), (64, 64, 192),
                                          (1 << 24, 2048, 8), (2048, 1 << 24, 8)]:
        for ok in (False, True):
            for cus in (R.CUS, 304, 8):
                p = R.plan(kind, M, N, K, dtype, ok, cus)
                assert p.slices >= 1
                if p.height:
                    # bf16, whole chunks, no 256 rows with a tail, whole panels
                    # across K, and every slice at least the four K blocks
                    # that the copies run ahead
                    assert dtype == "bf16" and ok and p.mid == 0
                    assert (p.height, p.width) in ((64, 128), (128, 256), (192, 256), (224, 256), (256, 256))
                    assert p.height < 256 or K % 64 == 0
                    assert kind[0] or p.height % 64 == 0
                    blocks = -(-K // 64)
                    assert p.per >= 4 and 4 <= blocks - p.per * (p.slices - 1) <= p.per
                elif p.mid:
                    assert kind == R.FORWARD and p.slices == 1 and p.mid in (1, 2, 3)
                    assert -(-M // (8 << p.mid)) * -(-N // 32) * 512 < 2 ** 32
                else:
                    bk = 64 if dtype == "bf16" else 32
                    assert p.per % bk == 0 and p.per * (p.slices - 1) < K <= p.per * p.slices
                if p.slices > 1:
                    need = p.slices * M * (-(-N // 8) * 8) * 4
                    assert need <= 64 << 20 and need <= R.workspace(kind, M, N, K, dtype, cus)


def test_empty_products():
    for M, N in ((0, 5), (5, 0)):
        assert R.plan(R.WEIGHT, M, N, 64).slices == 1 and R.workspace(R.WEIGHT, M, N, 64) == 0


def test_operands_of_the_tiles():
    assert R.tile_operand(1 << 20, 64, 64)
    for base, ld, row in ((8, 64, 64), (0, 65, 64), (0, 68, 64), (0, 64, 60), (0, (1 << 22) + 8, 64)):
        assert not R.tile_operand(base, ld, row)


@pytest.mark.parametrize("kind,M,N,K,ok,want", [
    (R.FORWARD, 8192, 8192, 5120, True, "tile256"), (R.FORWARD, 8192, 5120, 8192, True, "tile224"),
    (R.FORWARD, 4096, 5632, 2048, True, "tile192"), (R.INPUT, 4096, 2048, 5632, True, "tile128"),
    (R.WEIGHT, 5632, 2048, 4096, True, "tile192"), (R.FORWARD, 2048, 2048, 2048, True, "tile64"),
    (R.FORWARD, 128, 4096, 4096, True, "tile64+slices"), (R.FORWARD, 64, 512, 512, True, "mid1"),
    (R.FORWARD, 200, 1000, 2000, True, "mid2"), (R.FORWARD, 777, 1001, 1409, False, "any+slices"),
    (R.INPUT, 40, 2048, 4096, False, "any+slices"), (R.WEIGHT, 3001, 3001, 300, False, "any")])
def test_routes(kind, M, N, K, ok, want):
    assert R.route(kind, M, N, K, tiles_ok=ok) == want
