"""The plan of the gradients through MXFP4 weights, on the host: what its launches and partial sums need, and what the tests' sizes reach."""
import random

import pytest
import torch

import mx_plan as P
from paper_2608_08910_amd import tq

F32, BF16, F16 = tq.TQ_F32, tq.TQ_BF16, tq.TQ_F16
MAX_ROWS, MAX_K = 1 << 20, 16384


def sizes(seed, count, top_n, top_t, top_k=MAX_K):
    """Sizes spread over the logarithm of their range, a third with small counts, half with rows of whole 16-byte pieces."""
    rng = random.Random(seed)
    for i in range(count):
        n, t = (int(round(top ** rng.random())) if i % 3 else rng.randint(1, 600) for top in (top_n, top_t))
        k = 256 * (int(round((top_k // 256) ** rng.random())) if rng.random() < 0.5 else rng.randint(1, top_k // 256))
        yield (max(8, n // 8 * 8) if rng.random() < 0.5 else n), k, t


EDGES = [(n, k, t) for n in (1, 64, 65, MAX_ROWS) for k in (256, MAX_K) for t in (1, 32, 33, 256, 257, MAX_ROWS)]


@pytest.mark.parametrize("seed", range(4))
def test_partial_sums_and_launches_fit(seed):
    """Over the whole range of arguments: what a plan's kernels write of the workspace lies within it, a longer batch's workspace holds
    every shorter one's, and a launch has fewer than 2^31 threads and its grid's dimensions their limits."""
    so = P.lib()
    for n, k, t in [*(EDGES if seed == 0 else ()), *sizes(seed, 10000, MAX_ROWS, MAX_ROWS)]:
        for ty, parts, b in ((F32, 3, 4), (BF16, 1, 2), (F16, 2, 2)):
            for mats in (1, 2):
                p, what = P.plan(n, k, t, mats, ty), (n, k, t, ty, mats)
                pad = (n + 63) // 64 * 64
                assert so.pad_of(n) == pad and (p.tile != P.FEW or not (p.stacked or p.whole)) and p.splits >= 1, what
                planes = (2 * mats * parts * t * pad + 255) // 256 * 256
                assert mats * t * n * b <= planes, what  # (a copy of dy, where its pieces are not lined up)
                rows = t * parts if p.stacked else t
                tiles = (k // p.bc) * -(-rows // p.bn)
                threads = 512 if p.tile == P.FEW or p.bc * p.bn >= 128 * 128 else 256
                if p.whole:
                    others = tiles - p.whole
                    assert 0 < others < 256 and p.whole % 256 == 0 and p.splits > 1 and not p.stacked, what
                    used, groups = ((p.splits * others - 1) * p.bc * p.bn + min(p.bn, t) * p.bc) * 4, p.whole + others * p.splits
                else:
                    used, groups = (p.splits * rows * k * 4 if p.splits > 1 or p.stacked else 0), tiles * p.splits
                assert planes + used <= so.bytes(n, ty, t, mats), what
                assert groups * threads < 1 << 31 and p.splits <= 65535, what
                assert p.tile != P.FEW or -(-t // 32) <= 65535, what
                steps = -(-n // 64) * mats * (1 if p.stacked or p.in_type or p.tile == P.FEW else parts)
                assert p.splits <= steps and steps * p.splits < 1 << 31, what
                if t > 1:
                    assert so.bytes(n, ty, t - 1, mats) <= so.bytes(n, ty, t, mats), what


def test_sizes_take_every_way():
    """What ordinary sizes take of kernels, tiles, ways of parts and of splitting, the tests' sizes take too."""
    def ways(n, k, t):
        return {(ty, *P.way(P.plan(n, k, t, mats, ty))) for ty in (F32, BF16, F16) for mats in (1, 2)}
    reached = set().union(*(ways(*s) for s in P.SIZES))
    found = set().union(*(ways(*s) for s in sizes(17, 40000, 32768, 9000)))
    assert len(found) > 60 and found <= reached, sorted(found - reached)


def test_a_lost_part_shows():
    """The values that the exactness tests multiply: three bfloat16 parts hold an fp32 value; two hold one with its last bit set
    only where the second part begins at bit 7 or below, its bits 15 to 8 being zeros: one value of 256."""
    g = torch.Generator().manual_seed(4)
    x = ((torch.randint(1 << 23, 1 << 24, (4096,), generator=g) | 1).double() * 2.0 ** -23).float()
    parts, rest = [], x.clone()
    for _ in range(3):
        p = (rest.view(torch.int32) & -65536).view(torch.float32)
        assert torch.equal(p.bfloat16().float(), p)
        parts.append(p)
        rest = rest - p
    low = (x.view(torch.int32) & 0xff00) != 0
    assert bool((rest == 0).all()) and torch.equal(parts[0] + parts[1] != x, low) and float(low.float().mean()) > 0.98
    h = ((torch.randint(1 << 10, 1 << 11, (4096,), generator=g) | 1).double() * 2.0 ** -10).half().float()
    assert bool((h != (h.view(torch.int32) & -65536).view(torch.float32)).all())
