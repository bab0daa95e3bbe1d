"""What the 8-bit projections' outputs and workspaces may share memory with, on
the host: views of one buffer, never dereferenced."""
import itertools
import random

import pytest
import torch

import paper_2608_21229_amd as rc
from paper_2608_21229_amd import binding

BF16 = torch.bfloat16


def blocks_of(pool, at, rows, cols, t=None):
    """Fp8Blocks whose codes, then exponents, lie in a pool of bytes from `at` on."""
    pad, pitch = -(-cols // 128) * 128, -(-rows // 16) * 16
    codes, exps = pool[at:at + rows * pad], pool[at + rows * pad:at + rows * pad + pad // 128 * pitch]
    return rc.Fp8Blocks(codes.view(rows, pad), exps.view(pad // 128, pitch), (rows, cols), t)


@pytest.mark.parametrize("shift", [1, 3, 7])
def test_shifted_views_are_refused(shift):
    """By rows, by columns, and both, against the input and against the residual at one row stride."""
    m = torch.zeros(16, 512, dtype=BF16)
    out, far = m[:8, :128], torch.zeros(8, 128, dtype=BF16)
    for other in (m[shift:shift + 8, :128], m[:8, 8 * shift:8 * shift + 128], m[shift:shift + 8, 8 * shift:8 * shift + 128]):
        for a, b in ((out, other), (other, out)):
            with pytest.raises(ValueError, match="out may not be a"):
                binding._apart(a, "out", 512, b, "a", None, 0)
            with pytest.raises(ValueError, match="residual as it lies"):
                binding._apart(a, "out", 512, far, "a", b, 512)
    whole = torch.zeros(16, 128, dtype=BF16)
    with pytest.raises(ValueError, match="out may not be a"):
        binding._apart(whole[1:9], "out", 128, whole[:8], "a", None, 0)
    with pytest.raises(ValueError, match="residual as it lies"):
        binding._apart(whole[1:9], "out", 128, None, "a", whole[:8], 128)


def test_windows_side_by_side_are_taken():
    m = torch.zeros(16, 512, dtype=BF16)
    out, a, r = m[:8, 128:256], m[:8, :128], m[3:11, 256:384]
    binding._apart(out, "out", 512, a, "a", r, 512)
    binding._apart(m[:8], "out", 512, m[8:], "a", m[:8], 512)
    binding._apart(m[:1, :128], "out", 128, m[:1, 128:256], "a", m[1:2, :128], 128)
    binding._apart(m[4:5, :128], "out", 128, m[:8, 128:256], "a", None, 0)
    binding._apart(m[::2, :128], "out", 1024, m[:8, 128:256], "a", None, 0)
    with pytest.raises(ValueError, match="out may not be a"):
        binding._apart(m[::2, :128], "out", 1024, m[:8, 120:248], "a", None, 0)


def test_places_by_their_bytes():
    """Every pair of random windows of a buffer: equal strides are decided exactly, others never taken where they meet."""
    rng = random.Random(2)
    seen = {False: 0, True: 0}
    for _ in range(4000):
        places = []
        for stride in (rng.choice((24, 30)),) + (rng.choice((24, 30, 48)),):
            w, n = rng.randint(1, 24), rng.randint(1, 4)
            places.append(binding._place(rng.randint(0, 120), w, w if n == 1 else stride, n))
        a, b = places
        bytes_of = lambda t: {t[0] + i * t[2] + j for i in range(t[3]) for j in range(t[1])}  # noqa: E731
        meet = bool(bytes_of(a) & bytes_of(b))
        got = binding._meet(a, b)
        assert got == binding._meet(b, a) and (got or not meet)
        if a[2] == b[2] or 1 in (a[3], b[3]):
            assert got == meet
        seen[meet] += 1
    assert min(seen.values()) > 1000


def test_codes_and_exponents_in_one_pool():
    """Codes, exponents and what a call writes out of one allocation: apart, or refused."""
    pool = torch.zeros(1 << 16, dtype=torch.uint8)
    x = blocks_of(pool, 0, 40, 136)           # codes of 10240 bytes, exponents of 96
    end = 40 * 256 + 2 * 48
    after = pool[end:end + 40 * 136 * 2].view(BF16).view(40, 136)
    binding._apart_from(after, "out", x=x)
    for at in (end - 16, 10240 - 16, 4096):
        with pytest.raises(ValueError, match="out may not overlap x"):
            binding._apart_from(pool[at:at + 40 * 136 * 2].view(BF16).view(40, 136), "out", x=x)
    other = blocks_of(pool, end, 40, 136)
    binding._apart_from(other, "out", x=x, w=None)
    with pytest.raises(ValueError, match="out may not overlap x"):
        binding._apart_from(blocks_of(pool, end - 16, 40, 136), "out", x=x)
    # a workspace is what the call needs of it
    for need, fine in ((end, True), (end + 1, False)):
        place = (binding._place(pool.data_ptr(), need, need, 1),)
        if fine:
            binding._apart_from(place, "workspace", out=after)
        else:
            with pytest.raises(ValueError, match="workspace may not overlap out"):
                binding._apart_from(place, "workspace", out=after)


def test_nothing_meets_what_is_empty():
    m = torch.zeros(8, 128, dtype=BF16)
    for a, b in itertools.permutations((m[:0], m, m[:, :0]), 2):
        assert not binding._meet(binding._rows_at(a), binding._rows_at(b))
    empty = rc.Fp8Blocks(torch.zeros(0, 128, dtype=torch.uint8), torch.zeros(1, 0, dtype=torch.uint8), (0, 128))
    binding._apart_from(m, "out", x=empty)
    binding._apart_from(empty, "out", x=m)
