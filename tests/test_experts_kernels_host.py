"""Parts of the routed experts' kernels on host threads (tests/host/experts.cpp): what
keeps their accesses inside the caller's buffers."""
import os
import random
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_27888_gb300", "csrc")
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")


def struct(src, name):
    return re.search(rf"^(?:template <[^\n]*>\n)?struct {name} {{\n.*?^}};", src, re.M | re.S).group(0)


def function(src, name):
    return re.search(rf"^[^\n/#]*\b{name}\([^;{{]*\) {{(?:[^\n]*}}$|\n.*?^}})", src, re.M | re.S).group(0)


@pytest.fixture(scope="module")
def experts(tmp_path_factory):
    d = tmp_path_factory.mktemp("experts") / "csrc"
    d.mkdir()
    (d.parent / "include").symlink_to(os.path.join(ROOT, "include"))
    for f in ("experts.cpp", "cta.h"):
        (d / f).symlink_to(os.path.join(ROOT, "tests", "host", f))
    shared, linear = (open(os.path.join(CSRC, f)).read() for f in ("experts.cuh", "linear.cu"))
    parts = ["enum Mode { kForward = 0, kDx = 1, kDw = 2 };", "constexpr uint32_t kRows = 128;", function(shared, "offset_at")]
    parts += [function(linear, f) for f in ("scan_tiles", "hold_offsets", "make_table", "row_tiles_bound")]
    parts += [struct(linear, s) for s in ("Waiter", "Pack", "Packs", "Shape")]
    parts += [function(linear, f) for f in ("row_piece", "shifted", "pack_rows", "likely_tiles", "best_shape", "pitch_of",
                                            "round256", "tma_reads", "x_gathers", "x_packs", "w_packs", "x_bytes", "w_bytes",
                                            "operands")]
    (d / "parts.cuh").write_text("\n".join(parts) + "\n")
    exe = str(d / "experts")
    subprocess.run(["g++", "-O1", "-std=c++20", "-pthread", "-I", os.path.join(CUDA, "include"), "-I", str(d),
                    str(d / "experts.cpp"), "-o", exe], check=True)

    def run(*args):
        return subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=300, check=True).stdout
    return run


def wild(rng, E, n):
    """Offsets that are not what ntc_linear asks for: outside 0..n, decreasing, repeated."""
    kind = rng.randrange(4)
    if kind == 0:
        return [0 if e % 2 == 0 else n for e in range(E + 1)]
    if kind == 1:
        return [rng.randint(-n, 2 * n) for _ in range(E + 1)]
    if kind == 2:
        return sorted((rng.randint(0, n) for _ in range(E + 1)), reverse=True)
    return [rng.choice([-2 ** 31, 2 ** 31 - 1, 0, n, n // 2]) for _ in range(E + 1)]


@pytest.mark.parametrize("E", [1, 2, 3, 31, 32, 64, 700])
def test_wild_offsets_leave_no_more_tiles_than_workspaces_hold(experts, E):
    rng = random.Random(E)
    for _ in range(6):
        n, high = rng.randint(1, 5000), rng.choice([128, 256])
        offsets = wild(rng, E, n)
        off, tile, bound = ([int(x) for x in line.split()] for line in experts("table", high, n, *offsets).splitlines())
        least, want = n, [n]  # from the last on: held inside 0..n and by what follows
        for o in reversed(offsets):
            least = min(least, max(0, min(n, o)))
            want.insert(0, least)
        assert off == want
        tiles = [-(-(b - a) // high) for a, b in zip(want, want[1:])]
        assert tile == [sum(tiles[:e]) for e in range(E + 2)]
        if high == 128:  # the rows of `part`: a row of sums per tile of the experts
            assert tile[E] <= bound[0]


def test_offsets_as_asked_for_are_taken_as_they_are(experts):
    rng = random.Random(1)
    for E in (1, 5, 40, 300):
        n = rng.randint(1, 5000)
        offsets = [0] + sorted(rng.randint(0, n) for _ in range(E))
        off = experts("table", 128, n, *offsets).splitlines()[0]
        assert [int(x) for x in off.split()] == offsets + [n]


def test_a_wait_goes_on_while_its_cta_gets_on(experts):
    """A tile's contraction may take any time; only a CTA that stands still gives up."""
    opened, status, ms = map(int, experts("wait", 5000, 1).split())
    assert opened and status == 0 and ms == 5000
    opened, status, ms = map(int, experts("wait", 5000, 150).split())
    assert opened and status == 0
    opened, status, ms = map(int, experts("wait", 150, 0).split())
    assert opened and status == 0
    opened, status, ms = map(int, experts("wait", 5000, 0).split())
    assert not opened and status == 1 and 200 <= ms <= 210
    opened, status, ms = map(int, experts("wait", 5000, 300).split())
    assert not opened and status == 1 and 200 <= ms <= 310


# in_dim, out_dim, experts, rows, rows of x, then leading dimensions, offsets from 16 bytes, strides; with and without an
# index.  in_dim below 8: more rows than the first and the last reach past the matrix's ends in pieces of 16 bytes.
@pytest.mark.parametrize("K", [1, 2, 3, 5, 6, 7, 8, 9, 17, 100, 333, 1031])
@pytest.mark.parametrize("gap,off", [(0, 0), (0, 1), (0, 4), (1, 0), (1, 3), (3, 7), (8, 2)])
def test_copies_read_nothing_outside_their_operands(experts, K, gap, off):
    E, N, ld = 3, 5, K + gap
    for x_rows in (1, 40):
        out = experts("pack", K, N, E, x_rows, x_rows, ld, off, ld, N * ld + gap, off, 0)
        assert out.endswith("done\n") and len(out.splitlines()) == 2, out
    if K == 333:  # copied by an index: rows in any order, some of them none of x's (sizes from which dw's product asks for it)
        out = experts("pack", K, 1024, 16, 4500, 300, ld, off, ld, 1024 * ld, off, 1)
        assert out.endswith("copied 1 1\ndone\n") and len(out.splitlines()) == 2, out
