"""CPU check that the shapes at which the block's products are compared with the oracle reach every tile: the library's own
rules, compiled for the host, are asked for each."""
import os
import shutil
import subprocess

import pytest

from tests.block_shapes import REGISTERS, TILES, TOKENS, TWO_TERMS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_36662_amd", "csrc")
NAMES = ["256", "256 x 128", "128", "128 deep", "64"]
STAGES = {"256": 2, "256 x 128": 3, "128": 2, "128 deep": 4, "64": 4}
PROGRAM = r"""
#include <cstdio>
#include "product_tiles.hpp"
int main() {
    long long rows, cols, k, pair;
    while (std::scanf("%lld %lld %lld %lld", &rows, &cols, &k, &pair) == 4)
        std::printf("%d\n", (int)autoloco::tile_of_product(rows, cols, k, pair != 0));
}
"""


@pytest.fixture(scope="module")
def tile_of(tmp_path_factory):
    hipcc = next((c for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")) if c and os.path.exists(c)), None)
    if hipcc is None:
        pytest.skip("hipcc not available")
    tmp = tmp_path_factory.mktemp("tiles")
    src, exe = tmp / "tiles.hip", tmp / "tiles"
    src.write_text(PROGRAM)
    subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    f"-I{CSRC}", f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(exe)], check=True, stderr=subprocess.DEVNULL)

    def ask(products):
        text = "".join(f"{m} {n} {k} {int(pair)}\n" for m, n, k, pair in products)
        p = subprocess.run([str(exe)], input=text, stdout=subprocess.PIPE, text=True, check=True)
        return [NAMES[int(line)] for line in p.stdout.split()]
    return ask


def _products(shape):
    """rows, columns, summed elements and whether a pair, of each product that takes its operands straight into LDS."""
    rows, d, ffn, out = shape
    whole = lambda *v: all(x % 8 == 0 for x in v)  # noqa: E731
    p = {}
    if whole(d):
        p["projections"] = (rows, ffn, d, True)
    if whole(ffn):
        p["y"] = (rows, out, ffn, False)
    if whole(out, ffn):
        p["dh"], p["dw_down"] = (rows, ffn, out, False), (out, ffn, rows, False)
    if whole(d) and ffn % 64 == 0:
        p["dx"] = (rows, d, 2 * ffn, False)
    if whole(d, ffn):
        p["dw_gate"] = (ffn, d, rows, False)
    return p


def test_every_product_in_every_tile(tile_of):
    """Each in sums of more steps than are on their way at once, the last of them not a whole one."""
    want = {(p, t) for p in ("projections", "y", "dh", "dw_gate", "dw_down") for t in NAMES} - {("projections", "64")}
    got = set()
    for shape in TILES:
        p = _products(shape)
        for (name, (_, _, k, _)), tile in zip(p.items(), tile_of(p.values())):
            if k % 64 and k // 64 > STAGES[tile]:
                got.add((name, tile))
    assert want <= got, want - got


def test_two_terms_in_every_tile(tile_of):
    """The second term begins after the first loads have been used, and before the last are asked for."""
    shapes = [s for s in TWO_TERMS]
    tiles = {}
    for shape, tile in zip(shapes, tile_of([_products(s)["dx"] for s in shapes])):
        steps = shape[2] // 64
        tiles[tile] = max(tiles.get(tile, 0), steps - STAGES[tile])
    assert set(tiles) == set(NAMES) and all(v > 0 for v in tiles.values()), tiles


def test_registers():
    """Widths that are no whole pieces; both tiles and both kinds of loops of each product."""
    loops = {}
    for shape in REGISTERS:
        rows, d, ffn, out = shape
        for name, (m, n, k) in {"y": (rows, out, ffn), "dh": (rows, ffn, out), "dx": (rows, d, ffn), "dw_gate": (ffn, d, rows),
                                "dw_down": (out, ffn, rows)}.items():
            tile = 64 if -(-m // 128) * -(-n // 128) < 256 else 128
            steady = (k - 1) // 64 >= 2 * (4 if tile == 64 else 2)
            loops.setdefault((name, tile), set()).add(steady)
        assert not _products(shape)
    assert all(True in loops.get((name, tile), ()) for name in ("y", "dh", "dx", "dw_gate", "dw_down") for tile in (64, 128)), loops
    assert any((d - 1) // 64 >= 4 for rows, d, _, _ in REGISTERS if rows > 16)


def test_tokens():
    """Of both projections a round of the waves takes 512 summed elements, of y 2,048: sums of several rounds, and such as
    end within a piece of 32."""
    assert all(s[0] <= 16 for s in TOKENS)
    for at, whole in ((1, 512), (2, 2048)):
        sums = [s[at] for s in TOKENS]
        assert any(k >= 2 * whole for k in sums) and any(k >= whole and k % 32 for k in sums)
