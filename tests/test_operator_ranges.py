"""Without a GPU: the places that the few-token kernel reads of its input's rows (csrc/x_pieces.h), compiled for the host, up to the longest
rows that a call takes."""
import os
import subprocess

import paper_2602_01410_amd

CSRC = os.path.join(os.path.dirname(paper_2602_01410_amd.__file__), "csrc")

# All chunks of all shares, the one brought behind the last chunk included; what is read is in the row, and is dropped just where it is not of the chunk.
PIECES = r"""
#include <algorithm>
#include <cstdio>
#include "x_pieces.h"
using namespace snip;
int main()
{
    const long long ks[] = {32, 96, 128, 4096, 11008, 1 << 20, (1ll << 30) + 32, (1ll << 31) - 32768, (1ll << 31) - 32768 + 32, (1ll << 31) - 4096, (1ll << 31) - 128, (1ll << 31) - 32};
    long checks = 0;
    for (long long k : ks) for (int shares = 1; shares <= 8; shares *= 2) for (int chunk = 4; chunk <= 256; chunk += 4) {
        const int spans = (int)((k + 127) / 128), chunks = (spans + shares * chunk - 1) / (shares * chunk);
        for (int share = 0; share < shares; ++share) for (int c = 0; c < 6; ++c) {
            const int ch = c < 3 ? c : chunks + c - 5, begin = share * chunks * chunk;          // the first three and the last ones
            if (ch < 0 || ch > chunks) continue;
            for (int i : {0, 1, 15, 16 * chunk - 1}) {
                const long long wanted = ((long long)begin + (long long)ch * chunk) * 128 + i * 8;
                const int piece = x_piece(begin, ch, chunk, i), at = std::min(piece, x_pieces((int)k) - 1);
                const long long e = piece_element(at);
                ++checks;
                if (e < 0 || e + 8 > k || (wanted < k ? e != wanted : piece < x_pieces((int)k))) {
                    std::printf("k %lld, %d shares, chunk %d: share %d, chunk %d, piece %d: element %lld\n", k, shares, chunk, share, ch, i, e);
                    return 1;
                }
            }
        }
    }
    std::printf("%ld\n", checks);
    return 0;
}
"""


def run(tmp_path, program, include=CSRC):
    src, exe = tmp_path / "ranges.cpp", tmp_path / "ranges"
    src.write_text(program)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", f"-I{include}", str(src), "-o", str(exe)], check=True, timeout=120)
    return subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)


def test_input_pieces(tmp_path):
    res = run(tmp_path, PIECES)
    assert res.returncode == 0, res.stdout
    assert int(res.stdout) > 10000


def test_places_in_elements_are_noticed(tmp_path):
    """Counted in elements, in 32 bits, as the kernel once did: the chunk behind the last one wraps to the front of the row."""
    with open(os.path.join(CSRC, "x_pieces.h")) as f:
        text = f.read()
    wrong = text.replace("return (begin + ch * chunk) * (128 / kPieceElements) + i;", "return ((begin + ch * chunk) * 128 + i * 8) / 8;")
    assert wrong != text
    (tmp_path / "x_pieces.h").write_text(wrong)
    res = run(tmp_path, PIECES, tmp_path)
    assert res.returncode == 1 and "element -" in res.stdout, res.stdout


def test_threads_of_a_launch(tmp_path):
    """A launch counts its threads in 32 bits."""
    program = r"""
#include <cstdio>
#include "picks.h"
int main()
{
    for (int threads = 64; threads <= 1024; threads += 64)
        if (snip::most_blocks(threads) * threads >= 1ll << 32 || snip::most_blocks(threads) < 1 << 21) { std::printf("%d\n", threads); return 1; }
    return 0;
}
"""
    res = run(tmp_path, program)
    assert res.returncode == 0, res.stdout


def test_workspace_of_the_gradient_grows_with_the_matrix():
    """A workspace sized for a program's largest matrix serves the smaller ones: over the changes of the kernel's form, the size falls neither
    with the rows nor with the columns."""
    from paper_2602_01410_amd import snip
    rows = [0, 1, 2, 3, 4, 5, 8, 63, 64, 65, 200, 255, 256, 257, 260, 300, 511, 512, 513, 1023, 1024, 1025, 2047, 2048, 2049, 4096, 16384, 1 << 20, (1 << 31) - 1]
    cols = [1, 7, 8, 9, 505, 511, 512, 513, 520, 1016, 1023, 1024, 1025, 1032, 2047, 2048, 2049, 2056, 4095, 4096, 4097, 4104, 8184, 8191, 8192, 8193, 8200, 16383, 16384,
            16385, 16392, 40001, 1 << 20]
    size = snip.rms_norm_workspace_bytes
    for a, b in zip(rows, rows[1:]):
        for c in cols:
            assert size(a, c) <= size(b, c), (a, b, c)
    for a, b in zip(cols, cols[1:]):
        for r in rows:
            assert size(r, a) <= size(r, b), (r, a, b)
