"""What the thread that feeds group norm's ring waits for between two tiles (csrc/feed.h), compiled by itself and without a GPU.

Chunk w goes to stage w mod S and its release is completion number w / S (from 0) of that stage's barrier.  A wait for it by parity is over while exactly one
more completion than w / S has happened, and never is again once another one has: until a further one, which only a chunk that is not sent yet could bring.
The model below lets the threads that compute be as slow and as fast as they can be: everything between `one chunk behind what sending has waited for` and
`all that is sent` may be released when the feeder looks."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2205_12268_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "feed.h"

// completions of the barrier of stage s when the chunks 0 .. released-1 have been let go
static int completions(int s, int released, int stages) { return released <= s ? 0 : (released - 1 - s) / stages + 1; }
static bool over(int done, int phase) { return ((done & 1) ^ 1) == (phase & 1); }        // a wait for completion `phase`, by its parity

int main()
{
    int stuck = 0, early = 0, seen = 0;
    for (int stages = 2; stages <= 8; ++stages)
        for (int a = 1; a <= 20; ++a)
            for (int b = 1; b <= 20; ++b) {
                int sent = 0;
                const std::vector<int> tiles{a, b, a, 1, b, b};              // chunks of each
                for (int n : tiles) {
                    const int first = sent;
                    sent += n;
                    const int w = wcc::awaited_chunk(first, sent, stages);
                    if (w < 0) {
                        // nothing to wait for: sending has waited for the tile's first chunk
                        if (first > sent - 1 - stages) ++early;
                        continue;
                    }
                    ++seen;
                    // sending chunk sent-1 has waited for the release of sent-1-stages; all that is sent may be released
                    const int least = sent - stages > 0 ? sent - stages : 0;
                    if (w < first) ++early;
                    for (int released = least; released <= sent; ++released) {
                        const bool is = over(completions(w % stages, released, stages), w / stages);
                        if (is && released <= w) ++early;                    // taken for released, and is not
                        if (!is && released > w) ++stuck;                    // released, and waited for without end
                    }
                }
            }
    std::printf("%d %d %d\n", stuck, early, seen > 0);
}
"""


def test_no_wait_for_a_phase_that_is_over(tmp_path):
    src, exe = tmp_path / "feed.cpp", tmp_path / "feed"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout.split() == ["0", "0", "1"], out.stdout


def test_the_ring_asks_it():
    text = open(os.path.join(CSRC, "groupnorm_ring.cuh")).read()
    assert '#include "feed.h"' in text and "awaited_chunk(first, sent, stages)" in text
