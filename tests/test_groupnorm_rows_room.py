"""Group norm's backward pass on rows of tokens: the rows of partial sums that its CTAs write fit the workspace, and their number goes by the sizes alone (a
workspace is laid out without a device).  Host code of csrc/groupnorm.cuh, compiled by itself and without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#define WCC_TRAINING_UNIT
#include "groupnorm.cuh"
#include <cstdio>

namespace wcc { wcc_status status_address(int**) { return WCC_ERR_CUDA; } }
using namespace wcc;

int main()
{
    long long seen = 0, over = 0;
    const int Ns[] = {1, 2, 37, 147, 148, 149, 295, 296, 297, 310, 333, 400, 1000, 5000, 8192, 1 << 20};
    for (int es : {2, 4})
        for (int C = 16 / es; C <= 8192; C += 16 / es)
            for (int G : {1, 2, 3, 4, 8, 16, 32, 64, 96, C * es / 16})
                for (int kept = 0; kept < 2; ++kept) {
                    if (G < 1 || C % G || !gn::rows_path(1, C, G, es, kept)) continue;
                    for (int N : Ns) {
                        const gn::Plan q = gn::plan_of(N, 1, C, G, es, true, kept);
                        const gn::Layout l = gn::layout_of(q, N, C, G, true);
                        const long long room = (long long)(l.total - l.img) / (2LL * C * 4);
                        ++seen;
                        if (gn::rows_grid(N, C, es, true).blocks > room) ++over;
                    }
                }
    std::printf("%d %lld\n", seen > 10000, over);
}
"""


def test_rows_of_partial_sums_fit(tmp_path):
    src, exe = tmp_path / "rows.cu", tmp_path / "rows"
    src.write_text(PROGRAM)
    subprocess.check_call([os.environ.get("NVCC", "nvcc"), "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2205_12268_b200", "csrc"), "-o", str(exe), str(src)])
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.split() == ["1", "0"], out.stdout


def test_no_launch_goes_by_another_number():
    csrc = os.path.join(ROOT, "paper_2205_12268_b200", "csrc")
    text = open(os.path.join(csrc, "training.cu")).read()
    body = text[text.index("wcc_status wcc_groupnorm_bwd("):text.index("wcc_status wcc_gated_fwd(")]
    assert "di.sms" not in body
