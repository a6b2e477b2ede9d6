"""The header's statement of the orthogonalisation's accuracy names the figures
that test_gpu_ortho_steps.py checks."""
import os


def test_header_states_these_figures():
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "bk.h")) as f:
        text = " ".join(f.read().replace("\n *", " ").split())
    for figure in ("0.3 / sqrt(r) with BK_NS_F16", "4e-4 / sqrt(r) with BK_NS_F32", "2e-4 / sqrt(r) with a side of 64",
                   "0.1 to 0.5% with BK_NS_F16", "about 3e-6 with BK_NS_F32", "1.5e-8 sqrt(max(d, p))"):
        assert figure in text, figure
