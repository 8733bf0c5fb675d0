"""The rule by which a product with 8-bit weights takes its kernel (w8_pick of csrc/w8.hip), compiled for the host from the library's own source."""
import ctypes as C
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2408_05676_amd", "csrc")


def _cut(file, begin, end):
    text = open(os.path.join(CSRC, file)).read()
    at = text.index(begin)
    return text[at:text.index(end, at) + len(end)] + "\n"


def load(folder):
    """(pick(M, outs, Kd, gated) -> index, [shapes of the kernels of few rows (mt, nt, wk), then of the tiles (wm, wn)])."""
    few, tiles = _cut("w8_few.h", "constexpr W8Few kW8Few[]", ";"), _cut("w8_tile.h", "constexpr W8Shape kW8Shapes[]", ";")
    source = f"""
struct W8Args {{ int M, outs, rows, Kp; }};
struct W8Few {{ int mt, nt, wk; }};
struct W8Shape {{ int wm, wn; }};
{few}{tiles}
constexpr int kW8FewN = (int)(sizeof(kW8Few) / sizeof(kW8Few[0])), kW8ShapeN = (int)(sizeof(kW8Shapes) / sizeof(kW8Shapes[0]));
{_cut("w8.hip", "static int w8_pick(", chr(10) + "}")}
extern "C" int pick(int M, int outs, int Kd, int gated) {{
    return w8_pick(W8Args{{M, outs, (outs + 15) / 16 * 16 * (gated ? 2 : 1), (Kd + 255) / 256 * 256}}, gated);
}}
"""
    path, lib = os.path.join(folder, "rule.cpp"), os.path.join(folder, "rule.so")
    with open(path, "w") as f:
        f.write(source)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", path, "-o", lib], check=True)
    shapes = [tuple(int(v) for v in m.split(",")) for text in (few, tiles) for m in re.findall(r"\{([\d, ]+)\}", text)]
    return C.CDLL(lib).pick, shapes
