"""That the shapes of ``ff_paths`` take the ways they are listed for, by the rules themselves, and all ways there are (on the host)."""
import os
import subprocess

import ff_paths

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_shapes_take_every_way(tmp_path):
    exe = str(tmp_path / "show_cuts")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-o", exe, os.path.join(ROOT, "tests", "host", "show_cuts.cpp")], check=True)
    asked = "".join(" ".join(str(v) for v in shape[:4]) + "\n" for shape in ff_paths.SHAPES)
    told = subprocess.run([exe], input=asked, capture_output=True, text=True, check=True).stdout.splitlines()
    assert told == [shape[4] for shape in ff_paths.SHAPES]

    taken = set()
    for _, K, _, size, cut in ff_paths.SHAPES:
        words = cut.split()
        for what, kind, parts in zip(("forward", "dx", "dW"), words[::2], words[1::2]):
            taken.add((what, kind, "whole" if parts == "1" else "parts", size, K * size % 16 == 0))
    wanted = {("forward", kind, parts) for kind, parts in (("few1", "whole"), ("few2", "whole"), ("few4", "whole"), ("small", "whole"), ("small", "parts"),
                                                           ("large", "whole"))}
    wanted |= {(what, kind, parts) for what in ("dx", "dW") for kind in ("small", "large") for parts in ("whole", "parts")}
    assert taken == {way + (size, direct) for way in wanted for size in (2, 4) for direct in (False, True)}
