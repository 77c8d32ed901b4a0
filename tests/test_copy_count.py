"""What a producer that gives up waits for before its CTA may exit (no GPU: a wait that runs out is not brought about on one)."""

import pathlib
import re
import subprocess

HERE = pathlib.Path(__file__).parent
CSRC = HERE.parent / "paper_2606_00144_gb300" / "csrc"


def test_the_last_query_copy_is_waited_for_wherever_the_walk_ends(tmp_path):
    exe = tmp_path / "walk"
    subprocess.run(["g++", "-std=c++17", "-I", str(CSRC), "-o", str(exe), str(HERE / "copy_count_walk.cpp")], check=True)
    walks, left, left_by_segments, for_nothing, none = map(int, subprocess.run([str(exe)], capture_output=True, text=True,
                                                                              check=True).stdout.split())
    assert walks > 1000 and left == 0 and for_nothing == 0 and none == 0
    assert left_by_segments > 0          # (segments that were walked to their ends miss those that were begun)


def test_the_paged_producers_count_every_query_copy():
    source = (CSRC / "bd_verify_tc.cu").read_text()
    producers = source[source.index("// Two producers, of K"):source.index("tma_prefetch_map(&kmap);", source.index("// Two producers, of K"))]
    assert re.findall(r"load_q\([^)]*\);.*\n\s*queries\.add\(\);", producers) and producers.count("load_q(") == 1
    assert producers.count("next_q(unit)") == 2 and "queries.last_parity()" in producers
