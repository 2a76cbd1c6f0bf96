"""The search for the key blocks of highest score, run on the host with a wavefront's lanes as loops."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_candidates_fit_their_place_and_lists_are_right(tmp_path):
    """At most 64 candidates are written into a run's place, whatever the scores: one more would land in the next run's."""
    exe = tmp_path / "model"
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__host__=", "-D__device__=", "-D__forceinline__=inline", "-Wno-unknown-pragmas",
                    os.path.join(HERE, "select_search_model.cpp"), "-o", str(exe)], check=True, capture_output=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stdout[-1500:]
