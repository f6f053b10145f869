"""Geometry of the agent's update's launches up to the largest sizes its entry points take: calls that go all the way, with the HIP
entry points of a launch replaced by a driver that checks them.  No GPU is needed and none is used."""
import os
import subprocess

from paper_2001_08743_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_launch_is_one_that_the_hardware_takes(tmp_path):
    binding.load()
    exe = str(tmp_path / "explore_launch_check")
    subprocess.run(["gcc", "-O1", "-std=c11", "-Wall", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "paper_2001_08743_amd", "csrc", "explore_launch_check.c"), binding.LIB_PATH,
                    "-Wl,-rpath," + os.path.dirname(binding.LIB_PATH), "-Wl,-rpath,/opt/rocm/lib", "-L/opt/rocm/lib", "-lamdhip64", "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-4000:])
    assert "explore_launch_check ok" in r.stdout
