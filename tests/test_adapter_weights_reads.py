"""What is past an adapter's own rank is not read (include/cer.h): the many-token kernel's loads of weights, run on the CPU, with a page without access
right behind the last weight that the adapter has."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_nothing_past_the_adapters_rank_is_read(tmp_path):
    program = str(tmp_path / "reads")
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-O1", "-std=c++17", "-x", "hip", "--offload-host-only", "-w",
                           os.path.join(HERE, "adapter_weights_reads.cpp"), "-o", program])
    out = subprocess.run([program], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, (out.returncode, out.stdout[-200:].split("\r")[-2:])
