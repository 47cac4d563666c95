"""The addresses of the weight gradient's loads, formed by the kernel's own loaders on the host."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_weight_gradient_loads_stay_in_their_operand(tmp_path):
    # experts without rows, the last ones among them: nothing past the operand's last row is loaded
    exe = str(tmp_path / "expert_pieces")
    # host code only: nothing is compiled for the GPU, and nothing runs there
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-host-only", "-x", "hip", "-O1", "-std=c++17",
                    os.path.join(HERE, "expert_pieces.hip"), "-o", exe], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout.strip().splitlines()[-1:]
    assert "inside" in r.stdout
