"""The losses' products are the prefill kernel with other epilogues, unpacked weights and transposed reads of the LDS; what holds of its
inline assembly has to hold of them.  (The built code of all kernels, these among them, is checked in test_device_code.py and
test_counted_waits.py.)"""
import os
import subprocess

from paper_2603_18464_amd import build
from tests.test_device_code import built, ir_faults  # noqa: F401 (built: the fixture)


def test_products_in_flight_only_reach_the_wait(tmp_path):
    out = str(tmp_path / "device.ll")
    subprocess.run(["/opt/rocm/bin/hipcc", *build.FLAGS, "--cuda-device-only", "-S", "-emit-llvm",
                    os.path.join(build.CSRC, "head_loss.hip"), "-o", out], check=True, capture_output=True)
    ir = open(out).read()
    assert ir.count('asm sideeffect "v_mfma') > 100
    assert not ir_faults(ir)[:5]


def test_only_the_products_that_read_the_head_transposed_do_so(built):  # noqa: F811
    """grad_hidden of a head that is read as it is; nothing else pays for 8-byte reads."""
    with_tr = {n for n, code in built.items() if any(ins[1].startswith("ds_read_b64_tr_b16") for ins in code)}
    assert with_tr and all("EpiHiddenILi2E" in n for n in with_tr)
    assert len(with_tr) == sum("EpiHiddenILi2E" in n for n in built) == 5


def test_no_kernel_of_the_losses_spills_or_uses_scratch(built):  # noqa: F811
    names = [n for n in built if "loss_" in n or any(e in n for e in ("EpiStats", "EpiDz", "EpiHidden", "EpiHead", "EpiPlanes", "EpiGradients"))]
    assert len(names) > 40
    for n in names:
        assert not [ins[1] for ins in built[n] if ins[1].startswith("scratch_")], n
