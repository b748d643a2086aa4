"""Registers of the 4-bit attention kernels as the compiler reports them, and the distance that matrix instructions written by
hand keep from what writes their operands."""
import os
import re
import subprocess

import pytest

from paper_2603_12201_amd import build


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("kv4") / "kv4.s")
    p = subprocess.run(["hipcc"] + build.FLAGS + ["--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-S", os.path.join(build.CSRC, "ic_kv4.hip"), "-o", out],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, check=True)
    with open(out) as f:
        return p.stdout, f.read()


def test_no_vector_register_is_spilled(compiled):
    """A reload from scratch would wait for everything that the loop has asked for ahead."""
    seen = 0
    for name, body in re.findall(r"Function Name: (\S+)(.*?)(?=Function Name|\Z)", compiled[0], re.S):
        if not re.search(r"kv4_(attn|attn_few|probs)_kernel", name):
            continue
        seen += 1
        use = {k: int(v) for k, v in re.findall(r"(AGPRs|VGPRs Spill|VGPRs|ScratchSize \[bytes/lane\]): (\d+)", body)}
        assert use["VGPRs Spill"] == 0 and use["ScratchSize [bytes/lane]"] == 0, (name, use)
        assert use["VGPRs"] <= 256 and use["AGPRs"] <= 256, (name, use)
    assert seen == 4 + 4 + 8                      # dense and paged, below and behind 4 GB; the weights with one and four waves to a query


def _registers(text):
    m = re.match(r"([av])(?:\[(\d+):(\d+)\]|(\d+))", text.strip())
    return (m.group(1), int(m.group(2) or m.group(4)), int(m.group(3) or m.group(4))) if m else None


def test_products_are_two_wait_states_behind_what_writes_their_operands(compiled):
    """The compiler does not see that the asm statements hold matrix instructions: two instructions (or an s_nop 1) lie between
    a vector instruction and the product that reads its result."""
    before, products = [], 0
    for line in compiled[1].split("\n"):
        if re.match(r"_Z\S+:", line):
            before = []
        line = line.split(";")[0].strip()
        if not line or line.startswith(".") or line.endswith(":"):
            continue
        if line.startswith("v_mfma"):
            products += 1
            read = [_registers(x) for x in line.split(None, 1)[1].split(",")[1:3]]
            states = 0
            for p in reversed(before[-3:]):
                if states >= 2:
                    break
                if p.startswith("v_") and not p.startswith("v_mfma"):
                    w = _registers(p.split(None, 1)[1].split(",")[0])
                    assert not any(w and r and w[0] == r[0] and w[1] <= r[2] and w[2] >= r[1] for r in read), (p, line)
                m = re.match(r"s_nop (\d+)", p)
                states += int(m.group(1)) + 1 if m else 1
        before.append(line)
    assert products > 500
