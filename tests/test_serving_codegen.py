"""The generated code of the serving operators: no kernel has scratch memory (a reload would wait for the tiles that are on their way), LDS is of
fixed size, and the decode loop over whole tiles is what its comment counts.  CPU only (hipcc cross-compiles)."""
import os
import re
import subprocess

import pytest

from paper_2604_12798_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("codegen") / "serving.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([HIPCC] + flags + ["-S", "--cuda-device-only", "-o", str(out), os.path.join(build.CSRC, "serving.hip")], check=True, capture_output=True)
    text = out.read_text()
    bodies = dict(re.findall(r"^(_Z\S*_kernel\S*):[^\n]*\n(.*?)\.Lfunc_end", text, re.S | re.M))
    sizes = {m.group(1): (int(m.group(2)), int(m.group(3))) for m in re.finditer(
        r"\.amdhsa_kernel (\S+)\n\s*\.amdhsa_group_segment_fixed_size (\d+)\n\s*\.amdhsa_private_segment_fixed_size (\d+)", text)}
    return bodies, sizes


def test_no_scratch_and_fixed_lds(kernels):
    bodies, sizes = kernels
    for name in ("norm_rope_kernel", "kv8_append_kernel", "kv8_append_one_kernel", "kv8_read_kernel", "kv8_decode_kernel", "decode_merge_kernel"):
        assert any(name in n for n in bodies), name
    assert set(bodies) <= set(sizes)
    for n, (lds, scratch) in sizes.items():
        assert scratch == 0 and lds <= 160 * 1024, (n, lds, scratch)
        assert "scratch_" not in bodies[n], n
        assert not re.search(r"v_pk_(add|mul|fma)_f32", bodies[n]), n


def test_decode_loop(kernels):
    """The loop over whole tiles: all products of a tile, one request for each 16 bytes of codes, no wait for everything."""
    for n, body in kernels[0].items():
        m = re.search(r"kv8_decode_kernelILi(\d+)ELi(\d)ELi(\d)", n)
        if not m:
            continue
        d, rt = int(m.group(1)), int(m.group(2))
        lines = body.split("\n")
        labels = {x.group(1): i for i, l in enumerate(lines) if (x := re.match(r"^(\.LBB\d+_\d+):", l))}
        loops = []  # (the rescale lies apart and branches back into the loop, too; the tile at the end requests nothing)
        for i, l in enumerate(lines):
            x = re.search(r"s_c?branch\w* (\.LBB\d+_\d+)", l)
            if x and labels.get(x.group(1), i) < i:
                seg = lines[labels[x.group(1)]:i]
                if sum("v_mfma" in s for s in seg) == rt * d // 4 and any("buffer_load" in s for s in seg):
                    loops.append(seg)
        assert loops, n
        seg = min(loops, key=len)
        assert sum("buffer_load_dwordx4" in s for s in seg) == 2 * d // 16, n
        assert sum("v_cvt_scalef32_pk_bf16_fp8" in s for s in seg) == d, n
        assert not any(re.search(r"s_waitcnt vmcnt\(0\)", s) for s in seg), n
