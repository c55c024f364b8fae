"""The generated code of the paged cache and of masked attention: no scratch memory, LDS of fixed size that leaves room for the workgroups that the launches count
on, M0 written by the requests only, and the loops are what their comments count.  CPU only (hipcc cross-compiles)."""
import os
import re
import subprocess

import pytest

from paper_2604_12798_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("codegen") / "masked.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([HIPCC] + flags + ["-S", "--cuda-device-only", "-o", str(out), os.path.join(build.CSRC, "masked.hip")], check=True, capture_output=True)
    text = out.read_text()
    bodies = dict(re.findall(r"^(_Z\S*_kernel\S*):[^\n]*\n(.*?)\.Lfunc_end", text, re.S | re.M))
    sizes = {m.group(1): tuple(map(int, m.groups()[1:])) for m in re.finditer(
        r"\.amdhsa_kernel (\S+)\n\s*\.amdhsa_group_segment_fixed_size (\d+)\n\s*\.amdhsa_private_segment_fixed_size (\d+).*?\.amdhsa_next_free_vgpr (\d+)", text, re.S)}
    return bodies, sizes


def masked(bodies):
    for n, body in bodies.items():
        m = re.search(r"attn_masked_kernelILi(\d+)ELi(\d)ELi(\d)ELb(\d)ELb(\d)", n)
        if m:
            yield n, body, *map(int, m.groups())


def test_no_scratch_and_room(kernels):
    bodies, sizes = kernels
    for name in ("kvp_append_kernel", "kvp_decode_kernel", "row_ranges_kernel", "attn_masked_kernel", "decode_merge_kernel"):
        assert any(name in n for n in bodies), name
    assert set(bodies) <= set(sizes)
    for n, (lds, scratch, _) in sizes.items():
        assert scratch == 0 and lds <= 160 * 1024, (n, lds, scratch)
        assert "scratch_" not in bodies[n], n
        assert not re.search(r"v_pk_(add|mul|fma)_f32", bodies[n]), n
    for n, _, d, rw, kq, cap, bias in masked(bodies):
        lds, _, vgprs = sizes[n]
        places = 3 if d == 64 else 2  # workgroups of four waves on a unit
        assert places * lds <= 160 * 1024 and vgprs <= 512 // places // 8 * 8, (n, lds, vgprs)


def test_requests_alone_write_m0(kernels):
    """The requests say that they change M0 and do not put it back."""
    for n, body, *_ in masked(kernels[0]):
        outside = re.sub(r";;#ASMSTART.*?;;#ASMEND", "", body, flags=re.S)
        assert "s_mov_b32 m0" in body and not re.search(r"\bm0\b", outside), n


def test_loop_of_whole_rounds(kernels):
    """Four steps of 32 keys without a condition but the max's: all products, one exponential a score (two and a reciprocal with a cap), each fragment read
    once, no wait for all that is on its way."""
    for n, body, d, rw, kq, cap, bias in masked(kernels[0]):
        if kq != 1:
            continue
        lines = body.split("\n")
        labels = {x.group(1): i for i, l in enumerate(lines) if (x := re.match(r"^(\.LBB\d+_\d+):", l))}
        products = 4 * (2 * d // 16 + (1 if bias and not cap else 0))
        loops = []
        for i, l in enumerate(lines):
            x = re.search(r"s_c?branch\w* (\.LBB\d+_\d+)", l)
            if x and labels.get(x.group(1), i) < i:
                seg = lines[labels[x.group(1)]:i]
                if sum("v_mfma" in s for s in seg) == products and sum("buffer_load" in s for s in seg) == 4 * 2 * d // 64:
                    loops.append(seg)
        assert loops, n
        seg = min(loops, key=len)
        assert sum("v_exp_f32" in s for s in seg) == 64 * (2 if cap else 1), n
        assert sum("v_rcp_f32" in s for s in seg) == (64 if cap else 0), n
        assert sum("ds_read_b128" in s for s in seg) == 4 * d // 16 and sum("ds_read_b64_tr_b16" in s for s in seg) == 8 * d // 16, n
        assert not any(re.search(r"s_waitcnt vmcnt\(0\)", s) for s in seg), n
