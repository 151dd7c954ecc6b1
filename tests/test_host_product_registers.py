"""How many workgroups of each tile of the matrix products a CU holds, from the registers and the shared memory in the notes of the built library's own
code objects (CPU): the choice of tiles counts on these numbers."""
import os
import re
import shutil
import struct
import subprocess

import pytest

ROCM_LLVM = "/opt/rocm/llvm/bin"
A_CU = {(64, 64): 4, (128, 128): 2, (192, 256): 1, (256, 256): 1}       # plan_of() of csrc/qoda_linear.hip


@pytest.fixture(scope="module")
def products(tmp_path_factory):
    """[(type, form, rows, columns, waves, direct, vector registers, bytes of scratch memory a lane, bytes of shared memory)]"""
    readelf, objcopy = (os.path.join(ROCM_LLVM, "llvm-" + n) for n in ("readelf", "objcopy"))
    if not (os.path.exists(readelf) and os.path.exists(objcopy)):
        pytest.skip("no LLVM tools")
    from paper_2505_14371_amd import build, qoda

    if not os.path.exists(qoda.LIB_PATH):
        build.build()
    d = tmp_path_factory.mktemp("code")
    subprocess.check_call([objcopy, "--dump-section", f".hip_fatbin={d / 'fat'}", qoda.LIB_PATH, str(d / "rest")], stderr=subprocess.DEVNULL)
    data, out = (d / "fat").read_bytes(), []
    for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data):
        pos = m.start() + 32
        for _ in range(struct.unpack_from("<Q", data, m.start() + 24)[0]):
            off, size, n = struct.unpack_from("<QQQ", data, pos)
            target, pos = data[pos + 24:pos + 24 + n].decode(), pos + 24 + n
            if "gfx950" not in target:
                continue
            (d / "object").write_bytes(data[m.start() + off:m.start() + off + size])
            text = subprocess.run([readelf, "--notes", str(d / "object")], capture_output=True, text=True, check=True).stdout
            for block in text.split("- .agpr_count")[1:]:
                get = lambda k: re.search(r"\." + k + r":\s+(\S+)", block).group(1)  # noqa: E731
                kernel = re.search(r"k_productI(f|NS_4bf16E)Li(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELb(\d)E", get("name"))
                if kernel:
                    form, rows, columns, wm, wn, direct = (int(v) for v in kernel.groups()[1:])
                    out.append(("f32" if kernel.group(1) == "f" else "bf16", form, rows, columns, wm * wn, direct, int(get("vgpr_count")),
                                int(get("private_segment_fixed_size")), int(get("group_segment_fixed_size"))))
    assert len(out) == 2 * 3 * 3 * 2 + 3 * 2      # 32, 64 and 128 by type, form and loads; 192 and 256 in bf16 by direct loads
    return out


def test_as_many_workgroups_a_cu_as_the_choice_of_tiles_counts_on(products):
    for kind, form, rows, columns, waves, direct, registers, scratch, shared in products:
        assert scratch == 0, (kind, form, rows, columns, direct)
        if (rows, columns) in A_CU:
            a_simd = min(8, 512 // (-(-registers // 8) * 8))                     # waves
            fit = min(4 * a_simd // waves, (160 << 10) // shared)
            assert fit >= A_CU[rows, columns], (kind, form, rows, columns, direct, registers, shared)
