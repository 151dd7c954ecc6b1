"""How many workgroups of each kernel of the products in four bits, of the pairs' products and of the small updates a CU holds, from the registers and the
shared memory in the notes of the built library's own code objects (CPU): the choice of tiles counts on these numbers.  None of them keeps anything in scratch
memory."""
import os
import re
import struct
import subprocess

import pytest

ROCM_LLVM = "/opt/rocm/llvm/bin"
A_CU = {64: 4, 128: 2, 256: 1}       # kKinds of csrc/qoda_mx_product.hip and cut_of() of csrc/qoda_orthogonal.hip


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{mangled name: (vector registers, bytes of scratch memory a lane, bytes of shared memory)}"""
    readelf, objcopy = (os.path.join(ROCM_LLVM, "llvm-" + n) for n in ("readelf", "objcopy"))
    if not (os.path.exists(readelf) and os.path.exists(objcopy)):
        pytest.skip("no LLVM tools")
    from paper_2505_14371_amd import build, qoda

    if not os.path.exists(qoda.LIB_PATH):
        build.build()
    d = tmp_path_factory.mktemp("code")
    subprocess.check_call([objcopy, "--dump-section", f".hip_fatbin={d / 'fat'}", qoda.LIB_PATH, str(d / "rest")], stderr=subprocess.DEVNULL)
    data, out = (d / "fat").read_bytes(), {}
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
                out[get("name")] = tuple(int(get(k)) for k in ("vgpr_count", "private_segment_fixed_size", "group_segment_fixed_size"))
    return out


def fit(waves, registers, shared):
    return min(4 * min(8, 512 // (-(-registers // 8) * 8)) // waves, (160 << 10) // max(shared, 1))


def test_tiles(kernels):
    seen = 0
    for name, (registers, scratch, shared) in kernels.items():
        m = re.search(r"k_mx_productI.*Li\dELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)(E)EEv", name) or re.search(r"k_pair_productILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d)EEEv", name)
        if m:
            side, waves, steps = int(m.group(1)), int(m.group(3)) * int(m.group(4)), m.group(5)
            assert int(m.group(2)) == side and scratch == 0, name
            assert fit(waves, registers, shared) >= (1 if steps == "3" else A_CU[side]), (name, registers, shared)
            seen += 1
    assert seen == 3 * 5 + 5


def test_the_other_kernels_keep_nothing_in_scratch_memory(kernels):
    names = [n for n in kernels if re.search(r"k_(mx_rows|mx_columns|mx_values|mx_few_rows|small|squares|start|pair_join)", n)]
    assert len(names) >= 20
    for name in names:
        assert kernels[name][1] == 0, name


def test_small_updates(kernels):
    """Two or more workgroups of eight waves a CU where shared memory lets them in."""
    for name, (registers, _, shared) in kernels.items():
        m = re.search(r"k_smallI.*Li(\d+)ELi(\d+)EEEv", name)
        if m and int(m.group(2)) < 82000:
            assert fit(8, registers, shared) >= (160 << 10) // shared >= 2 or fit(8, registers, shared) >= 2, (name, registers)
