"""The benchmark's measured DRAM traffic is tied to the kernel that it was measured on, not to the host code in the same file."""
import os
import shutil

import bench

CSRC = os.path.join(bench.ROOT, "paper_2402_03694_b200", "csrc")


def edited(tmp_path, name, old, new):
    for f in ("gemm_tc.cu", "tc_common.cuh"):
        shutil.copy(os.path.join(CSRC, f), tmp_path / f)
    text = (tmp_path / name).read_text()
    assert old in text
    (tmp_path / name).write_text(text.replace(old, new, 1))
    return bench.src_hash("gemm_tc.cu", str(tmp_path))


def test_the_hash_follows_device_code_only(tmp_path):
    now = bench.src_hash("gemm_tc.cu")
    # host code: a launcher, the tensor-map helper, its declaration
    assert edited(tmp_path, "gemm_tc.cu", "int launch_head_tc(", "int launch_the_head_tc(") == now
    assert edited(tmp_path, "gemm_tc.cu", "CU_TENSOR_MAP_L2_PROMOTION_L2_256B", "CU_TENSOR_MAP_L2_PROMOTION_L2_128B") == now
    assert edited(tmp_path, "tc_common.cuh", "int encode_tmap_bf16_2d(", "int encode_tmap_bf16(") == now
    # device code: tile sizes, a kernel's body, a helper of the header
    assert edited(tmp_path, "gemm_tc.cu", "constexpr uint32_t BK = 64;", "constexpr uint32_t BK = 128;") != now
    assert edited(tmp_path, "gemm_tc.cu", "tmem_dealloc_pair(tmem_base", "tmem_dealloc_pair(0 + tmem_base") != now
    assert edited(tmp_path, "tc_common.cuh", "kWaitLimitNs = 2000000000ull", "kWaitLimitNs = 1000000000ull") != now
