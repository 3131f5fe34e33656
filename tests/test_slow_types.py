"""A config whose slow model has 4-bit layers: the library takes it; the oracle and the benchmark, which have no such model, refuse it."""
import dataclasses

import numpy as np
import pytest

import bench
import flowgen
import oracle
from workload import make_workload


def four_bit(c):
    return dataclasses.replace(flowgen.get_config(c), slow_dtype="mx4")


def test_the_oracle_has_no_four_bit_model():
    cfg = dataclasses.replace(four_bit(2), T=4, depth=4, n=64)
    wl = make_workload(cfg, n=64)
    with pytest.raises(ValueError):
        oracle.serve_batch(cfg, wl["fast"], wl["wide"], wl["forest"], wl["slow"], wl["tau"])
    with pytest.raises(ValueError):
        oracle.serve_batch3(cfg, wl["fast"], wl["wide"], wl["forest"], wl["forest"], wl["slow"], wl["tau"], wl["tau"])
    ref = oracle.serve_batch(dataclasses.replace(cfg, slow_dtype="bf16"), wl["fast"], wl["wide"], wl["forest"], wl["slow"], wl["tau"])
    assert ref["logits"].dtype == np.float32
    with pytest.raises(ValueError):
        bench.oracle_stage_run(wl, 1)


def test_the_benchmark_counts_no_bytes_for_it():
    peaks = {"hbm_gbs": 1.0, "bf16_tflops": 1.0, "bf16_tflops_sustained": 1.0}
    for cfg in (four_bit(2), four_bit(3)):
        with pytest.raises(ValueError):
            bench.kernel_launches_per_step(cfg, 1000)
        with pytest.raises(ValueError):
            bench.rooflines_for(cfg, 1000, 100, {"gemm": 1.0}, peaks, {})
    with pytest.raises(ValueError):
        bench.bench_batch(four_bit(2), 64, None, {k: None for k in ("torch", "sf", "hz", "ctx", "rank", "world", "local", "dist", "peaks")}, False, False, 0)
    assert flowgen.get_config(1).slow_bf16 is False and all(flowgen.get_config(c).slow_bf16 is True for c in (2, 3, 4, 5))
