"""Which kernels' spills fail the build (CPU only)."""
from paper_2401_12522_amd.build import _spilling_products


def test_every_product_is_looked_at():
    names = ["_Z18gemm_skinny_kernelILi5EEvv", "_Z21gemm_q8_skinny_kernelILi9ELi3EEvv", "_Z19gemm_q8_tile_kernelILi4EEvv"]
    assert _spilling_products({n: {"vgprs": 254, "scratch": 0} for n in names}) == []
    assert _spilling_products({n: {"vgprs": 256, "scratch": 8} for n in names}) == sorted(names)
    assert _spilling_products({"_Z15some_other_kernv": {"scratch": 8}, names[1]: {}}) == []
