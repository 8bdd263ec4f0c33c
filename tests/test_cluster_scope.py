"""CPU checks of the memory order between the CTAs of a cluster, from the kernels' source.

An arrive on another CTA's mbarrier, and a wait for one, are ordered towards that CTA only if they are of
cluster scope (the default is the CTA's); no run shows the difference reliably."""
import os
import re

from paper_2004_14696_gb300 import build as B


def read(name):
    with open(os.path.join(B.CSRC, name)) as f:
        return f.read()


def test_arrivals_at_another_cta_are_of_cluster_scope():
    found = 0
    for name in sorted(os.listdir(B.CSRC)):
        for ptx in re.findall(r"mbarrier\.arrive[\w.:]*", read(name)):
            if "shared::cluster" in ptx:
                found += 1
                assert re.match(r"mbarrier\.arrive\.(release|relaxed)\.cluster\.shared::cluster", ptx), (name, ptx)
    assert found >= 2


def test_the_pairs_of_the_8_bit_products_wait_at_cluster_scope():
    body = read("fp8_gemm.cu")
    body = body[body.index("    fp8_pair_kernel("):body.index("cudaError_t launch_fp8_pair(")]
    waits = re.findall(r"warp_wait(<true>)?\(smem_u32\((\w+)_bar", body)
    of_both = [scope for scope, bar in waits if bar in ("full", "empty", "tfull", "tempty", "asked")]
    assert len(of_both) >= 6 and all(of_both), waits
    assert re.search(r"mbarrier\.try_wait\.parity\.acquire\.cluster\.shared::cta", read("tc_ptx.cuh"))
