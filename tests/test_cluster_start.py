"""Another CTA's shared memory is there only once that CTA has started.  Read off the source, for what this prevents is a fault: the decode path's clusters arrive at
their barrier on entry and wait there ahead of the first exchange."""
import pathlib

CSRC = pathlib.Path(__file__).parents[1] / "paper_2609_17184_b200" / "csrc"


def test_the_gemm_of_a_decode_pass():
    body = (CSRC / "gemm.cuh").read_text().split("gemm_bf16_kernel(const __grid_constant__ GemmParams p) {")[1]
    arrive, wait = body.find("barrier.cluster.arrive"), body.find("barrier.cluster.wait")
    assert 0 <= arrive < wait < min(body.find(x) for x in ("gemm_push_tile<", "cluster.sync()"))


def test_the_selection():
    body = (CSRC / "select.cuh").read_text().split("select_kernel(const __grid_constant__ SelectParams p) {")[1]
    # what the kernel runs begins behind its helpers: at the wait for the logits
    start = body.index("  pdl_wait();\n  asm volatile(\"barrier.cluster.wait")
    assert 0 <= body.find("barrier.cluster.arrive") < start and "R." not in body[start:body.index("if (kind == RO_TARGET)", start)]
