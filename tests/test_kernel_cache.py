"""The directory of compiled kernels, which a program may change as it runs."""
import os

from paper_2205_13603_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_kernel_lies_in_the_directory_that_is_set(tmp_path):
    """One that the process has compiled before is no exception: it is there for the next process."""
    op = B.expert_order_op(64, 3, 2)
    try:
        for place in ("one", "other", "one"):
            B.set_cache_dir(str(tmp_path / place))
            before = B.jit_stats()
            B.Variant(op, op.space(), B.default_trace(op.space()))
            after = B.jit_stats()
            assert len(list((tmp_path / place).glob("*.hsaco"))) == 1
        assert after["compiled"] == before["compiled"] and after["from_memory"] == before["from_memory"] + 1
    finally:
        B.set_cache_dir(os.environ.get("MS_CACHE_DIR") or os.path.join(ROOT, "paper_2205_13603_amd", "kcache"))
