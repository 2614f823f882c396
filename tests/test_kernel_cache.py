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


def test_a_kernel_in_use_is_not_built_again_for_another_directory(tmp_path):
    """What a variant holds goes into the new directory as it is, into one without a place for it not at all; what lies there already stays."""
    op = B.expert_order_op(64, 3, 2)
    held = []

    def build():
        before = B.jit_stats()
        held.append(B.Variant(op, op.space(), B.default_trace(op.space())))
        after = B.jit_stats()
        return [after[k] - before[k] for k in ("compiled", "from_disk", "from_memory")]

    try:
        B.set_cache_dir(str(tmp_path / "one"))
        build()  # from wherever
        (first,) = (tmp_path / "one").iterdir()
        B.set_cache_dir(str(tmp_path / "other"))
        assert build() == [0, 0, 1]
        (second,) = (tmp_path / "other").iterdir()
        assert second.name == first.name and second.read_bytes() == first.read_bytes() and len(first.read_bytes()) > 64
        assert build() == [0, 0, 1]
        (tmp_path / "full").mkdir()
        kept = tmp_path / "full" / first.name
        kept.write_bytes(first.read_bytes())
        os.utime(kept, (1, 1))
        B.set_cache_dir(str(tmp_path / "full"))
        assert build() == [0, 0, 1] and kept.stat().st_mtime == 1 and len(list((tmp_path / "full").iterdir())) == 1
        (tmp_path / "file").write_bytes(b"")
        for place in (str(tmp_path / "file" / "none"), ""):
            B.set_cache_dir(place)
            assert build() == [0, 0, 1]
    finally:
        B.set_cache_dir(os.environ.get("MS_CACHE_DIR") or os.path.join(ROOT, "paper_2205_13603_amd", "kcache"))
