"""Which kernels the gated products run in.  CPU only: the rule is host code."""
import block_tiles as T


def test_the_shapes_run_where_they_are_meant_to(tmp_path):
    """A shape that has moved to another kernel leaves its own without a test on the device."""
    names = [(w, n) for w in ("linear", "dgrad") for n in T.SHAPES]
    want = [T.SHAPES[n][4][w == "dgrad"] for w, n in names]
    got = T.build(tmp_path)([T.shape(*n) for n in names])
    assert [(n, g) for n, g, w in zip(names, got, want) if g != w] == []
    for w in ("linear", "dgrad"):
        assert {g for (v, _), g in zip(names, got) if v == w} == {
            "64 all", "128 all", "256 all", "256 rounds and rest", "stream"} | (
                {"64 all once"} if w == "linear" else set())
