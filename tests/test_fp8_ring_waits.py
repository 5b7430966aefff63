"""The waits of the e4m3 ring tiles (csrc/fp8_ring.h) in the code the compiler made of them, followed as those of csrc/ring_k.h."""
from test_ring_waits import assembly, functions, weak_waits


def test_needed_stages_have_arrived(tmp_path):
    found = set()
    for name, lines in functions(assembly("fp8.hip", str(tmp_path / "kernels.s"))).items():
        weak, rings = weak_waits(lines)
        assert not weak, (name, weak)
        found |= rings
    assert found == {(4, 6), (3, 7)}                                # small and big tiles
