"""Sampling forms a token's weight for a sum, and again where the token that this sum's target falls on is looked for: no target
is missed as long as every compiled copy of the functions that form it gives the same bits.  Held to here: none of them leaves it
to the compiler whether a product is joined with a sum."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1810_08061_amd", "csrc", "sample.hip")


def test_weights_are_formed_with_written_out_roundings():
    with open(SOURCE) as f:
        source = f.read()
    weigh = source[source.index("struct Weigh {"):]
    weigh = weigh[:weigh.index("\n};")]
    bodies = re.findall(r"__device__ \w+ (\w+)\(float \w+\) const \{(.*?)\n    \}", weigh, re.S)
    assert [name for name, _ in bodies] == ["depth", "power", "weight"]
    for name, body in bodies:
        assert body.split("\n")[1].strip() == "#pragma clang fp contract(off)", name
    # and nothing else forms a weight
    assert len(re.findall(r"exp2f\(", source.replace("exp2f((float)a.bits - upto", ""))) == 1
