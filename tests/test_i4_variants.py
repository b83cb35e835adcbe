"""The shapes of the GPU tests reach every kernel of the products with 4-bit weights with every group, with zero points and without, aligned and not."""
import i4_checks
import i4_variants


def test_every_variant_is_reached():
    reached = set()
    for shape in i4_checks.SHAPES + i4_variants.SHAPES:
        reached |= set(i4_variants.reached(*shape))
    there = set(i4_variants.all_there_are())
    assert reached <= there, sorted(reached - there, key=str)
    assert there <= reached, sorted(there - reached, key=str)
