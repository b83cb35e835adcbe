"""Which kernel a product with 4-bit weights takes, and that the shapes of the GPU tests reach every one of them in every way: whole and ragged tiles, whole and ragged
ends of the contraction, aligned rows and others, every group, with zero points and without."""
import i4_checks


def calls():
    """(form, kernel, T, columns, n, group, zeros, aligned) of the GPU tests"""
    for T, d_in, d_out, group, zeros in i4_checks.SHAPES:
        for shifted in (False, True):
            for form, columns, n, planes, gated in (("linear", d_in, d_out, 1, False), ("gradient", d_out, d_in, 1, False), ("gated", d_in, d_out, 1, True),
                                                    ("gated gradient", d_out, d_in, 2, False)):
                aligned = not shifted and columns % 8 == 0
                yield form, i4_checks.kernel(T, columns, n, planes, gated, aligned, "gradient" in form, zeros and group == 32), T, columns, n, group, zeros, aligned


def test_every_kernel_is_reached():
    reached = {}
    for form, kernel, T, columns, n, group, zeros, aligned in calls():
        r = reached.setdefault((form, kernel, aligned), set())
        r |= {("whole columns", columns % 128 == 0), ("odd outputs", n % 2 == 1), ("zeros", zeros), ("group", group)}
        r.add(("one block", columns <= 128))
    for form in ("linear", "gradient", "gated", "gated gradient"):
        for kernel in i4_checks.KERNELS[:-1]:
            assert (form, kernel, True) in reached, (form, kernel)
        for kernel in i4_checks.KERNELS[:-1]:
            assert (form, kernel, False) in reached, (form, kernel)
        assert ((form, "square64", True) in reached) is (form == "linear") and (form, "square64", False) not in reached
        # both answers of each question somewhere among a form's kernels, every group
        both = set().union(*(r for (f, _, _), r in reached.items() if f == form))
        assert {("whole columns", True), ("whole columns", False), ("odd outputs", True), ("odd outputs", False), ("zeros", True), ("zeros", False), ("group", 32),
                ("group", 64), ("group", 128)} <= both


def test_limits():
    k = i4_checks.kernel
    assert k(1, 4096, 11008) == k(8, 13824, 13824) == "few"                      # a tile's other tokens would be none
    assert k(4096, 7, 4096) == k(100, (1 << 22) + 8, 64) == "few"                 # what the tiles do not take
    assert k(4096, 11008, 4096) == k(2048, 4096, 11008, gated=True) == "tile256"
    assert k(4096, 4096, 4096, aligned=False) == "tile256"
